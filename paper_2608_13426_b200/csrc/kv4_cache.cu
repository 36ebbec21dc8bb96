// Filling and reading the 4-bit cache of kv4.cuh.
//
// Append: a key is normalised and rotated (heads.cuh), rounded to bf16 as a 16-bit cache would hold it, and quantised; a value is
// quantised.  Bound: HBM, K and V read once and a quarter of that written (or five quarters, with the held values).  A warp takes the
// rows of neighbouring tokens of one head after another: eight lanes hold the 64 columns of a step, so least and largest value meet in
// three shuffles, each lane makes one word of codes, and no shared memory is used.
//
// The keys are rounded to bf16 before the codes are taken so that the codes follow from the 64-bit formula alone (norm_rope_row): the
// border of a code moves with the least value and the step, and an fp32 chain's last bits would decide it otherwise.
#include "kv4.cuh"

namespace rmm {
namespace {

constexpr int kWarps = 8;

struct CacheArgs {
    HeadRows k, v;
    kv4::View cache;
    RopeView rope;
    int64_t groups;             // groups of neighbouring tokens of one sequence, per sequence
    int64_t B, L;
    int D, lanes, heads_each;   // lanes of a row; heads of a warp
    int head_groups;
    int *status;
};

struct Quantised {
    uint32_t codes, pair;
};

__device__ __forceinline__ Quantised quantise8(const float (&x)[8])
{
    float lo = x[0], hi = x[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) {
        lo = fminf(lo, x[i]);
        hi = fmaxf(hi, x[i]);
    }
#pragma unroll
    for (int d = 4; d > 0; d >>= 1) {
        lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, d));
        hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, d));
    }
    const uint32_t step = (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(__fdiv_rn(__fsub_rn(hi, lo), 15.f)));
    const float s = bf16_bits(step);
    Quantised q;
    q.codes = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float n = s > 0.f ? fminf(rintf(__fdiv_rn(__fsub_rn(x[i], lo), s)), 15.f) : 0.f;
        q.codes |= (uint32_t)n << (4 * i);
    }
    q.pair = step | (__float_as_uint(lo) & 0xffff0000u);
    return q;
}

__device__ __forceinline__ void dequantise8(uint32_t codes, uint32_t pair, float (&x)[8])
{
    const float s = bf16_bits(pair & 0xffffu), m = __uint_as_float(pair & 0xffff0000u);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = fmaf(s, (float)(codes >> (4 * i) & 15u), m);
}

template <typename TI, bool HELD>
__global__ void __launch_bounds__(kWarps * 32) kv4_append_kernel(const __grid_constant__ CacheArgs a)
{
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, per = 32 / a.lanes, D = a.D;
    const int64_t unit = (int64_t)(blockIdx.x / a.head_groups) * kWarps + warp;
    if (unit >= a.B * a.groups) return;
    const int64_t b = unit / a.groups, i = (unit - b * a.groups) * per + lane / a.lanes;
    const int col = (lane & (a.lanes - 1)) * 8, chunk = col / 8;
    const int h0 = (int)(blockIdx.x % a.head_groups) * a.heads_each, h1 = min(a.k.heads, h0 + a.heads_each);
    int len, rows;
    kv4::sequence(a.cache, b, len, rows, a.status);
    const int64_t at = (int64_t)len - rows + i;
    const bool row = i < a.L;
    bool live = row && i < rows;
    if (live && (at < 0 || (a.rope.table != nullptr && at >= a.rope.rows))) {
        atomicExch(a.status, (int)RMM_ERR_BOUNDS);
        live = false;
    }
    uint8_t *base = live ? kv4::block_of(a.cache, b, h0, at / kv4::kBlock, D, a.status) : nullptr;
    const int t = (int)(at & (kv4::kBlock - 1));
    RowLane k;
    row_weights(k, a.k.weight, a.rope, col, D);
    row_angles(k, a.rope, live ? at : 0, col);
    const TI *ks = static_cast<const TI *>(a.k.src) + b * a.k.s_b + i * a.k.s_r + col;
    const TI *vs = static_cast<const TI *>(a.v.src) + b * a.v.s_b + i * a.v.s_r + col;
    for (int h = h0; h < h1; ++h) {
        float x[8], v[8], z[8];
        if (live) {
            load8(ks + h * a.k.s_h, a.k.vec_in != 0, x);
            load8(vs + h * a.v.s_h, a.v.vec_in != 0, v);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = v[e] = 0.f;
        }
        norm_rope_row<true>(x, k, a.lanes, D, a.rope.eps, z);
        if constexpr (sizeof(TI) == 4) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = __bfloat162float(__float2bfloat16_rn(v[e]));
        }
        const Quantised qk = quantise8(z), qv = quantise8(v);
        if (base != nullptr) {
            uint32_t *w = reinterpret_cast<uint32_t *>(base + (h - h0) * a.cache.head_stride);
            w[kv4::key_word(D, t, chunk)] = qk.codes;
            w[kv4::value_word(D, t, chunk)] = qv.codes;
            if ((chunk & 7) == 0) {
                w[kv4::key_pair_word(D, t, chunk >> 3)] = qk.pair;
                w[kv4::value_pair_word(D, t, chunk >> 3)] = qv.pair;
            }
        }
        if constexpr (HELD) {
            if (row) {
                dequantise8(qk.codes, qk.pair, x);   // (rows that are none: zeros)
                dequantise8(qv.codes, qv.pair, v);
                store8(static_cast<__nv_bfloat16 *>(a.k.dst) + b * a.k.d_b + h * a.k.d_h + i * a.k.d_r + col, a.k.vec_out != 0, x);
                store8(static_cast<__nv_bfloat16 *>(a.v.dst) + b * a.v.d_b + h * a.v.d_h + i * a.v.d_r + col, a.v.vec_out != 0, v);
            }
        }
    }
}

template <typename TO>
__global__ void __launch_bounds__(kWarps * 32) kv4_read_kernel(const __grid_constant__ CacheArgs a)
{
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, per = 32 / a.lanes, D = a.D;
    const int64_t unit = (int64_t)(blockIdx.x / a.head_groups) * kWarps + warp;
    if (unit >= a.B * a.groups) return;
    const int64_t b = unit / a.groups, i = (unit - b * a.groups) * per + lane / a.lanes;
    const int col = (lane & (a.lanes - 1)) * 8, chunk = col / 8;
    const int h0 = (int)(blockIdx.x % a.head_groups) * a.heads_each, h1 = min(a.k.heads, h0 + a.heads_each);
    int len, rows;
    kv4::sequence(a.cache, b, len, rows, a.status);
    if (i >= a.L) return;
    const int64_t at = (int64_t)len - rows + i;
    const uint8_t *base = nullptr;
    if (i < rows) {
        if (at < 0) atomicExch(a.status, (int)RMM_ERR_BOUNDS);
        else base = kv4::block_of(a.cache, b, h0, at / kv4::kBlock, D, a.status);
    }
    const int t = (int)(at & (kv4::kBlock - 1));
    for (int h = h0; h < h1; ++h) {
        float k[8] = {}, v[8] = {};
        if (base != nullptr) {
            const uint32_t *w = reinterpret_cast<const uint32_t *>(base + (h - h0) * a.cache.head_stride);
            dequantise8(w[kv4::key_word(D, t, chunk)], w[kv4::key_pair_word(D, t, chunk >> 3)], k);
            dequantise8(w[kv4::value_word(D, t, chunk)], w[kv4::value_pair_word(D, t, chunk >> 3)], v);
        }
        store8(static_cast<TO *>(a.k.dst) + b * a.k.d_b + h * a.k.d_h + i * a.k.d_r + col, a.k.vec_out != 0, k);
        store8(static_cast<TO *>(a.v.dst) + b * a.v.d_b + h * a.v.d_h + i * a.v.d_r + col, a.v.vec_out != 0, v);
    }
}

int fill(CacheArgs &a, const HeadRows &K, const HeadRows &V, const kv4::View &cache, int64_t B, int64_t L, int64_t D, int *status, int64_t &blocks)
{
    a.k = K;
    a.v = V;
    a.cache = cache;
    a.B = B;
    a.L = L;
    a.D = (int)D;
    a.lanes = (int)D / 8;
    a.groups = ceil_div(L, 32 / a.lanes);
    a.status = status;
    // All heads of a token by one warp, where that still leaves sixteen warps an SM
    const int64_t token_blocks = ceil_div(B * a.groups, kWarps), want = ceil_div((int64_t)sm_count() * 2, token_blocks);
    a.head_groups = (int)(want < K.heads ? want : K.heads);
    a.heads_each = (int)ceil_div(K.heads, a.head_groups);
    a.head_groups = (int)ceil_div(K.heads, a.heads_each);
    blocks = token_blocks * a.head_groups;
    return blocks > INT32_MAX ? fail(RMM_ERR_UNSUPPORTED, "kv4: more than 2^31 blocks of rows") : (int)RMM_OK;
}

}  // namespace

int launch_kv4_append(const HeadRows &K, const HeadRows &V, const kv4::View &cache, int in_bf16, const RopeView &rope, int64_t B, int64_t L, int64_t D,
                      int *status, cudaStream_t stream)
{
    CacheArgs a = {};
    int64_t blocks;
    a.rope = rope;
    if (int rc = fill(a, K, V, cache, B, L, D, status, blocks)) return rc;
    const bool held = K.dst != nullptr;
    auto kern = in_bf16 ? (held ? kv4_append_kernel<__nv_bfloat16, true> : kv4_append_kernel<__nv_bfloat16, false>)
                        : (held ? kv4_append_kernel<float, true> : kv4_append_kernel<float, false>);
    prof_begin("kv4_append_kernel", stream);
    launch_kernel(kern, dim3((unsigned)blocks), dim3(kWarps * 32), 0, stream, 1, a);
    return check_launch("kv4_append_kernel", stream);
}

int launch_kv4_read(const HeadRows &K, const HeadRows &V, const kv4::View &cache, int out_bf16, int64_t B, int64_t L, int64_t D, int *status,
                    cudaStream_t stream)
{
    CacheArgs a = {};
    int64_t blocks;
    if (int rc = fill(a, K, V, cache, B, L, D, status, blocks)) return rc;
    auto kern = out_bf16 ? kv4_read_kernel<__nv_bfloat16> : kv4_read_kernel<float>;
    prof_begin("kv4_read_kernel", stream);
    launch_kernel(kern, dim3((unsigned)blocks), dim3(kWarps * 32), 0, stream, 1, a);
    return check_launch("kv4_read_kernel", stream);
}

}  // namespace rmm
