// Attention of a few query rows over a paged cache held in 4 bits (kv4.cuh):  O = softmax(Q[:, I] K^[:, I]^T / sqrt(Dh)) V^,
// K^ = m + s n, V^ likewise, I the kept features of each query head (paper Sec. 3.3, rho_t = 1).
//
// Bound: HBM, 9/16 byte a value of K and V, as long as turning codes into matrix operands costs fewer instructions than the bytes
// take: at the copy rate an SM receives 41 values a cycle and can issue 128 lanes' worth of instructions, three a value.  So:
//   - codes are never multiplied out.  A code n in the low bits of a 16-bit word is the fp16 number n 2^-24 (or 16 n 2^-24, four
//     bits up), so one AND makes two operands of mma.m16n8k16: 5 instructions per 8 codes of K, 6 of V.  Products are exact, the sums
//     fp32.  Steps and least values come in afterwards, per key:  logit = sum_j s_j (q n)_j + m_j sum(q_j)  over the 64-column
//     groups j, and  O = sum_t (p_t s_t) n_t + sum_t p_t m_t.
//   - Q is scaled by a power of two to [2^14, 2^15) at its largest, so that what bf16 held is exact in fp16 down to 2^-28 of that.
//   - p_t s_t is rounded to fp16 (relative 2^-12, where the library's other forms round P to bf16).  The exponent's reference m is
//     that of p s, refreshed when p s would pass 2^14 and then set so that the largest is 2^6: what lies under 2^-14 loses bits gradually,
//     2^-25 against a largest weight of 2^6.
//   - S^T = K Q^T and O^T = V^T P^T, so that the 8 columns of an instruction are query rows that share a kv head and its 16 rows are
//     keys (or columns of V): the group's rows fill what 128-row tcgen05 tiles would pad.
// The 16-token blocks of all jobs (sequence, kv head, row tile) form one axis that is cut into equal shares, one a CTA, whatever the
// lengths are: they live on the device, so nothing is planned on the host and a captured call follows them.  Within a CTA every
// warp takes every eighth block through a ring of its own, filled by bulk copies of whole blocks, which runs on across jobs.  A job
// that ends in another CTA leaves its sums in the workspace; the last CTA of a job to arrive adds them up, in order.
#include <math.h>

#include <cuda_fp16.h>

#include "kv4.cuh"
#include "select.cuh"
#include "sm100_ptx.cuh"

namespace rmm {
namespace {

constexpr int kWarps = 8;
constexpr float kGrow = 14.f, kTop = 6.f, kLeastStep = -80.f;   // log2: see above; steps below 2^-80 weigh as 2^-80 in the reference

struct AttnArgs {
    const __nv_bfloat16 *q;
    __nv_bfloat16 *o;
    int64_t q_sb, q_sh, q_sr, o_sb, o_sh, o_sr;
    kv4::View cache;
    int B, Hkv, group, L, kd, causal, chunks;
    float scale_log2;
    int32_t *idx_feat;
    float *part;              // [2 CTAs][rows][D + 2]: sums, then (reference, sum of weights)
    unsigned *counters;
    int *status;
    unsigned long long wait_ns;
    int withhold;
};

template <int D, int NT>
struct Shape {
    static constexpr int kRows = 8 * NT, kBlockBytes = 18 * D, kGroups = D / 64;
    static constexpr int kCtas = D * NT <= 128 ? 2 : 1;                        // an SM
    static constexpr int kStages = D == 64 ? 8 : (D == 128 ? (NT == 1 ? 4 : 8) : 4);
    static constexpr int kPitchQ = D + 8, kPitchM = 66;
    static constexpr int kOffQ = kWarps * kStages * kBlockBytes;               // fp16 [rows][pitch]
    static constexpr int kOffMerge = kOffQ + kRows * kPitchQ * 2;              // fp32 [warp][row][pitch]
    static constexpr int kOffMl = kOffMerge + kWarps * kRows * kPitchM * 4;    // [warp][row]: (reference, sum), then the warp's factor
    static constexpr int kOffRow = kOffMl + kWarps * kRows * 8;                // [row]: scale, visible keys, then sums of q by group
    static constexpr int kOffKept = kOffRow + kRows * (2 + kGroups) * 4;       // [row's head][D / 32]
    static constexpr int kOffTot = kOffKept + kRows * (D / 32) * 4;            // [row]: reference, sum of the CTA
    static constexpr int kOffBar = (kOffTot + kRows * 8 + 15) / 16 * 16;       // barriers, then the tokens of each ring entry
    static constexpr int kSmem = kOffBar + kWarps * kStages * 12;
    static_assert(kSmem <= 227 * 1024 / kCtas - 2048, "shared memory");
};

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi)
{
    uint32_t y;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(y) : "f"(hi), "f"(lo));
    return y;
}
__device__ __forceinline__ float lg2(float x)
{
    float y;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// A place on the axis of all jobs' blocks.
struct Cursor {
    int b, len, rows, nb, valid;   // sequence, its tokens and rows, blocks of a job, row tiles that hold rows
    int hk, chunk;
    __device__ __forceinline__ int blocks() const { return chunk < valid ? nb : 1; }
    __device__ __forceinline__ bool reads() const { return chunk < valid && len > 0; }
};

template <int ROWS>
__device__ __forceinline__ void cursor_sequence(const AttnArgs &a, Cursor &c)
{
    kv4::sequence(a.cache, c.b, c.len, c.rows, a.status);
    c.nb = max(1, (c.len + kv4::kBlock - 1) / kv4::kBlock);
    c.valid = (c.rows * a.group + ROWS - 1) / ROWS;
}
template <int ROWS>
__device__ __forceinline__ int sequence_units(const AttnArgs &a, int b)
{
    Cursor c;
    c.b = b;
    cursor_sequence<ROWS>(a, c);
    return a.Hkv * (c.valid * c.nb + a.chunks - c.valid);
}
template <int ROWS>
__device__ __forceinline__ void cursor_next(const AttnArgs &a, Cursor &c)
{
    if (++c.chunk < a.chunks) return;
    c.chunk = 0;
    if (++c.hk < a.Hkv) return;
    c.hk = 0;
    if (++c.b < a.B) cursor_sequence<ROWS>(a, c);
}

// Kept features of the heads of a row tile (one warp a head) as bit masks; the rule of every other form: squares summed in fp64,
// rounded to fp32, the kd largest, the lower index first.
template <int D>
__device__ __noinline__ void keep_features(const AttnArgs &a, int b, int hk, int rows, int row0, int nrows, bool first, uint32_t *kept)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int idx = warp; idx < min(a.group, nrows); idx += kWarps) {
        const int64_t h = (int64_t)hk * a.group + (row0 + idx) % a.group;
        const __nv_bfloat16 *qp = a.q + b * a.q_sb + h * a.q_sh;
        uint32_t u[D / 32];
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
            double e = 0.0;
            for (int r = 0; r < rows; ++r) {
                const float x = __bfloat162float(qp[r * a.q_sr + i * 32 + lane]);
                e += (double)(x * x);
            }
            u[i] = sel::key_image((float)e);
        }
        uint32_t tau = 0;
#pragma unroll 1
        for (int bit = 30; bit >= 0; bit -= 2) {
            int n[3] = {0, 0, 0};
#pragma unroll
            for (int i = 0; i < D / 32; ++i)
#pragma unroll
                for (int v = 0; v < 3; ++v) n[v] += u[i] >= (tau | ((unsigned)(v + 1) << bit)) ? 1 : 0;
            unsigned digit = 0;
#pragma unroll
            for (int v = 0; v < 3; ++v) digit += __reduce_add_sync(0xffffffffu, n[v]) >= a.kd ? 1u : 0u;
            tau |= digit << bit;
        }
        int n = 0;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) n += u[i] > tau ? 1 : 0;
        int need = a.kd - __reduce_add_sync(0xffffffffu, n), at = 0;
        int32_t *out = first && a.idx_feat != nullptr && row0 + idx < a.group ? a.idx_feat + ((int64_t)b * a.Hkv * a.group + h) * a.kd : nullptr;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
            const unsigned eq = __ballot_sync(0xffffffffu, u[i] == tau), lt = (1u << lane) - 1u;
            const bool keep = u[i] > tau || (u[i] == tau && __popc(eq & lt) < need);
            need -= min(need, __popc(eq));
            const unsigned m = __ballot_sync(0xffffffffu, keep);
            if (out != nullptr && keep) out[at + __popc(m & lt)] = i * 32 + lane;
            at += __popc(m);
            if (lane == 0) kept[idx * (D / 32) + i] = m;
        }
    }
}

template <int D, int NT>
__global__ void __launch_bounds__(kWarps * 32, Shape<D, NT>::kCtas) kv4_attn_kernel(const __grid_constant__ AttnArgs a)
{
    using namespace ptx;
    using S = Shape<D, NT>;
    constexpr int ROWS = S::kRows, NG = S::kGroups, ST = S::kStages, W32 = D / 32;
    extern __shared__ __align__(1024) uint8_t smem[];
    __shared__ int s_scan[kWarps], s_begin[2], abort_flag, s_last;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t4 = lane & 3;
    const uint32_t ring = smem_u32(smem) + warp * ST * S::kBlockBytes, bars = smem_u32(smem) + S::kOffBar + warp * ST * 8;
    int *tokens = reinterpret_cast<int *>(smem + S::kOffBar + kWarps * ST * 8) + warp * ST;
    __half *qs = reinterpret_cast<__half *>(smem + S::kOffQ);
    float *merge = reinterpret_cast<float *>(smem + S::kOffMerge), *ml = reinterpret_cast<float *>(smem + S::kOffMl);
    float *row_scale = reinterpret_cast<float *>(smem + S::kOffRow), *row_sum = row_scale + 2 * ROWS, *tot = reinterpret_cast<float *>(smem + S::kOffTot);
    int *row_vis = reinterpret_cast<int *>(row_scale + ROWS);
    uint32_t *kept = reinterpret_cast<uint32_t *>(smem + S::kOffKept);

    if (lane == 0)
        for (int i = 0; i < ST; ++i) mbar_init(bars + 8 * i, 1);
    if (tid == 0) abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    __syncthreads();
    pdl_wait();

    // ---- this CTA's share of the axis
    auto scan = [&](int v, int &sum) {   // inclusive, over the block
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int o = __shfl_up_sync(0xffffffffu, v, d);
            if (lane >= d) v += o;
        }
        __syncthreads();
        if (lane == 31) s_scan[warp] = v;
        __syncthreads();
        int before = 0;
        sum = 0;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            if (w < warp) before += s_scan[w];
            sum += s_scan[w];
        }
        return v + before;
    };
    int total = 0, mine = 0, upto = 0;
    for (int b0 = 0; b0 < a.B; b0 += kWarps * 32) {
        int sum;
        mine = b0 + tid < a.B ? sequence_units<ROWS>(a, b0 + tid) : 0;
        upto = scan(mine, sum);
        total += sum;
    }
    const int ctas = min((int)gridDim.x, (total + kWarps - 1) / kWarps);   // eight blocks each at least
    if ((int)blockIdx.x >= ctas) return;
    int u = (int)((int64_t)total * blockIdx.x / ctas);
    const int u_end = (int)((int64_t)total * (blockIdx.x + 1) / ctas);
    for (int b0 = 0, base = 0; b0 < a.B; b0 += kWarps * 32) {
        int sum = 0;
        if (a.B > kWarps * 32) {
            mine = b0 + tid < a.B ? sequence_units<ROWS>(a, b0 + tid) : 0;
            upto = scan(mine, sum);
        }
        if (u >= base + upto - mine && u < base + upto) {
            s_begin[0] = b0 + tid;
            s_begin[1] = u - (base + upto - mine);
        }
        base += sum;
    }
    __syncthreads();

    Cursor cur;
    cur.b = s_begin[0];
    cursor_sequence<ROWS>(a, cur);
    int t_at;   // first block of the current job's part
    {
        const int per_head = cur.valid * cur.nb + a.chunks - cur.valid;
        int off = s_begin[1];
        cur.hk = off / per_head;
        off -= cur.hk * per_head;
        if (off < cur.valid * cur.nb) {
            cur.chunk = off / cur.nb;
            t_at = off - cur.chunk * cur.nb;
        } else {
            cur.chunk = cur.valid + off - cur.valid * cur.nb;
            t_at = 0;
        }
    }

    // ---- the warp's loads: blocks t_at + warp, + 8, .. of every part, ST of them under way
    Cursor pc = cur;
    int p_u = u, p_t0 = t_at, p_t = t_at + warp, p_page = 0, p_slot = 0;   // p_u: axis position of p_t0
    auto settle = [&]() {   // on to the next block that has something to load; its page number is fetched here, ahead of its use
        while (p_u < u_end) {
            const int end = min(pc.blocks(), p_t0 + u_end - p_u);
            if (pc.reads() && p_t < end) {
                p_page = __ldg(a.cache.pages + pc.b * a.cache.pages_stride + (p_t >> a.cache.page_shift));
                return;
            }
            p_u += end - p_t0;
            p_t0 = 0;
            p_t = warp;
            if (p_u < u_end) cursor_next<ROWS>(a, pc);
        }
    };
    auto request = [&]() {
        if (p_u >= u_end) return;
        if (lane == 0) {
            const uint32_t bar = bars + 8 * p_slot;
            const bool good = p_page >= 0 && p_page < a.cache.n_pages;
            tokens[p_slot] = good ? min(kv4::kBlock, pc.len - p_t * kv4::kBlock) : 0;
            if (!good) {
                atomicExch(a.status, (int)RMM_ERR_BOUNDS);
                mbar_arrive(bar);
            } else if (!(a.withhold && blockIdx.x == 0 && warp == 0)) {   // (test switch: these copies are never requested)
                const uint8_t *src = a.cache.pool + (int64_t)p_page * a.cache.page_stride + pc.hk * a.cache.head_stride +
                                     (int64_t)(p_t & ((1 << a.cache.page_shift) - 1)) * S::kBlockBytes;
                mbar_arrive_expect_tx(bar, S::kBlockBytes);
                asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                             ::"r"(ring + (uint32_t)p_slot * S::kBlockBytes), "l"(src), "r"((uint32_t)S::kBlockBytes), "r"(bar) : "memory");
            }
        }
        if (++p_slot == ST) p_slot = 0;
        p_t += kWarps;
        settle();
    };
    settle();
    for (int i = 0; i < ST; ++i) request();

    int slot = 0;
    uint32_t phases = 0;
    bool dead = false;
    while (u < u_end) {
        const int t_end = min(cur.blocks(), t_at + u_end - u);
        const int row0 = cur.chunk * ROWS, nrows = max(0, min(ROWS, cur.rows * a.group - row0));
        const bool whole = t_at == 0 && t_end == cur.blocks();

        // ---- Q of this row tile: row i * group + h of the kv head's rows, scaled to fp16
        if ((a.kd < D || a.idx_feat != nullptr) && nrows > 0) {
            keep_features<D>(a, cur.b, cur.hk, cur.rows, row0, nrows, t_at == 0, kept);
            __syncthreads();
        }
        for (int r = warp; r < ROWS; r += kWarps) {
            const int i = (row0 + r) / a.group, h = (row0 + r) - i * a.group;
            float x[W32], top = 0.f;
#pragma unroll
            for (int v = 0; v < W32; ++v) {
                x[v] = 0.f;
                if (r < nrows) {
                    const bool in = a.kd == D || (kept[(r % a.group) * W32 + v] >> lane & 1u);
                    if (in) x[v] = __bfloat162float(a.q[cur.b * a.q_sb + ((int64_t)cur.hk * a.group + h) * a.q_sh + (int64_t)i * a.q_sr + v * 32 + lane]);
                }
                top = fmaxf(top, fabsf(x[v]));
            }
            top = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(top)));
            // 2^e at top; a row of zeros, or one too small or large to scale, is taken as it is
            const int e = (int)(__float_as_uint(top) >> 23) - 127;
            const int shift = e < -100 || e > 100 ? 0 : 14 - e;
            const float up = __uint_as_float((uint32_t)(127 + shift) << 23);
#pragma unroll
            for (int v = 0; v < W32; ++v)   // odd columns meet codes that lie four bits up
                qs[r * S::kPitchQ + v * 32 + lane] = __float2half_rn(x[v] * up * (lane & 1 ? 0.0625f : 1.f));
#pragma unroll
            for (int j = 0; j < NG; ++j) {
                float sum = x[2 * j] + x[2 * j + 1];
#pragma unroll
                for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
                if (lane == 0) row_sum[r * NG + j] = sum * a.scale_log2;
            }
            if (lane == 0) {
                row_scale[r] = a.scale_log2 * __uint_as_float((uint32_t)(127 - shift + 24) << 23);
                row_vis[r] = r < nrows ? (a.causal ? max(0, min(cur.len, cur.len - cur.rows + i + 1)) : cur.len) : 0;
            }
        }
        __syncthreads();
        uint32_t qf[NT][D / 16][2];
        float cq[NT][2], qsum[NT][2][NG], m[NT][2], l[NT][2], low[NT][2][NG], o[NT][D / 16][4];
        int vis[NT][2], vis_least = cur.len;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) {
                // step ks: columns 32 (ks / 2) + 8 t4 + {0, 4} and {1, 5}, or {2, 6} and {3, 7}
                const __half *p = qs + (nt * 8 + g) * S::kPitchQ + (ks >> 1) * 32 + t4 * 8 + (ks & 1) * 2;
                qf[nt][ks][0] = (uint32_t)__half_as_ushort(p[0]) | (uint32_t)__half_as_ushort(p[4]) << 16;
                qf[nt][ks][1] = (uint32_t)__half_as_ushort(p[1]) | (uint32_t)__half_as_ushort(p[5]) << 16;
            }
#pragma unroll
            for (int mt = 0; mt < D / 16; ++mt)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[nt][mt][e] = 0.f;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int r = nt * 8 + 2 * t4 + e;
                cq[nt][e] = row_scale[r];
                vis[nt][e] = row_vis[r];
                m[nt][e] = -INFINITY;
                l[nt][e] = 0.f;
#pragma unroll
                for (int j = 0; j < NG; ++j) {
                    qsum[nt][e][j] = row_sum[r * NG + j];
                    low[nt][e][j] = 0.f;
                }
            }
        }
        for (int r = 0; r < nrows; ++r) vis_least = min(vis_least, row_vis[r]);

        if (cur.reads()) {
            for (int t = t_at + warp; t < t_end; t += kWarps) {
                dead = dead || !mbar_wait(bars + 8 * slot, phases >> slot & 1u, &abort_flag, a.status, a.wait_ns);
                if (dead) continue;   // (gave up: no more copies, but every meeting of the block and of the CTAs is kept)
                phases ^= 1u << slot;
                const uint8_t *blk = smem + (warp * ST + slot) * S::kBlockBytes;
                const int held = tokens[slot];
                // -- S^T = K Q^T
                float acc[NT][NG][4];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int j = 0; j < NG; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[nt][j][e] = 0.f;
                uint32_t k0[W32], k1[W32];
                {
                    const uint32_t *p0 = reinterpret_cast<const uint32_t *>(blk) + g * (D / 8) + t4 * W32, *p1 = p0 + D;
                    if constexpr (W32 == 2) {
                        const uint2 x = *reinterpret_cast<const uint2 *>(p0), y = *reinterpret_cast<const uint2 *>(p1);
                        k0[0] = x.x; k0[1] = x.y; k1[0] = y.x; k1[1] = y.y;
                    } else {
#pragma unroll
                        for (int i = 0; i < W32 / 4; ++i) {
                            const uint4 x = reinterpret_cast<const uint4 *>(p0)[i], y = reinterpret_cast<const uint4 *>(p1)[i];
                            k0[4 * i] = x.x; k0[4 * i + 1] = x.y; k0[4 * i + 2] = x.z; k0[4 * i + 3] = x.w;
                            k1[4 * i] = y.x; k1[4 * i + 1] = y.y; k1[4 * i + 2] = y.z; k1[4 * i + 3] = y.w;
                        }
                    }
                }
#pragma unroll
                for (int w = 0; w < W32; ++w) {
                    const uint32_t x = k0[w], y = k1[w], xs = x >> 8, ys = y >> 8;
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        mma_f16(acc[nt][w / 2], x & 0x000f000fu, y & 0x000f000fu, x & 0x00f000f0u, y & 0x00f000f0u, qf[nt][2 * w][0], qf[nt][2 * w][1]);
                        mma_f16(acc[nt][w / 2], xs & 0x000f000fu, ys & 0x000f000fu, xs & 0x00f000f0u, ys & 0x00f000f0u, qf[nt][2 * w + 1][0], qf[nt][2 * w + 1][1]);
                    }
                }
                // -- steps and least values of keys and values g and g + 8
                float ks[2][NG], km[2][NG], vs[2][NG], vm[2][NG], ls[2];
                const uint32_t *pairs = reinterpret_cast<const uint32_t *>(blk) + 4 * D;
                const bool edge = held < kv4::kBlock || (t + 1) * kv4::kBlock > vis_least;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float most = 0.f;
#pragma unroll
                    for (int j = 0; j < NG; ++j) {
                        const uint32_t x = pairs[(g + 8 * e) * NG + j];
                        uint32_t y = pairs[D / 4 + (g + 8 * e) * NG + j];
                        if (edge && g + 8 * e >= held) y = 0u;   // what lies behind the last token may be anything
                        ks[e][j] = bf16_bits(x & 0xffffu);
                        km[e][j] = __uint_as_float(x & 0xffff0000u);
                        vs[e][j] = bf16_bits(y & 0xffffu);
                        vm[e][j] = __uint_as_float(y & 0xffff0000u);
                        most = fmaxf(most, vs[e][j]);
                    }
                    ls[e] = fmaxf(lg2(most), kLeastStep);
                }
                float x[NT][4];
                bool grow = false;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float lin = ks[e >> 1][0] * acc[nt][0][e], off = km[e >> 1][0] * qsum[nt][e & 1][0];
#pragma unroll
                        for (int j = 1; j < NG; ++j) {
                            lin = fmaf(ks[e >> 1][j], acc[nt][j][e], lin);
                            off = fmaf(km[e >> 1][j], qsum[nt][e & 1][j], off);
                        }
                        x[nt][e] = fmaf(cq[nt][e & 1], lin, off);
                        if (edge && (g + (e >> 1) * 8 >= held || t * kv4::kBlock + g + (e >> 1) * 8 >= vis[nt][e & 1])) x[nt][e] = -INFINITY;
                        grow |= x[nt][e] + ls[e >> 1] > m[nt][e & 1] + kGrow;
                    }
                if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            float mx = fmaxf(x[nt][e] + ls[0], x[nt][e + 2] + ls[1]);
#pragma unroll
                            for (int d = 4; d < 32; d <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
                            mx = fmaxf(mx - kTop, m[nt][e]);
                            const float alpha = m[nt][e] > -INFINITY ? ex2(m[nt][e] - mx) : 1.f;
                            m[nt][e] = mx;
                            l[nt][e] *= alpha;
#pragma unroll
                            for (int j = 0; j < NG; ++j) low[nt][e][j] *= alpha;
#pragma unroll
                            for (int mt = 0; mt < D / 16; ++mt) {
                                o[nt][mt][e] *= alpha;
                                o[nt][mt][e + 2] *= alpha;
                            }
                        }
                }
                uint32_t pb[NT][NG][2];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    float p[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) p[e] = ex2(x[nt][e] + (m[nt][e & 1] > -INFINITY ? -m[nt][e & 1] : 0.f));
                    l[nt][0] += p[0] + p[2];
                    l[nt][1] += p[1] + p[3];
#pragma unroll
                    for (int j = 0; j < NG; ++j) {
                        low[nt][0][j] = fmaf(p[0], vm[0][j], fmaf(p[2], vm[1][j], low[nt][0][j]));
                        low[nt][1][j] = fmaf(p[1], vm[0][j], fmaf(p[3], vm[1][j], low[nt][1][j]));
                        pb[nt][j][0] = transpose8x8(pack_f16(p[0] * vs[0][j], p[1] * vs[0][j]));   // (key g, rows 2 t4) -> (row g, keys 2 t4)
                        pb[nt][j][1] = transpose8x8(pack_f16(p[2] * vs[1][j], p[3] * vs[1][j]));
                    }
                }
                // -- O^T += V^T P^T: lane (g, t4) has the columns 64 j + 8 g .. of tokens 2 t4, 2 t4 + 1 and those 8 on
                const uint32_t *vp = reinterpret_cast<const uint32_t *>(blk) + 2 * D;
                auto columns = [&](int j, uint32_t w0, uint32_t w1, uint32_t w2, uint32_t w3) {
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const uint32_t sel = half ? 0x7632u : 0x5410u;
                        uint32_t x = __byte_perm(w0, w1, sel), y = __byte_perm(w2, w3, sel);
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt)
                                mma_f16(o[nt][j * 4 + half * 2 + q], x & 0x000f000fu, x & 0x00f000f0u, y & 0x000f000fu, y & 0x00f000f0u, pb[nt][j][0], pb[nt][j][1]);
                            x >>= 8;
                            y >>= 8;
                        }
                    }
                };
                if constexpr (D == 64) {
                    const uint2 x = reinterpret_cast<const uint2 *>(vp)[lane], y = reinterpret_cast<const uint2 *>(vp)[32 + lane];
                    columns(0, x.x, x.y, y.x, y.y);
                } else {
#pragma unroll
                    for (int i = 0; i < D / 128; ++i) {
                        const uint4 x = reinterpret_cast<const uint4 *>(vp)[(2 * i) * 32 + lane], y = reinterpret_cast<const uint4 *>(vp)[(2 * i + 1) * 32 + lane];
                        columns(2 * i, x.x, x.z, y.x, y.z);
                        columns(2 * i + 1, x.y, x.w, y.y, y.w);
                    }
                }
                __syncwarp();   // every lane is done with this entry
                if (++slot == ST) slot = 0;
                request();
            }
        }

        // ---- the warps meet
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) {
                    l[nt][e] += __shfl_xor_sync(0xffffffffu, l[nt][e], d);
#pragma unroll
                    for (int j = 0; j < NG; ++j) low[nt][e][j] += __shfl_xor_sync(0xffffffffu, low[nt][e][j], d);
                }
                if (g == 0) {
                    ml[(warp * ROWS + nt * 8 + 2 * t4 + e) * 2] = m[nt][e];
                    ml[(warp * ROWS + nt * 8 + 2 * t4 + e) * 2 + 1] = l[nt][e];
                }
            }
        __syncthreads();
        if (tid < ROWS) {
            float mx = -INFINITY, sum = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) mx = fmaxf(mx, ml[(w * ROWS + tid) * 2]);
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float mw = ml[(w * ROWS + tid) * 2], lw = ml[(w * ROWS + tid) * 2 + 1];
                const float f = mw > -INFINITY ? ex2(mw - mx) : 0.f;
                // (a NaN among a row's logits is in its sum, though the reference may have passed it by)
                sum += mw > -INFINITY ? f * lw : lw;
                ml[(w * ROWS + tid) * 2] = f;
            }
            tot[tid * 2] = mx;
            tot[tid * 2 + 1] = tid < nrows ? sum : 0.f;   // (rows that are none have met keys all the same)
        }
        float *part = nullptr;
        if (!whole) part = a.part + (int64_t)(2 * blockIdx.x + (t_at == 0 ? 1 : 0)) * ROWS * (D + 2);
#pragma unroll
        for (int j = 0; j < NG; ++j) {
            if (j > 0) __syncthreads();
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float *dst = merge + (warp * ROWS + nt * 8 + 2 * t4 + e) * S::kPitchM + 8 * g;
#pragma unroll
                    for (int q = 0; q < 4; ++q)   // columns 8 g + 2 q and the next, whose codes lay four bits up
                        *reinterpret_cast<float2 *>(dst + 2 * q) = make_float2(fmaf(o[nt][j * 4 + q][e], 16777216.f, low[nt][e][j]),
                                                                               fmaf(o[nt][j * 4 + q][e + 2], 1048576.f, low[nt][e][j]));
                }
            __syncthreads();
            for (int i = tid; i < ROWS * 64; i += kWarps * 32) {
                const int r = i >> 6, c = i & 63;
                float sum = 0.f;
#pragma unroll
                for (int w = 0; w < kWarps; ++w) {
                    const float f = ml[(w * ROWS + r) * 2];
                    sum += f != 0.f ? f * merge[(w * ROWS + r) * S::kPitchM + c] : 0.f;
                }
                const float lsum = tot[r * 2 + 1];
                if (whole) {
                    const int row = row0 + r, qi = row / a.group;
                    if (qi < a.L)
                        a.o[cur.b * a.o_sb + ((int64_t)cur.hk * a.group + row - qi * a.group) * a.o_sh + (int64_t)qi * a.o_sr + j * 64 + c] =
                            __float2bfloat16_rn(lsum == 0.f ? 0.f : sum * (1.f / lsum));   // (0: the row sees no key; a NaN stays one)
                } else {
                    part[r * (D + 2) + j * 64 + c] = sum;
                    if (j == 0 && c < 2) part[r * (D + 2) + D + c] = tot[r * 2 + c];
                }
            }
        }
        __syncthreads();

        // ---- a job that other CTAs work on too: whichever comes last adds the parts up
        if (!whole) {
            const int job0 = u - t_at, job1 = job0 + cur.blocks() - 1;   // its first and last place on the axis
            const int c0 = (int)((((int64_t)job0 + 1) * ctas - 1) / total), c1 = (int)((((int64_t)job1 + 1) * ctas - 1) / total);
            const unsigned n = (unsigned)(c1 - c0 + 1);
            if (tid == 0) {
                __threadfence();
                s_last = atomicInc(a.counters + c0, n - 1u) == n - 1u;
                __threadfence();
            }
            __syncthreads();
            if (s_last) {
                for (int r = warp; r < ROWS; r += kWarps) {
                    const int row = row0 + r, qi = row / a.group;
                    if (qi >= a.L) continue;
                    const float *src = a.part + r * (D + 2);
                    auto at = [&](int c) { return src + (int64_t)(2 * c + (c == c0 ? 1 : 0)) * ROWS * (D + 2); };
                    float mx = -INFINITY;
                    for (int c = c0 + lane; c <= c1; c += 32) mx = fmaxf(mx, __ldcg(at(c) + D));
#pragma unroll
                    for (int d = 16; d > 0; d >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
                    float sum[W32], lsum = 0.f;
#pragma unroll
                    for (int i = 0; i < W32; ++i) sum[i] = 0.f;
#pragma unroll 4
                    for (int c = c0; c <= c1; ++c) {
                        const float mw = __ldcg(at(c) + D), lw = __ldcg(at(c) + D + 1), f = mw > -INFINITY ? ex2(mw - mx) : 0.f;
                        lsum += mw > -INFINITY ? f * lw : lw;
#pragma unroll
                        for (int i = 0; i < W32; ++i) {
                            const float v = __ldcg(at(c) + i * 32 + lane);
                            sum[i] += f != 0.f ? f * v : 0.f;
                        }
                    }
                    const float inv = lsum == 0.f ? 0.f : 1.f / lsum;
                    __nv_bfloat16 *o = a.o + cur.b * a.o_sb + ((int64_t)cur.hk * a.group + row - qi * a.group) * a.o_sh + (int64_t)qi * a.o_sr;
#pragma unroll
                    for (int i = 0; i < W32; ++i) o[i * 32 + lane] = __float2bfloat16_rn(lsum == 0.f ? 0.f : sum[i] * inv);
                }
            }
        }
        u += t_end - t_at;
        t_at = 0;
        if (u < u_end) cursor_next<ROWS>(a, cur);
    }
    if (dead) drain_copies();
}

// Row tiles of 8, or of 16 where a kv head has more rows: they read the cache half as often.
int row_tiles(const Kv4AttnProblem &p) { return p.Hq / p.Hkv * p.L <= 8 ? 1 : 2; }

template <int D, int NT>
int launch(const AttnArgs &a, cudaStream_t stream)
{
    using S = Shape<D, NT>;
    auto kern = kv4_attn_kernel<D, NT>;
    static PerDeviceOnce configured;
    if (cudaError_t e = configured.smem(S::kSmem, kern)) return fail(RMM_ERR_CUDA, "kv4_attn: cudaFuncSetAttribute: %s", cudaGetErrorString(e));
    prof_begin("kv4_attn_kernel", stream);
    launch_kernel(kern, dim3((unsigned)(sm_count() * S::kCtas)), dim3(kWarps * 32), S::kSmem, stream, 1, a);
    return check_launch("kv4_attn_kernel", stream);
}

}  // namespace

bool kv4_attn_fits(const Kv4AttnProblem &p, const kv4::View &cache)
{
    // the axis of all blocks is counted in 32 bits
    const double chunks = (double)ceil_div(p.Hq / p.Hkv * p.L, 8 * row_tiles(p));
    return (double)p.B * p.Hkv * chunks * ((double)(cache.max_pages << cache.page_shift) + 1.0) < 2147483647.0 && p.Hq / p.Hkv * p.L < INT32_MAX / 2;
}

size_t kv4_attn_workspace_bytes(const Kv4AttnProblem &p)
{
    return (size_t)sm_count() * 2 * 2 * 8 * row_tiles(p) * (p.D + 2) * 4;
}

int launch_kv4_attn(const Kv4AttnProblem &p, const kv4::View &cache, float *scratch, unsigned *counters, int *status, cudaStream_t stream)
{
    AttnArgs a = {};
    const int nt = row_tiles(p);
    a.q = static_cast<const __nv_bfloat16 *>(p.q);
    a.o = static_cast<__nv_bfloat16 *>(p.o);
    a.q_sb = p.q_sb; a.q_sh = p.q_sh; a.q_sr = p.q_sr;
    a.o_sb = p.o_sb; a.o_sh = p.o_sh; a.o_sr = p.o_sr;
    a.cache = cache;
    a.B = (int)p.B; a.Hkv = (int)p.Hkv; a.group = (int)(p.Hq / p.Hkv); a.L = (int)p.L; a.kd = (int)p.kd; a.causal = p.causal;
    a.chunks = (int)ceil_div((int64_t)a.group * a.L, 8 * nt);
    a.scale_log2 = (float)(1.4426950408889634 / sqrt((double)p.D));
    a.idx_feat = p.idx_feat;
    a.part = scratch;
    a.counters = counters;
    a.status = status;
    a.wait_ns = wait_limit_ns();
    a.withhold = debug_withhold() == WITHHOLD_KV4;
    if (p.D == 64) return nt == 1 ? launch<64, 1>(a, stream) : launch<64, 2>(a, stream);
    if (p.D == 128) return nt == 1 ? launch<128, 1>(a, stream) : launch<128, 2>(a, stream);
    return nt == 1 ? launch<256, 1>(a, stream) : launch<256, 2>(a, stream);
}

}  // namespace rmm
