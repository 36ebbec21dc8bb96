// RMS norm of every query and key head and the position rotation, in one pass (what a model does between its projections and
// rmm_reduced_attn):  y = x w / sqrt(mean x^2 + eps),  z_d = y_d cos - y_d' sin,  z_d' = y_d' cos + y_d sin.
//
// Bound: HBM, each head read and written once.  A row's columns sit in neighbouring lanes, eight each (16 bytes of bf16), so a
// row never leaves its lanes: squares meet by shuffles, pairs are exchanged by shuffles.  A warp takes one token and several heads: its
// cosines, sines and weights are read once and stay in registers (a table's row is as large as two heads).
#include "heads.cuh"

namespace rmm {
namespace {

constexpr int kWarps = 8, kTurns = 4;   // warps of a block: neighbouring tokens; rows of a lane

struct NormRopeArgs {
    HeadRows rows[2];
    RopeView rope;
    int64_t tokens, L;
    int D, lanes, groups[2];   // lanes of a row; warps that share a token's heads
    int *status;
};

template <typename TI, typename TO>
__global__ void __launch_bounds__(kWarps * 32) norm_rope_kernel(const __grid_constant__ NormRopeArgs a)
{
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, per = 32 / a.lanes;
    const int all = a.groups[0] + a.groups[1], g = blockIdx.x % all;
    const int64_t token = (int64_t)(blockIdx.x / all) * kWarps + warp;
    if (token >= a.tokens) return;
    const bool second = g >= a.groups[0];
    const HeadRows &h = a.rows[second];
    const int64_t b = token / a.L, i = token - b * a.L;
    const int first = (second ? g - a.groups[0] : g) * per * kTurns + lane / a.lanes, col = (lane & (a.lanes - 1)) * 8;
    const int64_t position = a.rope.positions != nullptr ? a.rope.positions[b * a.rope.p_b + i * a.rope.p_r] : i;
    if (a.rope.table != nullptr && (position < 0 || position >= a.rope.rows)) {   // such a row is not written
        if (lane == 0) atomicExch(a.status, (int)RMM_ERR_BOUNDS);
        return;
    }
    const TI *src = static_cast<const TI *>(h.src) + b * h.s_b + i * h.s_r + col;
    TO *dst = static_cast<TO *>(h.dst) + b * h.d_b + i * h.d_r + col;
    float x[kTurns][8];
#pragma unroll
    for (int t = 0; t < kTurns; ++t) {
        const int head = first + t * per;
        if (head < h.heads && col < a.D) {
            load8(src + head * h.s_h, h.vec_in != 0, x[t]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[t][e] = 0.f;
        }
    }
    RowLane k;
    row_weights(k, h.weight, a.rope, col, a.D);
    row_angles(k, a.rope, position, col);
#pragma unroll
    for (int t = 0; t < kTurns; ++t) {
        float z[8];
        norm_rope_row<false>(x[t], k, a.lanes, a.D, a.rope.eps, z);
        const int head = first + t * per;
        if (head < h.heads && col < a.D) store8(dst + head * h.d_h, h.vec_out != 0, z);
    }
}

}  // namespace

int launch_norm_rope(const HeadRows (&rows)[2], int in_bf16, int out_bf16, const RopeView &rope, int64_t B, int64_t L, int64_t D, int *status,
                     cudaStream_t stream)
{
    NormRopeArgs a = {};
    a.rows[0] = rows[0];
    a.rows[1] = rows[1];
    a.rope = rope;
    a.tokens = B * L;
    a.L = L;
    a.D = (int)D;
    for (a.lanes = 2; a.lanes * 8 < D;) a.lanes *= 2;
    for (int i = 0; i < 2; ++i) a.groups[i] = (int)ceil_div(rows[i].heads, 32 / a.lanes * kTurns);
    a.status = status;
    const int64_t blocks = ceil_div(a.tokens, kWarps) * (a.groups[0] + a.groups[1]);
    if (blocks > INT32_MAX) return fail(RMM_ERR_UNSUPPORTED, "qk_norm_rope: more than 2^31 blocks of rows");
    auto kern = in_bf16 ? (out_bf16 ? norm_rope_kernel<__nv_bfloat16, __nv_bfloat16> : norm_rope_kernel<__nv_bfloat16, float>)
                        : (out_bf16 ? norm_rope_kernel<float, __nv_bfloat16> : norm_rope_kernel<float, float>);
    prof_begin("norm_rope_kernel", stream);
    launch_kernel(kern, dim3((unsigned)blocks), dim3(kWarps * 32), 0, stream, 1, a);
    return check_launch("norm_rope_kernel", stream);
}

}  // namespace rmm
