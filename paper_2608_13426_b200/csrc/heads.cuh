// Rows of heads on their way from a projection to attention: RMS norm and position rotation (internal).
// A row of D columns belongs to `lanes` (a power of two) neighbouring lanes of a warp, eight columns c = 8 k .. 8 k + 7 each.
// Lane k of a row is turned against lane k +- rot/16 (pairs d, d + rot/2) or against itself (pairs 2 d, 2 d + 1).
#pragma once
#include "common.cuh"

namespace rmm {

struct HeadRows {
    const void *src;
    void *dst;
    const void *weight;     // [D] or NULL: no norm
    int64_t s_b, s_h, s_r, d_b, d_h, d_r;
    int heads;
    int vec_in, vec_out;    // rows start on 16-byte boundaries
};
struct RopeView {
    const float *table;     // [rows, rot]: cosines, then sines; NULL: no rotation
    int64_t rows, stride;
    const int32_t *positions;
    int64_t p_b, p_r;
    int rot, interleaved, weight_bf16;
    float eps;
};

__device__ __forceinline__ float bf16_bits(uint32_t x) { return __uint_as_float(x << 16); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}

// (plain loads: the rows may be written in place)
template <typename T>
__device__ __forceinline__ void load8(const T *p, bool vec, float (&x)[8])
{
    if constexpr (sizeof(T) == 2) {
        if (vec) {
            const uint4 v = *reinterpret_cast<const uint4 *>(p);
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[2 * i] = __uint_as_float(w[i] << 16);
                x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = __bfloat162float(p[i]);
        }
    } else {
        if (vec) {
            const float4 a = reinterpret_cast<const float4 *>(p)[0], b = reinterpret_cast<const float4 *>(p)[1];
            x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
            x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = p[i];
        }
    }
}

template <typename T>
__device__ __forceinline__ void store8(T *p, bool vec, const float (&x)[8])
{
    if constexpr (sizeof(T) == 2) {
        if (vec) {
            *reinterpret_cast<uint4 *>(p) = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) p[i] = __float2bfloat16_rn(x[i]);
        }
    } else {
        if (vec) {
            reinterpret_cast<float4 *>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
            reinterpret_cast<float4 *>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) p[i] = x[i];
        }
    }
}

// 64 bits to bf16 in one rounding, as an fp32 number.
__device__ __forceinline__ float bf16_of_double(double z)
{
    const float f = (float)z;
    uint32_t bits = __float_as_uint(f);
    const double d = z - (double)f;
    if ((bits & 0xffffu) == 0x8000u && d != 0.0) bits += (d > 0.0) == (f > 0.f) ? 1u : 0xffffffffu;   // fp32 rounded onto a tie
    return __bfloat162float(__float2bfloat16_rn(__uint_as_float(bits)));
}

// What a lane needs for every row of one position: its weights and its partner's, cosines, and sines with the sign of its side.
struct RowLane {
    float w[8], wp[8], c[8], s[8];
    int partner;            // lane whose columns turn against mine
    bool norm, rope, turns, self;
};

__device__ __forceinline__ void row_weights(RowLane &k, const void *weight, const RopeView &r, int col, int D)
{
    k.norm = weight != nullptr;
    k.rope = r.table != nullptr;
    const int chunk = col / 8, half = r.rot / 16;
    k.self = r.interleaved != 0;
    k.turns = k.rope && chunk < 2 * half;
    const int other = !k.turns || k.self ? chunk : (chunk < half ? chunk + half : chunk - half);
    k.partner = ((int)threadIdx.x & 31) + other - chunk;
    if (k.norm && col < D) {
        if (r.weight_bf16) {
            load8(static_cast<const __nv_bfloat16 *>(weight) + col, false, k.w);
            load8(static_cast<const __nv_bfloat16 *>(weight) + 8 * other, false, k.wp);
        } else {
            load8(static_cast<const float *>(weight) + col, false, k.w);
            load8(static_cast<const float *>(weight) + 8 * other, false, k.wp);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) k.w[i] = k.wp[i] = 1.f;
    }
}

__device__ __forceinline__ void row_angles(RowLane &k, const RopeView &r, int64_t position, int col)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        k.c[i] = 1.f;
        k.s[i] = 0.f;
    }
    if (!k.turns) return;
    const float *row = r.table + position * r.stride;
    const int half = r.rot / 2;
    if (k.self) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            k.c[i] = __ldg(row + (col + i) / 2);
            k.s[i] = i & 1 ? __ldg(row + half + (col + i) / 2) : -__ldg(row + half + (col + i) / 2);
        }
    } else {
        const int d = col < half ? col : col - half;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            k.c[i] = __ldg(row + d + i);
            k.s[i] = col < half ? -__ldg(row + half + d + i) : __ldg(row + half + d + i);
        }
    }
}

// One row: z = (norm and rotation of x).  All lanes of the warp take part; lanes past the row's columns hold zeros.
// ROUND: z is rounded to bf16 as the 64-bit result would be.  The fp32 chain is off by at most 2^-20 (|y c| + |y' s|): sum of up to
// 256 squares in 8-element chains and 5 exchanges (14 roundings of 2^-24, half of it after the root), rsqrtf (4), two scalings,
// product and sum (4).  Rows with a column that close to a border between two bf16 numbers (one in 20 or so) are done again in 64 bits.
template <bool ROUND>
__device__ __forceinline__ void norm_rope_row(const float (&x)[8], const RowLane &k, int lanes, int D, float eps, float (&z)[8])
{
    float r = 1.f;
    if (k.norm) {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum = fmaf(x[i], x[i], sum);
        for (int d = lanes >> 1; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        r = rsqrtf(sum / (float)D + eps);
    }
    float xp[8];
    bool near = false;
    if (k.rope && !k.self) {
#pragma unroll
        for (int i = 0; i < 8; ++i) xp[i] = __shfl_sync(0xffffffffu, x[i], k.partner);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) xp[i] = x[i ^ 1];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float y = x[i] * r * k.w[i];
        if (k.turns) {
            const float yp = xp[i] * r * (k.self ? k.w[i ^ 1] : k.wp[i]);
            const float t = yp * k.s[i];
            z[i] = fmaf(y, k.c[i], t);
            if constexpr (ROUND) {
                const uint32_t bits = __float_as_uint(z[i]);
                const float off = fabsf(__uint_as_float(0x4b000000u | (bits & 0xffffu)) - 8421376.f);   // from the tie, units of fp32
                near |= off * __uint_as_float(bits & 0x7f800000u) <= 8.f * fmaf(fabsf(y), fabsf(k.c[i]), fabsf(t));
            }
        } else {
            z[i] = y;
            if constexpr (ROUND) {
                const uint32_t bits = __float_as_uint(y);
                near |= k.norm && fabsf(__uint_as_float(0x4b000000u | (bits & 0xffffu)) - 8421376.f) <= 16.f;
            }
        }
    }
    if constexpr (ROUND) {
        if (__any_sync(0xffffffffu, near)) {
            double rd = 1.0;
            if (k.norm) {
                double sum = 0.0;
#pragma unroll
                for (int i = 0; i < 8; ++i) sum = fma((double)x[i], (double)x[i], sum);
                for (int d = lanes >> 1; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
                rd = 1.0 / sqrt(sum / (double)D + (double)eps);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const double y = (double)x[i] * rd * (double)k.w[i];
                const double yp = (double)xp[i] * rd * (double)(k.self ? k.w[i ^ 1] : k.wp[i]);
                z[i] = bf16_of_double(k.turns ? fma(y, (double)k.c[i], yp * (double)k.s[i]) : y);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) z[i] = __bfloat162float(__float2bfloat16_rn(z[i]));
        }
    }
}

int launch_norm_rope(const HeadRows (&rows)[2], int in_bf16, int out_bf16, const RopeView &rope, int64_t B, int64_t L, int64_t D, int *status,
                     cudaStream_t stream);

}  // namespace rmm
