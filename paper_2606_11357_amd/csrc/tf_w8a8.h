// The packed weights of the 8-bit by 8-bit matmuls, and what their kernels share.
#pragma once

#include "tf_internal.h"

namespace tf {

// Packed layout.  A weight [K, N] of int8 codes is cut into atoms of 64 rows by 16
// columns (1 KiB, one 16-byte load a lane): lane l = 16 g + c holds column
// 16 p + c, rows 64 a + 16 g + 0..15, lowest byte first, which is what a lane
// gives v_mfma_i32_16x16x64_i8.  Atom (panel p, a) is at (p * na + a) * 1024; na is
// even, rows past K and columns past N are zeros.  Then the columns' scales, fp32
// [16 np].  Experts follow each other, `total` bytes apart.
constexpr int kW8AtomK = 64, kW8Panel = 16, kW8AtomBytes = 1024;

struct W8Layout {
    int64_t K, N, np, na, s_off, total;
};
inline W8Layout w8_layout(int64_t K, int64_t N) {
    W8Layout L{K, N, (N + 15) / 16, (K + 127) / 128 * 2, 0, 0};
    L.s_off = L.np * L.na * kW8AtomBytes;
    L.total = align256(L.s_off + L.np * 16 * 4);
    return L;
}

// One matmul call.  Dense: experts 0.  By expert: the rows of C ("slots")
// offsets[e] .. offsets[e + 1] - 1 are rows of A (rows[slot], or slot) times weight e.
struct W8Args {
    const int8_t* A;
    const float* a_scale;
    const uint8_t* packed;
    uint16_t* C;
    const int32_t *offsets, *rows;
    int64_t M;               // rows of C
    int64_t a_rows;          // rows of A
    int64_t K, N, total, s_off;
    int na, np, experts;
    int bf;                  // C is bfloat16
    // K in parts, the sums of each in parts[part][M][N], added and scaled by a launch of
    // their own; 1: none
    int splits;
    int32_t* parts;
};

#ifdef __HIPCC__
// The slots of expert e (the same in all lanes of a wave): from the largest offset up
// to its own, within the call's, so that no two experts share one whatever the
// offsets hold.
__device__ __forceinline__ void w8_slots(const W8Args& a, int e, int& first, int& last) {
    const int lane = threadIdx.x & 63, M = (int)a.M;
    int top = 0;
    for (int i = lane; i <= e; i += 64) top = max(top, a.offsets[i]);
#pragma unroll
    for (int d = 32; d; d >>= 1) top = max(top, __shfl_xor(top, d));
    first = __builtin_amdgcn_readfirstlane(min(top, M));
    last = __builtin_amdgcn_readfirstlane(min(max(a.offsets[e + 1], first), M));
}

__device__ __forceinline__ uint2 w8_round(bool bf, const float (&v)[4]) {
    return bf ? uint2{round_out2<true>(v[0], v[1]), round_out2<true>(v[2], v[3])}
              : uint2{round_out2<false>(v[0], v[1]), round_out2<false>(v[2], v[3])};
}
// Outputs from four sums of one row (columns n .. n + 3): the sum as fp32, times the
// product of its two scales in fp32, rounded once more to the output's type.
//
// Scales whose product with another such one, and with any sum, loses nothing to the
// ends of fp32.
__device__ __forceinline__ bool w8_near(float s) {
    return (fabsf(s) >= 0x1p-60f && fabsf(s) <= 0x1p60f) || s == 0.f;
}
// For scales that are near.
__device__ __forceinline__ uint2 w8_scaled(bool bf, const i32x4& sum, float sa, const float4_t& sw) {
    float v[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = (float)sum[r] * (sa * sw[r]);
    return w8_round(bf, v);
}
// For any: products of significands, the exponents last (of near scales the same
// bits).  there: the row exists; else zeros, by columns that are not finite too.
__device__ __forceinline__ uint2 w8_scaled_far(bool bf, const i32x4& sum, float sa, const float4_t& sw, bool there) {
    float v[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const float p = (float)sum[r] * (__builtin_amdgcn_frexp_mantf(sa) * __builtin_amdgcn_frexp_mantf(sw[r]));
        v[r] = there ? ldexpf(p, __builtin_amdgcn_frexp_expf(sa) + __builtin_amdgcn_frexp_expf(sw[r])) : 0.f;
    }
    return w8_round(bf, v);
}
#endif

}  // namespace tf
