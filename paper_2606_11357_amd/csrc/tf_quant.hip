// Rows of 16-bit activations as int8 codes with one fp32 scale a row, and the
// rearrangement of int8 weights for the matmuls that take those codes.
//   h = x or silu(g) u,   s = max|h| / 127,   q = round(h * (127 / max|h|))
// x is read once (2 or 4 bytes a code), codes are written once; the row stays in
// registers between its maximum and its codes.  Many rows are bound by memory, with the
// vector unit 74% busy: 8192 rows of 4096 take 20.8 us (4.8 TB/s, inputs and outputs of
// ten calls in turn; 16.7 where one input lies in the MALL), 8192 of 14336 gated 122 us (4.8
// TB/s).  One row of 4096 takes 2.3 us, the latency of its loads and one reduction; 16
// gated ones of 14336 5.9 us, one compute unit's exponentials each.
#include "tf_w8a8.h"

namespace tf {
namespace {

typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));

struct QuantArgs {
    const uint16_t* x;
    int64_t stride, M;
    int N;
    int8_t* q;
    float* scale;
};

// g / (1 + e^-g) for g >= kFarGate.  The quotient is a reciprocal with one Newton step
// (with an IEEE division 16 gated rows of 14336 took 6.5 us, so 5.9; 2048 rows 37.8 and
// 33.7): within one unit in the last place.
__device__ __forceinline__ float silu(float g) {
    const float d = 1.0f + expf(-g);
    const float r = __builtin_amdgcn_rcpf(d);
    return g * fmaf(r, fmaf(-d, r, 1.0f), r);
}
// Below it silu(g) u = g e^g u: 1 + e^g is 1 in fp32.  e^g, or its reciprocal, leaves
// fp32 below -87, where g e^g u may still be far within it, so e^(g / 2) comes in
// twice, the second time last.
constexpr float kFarGate = -64.0f;
__device__ __forceinline__ float far_silu_mul(float g, float u) {
    const float w = expf(0.5f * g);
    return g * w * u * w;
}

// The largest |h| and a sum that is NaN where some h is not finite, over the WR
// waves of a row, the same in all threads.
template <int WR>
__device__ __forceinline__ void row_top(float& top, float& odd, float (*red)[2]) {
#pragma unroll
    for (int d = 32; d; d >>= 1) {
        top = fmaxf(top, __shfl_xor(top, d));
        odd += __shfl_xor(odd, d);
    }
    if constexpr (WR > 1) {
        if ((threadIdx.x & 63) == 0) {
            red[threadIdx.x >> 6][0] = top;
            red[threadIdx.x >> 6][1] = odd;
        }
        __syncthreads();
        top = odd = 0.f;
#pragma unroll
        for (int i = 0; i < WR; ++i) {
            top = fmaxf(top, red[i][0]);
            odd += red[i][1];
        }
    }
}

// WR waves a row, V vectors of 8 values a thread, as in the norm's kernel.
template <bool BF, bool GATED, int WR, int V>
__global__ __launch_bounds__(WR == 1 ? 256 : 64 * WR) void quantize_rows_kernel(QuantArgs a) {
    __shared__ float red[WR][2];
    const int lane = WR == 1 ? threadIdx.x & 63 : threadIdx.x;
    const int64_t row = WR == 1 ? (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6) : blockIdx.x;
    if (row >= a.M) return;
    const uint16_t* x = a.x + row * a.stride;
    u16x8 xv[V], uv[GATED ? V : 1];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int c = 8 * (lane + i * 64 * WR);
        xv[i] = u16x8{};
        if (GATED) uv[i] = u16x8{};
        if (c < a.N) {
            xv[i] = *reinterpret_cast<const u16x8*>(x + c);
            if (GATED) uv[i] = *reinterpret_cast<const u16x8*>(x + a.N + c);
        }
    }
    float h[V][8], top = 0.f, odd = 0.f;
    if constexpr (GATED) {
        float least = 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float g = scale_f32<BF>(xv[i][j]);
                least = fminf(least, g);
                h[i][j] = silu(g) * scale_f32<BF>(uv[i][j]);
            }
        if (least < kFarGate) {                      // (rare)
#pragma unroll
            for (int i = 0; i < V; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float g = scale_f32<BF>(xv[i][j]);
                    if (g < kFarGate) h[i][j] = far_silu_mul(g, scale_f32<BF>(uv[i][j]));
                }
        }
    }
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if constexpr (!GATED) h[i][j] = scale_f32<BF>(xv[i][j]);
            top = fmaxf(top, fabsf(h[i][j]));
            odd = fmaf(h[i][j], 0.f, odd);
        }
    row_top<WR>(top, odd, red);
    // A row under 2^-100 is one of zeros (127 / top would leave fp32); one with a
    // value that is not finite has the scale NaN.
    const bool none = !(top >= 0x1p-100f), bad = odd != odd;
    const float inv = none || bad ? 0.f : 127.0f / top;
    if (lane == 0) a.scale[row] = bad ? __builtin_nanf("") : none ? 0.f : top / 127.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int c = 8 * (lane + i * 64 * WR);
        if (c >= a.N) continue;
        uint32_t w[2] = {0, 0};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int q = bad ? 0 : (int)rintf(h[i][j] * inv);
            w[j / 4] |= (uint32_t)(q & 255) << (8 * (j % 4));
        }
        *reinterpret_cast<uint2*>(a.q + row * a.N + c) = uint2{w[0], w[1]};
    }
}

template <bool BF, bool GATED>
int launch_quant(const QuantArgs& a, hipStream_t s) {
    const int vecs = a.N / 8;
    const dim3 rows((unsigned)a.M), four((unsigned)((a.M + 3) / 4));
    if (vecs <= 64) return launch(quantize_rows_kernel<BF, GATED, 1, 1>, four, dim3(256), 0, s, a);
    if (vecs <= 128) return launch(quantize_rows_kernel<BF, GATED, 2, 1>, rows, dim3(128), 0, s, a);
    if (vecs <= 256) return launch(quantize_rows_kernel<BF, GATED, 4, 1>, rows, dim3(256), 0, s, a);
    if (vecs <= 512) return launch(quantize_rows_kernel<BF, GATED, 4, 2>, rows, dim3(256), 0, s, a);
    if (vecs <= 1024) return launch(quantize_rows_kernel<BF, GATED, 8, 2>, rows, dim3(512), 0, s, a);
    if (vecs <= 2048) return launch(quantize_rows_kernel<BF, GATED, 16, 2>, rows, dim3(1024), 0, s, a);
    return launch(quantize_rows_kernel<BF, GATED, 16, 8>, rows, dim3(1024), 0, s, a);
}

// One workgroup a block of 64 rows by 64 columns (four atoms) of one expert,
// turned in LDS.  The workgroups of the first block of rows copy the scales.
__global__ __launch_bounds__(256) void pack_w8a8_kernel(const int8_t* __restrict__ w, const void* __restrict__ scales,
                                                        int scale_dtype, W8Layout L, int64_t first,
                                                        uint8_t* __restrict__ packed) {
    __shared__ int8_t t[64][64 + 4];
    const int64_t e = first + blockIdx.z;
    const int a = blockIdx.x, n0 = blockIdx.y * 64, tid = threadIdx.x;
    const int8_t* src = w + e * L.K * L.N;
    uint8_t* dst = packed + e * L.total;
#pragma unroll
    for (int i = 0; i < 2; ++i) {                        // 8 bytes a thread and pass (N % 8 == 0)
        const int k = i * 32 + tid / 8, c = tid % 8 * 8;
        const int64_t row = (int64_t)a * 64 + k;
        uint2 v{0, 0};
        if (row < L.K && n0 + c < L.N) v = *reinterpret_cast<const uint2*>(src + row * L.N + n0 + c);
        *reinterpret_cast<uint32_t*>(&t[k][c]) = v.x;
        *reinterpret_cast<uint32_t*>(&t[k][c + 4]) = v.y;
    }
    __syncthreads();
    const int p = n0 / 16 + tid / 64, lane = tid & 63;
    if (p < L.np) {
        const int c = tid / 64 * 16 + (lane & 15), k = 16 * (lane >> 4);
        u32x4 v;
#pragma unroll
        for (int d = 0; d < 4; ++d)
            v[d] = (uint32_t)(uint8_t)t[k + 4 * d][c] | (uint32_t)(uint8_t)t[k + 4 * d + 1][c] << 8 |
                   (uint32_t)(uint8_t)t[k + 4 * d + 2][c] << 16 | (uint32_t)(uint8_t)t[k + 4 * d + 3][c] << 24;
        *reinterpret_cast<u32x4*>(dst + ((int64_t)p * L.na + a) * kW8AtomBytes + 16 * lane) = v;
    }
    if (a == 0 && tid < 64) {                            // (64 a block: to the end of the last 256 bytes)
        const int64_t n = n0 + tid;
        float s = 0.f;
        if (n < L.N) {
            const int64_t i = e * L.N + n;
            if (scale_dtype == TF_F32) s = static_cast<const float*>(scales)[i];
            else if (scale_dtype == TF_BF16) s = scale_f32<true>(static_cast<const uint16_t*>(scales)[i]);
            else s = scale_f32<false>(static_cast<const uint16_t*>(scales)[i]);
        }
        reinterpret_cast<float*>(dst + L.s_off)[n] = s;
    }
}

}  // namespace

int launch_quantize_rows(bool bf, const void* x, int64_t stride, int64_t M, int64_t N, bool gated, int8_t* q,
                         float* scale, hipStream_t s) {
    const QuantArgs a{static_cast<const uint16_t*>(x), stride, M, (int)N, q, scale};
    if (gated) return bf ? launch_quant<true, true>(a, s) : launch_quant<false, true>(a, s);
    return bf ? launch_quant<true, false>(a, s) : launch_quant<false, false>(a, s);
}

int launch_pack_w8a8(const int8_t* w, const void* scales, int scale_dtype, int64_t K, int64_t N, int64_t experts,
                     void* packed, hipStream_t s) {
    const W8Layout L = w8_layout(K, N);
    const int64_t columns = (N + 63) / 64, most = (int64_t(1) << 31) / (L.na * columns * 256);   // experts a launch
    for (int64_t e = 0; e < experts; e += most) {
        const dim3 grid((unsigned)L.na, (unsigned)columns, (unsigned)(experts - e < most ? experts - e : most));
        const int rc = launch(pack_w8a8_kernel, grid, dim3(256), 0, s, w, scales, scale_dtype, L, e,
                              static_cast<uint8_t*>(packed));
        if (rc) return rc;
    }
    return TF_OK;
}

}  // namespace tf
