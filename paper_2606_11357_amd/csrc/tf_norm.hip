// Residual sum and RMS norms between two blocks of a decoder layer:
//   y = x or rms(x) (post + o),  r = residual + scale * gate * y,
//   out = rms(r) (w + o),        rms(t) = t / sqrt(mean t^2 + eps)
// HBM-bound: x and residual are read once, r and out written once (8 bytes an
// element), the row staying in registers between its sums and its outputs.
// Sums are fp32; each output is rounded once, and the norm takes r before that
// rounding.  Outputs go past the L2: rows of 4096, inputs changing from call to call,
// us through and past it: 512 5.8 / 5.1, 1024 8.5 / 6.7, 2048 13.9 / 11.1, 4096 26.9 /
// 25.6, 8192 48.8 / 48.2 (5.6 TB/s; a copy of 1 GiB 5.1 to 5.2), 32768 184 / 181; a layer's
// step takes the same time either way.  One row of 4096 takes 2.9 us in the kernel,
// the latency of its loads and two sums.
#include "tf_internal.h"

namespace tf {
namespace {

typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));

struct NormArgs {
    const uint16_t *x, *residual, *post, *gate, *weight;
    uint16_t *r_out, *y;
    int64_t gate_stride, M;
    int N;
    float scale, offset, eps;
};

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

// The sum of v over the threads of one row (WR waves of 64), the same in all.
template <int WR>
__device__ __forceinline__ float row_sum(float v, float* red) {
    v = wave_sum(v);
    if constexpr (WR > 1) {
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int i = 0; i < WR; ++i) v += red[i];
    }
    return v;
}

// WR waves a row, V vectors of 8 elements a thread: element 8 (t + i * 64 WR).
// Rows of up to 512 take one wave each, four rows a workgroup; longer ones a
// workgroup each, of as many waves as give a thread one or two vectors (up to
// 16384 elements): all of a row's loads are then on their way at once.
template <bool BF, int WR, int V>
__global__ __launch_bounds__(WR == 1 ? 256 : 64 * WR) void add_rms_norm_kernel(NormArgs a) {
    __shared__ float red[2][WR];
    const int lane = WR == 1 ? threadIdx.x & 63 : threadIdx.x;
    const int64_t row = WR == 1 ? (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6) : blockIdx.x;
    if (row >= a.M) return;
    const float inv_n = 1.0f / (float)a.N;
    u16x8 xv[V], rv[V];
    float r[V][8];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int c = 8 * (lane + i * 64 * WR);
        if (c < a.N) {
            xv[i] = *reinterpret_cast<const u16x8*>(a.x + row * a.N + c);
            rv[i] = a.residual ? *reinterpret_cast<const u16x8*>(a.residual + row * a.N + c) : u16x8{};
        } else {
            xv[i] = rv[i] = u16x8{};
        }
    }
    float post_scale = 1.0f;
    if (a.post) {
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float t = scale_f32<BF>(xv[i][j]);
                ss = fmaf(t, t, ss);
            }
        post_scale = rsqrtf(row_sum<WR>(ss, red[0]) * inv_n + a.eps);
    }
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int c = 8 * (lane + i * 64 * WR);
        const bool in = c < a.N;
        u16x8 pv{}, gv{};
        if (in && a.post) pv = *reinterpret_cast<const u16x8*>(a.post + c);
        if (in && a.gate) gv = *reinterpret_cast<const u16x8*>(a.gate + row * a.gate_stride + c);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float t = scale_f32<BF>(xv[i][j]);
            if (a.post) t = t * post_scale * (scale_f32<BF>(pv[j]) + a.offset);
            if (a.gate) t *= scale_f32<BF>(gv[j]);
            t = fmaf(t, a.scale, scale_f32<BF>(rv[i][j]));
            r[i][j] = t;
            ss = in ? fmaf(t, t, ss) : ss;
        }
        if (in && a.r_out) {
            u16x8 o;
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] = round_out<BF>(r[i][j]);
            store_past(reinterpret_cast<u16x8*>(a.r_out + row * a.N + c), o);
        }
    }
    if (!a.y) return;
    const float norm = rsqrtf(row_sum<WR>(ss, red[1]) * inv_n + a.eps);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int c = 8 * (lane + i * 64 * WR);
        if (c >= a.N) continue;
        const u16x8 wv = *reinterpret_cast<const u16x8*>(a.weight + c);
        u16x8 o;
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] = round_out<BF>(r[i][j] * norm * (scale_f32<BF>(wv[j]) + a.offset));
        store_past(reinterpret_cast<u16x8*>(a.y + row * a.N + c), o);
    }
}

template <bool BF>
int launch_dt(const NormArgs& a, hipStream_t s) {
    const int vecs = a.N / 8;
    const dim3 rows((unsigned)a.M), four((unsigned)((a.M + 3) / 4));
    if (vecs <= 64) return launch(add_rms_norm_kernel<BF, 1, 1>, four, dim3(256), 0, s, a);
    if (vecs <= 128) return launch(add_rms_norm_kernel<BF, 2, 1>, rows, dim3(128), 0, s, a);
    if (vecs <= 256) return launch(add_rms_norm_kernel<BF, 4, 1>, rows, dim3(256), 0, s, a);
    if (vecs <= 512) return launch(add_rms_norm_kernel<BF, 4, 2>, rows, dim3(256), 0, s, a);
    if (vecs <= 1024) return launch(add_rms_norm_kernel<BF, 8, 2>, rows, dim3(512), 0, s, a);
    if (vecs <= 2048) return launch(add_rms_norm_kernel<BF, 16, 2>, rows, dim3(1024), 0, s, a);
    return launch(add_rms_norm_kernel<BF, 16, 8>, rows, dim3(1024), 0, s, a);
}

}  // namespace

int launch_add_rms_norm(bool bf, const void* x, const void* residual, const void* post, const void* gate,
                        int64_t gate_stride, float scale, const void* weight, float offset, float eps, int64_t M,
                        int64_t N, void* r_out, void* y, hipStream_t s) {
    auto in = [](const void* p) { return static_cast<const uint16_t*>(p); };
    const NormArgs a{in(x), in(residual), in(post), in(gate), in(weight), static_cast<uint16_t*>(r_out),
                     static_cast<uint16_t*>(y), gate_stride, M, (int)N, scale, offset, eps};
    return bf ? launch_dt<true>(a, s) : launch_dt<false>(a, s);
}

}  // namespace tf
