// Attention over whole packed prompts (prefill): causal or not, grouped heads,
// sequences of different lengths.
//
//   S = scale Q K^T, P = softmax(S), O = P V, one pass over the keys with the
//   running maximum and sum of the softmax.
//
// Bound by the matrix cores: 4 D flops a (query, key) pair against 4 D bytes a
// token and head.  Both products are taken transposed, S^T = K Q^T and
// O^T = V^T P^T, with 32 x 32 x 16 matrix instructions: a lane then holds one
// query's scores (its maximum and sum are the lane's own, joined with one other
// lane), and the scores it holds are, rounded, the very operand that the second
// product takes from it.
#include "tf_internal.h"

namespace tf {
namespace {

typedef float float16_t __attribute__((ext_vector_type(16)));
typedef short short4_t __attribute__((ext_vector_type(4)));

constexpr int kWaves = 4;
constexpr int kBM = 32 * kWaves;       // queries of a workgroup
constexpr int kBN = 64;                // keys of a step

struct PromptArgs {
    const uint16_t *q, *k, *v;
    int64_t q_stride, k_stride, v_stride;
    const int32_t *cu_q, *cu_k;
    int batch, q_heads, group;
    int64_t tokens_q, tokens_k;
    float scale2;
    int causal;
    uint16_t* out;
};

template <bool BF>
__device__ __forceinline__ float16_t mfma32(const u32x4& a, const u32x4& b, const float16_t& c) {
    if constexpr (BF)
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a),
                                                       __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8_t, a),
                                                      __builtin_bit_cast(half8_t, b), c, 0, 0, 0);
}

// 16-byte chunk at which chunk ch of row r is kept in LDS.
//  K: read 16 bytes a lane, neighbouring lanes in neighbouring rows: 16 rows of
//  one chunk land in 16 different 16-byte columns of the 256 bytes that the
//  banks span.
//  V: read by the transposing load, 64 bytes of each of four rows at a time:
//  the four land in different quarters of the banks.
template <int D>
__device__ __forceinline__ int k_chunk(int r, int ch) {
    return D == 64 ? ch ^ ((r >> 1) & 7) : ch ^ (r & 15);
}
template <int D>
__device__ __forceinline__ int v_chunk(int r, int ch) {
    return D == 64 ? ch ^ (((r >> 1) & 1) << 2) : ch ^ ((r & 3) << 2);
}

__device__ __forceinline__ u32x2 lds_read_tr16(const uint16_t* p) {
    typedef __attribute__((address_space(3))) short4_t lds_short4;
    const short4_t v = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (lds_short4*)(uintptr_t)(const __attribute__((address_space(3))) uint16_t*)p);
    return __builtin_bit_cast(u32x2, v);
}

template <bool BF, int D>
__global__ __launch_bounds__(64 * kWaves, D == 256 ? 1 : 2) void prompt_attn_kernel(PromptArgs a) {
    constexpr int CH = D / 8;             // 16-byte chunks of a row
    constexpr int KS = D / 16;            // K steps of S
    constexpr int DT = D / 32;            // output tiles
    __shared__ __align__(16) uint16_t ks[2][kBN * D];
    __shared__ __align__(16) uint16_t vs[2][kBN * D];
    __shared__ uint32_t wave_total[kWaves];
    __shared__ uint32_t before[64 * kWaves + 1];

    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, col = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

    // ---- which sequence, block of queries and head
    auto span = [&](const int32_t* cu, int b, int64_t tokens, int64_t& start) {
        start = cu[b];
        const int64_t n = (int64_t)cu[b + 1] - start;
        return start < 0 || n < 0 || start + n > tokens ? 0 : (int)n;
    };
    auto blocks_of = [&](int b) {
        int64_t s;
        return (uint32_t)((span(a.cu_q, b, a.tokens_q, s) + kBM - 1) / kBM);
    };
    const int seg = (a.batch + 64 * kWaves - 1) / (64 * kWaves);
    {
        uint32_t sum = 0;
        for (int b = tid * seg; b < (tid + 1) * seg && b < a.batch; ++b) sum += blocks_of(b);
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t o = __shfl_up(sum, d);
            if (lane >= d) sum += o;
        }
        if (lane == 63) wave_total[wave] = sum;
        __syncthreads();
        uint32_t base = 0;
        for (int w = 0; w < wave; ++w) base += wave_total[w];
        before[tid + 1] = base + sum;
        if (tid == 0) before[0] = 0;
        __syncthreads();
    }
    const uint32_t total = before[64 * kWaves];
    const uint32_t order = blockIdx.x / (uint32_t)a.q_heads;
    if (order >= total) return;
    // neighbouring workgroups (neighbouring XCDs) take different key/value
    // heads; the last, longest blocks go first
    const int kv_heads = a.q_heads / a.group;
    const int hx = (int)(blockIdx.x % (uint32_t)a.q_heads);
    const int hk = hx % kv_heads, hq = hk * a.group + hx / kv_heads;
    const uint32_t x = total - 1 - order;
    int b, block;
    {
        int s0 = 0, s1 = 64 * kWaves;
        while (s1 - s0 > 1) {
            const int mid = (s0 + s1) >> 1;
            if (before[mid] <= x) s0 = mid;
            else s1 = mid;
        }
        b = s0 * seg;
        uint32_t done = before[s0];
        for (;; ++b) {
            const uint32_t n = blocks_of(b);
            if (x < done + n) break;
            done += n;
        }
        b = __builtin_amdgcn_readfirstlane(b);
        block = __builtin_amdgcn_readfirstlane((int)(x - done));
    }
    int64_t q_start, k_start;
    const int n_q = span(a.cu_q, b, a.tokens_q, q_start);
    const int n_k = span(a.cu_k, b, a.tokens_k, k_start);
    const int q0 = block * kBM + wave * 32;               // the wave's first query
    const int qi = q0 + col;                              // the lane's query
    const int past = n_k - n_q;
    const int limit = a.causal ? (qi + past < n_k - 1 ? qi + past : n_k - 1) : n_k - 1;
    const int wave_low = a.causal ? (q0 + past < n_k - 1 ? q0 + past : n_k - 1) : n_k - 1;
    const int q_last = block * kBM + kBM < n_q ? block * kBM + kBM - 1 : n_q - 1;
    const int wave_q_last = q0 + 31 < n_q ? q0 + 31 : n_q - 1;
    const int wg_keys = a.causal ? (q_last + past + 1 < n_k ? q_last + past + 1 : n_k) : n_k;
    const int wave_keys = q0 >= n_q ? 0 : a.causal ? (wave_q_last + past + 1 < n_k ? wave_q_last + past + 1 : n_k) : n_k;
    const int steps = wg_keys > 0 ? (wg_keys + kBN - 1) / kBN : 0;

    u32x4 q[KS];
    {
        const int64_t row = q_start + (qi < n_q ? qi : n_q - 1);
        const uint16_t* src = a.q + row * a.q_stride + (int64_t)hq * D + half * 8;
#pragma unroll
        for (int s = 0; s < KS; ++s) q[s] = *reinterpret_cast<const u32x4*>(src + 16 * s);
    }
    // the keys' and values' rows straight into LDS, each lane 16 bytes in
    // order; the rearrangement is in which chunk of the row a lane fetches
    auto fetch = [&](int step) {
        const int buf = step & 1;
        constexpr int LOADS = kBN * CH / (64 * kWaves);
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int at = (wave * LOADS + i) * 64;       // the wave's first chunk
            const int r = (at + lane) / CH, ch = (at + lane) % CH;
            int key = step * kBN + r;
            key = key < n_k ? key : n_k - 1;              // rows past the end: masked scores
            const uint16_t* kp = a.k + (k_start + key) * a.k_stride + (int64_t)hk * D + 8 * k_chunk<D>(r, ch);
            const uint16_t* vp = a.v + (k_start + key) * a.v_stride + (int64_t)hk * D + 8 * v_chunk<D>(r, ch);
            typedef __attribute__((address_space(3))) void lds_void;
            typedef const __attribute__((address_space(1))) void global_void;
            __builtin_amdgcn_global_load_lds((global_void*)kp, (lds_void*)&ks[buf][at * 8], 16, 0, 0);
            __builtin_amdgcn_global_load_lds((global_void*)vp, (lds_void*)&vs[buf][at * 8], 16, 0, 0);
        }
    };

    float16_t o[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[t][i] = 0.f;
    float m = -__builtin_inff(), l = 0.f;

    if (steps > 0) fetch(0);
    for (int step = 0; step < steps; ++step) {
        __builtin_amdgcn_s_waitcnt(0);                    // this wave's part of the tiles is there
        __syncthreads();                                  // everyone's is, and the other buffer is free
        if (step + 1 < steps) fetch(step + 1);
        const int key0 = step * kBN;
        if (key0 >= wave_keys) continue;
        const uint16_t* kb = ks[step & 1];
        const uint16_t* vb = vs[step & 1];
        float16_t s[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
#pragma unroll
            for (int i = 0; i < 16; ++i) s[t][i] = 0.f;
#pragma unroll
            for (int j = 0; j < KS; ++j) {
                const int r = t * 32 + col;
                const u32x4 kf = *reinterpret_cast<const u32x4*>(kb + r * D + 8 * k_chunk<D>(r, 2 * j + half));
                s[t] = mfma32<BF>(kf, q[j], s[t]);
            }
        }
        if (key0 + kBN - 1 > wave_low) {                  // some key is hidden from some query
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (key0 + 32 * t + 8 * (i / 4) + 4 * half + i % 4 > limit) s[t][i] = -__builtin_inff();
        }
        float top = m;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, s[t][i]);
        top = fmaxf(top, __shfl_xor(top, 32));
        if (__any(top > m)) {
            const float f = top == -__builtin_inff() ? 1.f : __builtin_amdgcn_exp2f((m - top) * a.scale2);
            m = top;
            l *= f;
#pragma unroll
            for (int t = 0; t < DT; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[t][i] *= f;
        }
        const float base = m == -__builtin_inff() ? 0.f : m * a.scale2;
        u32x4 p[4];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
                const float e0 = __builtin_amdgcn_exp2f(fmaf(s[t][i], a.scale2, -base));
                const float e1 = __builtin_amdgcn_exp2f(fmaf(s[t][i + 1], a.scale2, -base));
                l += e0 + e1;
                p[2 * t + i / 8][(i % 8) / 2] = round_out2<BF>(e0, e1);
            }
        // keys 16 j + 4 half + 0..3 and + 8: the order in which p holds them
        const int l16 = lane & 15, sub = (lane >> 4) & 1;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int d = 32 * t + 16 * sub + 4 * (l16 & 3);
                const int r0 = 16 * j + 4 * half + (l16 >> 2), r1 = r0 + 8;
                const u32x2 v0 = lds_read_tr16(vb + r0 * D + 8 * v_chunk<D>(r0, d >> 3) + (d & 7));
                const u32x2 v1 = lds_read_tr16(vb + r1 * D + 8 * v_chunk<D>(r1, d >> 3) + (d & 7));
                o[t] = mfma32<BF>(u32x4{v0[0], v0[1], v1[0], v1[1]}, p[j], o[t]);
            }
    }
    l += __shfl_xor(l, 32);
    if (qi >= n_q) return;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    uint16_t* dst = a.out + ((q_start + qi) * a.q_heads + hq) * (int64_t)D + 4 * half;
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
            *reinterpret_cast<u32x2*>(dst + 32 * t + 2 * i) =
                u32x2{round_out2<BF>(o[t][i] * inv, o[t][i + 1] * inv),
                      round_out2<BF>(o[t][i + 2] * inv, o[t][i + 3] * inv)};
}

}  // namespace

int launch_prompt_attention(bool bf, const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v,
                            int64_t v_stride, const int32_t* cu_q, const int32_t* cu_k, int64_t batch,
                            int64_t tokens_q, int64_t tokens_k, int q_heads, int kv_heads, int D, float scale,
                            bool causal, void* out, hipStream_t s) {
    auto in = [](const void* p) { return static_cast<const uint16_t*>(p); };
    const PromptArgs a{in(q), in(k), in(v), q_stride, k_stride, v_stride, cu_q, cu_k, (int)batch, q_heads,
                       q_heads / kv_heads, tokens_q, tokens_k, scale * 1.4426950408889634f, causal ? 1 : 0,
                       static_cast<uint16_t*>(out)};
    // sum of ceil(n / kBM) over the sequences, at most
    const int64_t blocks = (tokens_q + (kBM - 1) * (batch < tokens_q ? batch : tokens_q)) / kBM;
    const dim3 grid((unsigned)(blocks * q_heads));
    auto go = [&](auto d) {
        constexpr int D_ = decltype(d)::value;
        return bf ? launch(prompt_attn_kernel<true, D_>, grid, dim3(64 * kWaves), 0, s, a)
                  : launch(prompt_attn_kernel<false, D_>, grid, dim3(64 * kWaves), 0, s, a);
    };
    if (D == 64) return go(std::integral_constant<int, 64>{});
    if (D == 128) return go(std::integral_constant<int, 128>{});
    return go(std::integral_constant<int, 256>{});
}

}  // namespace tf
