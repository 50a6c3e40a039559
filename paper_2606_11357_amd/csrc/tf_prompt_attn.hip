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
//
// Four waves of 32 queries share each step's 64 keys and values in LDS: with 128
// dims a wave reads 32 KB of them a step for 1024 cycles of matrix instructions.
// Measured (bf16, one causal prompt of 8192): 32 heads on 8 of 128 519 to 543 us, from
// card to card, 1.01 to 1.06 PFLOP/s, matrix cores busy 57% of the time and vector
// units 49%, at the 1.83 GHz at which a large matrix product starts too; 16 heads of 64
// 162 us, 848 TFLOP/s, vector units 70% busy; 8 of 256 325 us, 845, one wave a SIMD.
#include "tf_internal.h"

namespace tf {
namespace {

typedef float float16_t __attribute__((ext_vector_type(16)));
typedef short short4_t __attribute__((ext_vector_type(4)));

constexpr int kWaves = 4;
constexpr int kBM = 32 * kWaves;       // queries of a workgroup
constexpr int kBN = 64;                // keys of a step
// A weight may pass 1 by 2^kSlack before the sums move to a new maximum (0: 545 us
// instead of 527 for 32 heads of 128 on 8192; error against 64 bits 1.75e-3 and
// 1.93e-3, of which 1.65e-3 is the output's rounding).
constexpr float kSlack = 8.f;
// Powers of two that all weights carry besides (they leave with the sum of weights):
// fp16 has digits down to 2^-14, and weights below, of many keys beside one that takes
// most, would lose theirs (65536 keys, 0.3% outside that one: error up to 23% -> 6e-4).
// The largest weight stays under 2^15.  bf16 has the exponents of fp32.
template <bool BF> constexpr float kPlaces = BF ? 0.f : 7.f;
template <bool BF> constexpr uint32_t kOnes = BF ? 0x3F803F80u : 0x3C003C00u;
// Bytes of all parts up to which they are stored past the L2.  Measured, us through
// and past it: 13 MB (500 after 3000, 16 heads of 64) 25.1 / 22.9, 17 MB (2048, 16
// of 64) 32.3 / 29.1, 34 MB (500 after 3000, 32 of 128) 45.2 / 46.1, 67 MB (2048, 8
// of 256) 54.7 / 58.8.
constexpr int64_t kMostPast = 24 << 20;
constexpr int kSizedForCus = 256, kMostSplits = 16;

struct PromptArgs {
    const uint16_t *q, *k, *v;
    int64_t q_stride, k_stride, v_stride;
    const int32_t *cu_q, *cu_k;
    int batch, q_heads, group;
    int64_t tokens_q, tokens_k;
    float scale2;
    int causal;
    uint16_t* out;
    int splits;                        // parts that each block's keys are split into
    float* parts;                      // splits > 1: [part][slot] kBM rows of D sums, of a maximum, of a sum
    int64_t part_stride;               // floats of one part
    bool past;                         // parts past the L2
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

typedef __attribute__((address_space(3))) uint16_t Lds;

__device__ __forceinline__ u32x2 lds_read_tr16(const Lds* p) {
    typedef __attribute__((address_space(3))) short4_t lds_short4;
    const short4_t v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4*)p);
    return __builtin_bit_cast(u32x2, v);
}
__device__ __forceinline__ u32x4 lds_read16(const Lds* p) {
    typedef __attribute__((address_space(3))) const u32x4 lds_u32x4;
    return *(lds_u32x4*)p;
}

// Which sequence, block of queries and head a workgroup takes: slot counts
// (block, head) pairs, heads fastest, so that neighbouring workgroups
// (neighbouring XCDs) take different key/value heads; the last blocks of the
// packed sequences, the longest of each, go first.  Offsets that leave the
// tensors or run backwards make an empty sequence.
struct Block {
    int sequence = -1, block = 0, n_q = 0, n_k = 0, hq = 0, hk = 0, steps = 0, splits = 1;
    int64_t q_start = 0, k_start = 0;

    static __device__ __forceinline__ int span(const int32_t* cu, int b, int64_t tokens, int64_t& start) {
        start = cu[b];
        const int64_t n = (int64_t)cu[b + 1] - start;
        return start < 0 || n < 0 || start + n > tokens ? 0 : (int)n;
    }
    static __device__ __forceinline__ uint32_t blocks_of(const PromptArgs& a, int b) {
        int64_t s;
        return (uint32_t)((span(a.cu_q, b, a.tokens_q, s) + kBM - 1) / kBM);
    }
    // The first of the block's steps that part s takes.
    __device__ __forceinline__ int first_step(int s) const { return (int)((int64_t)steps * s / splits); }

    struct Found { int32_t sequence, block; int64_t q_start, k_start; int32_t n_q, n_k; };
    // All threads.  Each looks at its own sequences, and the one whose sequence
    // the block falls into tells the others.
    __device__ __forceinline__ Block(const PromptArgs& a, uint32_t slot, uint32_t* wave_total, Found* found) {
        const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
        const int seg = (a.batch + 64 * kWaves - 1) / (64 * kWaves), first = tid * seg;
        const int last = first + seg < a.batch ? first + seg : a.batch;
        Found mine{};
        uint32_t own = 0;
        for (int b = first; b < last; ++b) {
            // (with one sequence a thread all four offsets are loaded at once)
            mine.n_q = span(a.cu_q, b, a.tokens_q, mine.q_start);
            mine.n_k = span(a.cu_k, b, a.tokens_k, mine.k_start);
            own += (uint32_t)((mine.n_q + kBM - 1) / kBM);
        }
        uint32_t sum = own;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t o = __shfl_up(sum, d);
            if (lane >= d) sum += o;
        }
        if (lane == 63) wave_total[wave] = sum;
        __syncthreads();
        uint32_t total = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            if (w < wave) sum += wave_total[w];
            total += wave_total[w];
        }
        const uint32_t order = slot / (uint32_t)a.q_heads;
        if (order >= total) return;
        uint32_t x = total - 1 - order;
        if (x < sum && x >= sum - own) {
            x -= sum - own;
            mine.sequence = first;
            if (seg > 1) {
                for (;; ++mine.sequence) {
                    const uint32_t n = blocks_of(a, mine.sequence);
                    if (x < n) break;
                    x -= n;
                }
                mine.n_q = span(a.cu_q, mine.sequence, a.tokens_q, mine.q_start);
                mine.n_k = span(a.cu_k, mine.sequence, a.tokens_k, mine.k_start);
            }
            mine.block = (int)x;
            *found = mine;
        }
        __syncthreads();
        const int kv_heads = a.q_heads / a.group, hx = (int)(slot % (uint32_t)a.q_heads);
        hk = hx % kv_heads;
        hq = hk * a.group + hx / kv_heads;
        auto uniform = [](int64_t v) {
            return (int64_t)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32 |
                   (uint32_t)__builtin_amdgcn_readfirstlane((int)v);
        };
        sequence = __builtin_amdgcn_readfirstlane(found->sequence);
        block = __builtin_amdgcn_readfirstlane(found->block);
        n_q = __builtin_amdgcn_readfirstlane(found->n_q);
        n_k = __builtin_amdgcn_readfirstlane(found->n_k);
        q_start = uniform(found->q_start);
        k_start = uniform(found->k_start);
        const int q_end = (block + 1) * kBM < n_q ? (block + 1) * kBM : n_q;
        const int keys = a.causal ? (q_end + n_k - n_q < n_k ? q_end + n_k - n_q : n_k) : n_k;
        steps = keys > 0 ? (keys + kBN - 1) / kBN : 0;
        splits = a.splits;
    }
};

// 16 bytes a lane from base + off straight to LDS, lane i's at dst + 16 i.
__device__ __forceinline__ void direct_load16(const uint16_t* base, uint32_t off, Lds* dst) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(make_rsrc(base, 0x7FFFFFFFu),
                                             (__attribute__((address_space(3))) void*)dst, 16, off, 0, 0, 0);
}

template <bool BF, int D>
__global__ __launch_bounds__(64 * kWaves, D == 256 ? 1 : 2) void prompt_attn_kernel(PromptArgs a) {
    constexpr int CH = D / 8;             // 16-byte chunks of a row
    constexpr int KS = D / 16;            // K steps of S
    constexpr int DT = D / 32;            // output tiles
    __shared__ __align__(16) uint16_t ks[2][kBN * D];
    __shared__ __align__(16) uint16_t vs[2][kBN * D];
    __shared__ uint32_t wave_total[kWaves];
    __shared__ Block::Found found;
    __shared__ int not_finite;

    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, col = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

    if (tid == 0) not_finite = 0;
    const uint32_t slot = blockIdx.x / (uint32_t)a.splits, split = blockIdx.x % (uint32_t)a.splits;
    const Block bl(a, slot, wave_total, &found);
    if (bl.sequence < 0) return;
    const int n_q = bl.n_q, n_k = bl.n_k, past = n_k - n_q, hq = bl.hq, hk = bl.hk;
    const int64_t q_start = bl.q_start, k_start = bl.k_start;
    const int q0 = bl.block * kBM + wave * 32;            // the wave's first query
    const int qi = q0 + col;                              // the lane's query
    const int limit = a.causal ? (qi + past < n_k - 1 ? qi + past : n_k - 1) : n_k - 1;
    const int wave_low = a.causal ? (q0 + past < n_k - 1 ? q0 + past : n_k - 1) : n_k - 1;
    const int wave_q_last = q0 + 31 < n_q ? q0 + 31 : n_q - 1;
    const int wave_keys = q0 >= n_q ? 0 : a.causal ? (wave_q_last + past + 1 < n_k ? wave_q_last + past + 1 : n_k) : n_k;
    // this part's steps of the block's
    const int step0 = bl.first_step(split), steps = bl.first_step(split + 1);

    u32x4 q[KS];
    {
        const int64_t row = q_start + (qi < n_q ? qi : n_q - 1);
        const uint16_t* src = a.q + row * a.q_stride + (int64_t)hq * D + half * 8;
#pragma unroll
        for (int s = 0; s < KS; ++s) q[s] = *reinterpret_cast<const u32x4*>(src + 16 * s);
    }
    // The keys' (or values') rows of a step straight into LDS, each lane 16 bytes
    // in order; the rearrangement is in which chunk of the row a lane fetches.
    // A lane's offsets from the step's first row are the same in every step but
    // one that ends past the last key: there they stay on the last row (those
    // scores are hidden, and what is hidden has to be a number).
    constexpr int LOADS = kBN * CH / (64 * kWaves);
    const uint32_t k_row = (uint32_t)a.k_stride * 2, v_row = (uint32_t)a.v_stride * 2;
    const uint16_t* const k_base = a.k + k_start * a.k_stride + (int64_t)hk * D;
    const uint16_t* const v_base = a.v + k_start * a.v_stride + (int64_t)hk * D;
    uint32_t k_off[LOADS], v_off[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const int at = (wave * LOADS + i) * 64 + lane, r = at / CH, ch = at % CH;
        k_off[i] = r * k_row + 16 * k_chunk<D>(r, ch);
        v_off[i] = r * v_row + 16 * v_chunk<D>(r, ch);
    }
    auto fetch = [&](bool V, int step, const uint16_t* base, Lds* to) __attribute__((always_inline)) {
        Lds* const buf = to + wave * LOADS * 512;
        const int64_t key0 = (int64_t)step * kBN;
        const uint16_t* const rows = base + key0 * (V ? a.v_stride : a.k_stride);
        if (key0 + kBN <= n_k) {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) direct_load16(rows, V ? v_off[i] : k_off[i], buf + i * 512);
        } else {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const int at = (wave * LOADS + i) * 64 + lane, r = at / CH, ch = at % CH;
                const uint32_t row = min(r, (int)(n_k - 1 - key0));
                direct_load16(rows, V ? row * v_row + 16 * v_chunk<D>(r, ch) : row * k_row + 16 * k_chunk<D>(r, ch),
                              buf + i * 512);
            }
        }
    };

    float16_t o[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[t][i] = 0.f;
    float m = -__builtin_inff(), l = 0.f;
    // S^T of a step's 64 keys
    auto scores = [&](float16_t (&s)[2], const Lds* kb) __attribute__((always_inline)) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
#pragma unroll
            for (int i = 0; i < 16; ++i) s[t][i] = 0.f;
#pragma unroll
            for (int j = 0; j < KS; ++j) {
                const int r = t * 32 + col;
                const u32x4 kf = lds_read16(kb + r * D + 8 * k_chunk<D>(r, 2 * j + half));
                s[t] = mfma32<BF>(kf, q[j], s[t]);
            }
        }
    };

    // A step's scores are computed while the step before goes through its
    // softmax: the matrix cores and the vector units then work side by side.
    // Keys are fetched two steps ahead, values one.
    float16_t s[2];
    auto k_tile = [&](int step) { return (Lds*)ks[0] + (step & 1) * kBN * D; };
    auto v_tile = [&](int step) { return (Lds*)vs[0] + (step & 1) * kBN * D; };
    if (step0 < steps) {
        fetch(false, step0, k_base, k_tile(step0));
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();
        if (step0 + 1 < steps) fetch(false, step0 + 1, k_base, k_tile(step0 + 1));
        fetch(true, step0, v_base, v_tile(step0));
        scores(s, k_tile(step0));
    }
    // One step.  The tiles that it fills and those that it reads are apart, and
    // said to be: reads would wait for the loads on their way otherwise (one
    // prompt of 8192, 8 heads of 256: 338 -> 321 us; 2048, 32 heads of 128: 55 ->
    // 52.5).
    auto one_step = [&](int step, Lds* __restrict k_to, Lds* __restrict v_to, const Lds* __restrict kb,
                        const Lds* __restrict vb, const uint16_t* __restrict k_from,
                        const uint16_t* __restrict v_from) __attribute__((always_inline)) {
        if (step + 2 < steps) fetch(false, step + 2, k_from, k_to);
        if (step + 1 < steps) fetch(true, step + 1, v_from, v_to);
        const int key0 = step * kBN;
        if (key0 >= wave_keys) return;
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
        const SwapPair halves = swap32(top);
        top = fmaxf(halves.a, halves.b);
        // The sums move to a new maximum only where it outgrows the old one by
        // 2^kSlack; until then weights above 1 are as exact as those below.
        if (__any((top - m) * a.scale2 > kSlack || (m == -__builtin_inff() && top > m))) {
            const float f = top == -__builtin_inff() ? 1.f : __builtin_amdgcn_exp2f((m - top) * a.scale2);
            m = top;
            l *= f;
#pragma unroll
            for (int t = 0; t < DT; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[t][i] *= f;
        }
        const float base = m == -__builtin_inff() ? 0.f : fmaf(m, a.scale2, -kPlaces<BF>);
        u32x4 p[4];
        float16_t next[2];
        // (after the last step the scores of what the other tile holds are computed)
        auto weights = [&](int at) {                      // of scores at, at + 1 of 32
            const int t = at / 16, i = at % 16;
            const float e0 = __builtin_amdgcn_exp2f(fmaf(s[t][i], a.scale2, -base));
            const float e1 = __builtin_amdgcn_exp2f(fmaf(s[t][i + 1], a.scale2, -base));
            const uint32_t pair = round_out2<BF>(e0, e1);
            p[2 * t + i / 8][(i % 8) / 2] = pair;
            l = dot2<BF>(pair, kOnes<BF>, l);             // the weights as the matrix cores see them
        };
        // keys 16 j + 4 half + 0..3 and + 8: the order in which p holds them
        auto values = [&](int t, int j) {
            const int l16 = lane & 15, d = 32 * t + 16 * ((lane >> 4) & 1) + 4 * (l16 & 3);
            const int r0 = 16 * j + 4 * half + (l16 >> 2), r1 = r0 + 8;
            const u32x2 v0 = lds_read_tr16(vb + r0 * D + 8 * v_chunk<D>(r0, d >> 3) + (d & 7));
            const u32x2 v1 = lds_read_tr16(vb + r1 * D + 8 * v_chunk<D>(r1, d >> 3) + (d & 7));
            return u32x4{v0[0], v0[1], v1[0], v1[1]};
        };
        if constexpr (D == 256) {
            // One wave a SIMD: nothing but its own vector work hides a wait for LDS.
            // The operands come four at a time, a batch ahead of their instructions,
            // and the softmax is spread over the scores' batches (one prompt of 8192,
            // 8 heads: 462 -> 338 us; heads of 128 and 64, which have other waves to
            // run meanwhile, 525 -> 535 and 167 -> 176).
            auto keys = [&](int x) {                      // operand x of 2 KS: 16 dims of 32 keys
                const int r = (x & 1) * 32 + col;
                return lds_read16(kb + r * D + 8 * k_chunk<D>(r, (x & ~1) + half));
            };
            constexpr int B = 4, KB = 2 * KS / B;
            u32x4 f[2][B];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) next[t][i] = 0.f;
#pragma unroll
            for (int i = 0; i < B; ++i) f[0][i] = keys(i);
#pragma unroll
            for (int b = 0; b < KB; ++b) {
#pragma unroll
                for (int i = 0; i < B; ++i) f[(b + 1) & 1][i] = b + 1 < KB ? keys((b + 1) * B + i) : values(0, i);
#pragma unroll
                for (int i = 0; i < B; ++i) next[i & 1] = mfma32<BF>(f[b & 1][i], q[(b * B + i) / 2], next[i & 1]);
#pragma unroll
                for (int at = b * 32 / KB; at < (b + 1) * 32 / KB; at += 2) weights(at);
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int t = 0; t < DT; ++t) {
                if (t + 1 < DT)
#pragma unroll
                    for (int i = 0; i < B; ++i) f[(KB + t + 1) & 1][i] = values(t + 1, i);
#pragma unroll
                for (int i = 0; i < B; ++i) o[t] = mfma32<BF>(f[(KB + t) & 1][i], p[i], o[t]);
                __builtin_amdgcn_sched_barrier(0);
            }
        } else {
            scores(next, kb);
#pragma unroll
            for (int at = 0; at < 32; at += 2) weights(at);
#pragma unroll
            for (int t = 0; t < DT; ++t)
#pragma unroll
                for (int j = 0; j < 4; ++j) o[t] = mfma32<BF>(values(t, j), p[j], o[t]);
        }
        s[0] = next[0];
        s[1] = next[1];
    };
    // A hidden value's weight is 0, which a value that is not finite would make NaN.
    // Where some query of the block does not see all of a step's rows (the last row
    // repeats past the end) such values leave the tile, and those of them that a
    // query does see are added to its sums afterwards, from memory.  Whether the
    // tile (or one before it) has any.  Measured, us without and with it (bf16): one
    // prompt of 8192, 32 heads of 128, 529 / 529, 8 of 256 319 / 326; 2048, 16 of 64
    // 28.4 / 29.7; seven of up to 333, 16 of 64, 9.7 / 10.3.  Blocks computed again
    // with care only where their sums are not finite cost registers in every step:
    // 8192, 32 heads of 128, 529 / 539, 8 heads on 8 of 256 341 / 362.
    auto leave_out = [&](Lds* tile) __attribute__((always_inline)) {
        typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
        typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
        constexpr uint16_t INF = BF ? 0x7F80 : 0x7C00;
        lds_u32x4* const mine = (lds_u32x4*)tile + tid;
        u16x2 most = {0, 0};
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const u32x4 v = mine[i * 64 * kWaves];
#pragma unroll
            for (int j = 0; j < 4; ++j)
                most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, v[j] & 0x7FFF7FFFu));
        }
        if (__builtin_expect(most[0] >= INF || most[1] >= INF, false)) {
#pragma unroll 1
            for (int i = 0; i < LOADS; ++i) {
                u32x4 v = mine[i * 64 * kWaves];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if ((v[j] & 0x7FFFu) >= INF) v[j] &= 0xFFFF0000u;
                    if ((v[j] >> 16 & 0x7FFFu) >= INF) v[j] &= 0xFFFFu;
                }
                mine[i * 64 * kWaves] = v;
            }
            not_finite = 1;
        }
        __syncthreads();
        return not_finite != 0;
    };
    auto add_left_out = [&](int step) __attribute__((always_inline)) {
        asm volatile("" : "+s"(step));                      // (its addresses are nothing to keep ready)
        const int key0 = step * kBN, keys = wave_keys - key0 < kBN ? wave_keys - key0 : kBN;
        const uint16_t* row = v_base + (int64_t)key0 * a.v_stride + 4 * half;
#pragma unroll 1
        for (int j = 0; j < keys; ++j, row += a.v_stride) {
            const bool seen = key0 + j <= limit;
#pragma unroll
            for (int t = 0; t < DT; ++t)
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    const u32x2 v = *reinterpret_cast<const u32x2*>(row + 32 * t + 2 * i);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float x = scale_f32<BF>((uint16_t)(v[e / 2] >> (16 * (e % 2))));
                        if (seen && !(fabsf(x) < __builtin_inff())) o[t][i + e] += x;
                    }
                }
        }
    };
    const int block_low = a.causal ? bl.block * kBM + past : n_k - 1;     // last key that all its queries see
    for (int step = step0; step < steps; ++step) {
        __builtin_amdgcn_s_waitcnt(0);                    // this wave's part of the tiles is there
        __syncthreads();                                  // everyone's is, and the other buffers are free
        const bool left_out = step * kBN + kBN - 1 > block_low && leave_out(v_tile(step));
        one_step(step, k_tile(step), v_tile(step + 1), k_tile(step + 1), v_tile(step), k_base, v_base);
        if (__builtin_expect(left_out, false)) add_left_out(step);
    }
    const SwapPair sums = swap32(l);
    l = sums.a + sums.b;
    if (a.splits > 1) {
        // the sums as the lanes hold them, whole lines at a time; then the rows'
        // maxima and sums of weights
        float* part = a.parts + split * a.part_stride + (int64_t)slot * kBM * (D + 2);
        float4_t* dst = reinterpret_cast<float4_t*>(part) + wave * DT * 4 * 64 + lane;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const float4_t v = {o[t][i], o[t][i + 1], o[t][i + 2], o[t][i + 3]};
                store_past_if(a.past, &dst[(t * 4 + i / 4) * 64], v);
            }
        if (half == 0) {
            part[kBM * D + wave * 32 + col] = m * a.scale2;
            part[kBM * (D + 1) + wave * 32 + col] = l;
        }
        return;
    }
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

// Adds the parts of one block of queries in their order: workgroup (slot, y)
// takes 256 of the block's lanes' groups of four sums, one a thread.  Bound by
// reading the parts: 64 blocks of 8 parts, heads of 128 (34 MB), 7.8 us.
template <bool BF, int D>
__global__ __launch_bounds__(64 * kWaves) void prompt_join_kernel(PromptArgs a) {
    constexpr int DT = D / 32, AHEAD = 4;
    __shared__ uint32_t wave_total[kWaves];
    __shared__ Block::Found found;
    const Block bl(a, blockIdx.x, wave_total, &found);
    if (bl.sequence < 0) return;
    const int x = blockIdx.y * 64 * kWaves + threadIdx.x, lane = x % 64, t = x / 256 % DT, i = x / 64 % 4;
    const int r = x / (256 * DT) * 32 + lane % 32, qi = bl.block * kBM + r;
    if (qi >= bl.n_q) return;
    const float* part = a.parts + (int64_t)blockIdx.x * kBM * (D + 2);
    float top = -__builtin_inff(), sum = 0.f;
    float4_t v = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = 0; s0 < a.splits; s0 += AHEAD) {
        float ms[AHEAD], ls[AHEAD];
        float4_t vs[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const bool real = s0 + k < a.splits;
            const float* p = part + (real ? s0 + k : s0) * a.part_stride;
            ms[k] = real ? p[kBM * D + r] : -__builtin_inff();
            ls[k] = p[kBM * (D + 1) + r];
            vs[k] = reinterpret_cast<const float4_t*>(p)[x];
        }
        float next = top;
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) next = fmaxf(next, ms[k]);
        auto weight_of = [&](float m) { return m == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(m - next); };
        const float f = weight_of(top);
        top = next;
        sum *= f;
        v *= f;
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const float e = weight_of(ms[k]);
            sum = fmaf(ls[k], e, sum);
            v += vs[k] * e;
        }
    }
    v *= sum == 0.f ? 0.f : 1.f / sum;
    *reinterpret_cast<u32x2*>(a.out + ((bl.q_start + qi) * a.q_heads + bl.hq) * (int64_t)D + 32 * t + 8 * i +
                              4 * (lane / 32)) = u32x2{round_out2<BF>(v[0], v[1]), round_out2<BF>(v[2], v[3])};
}

// Blocks of queries times heads, at most: the sum of ceil(n / kBM) over sequences.
int64_t most_slots(int64_t batch, int64_t tokens_q, int q_heads) {
    return (tokens_q + (kBM - 1) * (batch < tokens_q ? batch : tokens_q)) / kBM * q_heads;
}
// Parts that the keys of a block are split into, for sequences taken to be of one
// length: as many as fill the chip (two workgroups a compute unit, one with heads
// of 256), of at least 8 steps of a block's mean, or 2.5 of the longer ones of
// heads of 256.  These also pay for parts where causal blocks are many enough but
// of lengths so different that the longest alone fill the end.  Measured (us,
// parts 1 / 2 / 4; the rule's in brackets): 16 heads of 128, 1 x 1024 [25.9] / 28.5
// / 25.4, 1 x 2048 45.9 / [43.1] / 49.2, 4096 [94.5] / 100.8 / 115; 500 after 3000
// 71.5 / 46.1 / 34.5 / [6: 32.7]; 8 heads of 256, 1 x 1024 46.3 / 36.1 / 30.1 [3:
// 32.4], 4096 151 / [113] / 135, 4 x 1000 [47.5] / 65.8 / 81.3.
int splits_for(int64_t slots, int64_t batch, int64_t tokens_q, int64_t tokens_k, int D, bool causal) {
    const int64_t n_k = tokens_k / batch, n_q = tokens_q / batch < n_k ? tokens_q / batch : n_k;
    const int64_t mean = causal ? n_k - n_q / 2 : n_k;
    int64_t wgs = D == 256 ? kSizedForCus : 2 * kSizedForCus;
    if (D == 256 && mean >= 16 * kBN) wgs = wgs * n_k / mean;
    const int64_t idle = wgs / slots, by_keys = mean / (D == 256 ? 5 * kBN / 2 : 8 * kBN);
    const int64_t s = idle < by_keys ? idle : by_keys;
    return s < 2 ? 1 : s > kMostSplits ? kMostSplits : (int)s;
}

}  // namespace

int64_t prompt_attention_workspace_bytes(int64_t batch, int64_t tokens_q, int64_t tokens_k, int q_heads, int D) {
    const int64_t slots = most_slots(batch, tokens_q, q_heads);
    const int full = splits_for(slots, batch, tokens_q, tokens_k, D, false);
    const int causal = splits_for(slots, batch, tokens_q, tokens_k, D, true), s = full > causal ? full : causal;
    return s == 1 ? 0 : align256(slots * s * kBM * (D + 2) * 4);
}

int launch_prompt_attention(bool bf, const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v,
                            int64_t v_stride, const int32_t* cu_q, const int32_t* cu_k, int64_t batch,
                            int64_t tokens_q, int64_t tokens_k, int q_heads, int kv_heads, int D, float scale,
                            bool causal, void* out, void* ws, hipStream_t s) {
    auto in = [](const void* p) { return static_cast<const uint16_t*>(p); };
    PromptArgs a{in(q), in(k), in(v), q_stride, k_stride, v_stride, cu_q, cu_k, (int)batch, q_heads,
                 q_heads / kv_heads, tokens_q, tokens_k, scale * 1.4426950408889634f, causal ? 1 : 0,
                 static_cast<uint16_t*>(out), 1, static_cast<float*>(ws), 0, false};
    const int64_t slots = most_slots(batch, tokens_q, q_heads);
    if (ws) a.splits = splits_for(slots, batch, tokens_q, tokens_k, D, causal);
    a.part_stride = slots * kBM * (D + 2);
    a.past = a.splits * a.part_stride * 4 <= kMostPast;
    const dim3 grid((unsigned)(slots * a.splits)), join_grid((unsigned)slots, (unsigned)(kBM * D / 4 / (64 * kWaves)));
    auto go = [&](auto d) {
        constexpr int D_ = decltype(d)::value;
        const int rc = bf ? launch(prompt_attn_kernel<true, D_>, grid, dim3(64 * kWaves), 0, s, a)
                          : launch(prompt_attn_kernel<false, D_>, grid, dim3(64 * kWaves), 0, s, a);
        if (rc || a.splits == 1) return rc;
        return bf ? launch(prompt_join_kernel<true, D_>, join_grid, dim3(64 * kWaves), 0, s, a)
                  : launch(prompt_join_kernel<false, D_>, join_grid, dim3(64 * kWaves), 0, s, a);
    };
    if (D == 64) return go(std::integral_constant<int, 64>{});
    if (D == 128) return go(std::integral_constant<int, 128>{});
    return go(std::integral_constant<int, 256>{});
}

}  // namespace tf
