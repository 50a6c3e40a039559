// Attention of single tokens over the 4-bit paged cache (decode).
//
// For the R = q_len * (q_heads / kv_heads) query rows that read one key/value
// head of one sequence:
//   S[j] = s_k[j] (Q . q_k[j] - z_k[j] sum(Q)),  P = softmax(scale S)
//   O    = sum_j P[j] s_v[j] (q_v[j] - z_v[j])
// The codes go to the matrix cores as they are: a code under a fixed exponent
// is a 16-bit float off + q (one and-or for two codes), and off and z leave as
// products with sum(Q) and with sums of P in fp32.
//
// The cache, D + 8 bytes a token and head, is read once, at the rate of a large
// copy where there is enough of it: 16 sequences of 8192, 32 heads on 32 of 128,
// 110 us, 5.2 TB/s; 64 of up to 8192, 32 heads on 8 of 128, 51 us, 3.9 TB/s, of
// which beginning and end take 8 us.  There the vector unit is 78% busy with codes
// and the softmax of 16 columns, of which q_len * group are real, but is not what
// is waited for: a copy with half the softmax ran 2% faster, one with shares that
// let all workgroups of a compute unit end together 1%.  Few tokens cost the chain
// lengths - table - tiles - sums: one sequence of 513 keys 8.9 us (fp16).
#include "tf_kv4.h"

namespace tf {

Kv4 kv4_view(const tf_kv4_cache& c);

namespace {

constexpr uint32_t kItemCost = 3;        // what beginning and ending an item costs, in rounds
constexpr uint32_t kLeastRounds = 3;     // rounds of an item that one workgroup takes before a second helps
constexpr uint32_t kFewParts = 16;       // parts that cost less to join than a second round of each
constexpr int kMostWgs = 1024;           // workgroups of a launch, at most (and counters in the workspace)
constexpr int kJoinThreads = 512;

struct AttnArgs {
    Kv4 cache;
    const uint16_t* q;
    int64_t q_stride;
    const int32_t* lens;
    int batch, q_len, group, row_blocks;  // group: query heads per key/value head
    Divisor by_batch, by_group, by_row_blocks, by_heads, by_tiles;        // heads: of keys, times row_blocks; tiles: of a page
    uint32_t wgs;                         // workgroups that share the rounds
    int32_t capacity;                     // positions a table row can hold
    float scale2;                         // softmax scale * log2(e)
    uint16_t* out;
    uint32_t* counters;                   // null: kv4_join_kernel adds the parts, as `spans` names them
    uint32_t* spans;                      // first and last workgroup of each item, by the first one
    float* parts;
};

// Offsets under which codes appear in the operands.  fp16 reads every second
// nibble without a shift, which gives it another exponent (64 instead of
// 1024).  Values of odd keys are stored as 15 - q and read with the sign set,
// -(off + 15 - q) = q - (off + 15): the offsets of neighbouring keys nearly
// cancel in the running sums, which so stay of the size of the codes instead of
// growing as off * sum(P) and losing the result's digits to it.
template <bool BF> constexpr float kOffA = BF ? 128.f : 1024.f;   // nibbles 0, 2
template <bool BF> constexpr float kOffB = BF ? 128.f : 64.f;     // nibbles 1, 3

// The weights go to the matrix cores as e s_v, e = 2^(scale2 x - base).  With base
// the maximum, e <= 1, fp16 has no room for them: under a scale of 2^-8 a key of
// 2^-6 of the largest weight would lose digits and one of 2^-17 be lost, in the
// numerator alone.  So base is the maximum less `places`, the most for which no e s_v
// passes 2^12 (2^15 is there: the maximum's own rounding may add some), by the
// exponent of the largest |s_v| that the row has seen: |s_v| < 2^(field - 14).  (8192
// keys, a sink of 91% of the weight, values of 0.1: error 1.2e-3 -> 1e-5 before the
// output's rounding; 65536, 10% outside the sink, of 0.05: 0.16 -> 5e-6.)  The sums of
// weights have the same power, which so leaves with them.  bf16 has fp32's exponents.
// It costs 1 or 2% (64 ragged sequences 50.2 -> 50.3 us, one of 513 keys 8.7 -> 8.9,
// two of 65537 with four tokens of one head of 256, for a spill, 27.1 -> 28.4).
constexpr int kMostPlaces = 12 + 14;

struct Magic { uint32_t a, b; };
template <bool BF>
__device__ __forceinline__ Magic magics(uint32_t sign) {
    Magic m{(BF ? 0x43004300u : 0x64006400u) | sign, (BF ? 0x43004300u : 0x54005400u) | sign};
    asm("" : "+v"(m.a), "+v"(m.b));       // in registers: one v_and_or_b32 each
    return m;
}
// The four pairs (nibbles e and e + 4) of a word.
template <bool BF>
__device__ __forceinline__ u32x4 code_pairs(uint32_t w, const Magic& m) {
    u32x4 o;
    if constexpr (BF) {
        o[0] = (w & 0x000F000Fu) | m.a;
        o[1] = (w >> 4 & 0x000F000Fu) | m.a;
        o[2] = (w >> 8 & 0x000F000Fu) | m.a;
        o[3] = (w >> 12 & 0x000F000Fu) | m.a;
    } else {
        const uint32_t w8 = w >> 8;
        o[0] = (w & 0x000F000Fu) | m.a;
        o[1] = (w & 0x00F000F0u) | m.b;
        o[2] = (w8 & 0x000F000Fu) | m.a;
        o[3] = (w8 & 0x00F000F0u) | m.b;
    }
    return o;
}

// Sum and maximum over the four 16-lane groups, the same in all of them.
__device__ __forceinline__ float over_groups(float v) {
    const SwapPair r = swap16(v);
    const SwapPair h = swap32(r.a + r.b);
    return h.a + h.b;
}
__device__ __forceinline__ float max_over_groups(float v) {
    const SwapPair r = swap16(v);
    const SwapPair h = swap32(fmaxf(r.a, r.b));
    return fmaxf(h.a, h.b);
}

__device__ __forceinline__ uint32_t max_over_groups(uint32_t v) {
    auto most = [](auto r) { return r[0] > r[1] ? r[0] : r[1]; };
    v = most(__builtin_amdgcn_permlane16_swap(v, v, false, false));
    return most(__builtin_amdgcn_permlane32_swap(v, v, false, false));
}

// What lane % 16 of the first group holds.
__device__ __forceinline__ float of_group0(float v) { return swap32(swap16(v).a).a; }

// 16-byte pieces of a lane's K (or V) codes, and word w of key half u in them
// as kv4_word places it.
template <int D> constexpr int kPieces = D == 64 ? 1 : D / 64;
template <int D>
__device__ __forceinline__ uint32_t code_word(const u32x4* x, int u, int w) {
    if constexpr (D == 64) return x[0][2 * u + w];
    else return x[u * (D / 128) + w / 4][w % 4];
}

// Reads of N 16-byte pieces, `step` bytes apart, from LDS that direct loads
// fill, waited for in the same statement.  (As statements of the language the
// compiler would put a wait for every direct load in flight before them.)
template <int N, int STEP>
__device__ __forceinline__ void lds_read(u32x4* x, uint32_t at) {
    if constexpr (N == 1) {
        asm volatile("ds_read_b128 %0, %1\n\ts_waitcnt lgkmcnt(0)" : "=&v"(x[0]) : "v"(at) : "memory");
    } else if constexpr (N == 2) {
        asm volatile("ds_read_b128 %0, %2\n\tds_read_b128 %1, %2 offset:%3\n\ts_waitcnt lgkmcnt(0)"
                     : "=&v"(x[0]), "=&v"(x[1]) : "v"(at), "i"(STEP) : "memory");
    } else {
        static_assert(N == 4, "one, two or four pieces");
        asm volatile("ds_read_b128 %0, %4\n\tds_read_b128 %1, %4 offset:%5\n\tds_read_b128 %2, %4 offset:%6\n\t"
                     "ds_read_b128 %3, %4 offset:%7\n\ts_waitcnt lgkmcnt(0)"
                     : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3])
                     : "v"(at), "i"(STEP), "i"(2 * STEP), "i"(3 * STEP) : "memory");
    }
}
typedef const __attribute__((address_space(1))) uint8_t* GlobalBytes;
// 16 (or 4) bytes a lane from its p straight to LDS: lane i's at dst + 16 i (4 i).
typedef const __attribute__((address_space(1))) void* GlobalVoid;
typedef __attribute__((address_space(3))) void* LdsVoid;
__device__ __forceinline__ void direct_load16(GlobalBytes p, uint32_t dst) {
    __builtin_amdgcn_global_load_lds((GlobalVoid)p, (LdsVoid)(uintptr_t)dst, 16, 0, 0);
}
__device__ __forceinline__ void direct_load4(GlobalBytes p, uint32_t dst) {
    __builtin_amdgcn_global_load_lds((GlobalVoid)p, (LdsVoid)(uintptr_t)dst, 4, 0, 0);
}

// Value i (0..7) of eight packed 16-bit floats.
template <bool BF>
__device__ __forceinline__ float meta_f32(const u32x4& m, int i) {
    const uint32_t w = m[i / 2];
    if constexpr (BF) return __builtin_bit_cast(float, i & 1 ? w & 0xFFFF0000u : w << 16);
    else return scale_f32<false>(i & 1 ? w >> 16 : w & 0xFFFFu);
}

__device__ __forceinline__ uint32_t lds_address(const void* p) {
    return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p;
}

// A pointer to memory that no kernel writes while this one runs, as the scalar
// loads take it.
__device__ __forceinline__ const __attribute__((address_space(4))) int32_t* as_constant(const int32_t* p) {
    return (const __attribute__((address_space(4))) int32_t*)(uintptr_t)p;
}

// How the rounds of all items are shared out.  An item is one (sequence,
// key/value head, block of query rows); its rounds are 32 keys for each of W
// waves, at least one (which writes the zeros of an empty row), and it counts
// kItemCost units of its own before them.  Workgroup w of `wgs` takes a
// contiguous share of all units, in the order of sequence, head and block, and
// shares differ by at most one unit whatever the lengths are.  Where there are
// fewer items than workgroups, no more of these work than an item of average
// length is worth: one where no item has more than kLeastRounds rounds (they cost
// less than joining parts), else one a round, or one for two rounds past kFewParts
// (items of one length then end where shares do).
template <int W, int THREADS>
struct Shares {
    static constexpr int WAVES = THREADS / 64, KEYS = kKvTile * W;
    const AttnArgs& a;
    int first_b, last_b;                  // this thread's sequences
    uint32_t own_len, own, until;         // the last one's length; units of one head of them, and with all before
    uint32_t heads, total, wgs;
    uint32_t share, rest;                 // total / wgs and what that leaves
    float inv_wgs, wgs_per_unit;

    __device__ __forceinline__ static uint32_t clamped(const AttnArgs& a, int32_t n) {
        return (uint32_t)(n < 0 ? 0 : n > a.capacity ? a.capacity : n);
    }
    __device__ __forceinline__ static uint32_t length_of(const AttnArgs& a, int b) { return clamped(a, a.lens[b]); }
    // the same for a b that all lanes share
    __device__ __forceinline__ static uint32_t uniform_length(const AttnArgs& a, int b) {
        return clamped(a, as_constant(a.lens)[b]);
    }
    __device__ __forceinline__ static uint32_t rounds_of(uint32_t n) {
        return n == 0 ? 1u : (n + KEYS - 1) / KEYS;
    }
    __device__ __forceinline__ static uint32_t units_of(uint32_t n) { return kItemCost + rounds_of(n); }
    // All THREADS threads, each with its part of the sequences; scratch: WAVES
    // words of LDS.
    __device__ __forceinline__ Shares(const AttnArgs& args, uint32_t* scratch) : a(args), own_len(0), own(0) {
        const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
        const int seg = (a.batch + THREADS - 1) / THREADS;
        first_b = tid * seg;
        last_b = first_b + seg < a.batch ? first_b + seg : a.batch;
        uint32_t longest = 0;
        for (int b = first_b; b < last_b; ++b) {
            own_len = length_of(a, b);
            own += units_of(own_len);
            longest = own_len > longest ? own_len : longest;
        }
        // units of all heads fit 31 bits: the 32nd carries whether an item is long
        const uint32_t is_long = __any(longest > kLeastRounds * KEYS) ? 1u << 31 : 0;
        until = own;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t o = __shfl_up(until, d);
            if (lane >= d) until += o;
        }
        if (lane == 63) scratch[wave] = until | is_long;
        __syncthreads();
        uint32_t all = 0, any_long = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const uint32_t n = scratch[w] & ~(1u << 31);
            if (w < wave) until += n;
            all += n;
            any_long |= scratch[w] >> 31;
        }
        all = __builtin_amdgcn_readfirstlane(all);
        heads = a.by_heads.d;
        total = all * heads;
        const uint32_t items = heads * a.batch;
        uint32_t pieces = 1;
        if (__builtin_amdgcn_readfirstlane(any_long)) {
            const uint32_t mean = a.by_batch.of(all - kItemCost * a.batch);
            pieces = mean <= kFewParts ? mean : (mean + 1) / 2;
        }
        wgs = items < a.wgs && items * pieces < a.wgs ? items * pieces : a.wgs;
        share = total / wgs;
        rest = total - share * wgs;
        inv_wgs = __builtin_amdgcn_rcpf((float)wgs);
        wgs_per_unit = (float)wgs * __builtin_amdgcn_rcpf((float)total);
    }
    // n / d for quotients below 2^20, of which the approximation is one off at most
    __device__ __forceinline__ static uint32_t small_quotient(uint32_t n, uint32_t d, float inv) {
        const uint32_t q = (uint32_t)((float)n * inv);
        const int32_t r = (int32_t)(n - q * d);
        return r < 0 ? q - 1 : r >= (int32_t)d ? q + 1 : q;
    }
    // floor(w total / wgs) (w is at most kMostWgs and rest below it)
    __device__ __forceinline__ uint32_t begin_of(uint32_t w) const {
        return w * share + small_quotient(w * rest, wgs, inv_wgs);
    }
    // the workgroup that takes unit x: the last w with begin_of(w) <= x
    __device__ __forceinline__ uint32_t owner(uint32_t x) const {
        uint32_t w = (uint32_t)((float)x * wgs_per_unit);                     // one off at most
        w = w < wgs ? w : wgs - 1;
        if (begin_of(w) > x) return w - 1;
        return w + 1 < wgs && begin_of(w + 1) <= x ? w + 1 : w;
    }
    struct Found { int32_t b; uint32_t start, len; };
    // The sequence of unit x, the units (of all heads) before it and its length,
    // told by the thread that has it.
    __device__ __forceinline__ Found sequence_of_unit(uint32_t x, Found* lds) const {
        x = a.by_heads.of(x);
        if (x < until && x >= until - own) {
            Found f{first_b, until - own, own_len};
            if (last_b - first_b > 1)
                for (;; ++f.b) {
                    f.len = length_of(a, f.b);
                    const uint32_t n = units_of(f.len);
                    if (x < f.start + n) break;
                    f.start += n;
                }
            *lds = f;
        }
        return told(lds);
    }

private:
    __device__ __forceinline__ Found told(const Found* lds) const {
        __syncthreads();
        return {__builtin_amdgcn_readfirstlane(lds->b), (uint32_t)__builtin_amdgcn_readfirstlane(lds->start) * heads,
                (uint32_t)__builtin_amdgcn_readfirstlane(lds->len)};
    }
};

// One part of an item that several workgroups share: `rows` rows of D sums,
// their maxima and their sums of weights.  A workgroup has at most two: of the
// item that it ends (slot 0) and of the one that it begins (slot 1).
template <int D, int ROWS>
struct Parts {
    static constexpr int64_t kSlot = (int64_t)ROWS * (D + 2);
    static __device__ __forceinline__ float* at(float* parts, uint32_t w, uint32_t first) {
        return parts + ((int64_t)w * 2 + (w == first ? 1 : 0)) * kSlot;
    }
};

// What sums under the maximum m weigh under the maximum `to`; nothing where
// they hold nothing (a NaN among them stays one: it is multiplied, not skipped).
__device__ __forceinline__ float weight_of(float m, float to) {
    return m == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(m - to);
}

// Adds the parts of workgroups first..final, in their order, at U pairs of
// neighbouring sums (d[u] of row r[u]), AHEAD parts at a time; v[u] are the
// outputs.  load2: two floats at an even address.
template <int D, int ROWS, int AHEAD, int U, typename Load2, typename Load1>
__device__ __forceinline__ void join_parts(float* parts, uint32_t first, uint32_t final, const int (&r)[U],
                                           const int (&d)[U], float2_t (&v)[U], Load2 load2, Load1 load1) {
    using P = Parts<D, ROWS>;
    float top[U], sum[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        top[u] = -__builtin_inff();
        sum[u] = 0.f;
        v[u] = float2_t{0.f, 0.f};
    }
    for (uint32_t w0 = first; w0 <= final; w0 += AHEAD) {
        float mw[U][AHEAD], lw[U][AHEAD];
        float2_t vw[U][AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const float* p = P::at(parts, w0 + i <= final ? w0 + i : final, first);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                mw[u][i] = load1(p + ROWS * D + r[u]);
                lw[u][i] = load1(p + ROWS * (D + 1) + r[u]);
                vw[u][i] = load2(p + r[u] * D + d[u]);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float next = top[u];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i)
                if (w0 + i <= final) next = fmaxf(next, mw[u][i]);
            const float f = weight_of(top[u], next);
            top[u] = next;
            sum[u] *= f;
            v[u] *= f;
#pragma unroll
            for (int i = 0; i < AHEAD; ++i)
                if (w0 + i <= final) {
                    const float e = weight_of(mw[u][i], next);
                    sum[u] = fmaf(lw[u][i], e, sum[u]);
                    v[u][0] = fmaf(vw[u][i][0], e, v[u][0]);
                    v[u][1] = fmaf(vw[u][i][1], e, v[u][1]);
                }
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] *= sum[u] == 0.f ? 0.f : 1.f / sum[u];
}

// Output row `row` (of the q_len * group that read one head) of an item.
template <int D>
__device__ __forceinline__ uint16_t* out_row(const AttnArgs& a, int b, int h, int row) {
    const int tq = (int)a.by_group.of(row);
    return a.out + ((int64_t)b * a.q_len + tq) * ((int64_t)a.cache.kv_heads * a.group * D) +
           (int64_t)(h * a.group + row - tq * a.group) * D;
}

// A barrier for what the workgroup shares in LDS: unlike __syncthreads it does
// not wait for stores to memory.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// Half of 2 N groups of four sums goes to the wave that keeps that half, and this
// wave adds what that one holds of its own half.
template <int N>
__device__ __forceinline__ void exchange(float4_t* v, bool upper, float4_t* out, const float4_t* in) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float4_t lo = v[i], hi = v[N + i];
        out[i * 64] = upper ? lo : hi;
        v[i] = upper ? hi : lo;
    }
    lds_barrier();
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += in[i * 64];
}

// Waves that a SIMD holds, as the registers of the sums allow.
constexpr int waves_per_simd(int D, int nr) { return D <= 128 && nr == 1 ? 4 : 2; }

// One workgroup of W waves on its share of the rounds (see Shares), a tile for
// each wave a round.  Items that lie inside one share are written directly; the
// others' partial sums go through the workspace, and the workgroup that arrives
// last adds them in order (or kv4_join_kernel does).
template <bool BF, int D, int NR, int W>
__global__ __launch_bounds__(64 * W, waves_per_simd(D, NR)) void kv4_attn_kernel(AttnArgs a) {
    constexpr int THREADS = 64 * W;
    using Shares = tf::Shares<W, THREADS>;
    constexpr int NT = D / 16;            // 16-dim tiles of the output
    constexpr int NW = D / 32;            // words of codes per lane and key half
    constexpr int ROWS = 16 * NR;
    constexpr int SUMS = NR * NT;         // groups of four sums of a lane, and what a wave keeps of them
    constexpr int KEEP = SUMS >= W ? SUMS / W : 1;
    constexpr int64_t TB = kv4_tile_bytes(D);
    using P = Parts<D, ROWS>;
    // Each wave keeps RING tiles in LDS, fetched by direct loads: what it
    // multiplies and RING - 1 on the way, without a register.  The same memory
    // takes the waves' sums once an item's tiles are done.
    constexpr int RING = D == 64 ? 4 : 2, LOADS = 2 * kPieces<D> + 1;
    constexpr int kRingBytes = W * RING * (int)TB, kSumBytes = SUMS / 2 * 1024;
    static_assert(W * kSumBytes <= kRingBytes, "the waves' sums fit the ring");
    __shared__ __align__(1024) uint8_t pool[kRingBytes];
    __shared__ uint32_t scratch[W];
    __shared__ typename Shares::Found found;
    __shared__ __align__(16) float ms[ROWS][W], ls[ROWS][W];
    __shared__ __align__(16) float2_t q_sums[NR][16][NW];
    __shared__ u32x4 qs[NR][NW][64];
    __shared__ int last;

    const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const Shares sh(a, scratch);
    const uint32_t wg = blockIdx.x;
    if (wg >= sh.wgs) return;
    uint32_t at = __builtin_amdgcn_readfirstlane(sh.begin_of(wg));
    const uint32_t end = __builtin_amdgcn_readfirstlane(sh.begin_of(wg + 1));
    if (at >= end) return;
    const typename Shares::Found at_first = sh.sequence_of_unit(at, &found);
    int b = at_first.b;
    uint32_t seq_start = at_first.start;  // units (of all heads) before sequence b
    uint32_t b_len = at_first.len;

    const uint32_t ring = lds_address(pool) + wave * RING * (uint32_t)TB;
    const uint32_t q_at = lds_address(qs) + lane * 16;
    const Magic mk = magics<BF>(0), mv = magics<BF>(0x80000000u);
    // Row 0 of a further operand beside the values' codes takes the values'
    // zero-points, row 1 and 2 the offsets of the low and high dims' codes: one
    // matrix instruction sums the rounded weights with each of them.
    const uint32_t off_a = BF ? 0xC30F4300u : 0xE40F6400u;    // -(off + 15), off
    const uint32_t off_b = BF ? 0xC30F4300u : 0xD4F05400u;
    const uint32_t off_row = c == 1 ? off_a : c == 2 ? off_b : 0u;
    const int q_rows = a.q_len * a.group;

    while (at < end) {
        // ---- the item at `at`
        const uint32_t len = b_len;
        const uint32_t n_rounds = Shares::rounds_of(len), n_units = Shares::units_of(len);
        const uint32_t item = Shares::small_quotient(at - seq_start, n_units, __builtin_amdgcn_rcpf((float)n_units));
        const uint32_t item_rounds = seq_start + item * n_units + kItemCost;      // unit of its first round
        const int h = (int)a.by_row_blocks.of(item), rb = (int)item - h * a.row_blocks;
        const uint32_t r0 = at > item_rounds ? at - item_rounds : 0;
        const uint32_t item_end = item_rounds + n_rounds;
        const uint32_t r1 = (end < item_end ? end : item_end) - item_rounds;
        at = end < item_end ? end : item_end;
        const int this_b = b;
        if (item + 1 == sh.heads && at == item_end) {
            seq_start += sh.heads * n_units;
            ++b;
            if (at < end) b_len = Shares::uniform_length(a, b);
        }
        if (at <= item_rounds) continue;  // the share ends before the item's rounds

        // The queries as the matrix cores take them, by way of LDS, each wave some of
        // their 32-dim pieces (all waves asking for all of them cost 4 us of 30 for 32
        // rows of 256).  Requested before anything waits for the page table.
        int limit[NR];                    // last visible position of the lane's row
        const uint16_t* q_src[NR];
#pragma unroll
        for (int n = 0; n < NR; ++n) {
            const int row = rb * ROWS + n * 16 + c;
            const bool real = row < q_rows;
            const int tq = real ? (int)a.by_group.of(row) : 0, hq = h * a.group + (real ? row - tq * a.group : 0);
            q_src[n] = a.q + ((int64_t)this_b * a.q_len + tq) * a.q_stride + (int64_t)hq * D + 8 * g;
            limit[n] = (int)len - a.q_len + tq;
        }
        constexpr int WORDS = NR * NW, OWN = (WORDS + W - 1) / W;
        u32x4 q[OWN];
#pragma unroll
        for (int i = 0; i < OWN; ++i) {
            const int x = wave + i * W, n = x / NW;
            q[i] = u32x4{0, 0, 0, 0};
            if (x < WORDS && rb * ROWS + n * 16 + c < q_rows)
                q[i] = *reinterpret_cast<const u32x4*>((NR == 2 && n ? q_src[NR - 1] : q_src[0]) + 32 * (x % NW));
        }

        // ---- the wave's tiles: W r + wave for r0 <= r < r1, those that begin before len
        const uint32_t tiles = (len + kKvTile - 1) / kKvTile;
        // Table entries are read through the scalar cache, an iteration ahead: a
        // vector load would wait in line behind the codes.  A tile without a
        // page is some memory of the cache, and every key of it hidden.
        const auto* row = as_constant(a.cache.table) + this_b * a.cache.table_stride;
        auto entry_of = [&](uint32_t t) { return row[a.by_tiles.of(t)]; };
        auto tile_at = [&](uint32_t t, int32_t page, bool& found) {
            found = page >= 0 && page < a.cache.pages;
            const uint32_t in_page = t - a.by_tiles.of(t) * a.by_tiles.d;
            const uint8_t* p = a.cache.data + (found ? (int64_t)page * a.cache.page_bytes +
                                                           ((int64_t)h * a.by_tiles.d + in_page) * TB : 0);
            asm("" : "+s"(p));            // in scalar registers, the lanes' offsets beside it
            return (GlobalBytes)(uintptr_t)p;
        };
        auto fetch = [&](GlobalBytes tile, uint32_t slot) {
            const uint32_t dst = __builtin_amdgcn_readfirstlane(ring + slot * (uint32_t)TB);
            const uint32_t off = lane * 16;
#pragma unroll
            for (int p = 0; p < 2 * kPieces<D>; ++p) direct_load16(tile + p * 1024 + off, dst + p * 1024);
            direct_load4(tile + 32 * D + lane * 4, dst + 32 * D);
        };
        uint32_t t = W * r0 + wave;
        const uint32_t t_end = W * r1 < tiles ? W * r1 : tiles;
        // Tiles are fetched RING - 1 ahead, and past the end some memory of the
        // cache, so that the number of loads in flight is always the same.
        bool found[RING];
        int32_t entry;
#pragma unroll
        for (int i = 0; i < RING; ++i) {
            const uint32_t ti = t + i * W;
            entry = ti < t_end ? entry_of(ti) : -1;
            fetch(tile_at(ti, entry, found[i]), i);
        }
        entry = t + RING * W < t_end ? entry_of(t + RING * W) : -1;

        const uint32_t first = __builtin_amdgcn_readfirstlane(sh.owner(item_rounds));
        const uint32_t final = __builtin_amdgcn_readfirstlane(sh.owner(item_end - 1));

#pragma unroll
        for (int i = 0; i < OWN; ++i) {
            const int x = wave + i * W, n = x / NW, w = x % NW;
            if (x >= WORDS) continue;
            const u32x4& v = q[i];
            const int ch = 4 * w + g;     // the lane's 8 dims: word ch % NW of lane group ch / NW
            qs[n][ch % NW][ch / NW * 16 + c] = v;
            const float sa = meta_f32<BF>(v, 0) + meta_f32<BF>(v, 1) + meta_f32<BF>(v, 4) + meta_f32<BF>(v, 5);
            const float sb = meta_f32<BF>(v, 2) + meta_f32<BF>(v, 3) + meta_f32<BF>(v, 6) + meta_f32<BF>(v, 7);
            const float2_t both = {over_groups(sa), over_groups(sb)};
            if (g == 0) q_sums[n][c][w] = both;
        }
        lds_barrier();
        float sum_q[NR], off_q[NR];
#pragma unroll
        for (int n = 0; n < NR; ++n) {
            u32x4 x[NW / 2];
            lds_read<NW / 2, 16>(x, lds_address(q_sums[n][c]));
            float sa = 0.f, sb = 0.f;
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                sa += __builtin_bit_cast(float, (uint32_t)x[w / 2][2 * (w % 2)]);
                sb += __builtin_bit_cast(float, (uint32_t)x[w / 2][2 * (w % 2) + 1]);
            }
            sum_q[n] = sa + sb;
            off_q[n] = sa * kOffA<BF> + sb * kOffB<BF>;
        }
        float4_t o[SUMS], osum[NR];       // osum: rows 0..2 of the further operand
        float m[NR], l[NR];               // maximum of scale-free scores; sum of weights
        int places[NR];                   // the weights' powers of two (see kMostPlaces)
#pragma unroll
        for (int n = 0; n < NR; ++n) {
            places[n] = BF ? 0 : kMostPlaces;
            m[n] = -__builtin_inff();
            l[n] = 0.f;
            osum[n] = float4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < NT; ++k) o[n * NT + k] = float4_t{0.f, 0.f, 0.f, 0.f};
        }

        for (uint32_t slot = 0; t < t_end; t += W, slot = (slot + 1) % RING) {
            const bool here = found[0];
            const uint32_t buf = ring + slot * (uint32_t)TB;
            asm volatile("s_waitcnt vmcnt(%0)" ::"i"((RING - 1) * LOADS) : "memory");     // this tile has landed
            {
                float4_t s[NR][2];
                u32x4 kc[kPieces<D>];
                lds_read<kPieces<D>, 1024>(kc, buf + lane * 16);
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int n = 0; n < NR; ++n) s[n][u] = float4_t{-off_q[n], -off_q[n], -off_q[n], -off_q[n]};
                constexpr int QW = NW < 4 ? NW : 4;         // words of queries at a time
#pragma unroll
                for (int w0 = 0; w0 < NW; w0 += QW) {
                    u32x4 qf[NR][QW];
#pragma unroll
                    for (int n = 0; n < NR; ++n) lds_read<QW, 1024>(qf[n], q_at + (n * NW + w0) * 1024);
#pragma unroll
                    for (int w = 0; w < QW; ++w)
#pragma unroll
                        for (int u = 0; u < 2; ++u) {
                            const u32x4 kf = code_pairs<BF>(code_word<D>(kc, u, w0 + w), mk);
#pragma unroll
                            for (int n = 0; n < NR; ++n) s[n][u] = mfma16<BF>(kf, qf[n][w], s[n][u]);
                        }
                }
                u32x4 meta[4];            // k scale, k zero, v scale, v zero
                lds_read<4, 16>(meta, buf + 32 * D + g * 64);
                // slot i of the lane: key 16 (i / 4) + 4 g + i % 4 of the tile
                const int key0 = (int)(t * kKvTile) + 4 * g;
                const bool edge = !here || (int)(t * kKvTile) + kKvTile - 1 > (int)len - a.q_len;
                uint32_t scale_bits = 0;  // fp16: of the largest |s_v| of the lane's keys
                if constexpr (!BF) {
                    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
                    u16x2 most = {0, 0};
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, meta[2][i] & 0x7FFF7FFFu));
                    scale_bits = most[0] > most[1] ? most[0] : most[1];
                }
                u32x4 p[NR], zrow = meta[3];
                if (edge) {               // no zero-points of positions that were never written
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (!here || key0 + 16 * (i / 4) + i % 4 >= (int)len)
                            zrow[i / 2] &= i & 1 ? 0xFFFFu : 0xFFFF0000u;
                }
#pragma unroll
                for (int n = 0; n < NR; ++n) {
                    float x[8], top = m[n];
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        x[i] = fmaf(-meta_f32<BF>(meta[1], i), sum_q[n], s[n][i / 4][i % 4]) *
                               meta_f32<BF>(meta[0], i);
                    uint32_t bits = scale_bits;             // ... that the row sees
                    if (edge) {
                        const int seen = (here ? limit[n] : -1) - key0;
                        bits = 0;
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            if (16 * (i / 4) + i % 4 > seen) {
                                x[i] = -__builtin_inff();
                            } else if constexpr (!BF) {
                                const uint32_t sv = meta[2][i / 2] >> 16 * (i % 2) & 0x7FFFu;
                                bits = sv > bits ? sv : bits;
                            }
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i) top = fmaxf(top, x[i]);
                    top = max_over_groups(top);
                    if (__any(top > m[n] || (!BF && (int)(bits >> 10) > kMostPlaces - places[n]))) {
                        int fewer = 0;
                        if constexpr (!BF) {                // (a NaN among the scales makes the row NaN)
                            const int room = kMostPlaces - (int)(max_over_groups(bits) >> 10);
                            fewer = room < places[n] ? places[n] - room : 0;
                            places[n] -= fewer;
                        }
                        const float f =
                            top == -__builtin_inff() ? 1.f : __builtin_amdgcn_exp2f((m[n] - top) * a.scale2 - fewer);
                        const bool sums_yet = __any(m[n] != -__builtin_inff());
                        m[n] = top;
                        if (sums_yet) {
                            l[n] *= f;
                            osum[n] *= f;
#pragma unroll
                            for (int k = 0; k < NT; ++k) o[n * NT + k] *= f;
                        }
                    }
                    const float base = m[n] == -__builtin_inff() ? 0.f : fmaf(m[n], a.scale2, -places[n]);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float e = __builtin_amdgcn_exp2f(fmaf(x[i], a.scale2, -base));
                        l[n] += e;
                        x[i] = e * meta_f32<BF>(meta[2], i);
                    }
                    if (edge) {           // a hidden value's scale may be anything
                        const int seen = (here ? limit[n] : -1) - key0;
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            if (16 * (i / 4) + i % 4 > seen) x[i] = 0.f;
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) p[n][i] = round_out2<BF>(x[2 * i], x[2 * i + 1]);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) zrow[i] = c == 0 ? zrow[i] : off_row;
                u32x4 vc[kPieces<D>];
                lds_read<kPieces<D>, 1024>(vc, buf + 16 * D + lane * 16);
                // everything of the tile is in registers: its place takes another
#pragma unroll
                for (int i = 0; i + 1 < RING; ++i) found[i] = found[i + 1];
                fetch(tile_at(t + RING * W, entry, found[RING - 1]), slot);
                if (t + (RING + 1) * W < t_end) entry = entry_of(t + (RING + 1) * W);
                else entry = -1;
#pragma unroll
                for (int n = 0; n < NR; ++n) osum[n] = mfma16<BF>(zrow, p[n], osum[n]);
#pragma unroll
                for (int w = 0; w < NW; ++w) {
                    const u32x4 a0 = code_pairs<BF>(code_word<D>(vc, 0, w), mv);
                    const u32x4 a1 = code_pairs<BF>(code_word<D>(vc, 1, w), mv);
                    const u32x4 lo{a0[0], a0[2], a1[0], a1[2]}, hi{a0[1], a0[3], a1[1], a1[3]};
#pragma unroll
                    for (int n = 0; n < NR; ++n) {
                        o[n * NT + w] = mfma16<BF>(lo, p[n], o[n * NT + w]);
                        o[n * NT + NW + w] = mfma16<BF>(hi, p[n], o[n * NT + NW + w]);
                    }
                }
            }
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // nothing lands in the ring any more

        // ---- the wave's sums: offsets and zero-points leave
#pragma unroll
        for (int n = 0; n < NR; ++n) {
            l[n] = over_groups(l[n]);
            // the three sums of column c are in lane c (group 0)
            const float z = of_group0(osum[n][0]);
            const float ca = z + of_group0(osum[n][1]), cb = z + of_group0(osum[n][2]);
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                o[n * NT + w] -= ca;
                o[n * NT + NW + w] -= cb;
            }
            m[n] = fmaf(m[n], a.scale2, -places[n]);
            if (g == 0) {
                ms[n * 16 + c][wave] = m[n];
                ls[n * 16 + c][wave] = l[n];
            }
        }
        // ---- the waves' sums under a common maximum: each wave keeps its W-th of
        // them, halving what it holds with one wave after another (32 rows of 256:
        // 3 us; some rows of all waves at a time, four times, took 7)
        lds_barrier();                    // the tiles are read; maxima and sums are there
        float tops[NR], sums[NR];
#pragma unroll
        for (int n = 0; n < NR; ++n) {
            const float *mr = ms[n * 16 + c], *lr = ls[n * 16 + c];
            float mw[W], lw[W];
#pragma unroll
            for (int w = 0; w < W; ++w) {
                mw[w] = mr[w];
                lw[w] = lr[w];
            }
            tops[n] = mw[0];
#pragma unroll
            for (int w = 1; w < W; ++w) tops[n] = fmaxf(tops[n], mw[w]);
            sums[n] = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w) sums[n] = fmaf(lw[w], weight_of(mw[w], tops[n]), sums[n]);
            const float f = weight_of(m[n], tops[n]);
#pragma unroll
            for (int k = 0; k < NT; ++k) o[n * NT + k] *= f;
        }
        // What wave w writes only the wave it exchanges with reads, which writes
        // its next half in the same place: one barrier an exchange.
        auto sums_of = [&](int w) { return reinterpret_cast<float4_t*>(pool + w * kSumBytes) + lane; };
        exchange<SUMS / 2>(o, wave & W / 2, sums_of(wave), sums_of(wave ^ W / 2));
        if constexpr (W == 8) {
            exchange<SUMS / 4>(o, wave & 2, sums_of(wave ^ 4), sums_of(wave ^ 6));
            if constexpr (SUMS >= 8) {
                exchange<SUMS / 8>(o, wave & 1, sums_of(wave ^ 6), sums_of(wave ^ 7));
            } else {                      // half of the four sums that are left
                const float4_t v = o[0];
                float2_t* mine = reinterpret_cast<float2_t*>(sums_of(wave ^ 6));
                *mine = wave & 1 ? float2_t{v[0], v[1]} : float2_t{v[2], v[3]};
                lds_barrier();
                const float2_t other = *reinterpret_cast<const float2_t*>(sums_of(wave ^ 7));
                o[0][0] = (wave & 1 ? v[2] : v[0]) + other[0];
                o[0][1] = (wave & 1 ? v[3] : v[1]) + other[1];
            }
        } else {
            exchange<SUMS / 4>(o, wave & 1, sums_of(wave ^ 2), sums_of(wave ^ 3));
        }
        // the wave's sums: KEEP groups of four (or half of one) of one row a lane
        constexpr int VALUES = 4 * SUMS / W < 4 ? 2 : 4;
        const int kept_at = wave * (4 * SUMS / W), kept_n = kept_at / (4 * NT);
        const int r = kept_n * 16 + c, d0 = kept_at % (4 * NT) / 4 * 16 + 4 * g + kept_at % 4;
        const int rows_here = q_rows - rb * ROWS < ROWS ? q_rows - rb * ROWS : ROWS;
        float* const slot = P::at(a.parts, wg, first);
        if (r < rows_here && first == final) {
            const float sum = NR == 2 && kept_n ? sums[NR - 1] : sums[0], inv = sum == 0.f ? 0.f : 1.f / sum;
            uint16_t* dst = out_row<D>(a, this_b, h, rb * ROWS + r) + d0;
#pragma unroll
            for (int i = 0; i < KEEP; ++i) {
                const float4_t v = o[i] * inv;
                if constexpr (VALUES == 4)
                    *reinterpret_cast<u32x2*>(dst + 16 * i) =
                        u32x2{round_out2<BF>(v[0], v[1]), round_out2<BF>(v[2], v[3])};
                else
                    *reinterpret_cast<uint32_t*>(dst) = round_out2<BF>(v[0], v[1]);
            }
        } else if (r < rows_here) {
            // Where the last workgroup adds the parts, they and the counters are
            // touched only by agent-scope atomic accesses, which pass the per-XCD L2,
            // and the stores complete before the arrival is counted.
            float* dst = slot + r * D + d0;
#pragma unroll
            for (int i = 0; i < KEEP; ++i) {
                if (a.counters || VALUES == 2) {
#pragma unroll
                    for (int j = 0; j < VALUES; j += 2)
                        __hip_atomic_store(reinterpret_cast<uint64_t*>(dst + 16 * i + j),
                                           __builtin_bit_cast(uint64_t, float2_t{o[i][j], o[i][j + 1]}),
                                           __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                } else {
                    *reinterpret_cast<float4_t*>(dst + 16 * i) = o[i];
                }
            }
        }
        if (!a.counters && wg == first && tid == 0)
            *reinterpret_cast<u32x2*>(a.spans + 2 * (this_b * sh.heads + item)) = u32x2{first, final};
        if (first != final && wave == 0 && g == 0) {
#pragma unroll
            for (int n = 0; n < NR; ++n)
                if (n * 16 + c < rows_here) {
                    __hip_atomic_store(slot + ROWS * D + n * 16 + c, tops[n], __ATOMIC_RELAXED,
                                       __HIP_MEMORY_SCOPE_AGENT);
                    __hip_atomic_store(slot + ROWS * (D + 1) + n * 16 + c, sums[n], __ATOMIC_RELAXED,
                                       __HIP_MEMORY_SCOPE_AGENT);
                }
        }
        if (first != final && a.counters) {
            __builtin_amdgcn_s_waitcnt(0);          // this thread's stores have completed
            __syncthreads();
            if (tid == 0)
                last = __hip_atomic_fetch_add(&a.counters[first], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) ==
                       final - first;
            __syncthreads();
            if (last) {
                auto load1 = [](const float* p) {
                    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                };
                auto load2 = [](const float* p) {
                    return __builtin_bit_cast(float2_t, __hip_atomic_load(reinterpret_cast<const uint64_t*>(p),
                                                                          __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
                };
                auto join = [&](auto ahead, auto u_) {
                    constexpr int U = decltype(u_)::value;
                    const int pairs = rows_here * D / 2;
                    for (int i0 = tid; i0 < pairs; i0 += U * THREADS) {
                        int jr[U], jd[U];
                        float2_t v[U];
#pragma unroll
                        for (int u = 0; u < U; ++u) {
                            const int i = i0 + u * THREADS < pairs ? i0 + u * THREADS : i0;
                            jr[u] = i / (D / 2);
                            jd[u] = i % (D / 2) * 2;
                        }
                        join_parts<D, ROWS, decltype(ahead)::value>(a.parts, first, final, jr, jd, v, load2, load1);
#pragma unroll
                        for (int u = 0; u < U; ++u)
                            *reinterpret_cast<uint32_t*>(out_row<D>(a, this_b, h, rb * ROWS + jr[u]) + jd[u]) =
                                round_out2<BF>(v[u][0], v[u][1]);
                    }
                };
                if constexpr (NR == 2)
                    join(std::integral_constant<int, 4>{}, std::integral_constant<int, 4>{});
                else if (rows_here * D / 2 > THREADS)
                    join(std::integral_constant<int, 4>{}, std::integral_constant<int, 2>{});
                else
                    join(std::integral_constant<int, 8>{}, std::integral_constant<int, 1>{});
                if (tid == 0)
                    __hip_atomic_store(&a.counters[first], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
        }
        lds_barrier();                    // the sums in LDS and `last` are read before the next item's
    }
}

// The parts of items that several workgroups share, added by a launch of its
// own: workgroup (i, y) takes 128 sums, from 128 y on, of item i, its 16
// groups of 32 threads every sixteenth part each.  Latency-bound: 2 items of 128
// parts, 32 rows of 256 (8.4 MB), 4.7 us.
template <bool BF, int D, int NR>
__global__ __launch_bounds__(kJoinThreads) void kv4_join_kernel(AttnArgs a) {
    constexpr int ROWS = 16 * NR, AHEAD = 4, SLICES = kJoinThreads / 32;
    using P = Parts<D, ROWS>;
    __shared__ float4_t vals[SLICES][32];
    __shared__ float m8[SLICES][32], l8[SLICES][32];
    const uint32_t first = a.spans[2 * blockIdx.x], final = a.spans[2 * blockIdx.x + 1];
    if (first == final) return;
    const int tid = threadIdx.x, slice = tid >> 5;
    const int b = (int)a.by_heads.of(blockIdx.x);
    const uint32_t item = blockIdx.x - b * a.by_heads.d;
    const int h = (int)a.by_row_blocks.of(item), rb = (int)item - h * a.row_blocks;
    const int q_rows = a.q_len * a.group;
    const int i = blockIdx.y * 128 + 4 * (tid & 31), r = i / D, d = i % D;
    if (blockIdx.y * 128 / D >= q_rows - rb * ROWS) return;   // the group of 128 lies in one row but for D = 64
    float top = -__builtin_inff(), sum = 0.f;
    float4_t v = {0.f, 0.f, 0.f, 0.f};
    for (uint32_t w0 = first + slice; w0 <= final; w0 += SLICES * AHEAD) {
        float mw[AHEAD], lw[AHEAD];
        float4_t vw[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const uint32_t w = w0 + SLICES * k <= final ? w0 + SLICES * k : w0;
            const float* p = P::at(a.parts, w, first);
            mw[k] = w0 + SLICES * k <= final ? p[ROWS * D + r] : -__builtin_inff();
            lw[k] = p[ROWS * (D + 1) + r];
            vw[k] = *reinterpret_cast<const float4_t*>(p + r * D + d);
        }
        float next = top;
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) next = fmaxf(next, mw[k]);
        const float f = weight_of(top, next);
        top = next;
        sum *= f;
        v *= f;
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const float e = weight_of(mw[k], top);
            sum = fmaf(lw[k], e, sum);
            v += vw[k] * e;
        }
    }
    m8[slice][tid & 31] = top;
    l8[slice][tid & 31] = sum;
    vals[slice][tid & 31] = v;
    __syncthreads();
    if (slice != 0) return;
    float all = -__builtin_inff();
#pragma unroll
    for (int k = 0; k < SLICES; ++k) all = fmaxf(all, m8[k][tid]);
    sum = 0.f;
    v = float4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < SLICES; ++k) {
        const float e = weight_of(m8[k][tid], all);
        sum = fmaf(l8[k][tid], e, sum);
        v += vals[k][tid] * e;
    }
    if (rb * ROWS + r >= q_rows) return;
    v *= sum == 0.f ? 0.f : 1.f / sum;
    *reinterpret_cast<u32x2*>(out_row<D>(a, b, h, rb * ROWS + r) + d) =
        u32x2{round_out2<BF>(v[0], v[1]), round_out2<BF>(v[2], v[3])};
}

// Rows per workgroup (16 or 32) and the blocks of them that q_rows need.
int row_tiles(int q_rows) { return q_rows <= 16 ? 1 : 2; }
// Workgroups of `waves` waves that a compute unit holds on its four SIMDs.
int wgs_per_cu(int D, int nr, int waves) { return waves_per_simd(D, nr) * 4 / waves; }
// Workgroups of a launch, at most: what 256 compute units hold, four waves each.
int most_wgs(int D, int nr) { return kMostWgs / 4 * waves_per_simd(D, nr); }
// Waves of a workgroup: eight, whose sums meet in LDS, where items are few; four
// where there are two items and more a compute unit, so that more items are on
// their way at once.  Measured (8 heads of 128, up to 300 keys, us, 8 -> 4 waves):
// 32 sequences 12.0 -> 13.9, 64 16.9 -> 15.1, 128 23.6 -> 18.6; 32 heads, 128
// sequences of up to 2000: 118 -> 90.
// 32 rows of 256 keep eight: their queries and rings let a compute unit hold one
// workgroup, of either size.
constexpr bool four_waves_fit(int D, int nr) { return D < 256 || nr == 1; }
int waves_for(int64_t items, int cus, int D, int nr) { return items >= 2 * cus && four_waves_fit(D, nr) ? 4 : 8; }

}  // namespace

int64_t kv4_attention_workspace_bytes(int64_t batch, int q_len, int q_heads, int kv_heads, int D) {
    (void)batch;
    const int nr = row_tiles(q_len * (q_heads / kv_heads));
    return align256(kMostWgs * 12) + align256((int64_t)most_wgs(D, nr) * 2 * 16 * nr * (D + 2) * 4);
}

int launch_kv4_attention(const tf_kv4_cache& c, const void* q, int64_t q_stride, const int32_t* lens, int64_t batch,
                         int q_len, int q_heads, float scale, void* out, void* ws, hipStream_t s) {
    const int group = q_heads / c.kv_heads, q_rows = q_len * group, nr = row_tiles(q_rows);
    AttnArgs a{};
    a.cache = kv4_view(c);
    a.q = static_cast<const uint16_t*>(q);
    a.q_stride = q_stride;
    a.lens = lens;
    a.batch = (int)batch;
    a.q_len = q_len;
    a.group = group;
    a.row_blocks = (q_rows + 16 * nr - 1) / (16 * nr);
    a.capacity = (int32_t)(c.max_pages * c.page_size);
    a.by_batch = Divisor((uint32_t)batch);
    a.by_group = Divisor((uint32_t)group);
    a.by_row_blocks = Divisor((uint32_t)a.row_blocks);
    a.by_heads = Divisor((uint32_t)(c.kv_heads * a.row_blocks));
    a.by_tiles = Divisor((uint32_t)(c.page_size / kKvTile));
    a.scale2 = scale * 1.4426950408889634f;
    a.out = static_cast<uint16_t*>(out);
    a.counters = static_cast<uint32_t*>(ws);
    a.spans = a.counters + kMostWgs;
    a.parts = reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + align256(kMostWgs * 12));
    // no more workgroups than rounds there can be
    const int cus = device_cus(s);
    const int64_t items = batch * c.kv_heads * a.row_blocks;
    const int waves = waves_for(items, cus, c.head_dim, nr);
    const int64_t item_rounds = ((int64_t)a.capacity + kKvTile * waves - 1) / (kKvTile * waves);
    int64_t wgs = (int64_t)cus * wgs_per_cu(c.head_dim, nr, waves);
    if (wgs > most_wgs(c.head_dim, nr)) wgs = most_wgs(c.head_dim, nr);
    if (wgs > items * item_rounds) wgs = items * item_rounds;
    a.wgs = (uint32_t)wgs;
    // Parts of one item, at most: as many as one long sequence among empty ones
    // makes.  Many large ones are added by a launch of its own, many workgroups
    // to an item.
    const int64_t most = wgs / (c.kv_heads * a.row_blocks) < item_rounds ? wgs / (c.kv_heads * a.row_blocks) : item_rounds;
    const int64_t part_rows = q_rows < 16 * nr ? q_rows : 16 * nr;
    const bool join = most * part_rows * c.head_dim * 4 > 256 * 1024 && items <= wgs;
    if (join) a.counters = nullptr;
    const dim3 grid((unsigned)wgs), join_grid((unsigned)items, (unsigned)((part_rows * c.head_dim + 127) / 128));
    auto go_waves = [&](auto d, auto n, auto bf, auto w) {
        constexpr int D = decltype(d)::value, NR = decltype(n)::value, W = decltype(w)::value;
        constexpr bool BF = decltype(bf)::value;
        const int rc = launch(kv4_attn_kernel<BF, D, NR, W>, grid, dim3(64 * W), 0, s, a);
        if (rc || !join) return rc;
        return launch(kv4_join_kernel<BF, D, NR>, join_grid, dim3(kJoinThreads), 0, s, a);
    };
    auto go = [&](auto d, auto n, auto bf) {
        if constexpr (four_waves_fit(decltype(d)::value, decltype(n)::value))
            if (waves == 4) return go_waves(d, n, bf, std::integral_constant<int, 4>{});
        return go_waves(d, n, bf, std::integral_constant<int, 8>{});
    };
    auto by_rows = [&](auto d, auto bf) {
        return nr == 1 ? go(d, std::integral_constant<int, 1>{}, bf) : go(d, std::integral_constant<int, 2>{}, bf);
    };
    auto by_type = [&](auto d) {
        return c.dtype == TF_BF16 ? by_rows(d, std::true_type{}) : by_rows(d, std::false_type{});
    };
    if (c.head_dim == 64) return by_type(std::integral_constant<int, 64>{});
    if (c.head_dim == 128) return by_type(std::integral_constant<int, 128>{});
    return by_type(std::integral_constant<int, 256>{});
}

}  // namespace tf
