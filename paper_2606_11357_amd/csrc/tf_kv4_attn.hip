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
// HBM-bound: D + 8 bytes of cache a token and head, of which each is read once.
#include "tf_kv4.h"

namespace tf {

Kv4 kv4_view(const tf_kv4_cache& c);

namespace {

constexpr int kRoundKeys = 128;          // keys of one round: a tile of 32 for each of 4 waves
constexpr int kWgPerCu = 4;

struct AttnArgs {
    Kv4 cache;
    const uint16_t* q;
    int64_t q_stride;
    const int32_t* lens;
    int batch, q_len, group, row_blocks;  // group: query heads per key/value head
    int64_t capacity;                     // positions a table row can hold
    float scale2;                         // softmax scale * log2(e)
    uint16_t* out;
    uint32_t* counters;
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
        o[1] = (w >> 4 & 0x000F000Fu) | m.b;
        o[2] = (w >> 8 & 0x000F000Fu) | m.a;
        o[3] = (w >> 12 & 0x000F000Fu) | m.b;
    } else {
        const uint32_t w8 = w >> 8;
        o[0] = (w & 0x000F000Fu) | m.a;
        o[1] = (w & 0x00F000F0u) | m.b;
        o[2] = (w8 & 0x000F000Fu) | m.a;
        o[3] = (w8 & 0x00F000F0u) | m.b;
    }
    return o;
}

__device__ __forceinline__ float over_groups(float v) {       // sum over the four 16-lane groups
    v += __shfl_xor(v, 16);
    return v + __shfl_xor(v, 32);
}

template <int D>
struct TileRegs {
    static constexpr int P = D == 64 ? 1 : D / 64;    // 16-byte pieces of a lane
    u32x4 k[P], v[P], meta[4];                        // meta: k scale, k zero, v scale, v zero
    __device__ __forceinline__ void load(const uint8_t* tile, int lane) {
#pragma unroll
        for (int p = 0; p < P; ++p) k[p] = *reinterpret_cast<const u32x4*>(tile + p * 1024 + lane * 16);
#pragma unroll
        for (int p = 0; p < P; ++p) v[p] = *reinterpret_cast<const u32x4*>(tile + 16 * D + p * 1024 + lane * 16);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            meta[i] = *reinterpret_cast<const u32x4*>(tile + 32 * D + (lane >> 4) * 64 + i * 16);
    }
    // word w of key half u, as kv4_word places it
    static __device__ __forceinline__ uint32_t word(const u32x4* x, int u, int w) {
        if constexpr (D == 64) return x[0][2 * u + w];
        else return x[u * (D / 128) + w / 4][w % 4];
    }
};

// Value i (0..7) of eight packed 16-bit floats.
template <bool BF>
__device__ __forceinline__ float meta_f32(const u32x4& m, int i) {
    const uint32_t w = m[i / 2];
    if constexpr (BF) return __builtin_bit_cast(float, i & 1 ? w & 0xFFFF0000u : w << 16);
    else return scale_f32<false>(i & 1 ? w >> 16 : w & 0xFFFFu);
}

// One workgroup of four waves takes a contiguous share of all rounds of all
// items, an item being one (sequence, key/value head, block of 16 NR query
// rows) and a round 128 keys of it, a tile for each wave.  Shares differ by at
// most one round whatever the lengths are.  Items that lie inside one share are
// written directly; the others' partial sums go through the workspace, and the
// workgroup that arrives last adds them in order.
template <bool BF, int D, int NR>
__global__ __launch_bounds__(256) void kv4_attn_kernel(AttnArgs a) {
    constexpr int NT = D / 16;            // 16-dim tiles of the output
    constexpr int NW = D / 32;            // words of codes per lane and key half
    constexpr int ROWS = 16 * NR;
    constexpr int PITCH = D + 4;
    constexpr int64_t TB = kv4_tile_bytes(D);
    constexpr int64_t SLOT = (int64_t)ROWS * (D + 2);
    __shared__ uint32_t wave_total[4];
    __shared__ uint32_t before[257];      // rounds of one head before each thread's sequences
    __shared__ float ms[4][ROWS], ls[2][ROWS];
    __shared__ float acc[2][ROWS * PITCH];
    __shared__ int last;

    const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

    // ---- this workgroup's share
    const int seg = (a.batch + 255) / 256;
    auto length_of = [&](int b) {
        const int64_t n = a.lens[b];
        return (uint32_t)(n < 0 ? 0 : n > a.capacity ? a.capacity : n);
    };
    auto rounds_of = [&](uint32_t n) { return n == 0 ? 1u : (n + kRoundKeys - 1) / kRoundKeys; };
    {
        uint32_t mine = 0;
        for (int b = tid * seg; b < (tid + 1) * seg && b < a.batch; ++b) mine += rounds_of(length_of(b));
        uint32_t sum = mine;
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
    const uint32_t heads = (uint32_t)a.cache.kv_heads * a.row_blocks;
    const uint32_t total = before[256] * heads;
    const uint32_t share = total / gridDim.x, extra = total % gridDim.x;
    const uint32_t wg = blockIdx.x;
    uint32_t at = wg * share + (wg < extra ? wg : extra);
    const uint32_t end = at + share + (wg < extra ? 1 : 0);
    if (at >= end) return;
    auto owner_wg = [&](uint32_t x) {
        const uint32_t big = extra * (share + 1);
        return x < big ? x / (share + 1) : extra + (x - big) / share;
    };
    int b;
    uint32_t seq_start;                   // rounds (of all heads) before sequence b
    {
        const uint32_t x = at / heads;
        int s0 = 0, s1 = 256;
        while (s1 - s0 > 1) {
            const int mid = (s0 + s1) >> 1;
            if (before[mid] <= x) s0 = mid;
            else s1 = mid;
        }
        b = s0 * seg;
        uint32_t done = before[s0];
        for (;; ++b) {
            const uint32_t n = rounds_of(length_of(b));
            if (x < done + n) break;
            done += n;
        }
        seq_start = done * heads;
        b = __builtin_amdgcn_readfirstlane(b);
        seq_start = __builtin_amdgcn_readfirstlane(seq_start);
    }

    const Magic mk = magics<BF>(0), mv = magics<BF>(0x80000000u);
    const int q_rows = a.q_len * a.group;

    while (at < end) {
        // ---- the item at `at`
        const uint32_t len = __builtin_amdgcn_readfirstlane(length_of(b));
        const uint32_t n_rounds = rounds_of(len);
        const uint32_t item = (at - seq_start) / n_rounds;
        const uint32_t item_start = seq_start + item * n_rounds;
        const int h = (int)(item / a.row_blocks), rb = (int)(item % a.row_blocks);
        const uint32_t r0 = at - item_start;
        const uint32_t r1 = end - item_start < n_rounds ? end - item_start : n_rounds;

        u32x4 q[NR][NW];
        float sum_q[NR], off_q[NR];
        int limit[NR];                    // last visible position of the lane's row
#pragma unroll
        for (int n = 0; n < NR; ++n) {
            const int row = rb * ROWS + n * 16 + c;
            const bool real = row < q_rows;
            const int tq = real ? row / a.group : 0, hq = h * a.group + (real ? row - tq * a.group : 0);
            const uint16_t* src = a.q + ((int64_t)b * a.q_len + tq) * a.q_stride + (int64_t)hq * D + g * (D / 4);
            limit[n] = (int)len - a.q_len + tq;
            float sa = 0.f, sb = 0.f;
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                u32x4 v = *reinterpret_cast<const u32x4*>(src + 8 * w);
                if (!real) v = u32x4{0, 0, 0, 0};
                q[n][w] = v;
                sa += meta_f32<BF>(v, 0) + meta_f32<BF>(v, 1) + meta_f32<BF>(v, 4) + meta_f32<BF>(v, 5);
                sb += meta_f32<BF>(v, 2) + meta_f32<BF>(v, 3) + meta_f32<BF>(v, 6) + meta_f32<BF>(v, 7);
            }
            sa = over_groups(sa);
            sb = over_groups(sb);
            sum_q[n] = sa + sb;
            off_q[n] = sa * kOffA<BF> + sb * kOffB<BF>;
        }
        float4_t o[NR][NT];
        float m[NR], l[NR], pe[NR], po[NR], pz[NR];   // max; sums of P, P' over even and odd keys, P' z
#pragma unroll
        for (int n = 0; n < NR; ++n) {
            m[n] = -__builtin_inff();
            l[n] = pe[n] = po[n] = pz[n] = 0.f;
#pragma unroll
            for (int t = 0; t < NT; ++t) o[n][t] = float4_t{0.f, 0.f, 0.f, 0.f};
        }

        // ---- the wave's tiles: 4 r + wave for r0 <= r < r1, those that begin before len
        const uint32_t tiles = (len + kKvTile - 1) / kKvTile;
        auto tile_at = [&](uint32_t t) { return kv4_tile(a.cache, b, t * kKvTile, h, TB); };
        uint32_t t = 4 * r0 + wave;
        const uint32_t t_end = 4 * r1 < tiles ? 4 * r1 : tiles;
        TileRegs<D> cur, nxt;
        const uint8_t* cur_p = t < t_end ? tile_at(t) : nullptr;
        if (cur_p) cur.load(cur_p, lane);
        for (; t < t_end; t += 4) {
            const uint8_t* nxt_p = t + 4 < t_end ? tile_at(t + 4) : nullptr;
            if (nxt_p) nxt.load(nxt_p, lane);
            if (cur_p) {
                float4_t s[NR][2];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
#pragma unroll
                    for (int n = 0; n < NR; ++n) s[n][u] = float4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int w = 0; w < NW; ++w) {
                        const u32x4 kc = code_pairs<BF>(TileRegs<D>::word(cur.k, u, w), mk);
#pragma unroll
                        for (int n = 0; n < NR; ++n) s[n][u] = mfma16<BF>(kc, q[n][w], s[n][u]);
                    }
                }
                // slot i of the lane: key 16 (i / 4) + 4 g + i % 4 of the tile
                float sk[8], zk[8], sv[8], zv[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    sk[i] = meta_f32<BF>(cur.meta[0], i) * a.scale2;
                    zk[i] = meta_f32<BF>(cur.meta[1], i);
                    sv[i] = meta_f32<BF>(cur.meta[2], i);
                    zv[i] = meta_f32<BF>(cur.meta[3], i);
                }
                const int key0 = (int)(t * kKvTile) + 4 * g;
                const bool masked = (int)(t * kKvTile) + kKvTile - 1 > (int)len - a.q_len;
                u32x4 p[NR];
#pragma unroll
                for (int n = 0; n < NR; ++n) {
                    float x[8];
                    float top = -__builtin_inff();
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        x[i] = fmaf(-zk[i], sum_q[n], s[n][i / 4][i % 4] - off_q[n]) * sk[i];
                        if (masked && key0 + 16 * (i / 4) + i % 4 > limit[n]) x[i] = -__builtin_inff();
                        top = fmaxf(top, x[i]);
                    }
                    top = fmaxf(top, __shfl_xor(top, 16));
                    top = fmaxf(top, __shfl_xor(top, 32));
                    if (__any(top > m[n])) {
                        const float next = fmaxf(m[n], top);
                        const float f = next == -__builtin_inff() ? 1.f : __builtin_amdgcn_exp2f(m[n] - next);
                        m[n] = next;
                        l[n] *= f;
                        pe[n] *= f;
                        po[n] *= f;
                        pz[n] *= f;
#pragma unroll
                        for (int k = 0; k < NT; ++k) o[n][k] *= f;
                    }
                    const float base = m[n] == -__builtin_inff() ? 0.f : m[n];
#pragma unroll
                    for (int i = 0; i < 8; i += 2) {
                        float w2[2], z2[2];
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            const float e = __builtin_amdgcn_exp2f(x[i + j] - base);
                            l[n] += e;
                            const bool hidden = masked && key0 + 16 * (i / 4) + (i + j) % 4 > limit[n];
                            w2[j] = hidden ? 0.f : e * sv[i + j];
                            z2[j] = hidden ? 0.f : zv[i + j];
                        }
                        const uint32_t pr = round_out2<BF>(w2[0], w2[1]);
                        p[n][i / 2] = pr;
                        // the sums use P' as the matrix cores see it
                        const float ra = scale_f32<BF>(pr & 0xFFFFu), rc = scale_f32<BF>(pr >> 16);
                        pe[n] += ra;
                        po[n] += rc;
                        pz[n] = fmaf(ra, z2[0], fmaf(rc, z2[1], pz[n]));
                    }
                }
#pragma unroll
                for (int w = 0; w < NW; ++w) {
                    const u32x4 a0 = code_pairs<BF>(TileRegs<D>::word(cur.v, 0, w), mv);
                    const u32x4 a1 = code_pairs<BF>(TileRegs<D>::word(cur.v, 1, w), mv);
                    const u32x4 lo{a0[0], a0[2], a1[0], a1[2]}, hi{a0[1], a0[3], a1[1], a1[3]};
#pragma unroll
                    for (int n = 0; n < NR; ++n) {
                        o[n][w] = mfma16<BF>(lo, p[n], o[n][w]);
                        o[n][NW + w] = mfma16<BF>(hi, p[n], o[n][NW + w]);
                    }
                }
            }
            cur = nxt;
            cur_p = nxt_p;
        }

        // ---- the wave's sums: offsets and zero-points leave
#pragma unroll
        for (int n = 0; n < NR; ++n) {
            l[n] = over_groups(l[n]);
            pe[n] = over_groups(pe[n]);
            po[n] = over_groups(po[n]);
            pz[n] = over_groups(pz[n]);
            const float ca = kOffA<BF> * pe[n] - (kOffA<BF> + 15.f) * po[n] + pz[n];
            const float cb = kOffB<BF> * pe[n] - (kOffB<BF> + 15.f) * po[n] + pz[n];
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                o[n][w] -= ca;
                o[n][NW + w] -= cb;
            }
            if (g == 0) ms[wave][n * 16 + c] = m[n];
        }
        __syncthreads();
        // ---- the four waves' sums under a common maximum, added in a tree
#pragma unroll
        for (int n = 0; n < NR; ++n) {
            const int r = n * 16 + c;
            const float all = fmaxf(fmaxf(ms[0][r], ms[1][r]), fmaxf(ms[2][r], ms[3][r]));
            const float f = m[n] == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(m[n] - all);
            m[n] = all;
            l[n] *= f;
#pragma unroll
            for (int k = 0; k < NT; ++k) o[n][k] *= f;
        }
#pragma unroll
        for (int step = 2; step >= 1; --step) {
            if (wave >= step && wave < 2 * step) {
#pragma unroll
                for (int n = 0; n < NR; ++n) {
                    float* dst = acc[wave - step] + (n * 16 + c) * PITCH + 4 * g;
#pragma unroll
                    for (int k = 0; k < NT; ++k) *reinterpret_cast<float4_t*>(dst + 16 * k) = o[n][k];
                    if (g == 0) ls[wave - step][n * 16 + c] = l[n];
                }
            }
            __syncthreads();
            if (wave < step) {
#pragma unroll
                for (int n = 0; n < NR; ++n) {
                    const float* src = acc[wave] + (n * 16 + c) * PITCH + 4 * g;
#pragma unroll
                    for (int k = 0; k < NT; ++k) o[n][k] += *reinterpret_cast<const float4_t*>(src + 16 * k);
                    l[n] += ls[wave][n * 16 + c];
                }
            }
            __syncthreads();
        }

        auto out_row = [&](int row) {
            const int tq = row / a.group;
            return a.out + ((int64_t)b * a.q_len + tq) * ((int64_t)a.cache.kv_heads * a.group * D) +
                   (int64_t)(h * a.group + row - tq * a.group) * D;
        };
        const int rows_here = q_rows - rb * ROWS < ROWS ? q_rows - rb * ROWS : ROWS;
        const uint32_t first = owner_wg(item_start), final_wg = owner_wg(item_start + n_rounds - 1);
        if (first == final_wg) {
            if (wave == 0) {
#pragma unroll
                for (int n = 0; n < NR; ++n) {
                    if (n * 16 + c >= rows_here) continue;
                    uint16_t* dst = out_row(rb * ROWS + n * 16 + c) + 4 * g;
                    const float inv = l[n] == 0.f ? 0.f : 1.f / l[n];
#pragma unroll
                    for (int k = 0; k < NT; ++k) {
                        const float4_t v = o[n][k] * inv;
                        *reinterpret_cast<u32x2*>(dst + 16 * k) =
                            u32x2{round_out2<BF>(v[0], v[1]), round_out2<BF>(v[2], v[3])};
                    }
                }
            }
        } else {
            // Partial sums and counters are touched only by agent-scope atomic
            // accesses, which pass the per-XCD L2; the stores complete before
            // the arrival is counted.
            if (wave == 0) {
                float* slot = a.parts + ((int64_t)wg * 2 + (wg == first ? 1 : 0)) * SLOT;
#pragma unroll
                for (int n = 0; n < NR; ++n) {
                    const int r = n * 16 + c;
                    if (r >= rows_here) continue;
                    float* dst = slot + r * D + 4 * g;
#pragma unroll
                    for (int k = 0; k < NT; ++k)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            __hip_atomic_store(dst + 16 * k + i, o[n][k][i], __ATOMIC_RELAXED,
                                               __HIP_MEMORY_SCOPE_AGENT);
                    if (g == 0) {
                        __hip_atomic_store(slot + ROWS * D + r, m[n], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                        __hip_atomic_store(slot + ROWS * (D + 1) + r, l[n], __ATOMIC_RELAXED,
                                           __HIP_MEMORY_SCOPE_AGENT);
                    }
                }
                __builtin_amdgcn_s_waitcnt(0);
                if (lane == 0)
                    last = __hip_atomic_fetch_add(&a.counters[first], 1u, __ATOMIC_RELAXED,
                                                  __HIP_MEMORY_SCOPE_AGENT) == final_wg - first;
            }
            __syncthreads();
            if (last) {
                auto part = [&](uint32_t w) {
                    return a.parts + ((int64_t)w * 2 + (w == first ? 1 : 0)) * SLOT;
                };
                auto load = [](const float* p) {
                    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                };
                for (int i = tid; i < rows_here * D; i += 256) {
                    const int r = i / D, d = i % D;
                    float top = -__builtin_inff();
                    for (uint32_t w = first; w <= final_wg; ++w) top = fmaxf(top, load(part(w) + ROWS * D + r));
                    float sum = 0.f, v = 0.f;
                    for (uint32_t w = first; w <= final_wg; ++w) {
                        const float* p = part(w);
                        const float mw = load(p + ROWS * D + r);
                        const float f = mw == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(mw - top);
                        sum = fmaf(load(p + ROWS * (D + 1) + r), f, sum);
                        v = fmaf(load(p + r * D + d), f, v);
                    }
                    out_row(rb * ROWS + r)[d] = round_out<BF>(sum == 0.f ? 0.f : v / sum);
                }
                if (tid == 0)
                    __hip_atomic_store(&a.counters[first], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
            __syncthreads();              // `last` is read before the next item sets it
        }

        at = item_start + r1;
        if (item + 1 == heads && r1 == n_rounds) {
            seq_start += heads * n_rounds;
            ++b;
        }
    }
}

// Rows per workgroup (16 or 32) and the blocks of them that q_rows need.
int row_tiles(int q_rows) { return q_rows <= 16 ? 1 : 2; }

// Most workgroups of a launch: the workspace is sized for them.
constexpr int kMostCus = 304;
int64_t most_wgs(int64_t items) {
    (void)items;
    return (int64_t)kMostCus * kWgPerCu;
}

}  // namespace

int64_t kv4_attention_workspace_bytes(int64_t batch, int q_len, int q_heads, int kv_heads, int D) {
    const int rows = 16 * row_tiles(q_len * (q_heads / kv_heads));
    const int64_t w = most_wgs(batch * kv_heads);
    return align256(w * 4) + align256(w * 2 * rows * (D + 2) * 4);
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
    a.capacity = c.max_pages * c.page_size;
    a.scale2 = scale * 1.4426950408889634f;
    a.out = static_cast<uint16_t*>(out);
    const int64_t most = most_wgs(batch * c.kv_heads);
    a.counters = static_cast<uint32_t*>(ws);
    a.parts = reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + align256(most * 4));
    // no more workgroups than rounds there can be
    const int64_t rounds = batch * c.kv_heads * a.row_blocks * ((a.capacity + kRoundKeys - 1) / kRoundKeys);
    int64_t wgs = (int64_t)device_cus(s) * kWgPerCu;
    if (wgs > most) wgs = most;
    if (wgs > rounds) wgs = rounds;
    const dim3 grid((unsigned)wgs);
    auto go = [&](auto d) {
        constexpr int D = decltype(d)::value;
        if (c.dtype == TF_BF16)
            return nr == 1 ? launch(kv4_attn_kernel<true, D, 1>, grid, dim3(256), 0, s, a)
                           : launch(kv4_attn_kernel<true, D, 2>, grid, dim3(256), 0, s, a);
        return nr == 1 ? launch(kv4_attn_kernel<false, D, 1>, grid, dim3(256), 0, s, a)
                       : launch(kv4_attn_kernel<false, D, 2>, grid, dim3(256), 0, s, a);
    };
    if (c.head_dim == 64) return go(std::integral_constant<int, 64>{});
    if (c.head_dim == 128) return go(std::integral_constant<int, 128>{});
    return go(std::integral_constant<int, 256>{});
}

}  // namespace tf
