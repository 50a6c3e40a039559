// Choice of experts, the order in which their products take the tokens, and the
// weighted sum of their outputs.
#include "tf_internal.h"
#include "tf_route.h"

namespace tf {
namespace {

typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ double wave_max(double v) {
#pragma unroll
    for (int d = 32; d; d >>= 1) v = fmax(v, __shfl_xor(v, d));
    return v;
}
__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

// Token t's logits of experts lane + 64 i (past the last: that one's again), all loads
// on their way at once.
template <int V>
__device__ __forceinline__ void load_logits(const RouteArgs& a, int64_t t, int lane, double (&x)[V]) {
    if (a.dtype == TF_F32) {
        const float* p = static_cast<const float*>(a.logits) + t * a.stride;
        float v[V];
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = p[min(lane + 64 * i, a.E - 1)];
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = (double)v[i];
        return;
    }
    const uint16_t* p = static_cast<const uint16_t*>(a.logits) + t * a.stride;
    uint16_t v[V];
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = p[min(lane + 64 * i, a.E - 1)];
#pragma unroll
    for (int i = 0; i < V; ++i)
        x[i] = (double)(a.dtype == TF_BF16 ? scale_f32<true>(v[i]) : scale_f32<false>(v[i]));
}

// The two largest of a set of values, the absent ones -infinity.
struct Two { double a, b; };
__device__ __forceinline__ Two with(Two t, double v) {
    return v > t.a ? Two{v, t.a} : Two{t.a, fmax(t.b, v)};
}

// An order of doubles as unsigned numbers (no NaN; all above 0, which is for closed).
__device__ __forceinline__ uint64_t key_of(double v) {
    const uint64_t b = __builtin_bit_cast(uint64_t, v + 0.0);            // (-0 as 0)
    return b >> 63 ? ~b : b | 0x8000000000000000ull;
}

// The largest of v over the wave, in every lane's scalar copy: neighbours' values by
// row shifts and broadcasts, the last lane has them all.
__device__ __forceinline__ uint32_t wave_top(uint32_t v) {
#define TF_STEP(ctrl, rows) \
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, ctrl, rows, 0xF, false))
    TF_STEP(0x111, 0xF);
    TF_STEP(0x112, 0xF);
    TF_STEP(0x114, 0xF);
    TF_STEP(0x118, 0xF);
    TF_STEP(0x142, 0xA);
    TF_STEP(0x143, 0xC);
#undef TF_STEP
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}

__device__ __forceinline__ double from_lane(double v, int lane) {
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)b, lane);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), lane);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// One wave a token, V experts a lane: expert lane + 64 i.  Scores and choices are
// fp64: what is compared here decides which weights are read, and rounded to 32
// bits unequal scores would tie.  The vector unit bounds it: an exponential and a
// quotient an expert in fp64, then for each of the top k a search over the lanes, by
// the upper halves of the choices alone unless these tie (by 64-bit shuffles twice as
// long).  8192 tokens, 8 of 256 experts in 4 of 8 groups: 18.7 us; 64 tokens, 2 of 8: 3.6.
template <int V>
__global__ __launch_bounds__(256) void route_kernel(RouteArgs a) {
    extern __shared__ double grouped[];              // [4][E] where experts are grouped
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t t = (int64_t)blockIdx.x * 4 + wave;
    if (t >= a.T) return;                            // (whole waves; no barrier follows)
    double x[V], score[V];
    double top = -INFINITY;
    load_logits<V>(a, t, lane, x);
    float bias[V];
#pragma unroll
    for (int i = 0; i < V; ++i) bias[i] = a.bias ? a.bias[min(lane + 64 * i, a.E - 1)] : 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        if (lane + 64 * i >= a.E || x[i] != x[i]) x[i] = -INFINITY;      // NaN: masked
        top = fmax(top, x[i]);
    }
    if (a.sigmoid) {
#pragma unroll
        for (int i = 0; i < V; ++i) score[i] = 1.0 / (1.0 + exp(-x[i]));
    } else {
        top = wave_max(top);
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < V; ++i) {                // exp(x - top), equal ones (infinite ones too) 1
            score[i] = x[i] == -INFINITY ? 0.0 : x[i] == top ? 1.0 : exp(x[i] - top);
            sum += score[i];
        }
        sum = wave_sum(sum);
        const double part = sum > 0.0 ? 1.0 / sum : 0.0;
#pragma unroll
        for (int i = 0; i < V; ++i) score[i] *= part;
    }
    double choice[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const double c = score[i] + (double)bias[i];
        choice[i] = x[i] == -INFINITY || c != c ? -INFINITY : c;
    }
    uint64_t key[V];                                 // 0: not to be chosen, or chosen already
#pragma unroll
    for (int i = 0; i < V; ++i) key[i] = lane + 64 * i < a.E ? key_of(choice[i]) : 0;
    if (a.top_groups < a.groups) {
        const int gs = a.E / a.groups;
        const float per_gs = 1.0f / (float)gs;
        double* mine = grouped + wave * a.E;
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (lane + 64 * i < a.E) mine[lane + 64 * i] = choice[i];
        __builtin_amdgcn_wave_barrier();
        // `per` lanes a group: each the two largest of its part, then of their parts
        const int per = a.lanes_per_group, gr = lane / per, sub = lane % per;
        Two two{-INFINITY, -INFINITY};
        if (gr < a.groups)
            for (int i = sub; i < gs; i += per) two = with(two, mine[gr * gs + i]);
        for (int d = 1; d < per; d <<= 1) {
            const Two o{__shfl_xor(two.a, d), __shfl_xor(two.b, d)};
            two = with(with(two, o.a), o.b);
        }
        double value = two.a;
        if (a.group_top2 && two.b != -INFINITY) value += two.b;
        int rank = 0;                                // groups before this one
        for (int o = 0; o < a.groups; ++o) {
            const double v = from_lane(value, o * per);
            rank += v > value || (v == value && o < gr) ? 1 : 0;
        }
        // bit g * per: group g takes part
        const uint64_t kept = __ballot(gr < a.groups && rank < a.top_groups);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int e = lane + 64 * i;
            const int g = (int)(((float)e + 0.5f) * per_gs);         // e / gs: e under 1024
            if (e < a.E && !(kept >> (g * per) & 1)) key[i] = 0;
        }
    }
    // top k: the largest choice, of equal ones the lowest index
    double w_of = 0.0, total = 0.0;                  // of choice number `lane`
    int e_of = 0;
    for (int j = 0; j < a.k; ++j) {
        uint64_t best = key[0];                      // this lane's, of equal ones the first
        double s = score[0];
        int at = 0;
#pragma unroll
        for (int i = 1; i < V; ++i)
            if (key[i] > best) best = key[i], s = score[i], at = i;
        const uint32_t hi = (uint32_t)(best >> 32), hi_top = wave_top(hi);
        uint64_t who = __ballot(hi == hi_top);
        if (who & (who - 1)) {
            asm volatile("");                        // (a branch: ties are rare)
            const uint32_t lo = hi == hi_top ? (uint32_t)best : 0, lo_top = wave_top(lo);
            who = __ballot(hi == hi_top && lo == lo_top);
            if (who & (who - 1)) {                   // equal choices: the lowest of 64 at + lane
                const uint32_t last = who >> lane & 1 ? 65535u - (uint32_t)(64 * at + lane) : 0;
                who = __ballot(last == wave_top(last));
            }
        }
        const int winner = __builtin_ctzll(who);
        const int i_won = __builtin_amdgcn_readlane(at, winner);
        // (-infinity: masked, chosen for want of others)
        const bool masked = (uint32_t)__builtin_amdgcn_readlane((int)hi, winner) < 0x00100000u;
        const double s_won = masked ? 0.0 : from_lane(s, winner);
        total += s_won;
        if (lane == j) w_of = s_won, e_of = 64 * i_won + winner;
        if (lane == winner) {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (i == i_won) key[i] = 0;
        }
    }
    if (lane < a.k) {
        if (a.renormalize) w_of = total > 0.0 ? w_of / total : 0.0;
        a.weights[t * a.k + lane] = (float)(w_of * a.scale);
        a.chosen[t * a.k + lane] = e_of;
    }
}

// The order by expert: workgroup e looks through all choices, counts those of lower
// experts (its offset) and its own, and then writes its own in order.  Wave w has the
// w-th part of the choices, 256 of them (four a lane, in order) at a time; counts come
// from ballots.  No counter is shared, so the order is always the same.  per_k is 2^32 / k
// rounded up: exact here, choices being under 2^25 and k at most 32; 0 for 1.
// Every workgroup reads all choices, four blocks at a time (L2; one at a time 17.7 us):
// 65536 choices of 256 experts take 14.5 us, 128 of 8 4.0.
constexpr int kPlanThreads = 1024, kPlanWaves = kPlanThreads / 64;
__global__ __launch_bounds__(kPlanThreads) void plan_kernel(const int32_t* __restrict__ chosen, int64_t S,
                                                            uint32_t per_k, int E, int32_t* __restrict__ offsets, int32_t* __restrict__ tokens,
                                                            int32_t* __restrict__ places) {
    __shared__ int before[kPlanWaves], own[kPlanWaves];
    const int e = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t run = (S + 256 * kPlanWaves - 1) / (256 * kPlanWaves) * 256;
    const int64_t i0 = min(S, wave * run), i1 = min(S, i0 + run);
    // choices i + 256 b + 4 lane .. + 3 of kAtOnce blocks b, those past the end E
    constexpr int kAtOnce = 4;
    const bool whole = (reinterpret_cast<uintptr_t>(chosen) & 15) == 0;
    auto load = [&](int64_t i, int (&c)[kAtOnce][4]) {
#pragma unroll
        for (int b = 0; b < kAtOnce; ++b) {
            const int64_t at = i + 256 * b + 4 * lane;
            int4 v{E, E, E, E};
            if (whole && at + 4 <= i1) {
                v = *reinterpret_cast<const int4*>(chosen + at);
            } else {
                if (at < i1) v.x = chosen[at];
                if (at + 1 < i1) v.y = chosen[at + 1];
                if (at + 2 < i1) v.z = chosen[at + 2];
                if (at + 3 < i1) v.w = chosen[at + 3];
            }
            c[b][0] = v.x, c[b][1] = v.y, c[b][2] = v.z, c[b][3] = v.w;
        }
    };
    int lower = 0, mine = 0;
    for (int64_t i = i0; i < i1; i += 256 * kAtOnce) {
        int c[kAtOnce][4];
        load(i, c);
#pragma unroll
        for (int b = 0; b < kAtOnce; ++b)
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                lower += __builtin_popcountll(__ballot(c[b][u] < e));
                mine += __builtin_popcountll(__ballot(c[b][u] == e));
            }
    }
    if (lane == 0) before[wave] = lower, own[wave] = mine;
    __syncthreads();
    int first = 0, count = 0, at = 0;
    for (int w = 0; w < kPlanWaves; ++w) {
        first += before[w];
        at += w < wave ? own[w] : 0;
        count += own[w];
    }
    if (tid == 0) {
        offsets[e] = first;
        if (e == E - 1) offsets[E] = first + count;
    }
    if (!mine) return;
    at += first;
    for (int64_t i = i0; i < i1; i += 256 * kAtOnce) {
        int c[kAtOnce][4];
        load(i, c);
#pragma unroll
        for (int b = 0; b < kAtOnce; ++b) {
            int slot = at;
            uint64_t any = 0;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const uint64_t who = __ballot(c[b][u] == e);
                slot += (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0));
                at += __builtin_popcountll(who);
                any |= who;
            }
            if (!any) continue;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if (c[b][u] != e) continue;
                const int64_t j = i + 256 * b + 4 * lane + u;
                tokens[slot] = per_k ? (int)__umulhi((uint32_t)j, per_k) : (int)j;
                places[j] = slot++;
            }
        }
    }
}

// y[t] = add[t] + sum_j w[t, j] Y[places[t, j]], a thread eight columns of a token.
// HBM-bound: every row of Y is read once.  8192 tokens of 8 rows of 4096, with add: 136 us
// (4.95 TB/s; a copy of 1 GiB 5.2), 16 tokens of 2: 2.9.
template <bool BF>
__global__ __launch_bounds__(256) void combine_kernel(CombineArgs a) {
    const int per_row = a.N / 8;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= a.T * per_row) return;
    const int64_t t = i / per_row;
    const int c = (int)(i - t * per_row) * 8;
    float y[8] = {};
    for (int j = 0; j < a.k; ++j) {
        const float w = a.weights[t * a.k + j];
        const int at = a.places[t * a.k + j];
        if (w == 0.f || at < 0 || at >= a.S) continue;
        const u16x8 v = *reinterpret_cast<const u16x8*>(a.Y + (int64_t)at * a.N + c);
#pragma unroll
        for (int u = 0; u < 8; ++u) y[u] = fmaf(w, scale_f32<BF>(v[u]), y[u]);
    }
    if (a.add) {
        const u16x8 v = *reinterpret_cast<const u16x8*>(a.add + t * a.N + c);
#pragma unroll
        for (int u = 0; u < 8; ++u) y[u] += scale_f32<BF>(v[u]);
    }
    u16x8 o;
#pragma unroll
    for (int u = 0; u < 8; ++u) o[u] = round_out<BF>(y[u]);
    *reinterpret_cast<u16x8*>(a.out + t * a.N + c) = o;
}

}  // namespace

int launch_route_experts(const RouteArgs& a, int32_t* offsets, int32_t* tokens, int32_t* places, hipStream_t s) {
    const dim3 grid((unsigned)((a.T + 3) / 4)), block(256);
    const size_t lds = a.top_groups < a.groups ? 4 * a.E * sizeof(double) : 0;
    int rc;
    if (a.E <= 64) rc = launch(route_kernel<1>, grid, block, lds, s, a);
    else if (a.E <= 128) rc = launch(route_kernel<2>, grid, block, lds, s, a);
    else if (a.E <= 256) rc = launch(route_kernel<4>, grid, block, lds, s, a);
    else if (a.E <= 512) rc = launch(route_kernel<8>, grid, block, lds, s, a);
    else rc = launch(route_kernel<16>, grid, block, lds, s, a);
    if (rc) return rc;
    return launch(plan_kernel, dim3((unsigned)a.E), dim3(kPlanThreads), 0, s, (const int32_t*)a.chosen, a.T * a.k,
                  a.k == 1 ? 0u : (uint32_t)((0x100000000ull + a.k - 1) / a.k), a.E, offsets, tokens, places);
}

int launch_combine_experts(const CombineArgs& a, bool bf, hipStream_t s) {
    const dim3 grid((unsigned)((a.T * (a.N / 8) + 255) / 256));
    return bf ? launch(combine_kernel<true>, grid, dim3(256), 0, s, a)
              : launch(combine_kernel<false>, grid, dim3(256), 0, s, a);
}

}  // namespace tf
