// Choice of experts, the order in which their products take the tokens, and the
// weighted sum of their outputs.
#include "tf_internal.h"
#include "tf_route.h"

namespace tf {
namespace {

typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ double lane_value(double v, int lane) { return __shfl(v, lane); }

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

__device__ __forceinline__ double logit(const RouteArgs& a, int64_t t, int e) {
    const int64_t i = t * a.stride + e;
    if (a.dtype == TF_F32) return (double)static_cast<const float*>(a.logits)[i];
    const uint16_t b = static_cast<const uint16_t*>(a.logits)[i];
    return a.dtype == TF_BF16 ? (double)scale_f32<true>(b) : (double)scale_f32<false>(b);
}

// The two largest of a set of values, the absent ones -infinity.
struct Two { double a, b; };
__device__ __forceinline__ Two with(Two t, double v) {
    return v > t.a ? Two{v, t.a} : Two{t.a, fmax(t.b, v)};
}

// One wave a token, V experts a lane: expert lane + 64 i.  Scores and choices are
// fp64: what is compared here decides which weights are read, and rounded to 32
// bits unequal scores would tie.
template <int V>
__global__ __launch_bounds__(256) void route_kernel(RouteArgs a) {
    extern __shared__ double grouped[];              // [4][E] where experts are grouped
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t t = (int64_t)blockIdx.x * 4 + wave;
    if (t >= a.T) return;                            // (whole waves; no barrier follows)
    double x[V], score[V], choice[V];
    double top = -INFINITY;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int e = lane + 64 * i;
        double v = e < a.E ? logit(a, t, e) : -INFINITY;
        v = v == v ? v : -INFINITY;                  // NaN: masked
        x[i] = v;
        top = fmax(top, v);
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
#pragma unroll
        for (int i = 0; i < V; ++i) score[i] = sum > 0.0 ? score[i] / sum : 0.0;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int e = lane + 64 * i;
        double c = score[i];
        if (a.bias && e < a.E) c += (double)a.bias[e];
        choice[i] = x[i] == -INFINITY || c != c ? -INFINITY : c;
    }
    const int gs = a.E / a.groups;
    uint64_t kept = ~0ull;
    if (a.top_groups < a.groups) {
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
            const double v = lane_value(value, o * per);
            rank += v > value || (v == value && o < gr) ? 1 : 0;
        }
        // bit g * per of `kept`: group g takes part
        kept = __ballot(gr < a.groups && rank < a.top_groups);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int e = lane + 64 * i;
            if (e < a.E && !(kept >> (e / gs * per) & 1)) x[i] = NAN;      // not to be chosen at all
        }
    }
    // top k: the largest choice, of equal ones the lowest index
    double w_of = 0.0, total = 0.0;                  // of choice number `lane`
    int e_of = 0;
    for (int j = 0; j < a.k; ++j) {
        double best = -INFINITY, s = 0.0;
        int at = INT32_MAX;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int e = lane + 64 * i;
            const bool open = e < a.E && x[i] == x[i];
            if (open && (choice[i] > best || at == INT32_MAX)) best = choice[i], at = e, s = score[i];
        }
#pragma unroll
        for (int d = 32; d; d >>= 1) {
            const double ob = __shfl_xor(best, d), os = __shfl_xor(s, d);
            const int oa = __shfl_xor(at, d);
            if (oa != INT32_MAX && (at == INT32_MAX || ob > best || (ob == best && oa < at))) best = ob, at = oa, s = os;
        }
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (lane + 64 * i == at) x[i] = NAN;
        if (best == -INFINITY) s = 0.0;              // masked: chosen for want of others
        total += s;
        if (lane == j) w_of = s, e_of = at;
    }
    if (lane < a.k) {
        if (a.renormalize) w_of = total > 0.0 ? w_of / total : 0.0;
        a.weights[t * a.k + lane] = (float)(w_of * a.scale);
        a.chosen[t * a.k + lane] = e_of;
    }
}

// The order by expert: workgroup e looks through all choices, counts those of lower
// experts (its offset) and its own, and writes its own in order.  Each thread has a
// run of choices; a second look at them follows the counts.
constexpr int kPlanThreads = 1024;
__global__ __launch_bounds__(kPlanThreads) void plan_kernel(const int32_t* __restrict__ chosen, int64_t S, int k, int E,
                                                            int32_t* __restrict__ offsets, int32_t* __restrict__ tokens,
                                                            int32_t* __restrict__ places) {
    __shared__ int before[kPlanThreads / 64], own[kPlanThreads / 64];
    const int e = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t run = (S + kPlanThreads - 1) / kPlanThreads, i0 = min(S, tid * run), i1 = min(S, i0 + run);
    int lower = 0, mine = 0;
    for (int64_t i = i0; i < i1; ++i) {
        const int c = chosen[i];
        lower += c < e;
        mine += c == e;
    }
    int scan = mine, all = lower;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(scan, d);
        if (lane >= d) scan += o;
        all += __shfl_xor(all, d);
    }
    if (lane == 63) own[wave] = scan;
    if (lane == 0) before[wave] = all;
    __syncthreads();
    int at = scan - mine, first = 0, count = 0;
    for (int w = 0; w < kPlanThreads / 64; ++w) {
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
    for (int64_t i = i0; i < i1; ++i)
        if (chosen[i] == e) {
            tokens[at] = (int)(i / k);
            places[i] = at++;
        }
}

// y[t] = add[t] + sum_j w[t, j] Y[places[t, j]], a thread eight columns of a token.
// HBM-bound: every row of Y is read once.
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
    return launch(plan_kernel, dim3((unsigned)a.E), dim3(kPlanThreads), 0, s, (const int32_t*)a.chosen, a.T * a.k, a.k,
                  a.E, offsets, tokens, places);
}

int launch_combine_experts(const CombineArgs& a, bool bf, hipStream_t s) {
    const dim3 grid((unsigned)((a.T * (a.N / 8) + 255) / 256));
    return bf ? launch(combine_kernel<true>, grid, dim3(256), 0, s, a)
              : launch(combine_kernel<false>, grid, dim3(256), 0, s, a);
}

}  // namespace tf
