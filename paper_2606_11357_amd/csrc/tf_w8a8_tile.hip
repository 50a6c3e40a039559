// The 8-bit matrix product for many rows (dense, or of each expert): C tiles of
// 256 x 256, K in steps of 64.
//
// One workgroup of four waves a compute unit, one wave a SIMD with the whole
// register file: each has all 256 rows by 64 columns (256 accumulators) of
// v_mfma_i32_16x16x64_i8, 64 of them a step.
//  - A goes global -> LDS by direct loads, two steps (128 bytes of a row, whole cache
//    lines) at a time into one of four buffers, three such pairs ahead; 16-byte
//    chunks are XOR-swizzled by row, so that fragment reads meet no bank twice.
//  - A fragments are read half a step ahead of their use, in two bursts a step.
//  - Weights are stored in the order of the matrix instruction's operand: a wave
//    loads its own columns straight into a ring of registers, three steps ahead.
//  - Workgroups are dealt to the XCDs so that the 32 tiles that one runs at a time
//    are about 8 by 4: each L2 then serves 12 operand tiles to 32.
// The two bytes an element that rows and columns take in bf16 are one here and the
// matrix instruction does twice the work in the same 16 cycles, so a step asks for
// as many bytes a cycle as the 16-bit kernel's.
#include <algorithm>

#include "tf_w8a8.h"

namespace tf {
namespace {

constexpr int kThreads = 256, kXcds = 8;

// A form: RB row blocks of 16, CB column blocks of 16 a wave; P buffers of A, each of
// two steps (a pair); weights R steps deep in registers; WGS workgroups a compute
// unit.
template <int RB_, int CB_, int P_, int R_, int WGS_>
struct Form {
    static constexpr int RB = RB_, CB = CB_, P = P_, R = R_, WGS = WGS_;
    static constexpr int BM = 16 * RB, BN = 64 * CB;
    static constexpr int kPairBytes = BM * 128;
    static constexpr int kDma = RB / 4;                      // direct loads of a wave and step
    static constexpr int kSlots = RB * CB;                   // matrix instructions of a wave and step
    static constexpr bool kAhead = kSlots <= 8;              // two sets of fragments
    static constexpr bool kOften = kSlots >= 64;             // a barrier every step: see the loop
    static constexpr int kRowGroup = 2048 / BM;              // row tiles that share the columns' order
    static_assert((P & (P - 1)) == 0 && R % 4 == 0, "buffers by a mask, whole pairs a pass of the loop");
};

__device__ __forceinline__ int a_swz(int row) { return row & 7; }

// LDS reads as asm statements with waits of their own (lds_wait), so that the compiler
// waits neither for them nor for the direct loads on their way to other buffers.
template <int OFF>
__device__ __forceinline__ u32x4 lds_read16_at(uint32_t addr) {
    u32x4 v;
    asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "i"(OFF));
    return v;
}
__device__ __forceinline__ u32x4 lds_read_block(uint32_t addr, int i) {
    switch (i) {
#define TF_BLOCK(n) \
    case n: return lds_read16_at<(n) * 16 * 128>(addr);
        TF_BLOCK(0) TF_BLOCK(1) TF_BLOCK(2) TF_BLOCK(3) TF_BLOCK(4) TF_BLOCK(5) TF_BLOCK(6) TF_BLOCK(7)
        TF_BLOCK(8) TF_BLOCK(9) TF_BLOCK(10) TF_BLOCK(11) TF_BLOCK(12) TF_BLOCK(13) TF_BLOCK(14) TF_BLOCK(15)
#undef TF_BLOCK
        default: return lds_read16_at<0>(addr);
    }
}
__device__ __forceinline__ void lds_wait() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
// All but the last NOW of this wave's reads are done (they return in order).
template <int NOW>
__device__ __forceinline__ void lds_wait_but() {
    static_assert(NOW >= 0 && NOW < 16, "lgkmcnt holds 4 bits");
    asm volatile("s_waitcnt lgkmcnt(%0)" ::"i"(NOW) : "memory");
}

__device__ __forceinline__ u32x4 load16(__amdgpu_buffer_rsrc_t r, uint32_t voff) {
    return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, voff, 0, 0));
}

// A direct load: 16 bytes from each lane's offset to `to` + 16 lane in LDS.
__device__ __forceinline__ void dma16(__amdgpu_buffer_rsrc_t r, void* to, uint32_t voff) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)to, 16, voff, 0, 0, 0);
}

// Accumulators are pinned to AGPRs; mfma_hazard_gap() stands between their
// initialisation and the first, and between the last and their first read.
__device__ __forceinline__ void mfma_i8(i32x4& acc, const u32x4& a, const u32x4& b) {
    asm("v_mfma_i32_16x16x64_i8 %0, %1, %2, %0" : "+a"(acc) : "v"(a), "v"(b));
}

__device__ __forceinline__ void barrier_only() {
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
}
// A barrier after all but this wave's last NOW vector-memory operations are done
// (they complete in order).
template <int NOW>
__device__ __forceinline__ void barrier_after_loads() {
    static_assert(NOW >= 0 && NOW < 64, "vmcnt holds 6 bits");
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(0x0F70 | (NOW & 15) | ((NOW >> 4) << 14));
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
}

template <class F>
struct TileShared {
    uint8_t a[F::P * F::kPairBytes];
    float scale[F::BM];
};

// Tile number `at` of row tiles x column tiles, rows in groups of kRowGroup.
template <class F>
__device__ __forceinline__ void tile_of(int at, int tiles_m, int tiles_n, int& tm, int& tn) {
    const int group = at / (F::kRowGroup * tiles_n), rest = at - group * F::kRowGroup * tiles_n;
    const int height = min(F::kRowGroup, tiles_m - group * F::kRowGroup);
    tn = rest / height;
    tm = group * F::kRowGroup + rest - tn * height;
}

// Rows row0 .. row0 + rows - 1 of C (A's, or those that a.rows names) by columns
// col0 .. col0 + BN - 1 of `packed`.
template <class F, bool GATHER>
__device__ __forceinline__ void tile_product(const W8Args& a, const uint8_t* packed, int64_t row0, int rows,
                                             int64_t col0, TileShared<F>& sm) {
    constexpr int RB = F::RB, CB = F::CB, P = F::P, R = F::R, S = F::kSlots;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 15, kg = lane >> 4;
    const int steps = a.na, pairs = steps / 2;

    // A: rows that are not there repeat one that is; they are not stored.
    // Rows of A are counted from `base`, of which `there` are.
    const int64_t base = GATHER ? 0 : row0;
    const int there = GATHER ? (int)a.a_rows : (int)max(min(a.a_rows - row0, (int64_t)rows), (int64_t)0);
    const __amdgpu_buffer_rsrc_t ar =
        make_rsrc(a.A + base * a.K, (uint32_t)min((a.a_rows - base) * a.K, (int64_t)0xFFFFFF00));
    auto row_of = [&](int r) {                        // a row of C as one of A; not there: negative or past `there`
        return GATHER ? a.rows[row0 + min(r, rows - 1)] : r;
    };
    auto in = [&](int at) { return (uint32_t)at < (uint32_t)there; };
    // Direct load r of wave w fills rows 4 RB w + 8 r .. + 7 of a buffer, eight lanes a row.
    uint32_t avoff[RB / 2];
#pragma unroll
    for (int r = 0; r < RB / 2; ++r) {
        const int row = 4 * RB * wave + 8 * r + (lane >> 3);
        const int at = row_of(row);
        avoff[r] = (uint32_t)(in(at) ? at : 0) * (uint32_t)a.K + (uint32_t)((lane & 7) ^ a_swz(row)) * 16u;
    }
    auto dma_a = [&](int pair, int buf, int r) {
        dma16(ar, sm.a + buf * F::kPairBytes + (RB / 2 * wave + r) * 1024, avoff[r] + (uint32_t)min(pair, pairs - 1) * 128u);
    };
    const uint32_t lds = (uint32_t)reinterpret_cast<uintptr_t>(sm.a);
    uint32_t a_lane[2];
#pragma unroll
    for (int odd = 0; odd < 2; ++odd) a_lane[odd] = lds + (uint32_t)(c * 128 + ((kg + 4 * odd) ^ a_swz(c)) * 16);

    // B: this wave's panels; one past N is empty, and so is what follows K.
    __amdgpu_buffer_rsrc_t wr[CB];
#pragma unroll
    for (int t = 0; t < CB; ++t) {
        const int64_t panel = col0 / kW8Panel + CB * wave + t;
        const bool here = panel < a.np;
        wr[t] = make_rsrc(packed + (here ? panel : 0) * a.na * kW8AtomBytes, here ? (uint32_t)a.na * kW8AtomBytes : 0u);
    }
    u32x4 ring[R][CB];
    auto load_b = [&](int step, int t, u32x4& v) { v = load16(wr[t], (uint32_t)(lane * 16 + step * kW8AtomBytes)); };

    float row_scale = 0.f;
    if (tid < F::BM) {
        const int at = row_of(tid);
        const float s = a.a_scale[in(at) ? base + at : 0];
        row_scale = in(at) ? s : 0.f;
    }
    // What is on its way when the loop begins: its own loads of the R - 1 steps before it,
    // in its order (so that the same counts tell what has landed), and before them the
    // halves of pairs that earlier steps would have brought, which are waited for.
    constexpr int kOps = F::kDma + CB;                // vector-memory operations of a wave and step
    constexpr int kHalf0 = F::kOften ? 2 * P - 2 : 2 * P - 3;      // half of a pair that step 0 brings
    constexpr int kBefore = kHalf0 - (R - 1);
    static_assert(kBefore >= 2, "the first pair is among those waited for");
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int h = 0; h < kBefore; ++h)
#pragma unroll
        for (int r = 0; r < F::kDma; ++r) dma_a(h / 2, h / 2, F::kDma * (h % 2) + r);
#pragma unroll
    for (int j = 0; j < R - 1; ++j) {
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int r = 0; r < F::kDma; ++r)
            dma_a((kBefore + j) / 2, (kBefore + j) / 2, F::kDma * ((kBefore + j) % 2) + r);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int t = 0; t < CB; ++t) load_b(j, t, ring[j][t]);
    }
    __builtin_amdgcn_sched_barrier(0);
    i32x4 acc[RB][CB];
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int t = 0; t < CB; ++t) acc[i][t] = i32x4{0, 0, 0, 0};
    if (tid < F::BM) sm.scale[tid] = row_scale;
    lds_wait();
    barrier_after_loads<(R - 1) * kOps < 63 ? (R - 1) * kOps : 63>();
    u32x4 af[F::kAhead ? 2 : 1][RB];
#pragma unroll
    for (int i = 0; i < (F::kAhead ? RB : RB - 1); ++i) af[0][i] = lds_read_block(a_lane[0], i);
    mfma_hazard_gap();

    // Steps in turn, R to a pass of the loop (so that the ring has fixed places; steps
    // past K multiply zeros), S slots each of one matrix instruction (row block q / CB,
    // column block q % CB) and at most one of the others beside it, which are spread over
    // the step: four waves at once ask LDS and the memory pipe for four times what one
    // does, and an instruction that has to wait for its turn holds up those behind it.
    //  - before slot CB i: wait for the fragment of row block i
    //  - at slot CB i: read that of block i - 1 for the next step (block RB - 1 of this
    //    step at slot 0).  Small forms (kAhead) read all of the next step's into a second
    //    set.
    //  - every S / kOps slots: a direct load (half a pair a step) or one of the weights of
    //    step s + R - 1.
    // Pair p is read from step 2 p - 1 on: at the end of step 2 p - 2 its direct loads
    // have to have landed, which leaves this wave's later operations on their way (they
    // complete in order).  After the barrier there no wave reads pair p - 2 any more, and
    // the next two steps fill its buffer with pair p - 2 + P: one barrier for two steps.
    // With kOften a second barrier ends the odd steps, after which pair p - 1 is done, and
    // steps 2 p and 2 p + 1 fill its buffer: a step earlier, where four buffers of 32 KB
    // are all there is.
    constexpr int kLater = CB + (F::kOften ? 2 * P - 5 : 2 * P - 6) * kOps;
    for (int s0 = 0; s0 < steps; s0 += R) {
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int step = s0 + j, odd = j & 1;
            auto place = [&](int pair) { return (uint32_t)((s0 / 2 + pair) & (P - 1)) * F::kPairBytes; };
            const uint32_t cur = place(j / 2), next = place((j + 1) / 2);
            // the pair whose half is filled in this step
            const int fill = s0 / 2 + (F::kOften ? j / 2 + P - 1 : (j + 1) / 2 + P - 2);
            const int half = F::kOften ? odd : odd ^ 1;
            constexpr int kSets = F::kAhead ? 2 : 1;
            u32x4 (&now)[RB] = af[j % kSets];
            u32x4 (&nxt)[RB] = af[(j + 1) % kSets];
#pragma unroll
            for (int q = 0; q < S; ++q) {
                const int i = q / CB, t = q % CB;
                __builtin_amdgcn_sched_barrier(0);
                if constexpr (F::kAhead) {
                    if (q == 0) lds_wait();
                } else {
                    if (t == 0) lds_wait_but<RB - 2>();
                }
                mfma_i8(acc[i][t], ring[j % R][t], now[i]);
                if constexpr (F::kAhead) {
#pragma unroll
                    for (int r = q * RB / S; r < (q + 1) * RB / S; ++r) nxt[r] = lds_read_block(a_lane[odd ^ 1] + next, r);
                } else if (t == 0) {
                    if (i == 0) now[RB - 1] = lds_read_block(a_lane[odd] + cur, RB - 1);
                    else nxt[i - 1] = lds_read_block(a_lane[odd ^ 1] + next, i - 1);
                }
#pragma unroll
                for (int o = 0; o < kOps; ++o) {
                    if (q != o * S / kOps + CB / 2) continue;
                    if (o < F::kDma) dma_a(fill, fill & (P - 1), F::kDma * half + o);
                    else load_b(step + R - 1, o - F::kDma, ring[(j + R - 1) % R][o - F::kDma]);
                }
            }
            if (!odd) barrier_after_loads<kLater < 63 ? kLater : 63>();
            else if (F::kOften) barrier_only();
        }
    }
    // The last step's reads, which nothing uses, keep their registers until they are done.
    lds_wait();
#pragma unroll
    for (int i = 0; i < RB; ++i) asm volatile("" ::"v"(af[0][i]), "v"(af[F::kAhead ? 1 : 0][i]));
    mfma_hazard_gap();
    __builtin_amdgcn_s_waitcnt(0);       // the direct loads past the end have landed
    __syncthreads();                     // and no wave reads the buffers, which the output passes through

    // A row block at a time through LDS (rows padded by 16 bytes), stored as 16 bytes a
    // lane, 2 CB lanes a row.
    const float* scales = reinterpret_cast<const float*>(packed + a.s_off);
    const int64_t wcol = col0 + 16 * CB * wave;
    float4_t sw[CB];
#pragma unroll
    for (int t = 0; t < CB; ++t) {
        const int64_t n = wcol + 16 * t + 4 * kg;
        sw[t] = n < a.np * 16 ? *reinterpret_cast<const float4_t*>(scales + n) : float4_t{0.f, 0.f, 0.f, 0.f};
    }
    constexpr int kStageRow = 32 * CB + 16, kLanes = 2 * CB, kAtOnce = 64 / kLanes;
    uint8_t* stage = sm.a + wave * 16 * kStageRow;
    const int rr = lane / kLanes, cc = lane % kLanes;
#pragma unroll
    for (int i = 0; i < RB; ++i) {
        __builtin_amdgcn_sched_barrier(0);
        const float sa = sm.scale[16 * i + c];
#pragma unroll
        for (int t = 0; t < CB; ++t)
            *reinterpret_cast<uint2*>(stage + c * kStageRow + 32 * t + 8 * kg) = w8_scaled(a.bf, acc[i][t], sa, sw[t]);
        __builtin_amdgcn_s_waitcnt(0xC07F);       // lgkmcnt(0): this wave's stores landed
        constexpr int kTimes = kAtOnce > 16 ? 1 : 16 / kAtOnce;
        u32x4 v[kTimes];
#pragma unroll
        for (int h = 0; h < kTimes; ++h)
            v[h] = *reinterpret_cast<const u32x4*>(stage + (rr % 16 + kAtOnce * h) * kStageRow + 16 * cc);
        __builtin_amdgcn_s_waitcnt(0xC07F);       // read before the area is written again
#pragma unroll
        for (int h = 0; h < kTimes; ++h) {
            const int r = 16 * i + rr + kAtOnce * h;
            const int64_t n = wcol + 8 * cc;
            if (rr < 16 && r < rows && n < a.N) *reinterpret_cast<u32x4*>(a.C + (row0 + r) * a.N + n) = v[h];
        }
    }
}

// The place in the list of workgroup b's tile: each XCD (workgroups go to the eight in
// turn) has a contiguous part of the list.  Past the end: -1.
__device__ __forceinline__ int place_of(int b, int total) {
    const int per = total / kXcds, rem = total % kXcds, x = b % kXcds, i = b / kXcds;
    return i < per + (x < rem ? 1 : 0) ? x * per + min(x, rem) + i : -1;
}

template <class F>
__global__ __launch_bounds__(kThreads, F::WGS) void w8a8_tile_kernel(W8Args a, int tiles_m, int tiles_n) {
    __shared__ __align__(16) TileShared<F> sm;
    const int at = place_of(blockIdx.x, tiles_m * tiles_n);
    if (at < 0) return;
    int tm, tn;
    tile_of<F>(at, tiles_m, tiles_n, tm, tn);
    tm = __builtin_amdgcn_readfirstlane(tm);
    tn = __builtin_amdgcn_readfirstlane(tn);
    const int64_t row0 = (int64_t)tm * F::BM;
    tile_product<F, false>(a, a.packed, row0, (int)min((int64_t)F::BM, a.M - row0), (int64_t)tn * F::BN, sm);
}

// By expert: the row tiles of all experts in one list, found from the offsets by
// every workgroup (thread t has experts 4 t .. 4 t + 3).
template <class F, bool GATHER>
__global__ __launch_bounds__(kThreads, F::WGS) void w8a8_tile_experts_kernel(W8Args a, int tiles_n) {
    __shared__ __align__(16) TileShared<F> sm;
    int* ints = reinterpret_cast<int*>(sm.a);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    // offsets with a running maximum within the call's slots
    int end[4], top = 0;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int e = 4 * tid + u;
        top = max(top, e < a.experts ? min(max(a.offsets[e + 1], 0), (int)a.M) : 0);
        end[u] = top;
    }
    int before = top;                                 // largest end up to this thread's last
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(before, d);
        if (lane >= d) before = max(before, o);
    }
    if (lane == 63) ints[wave] = before;
    __syncthreads();
    before = __shfl_up(before, 1);
    if (lane == 0) before = 0;
    int first = min(max(a.offsets[0], 0), (int)a.M);
    before = max(before, first);
    for (int w = 0; w < wave; ++w) before = max(before, ints[w]);
    int start[4], tiles[4], mine = 0;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        start[u] = before;
        end[u] = max(end[u], before);
        if (4 * tid + u >= a.experts) end[u] = before;
        before = end[u];
        tiles[u] = (end[u] - start[u] + F::BM - 1) / F::BM;
        mine += tiles[u];
    }
    int scan = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(scan, d);
        if (lane >= d) scan += o;
    }
    if (lane == 63) ints[8 + wave] = scan;
    __syncthreads();
    int total = 0, from = scan - mine;
    for (int w = 0; w < 4; ++w) {
        if (w < wave) from += ints[8 + w];
        total += ints[8 + w];
    }
    const int at = place_of(blockIdx.x, total * tiles_n);
    if (at < 0) return;                               // (the whole workgroup)
    int tm, tn;
    tile_of<F>(at, total, tiles_n, tm, tn);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        if (tm >= from && tm < from + tiles[u]) {
            ints[16] = 4 * tid + u;
            ints[17] = start[u] + (tm - from) * F::BM;
            ints[18] = end[u];
        }
        from += tiles[u];
    }
    __syncthreads();
    const int e = __builtin_amdgcn_readfirstlane(ints[16]), row0 = __builtin_amdgcn_readfirstlane(ints[17]);
    const int rows = min(F::BM, __builtin_amdgcn_readfirstlane(ints[18]) - row0);
    tn = __builtin_amdgcn_readfirstlane(tn);
    __syncthreads();                                  // the buffers take this place
    tile_product<F, GATHER>(a, a.packed + e * a.total, row0, rows, (int64_t)tn * F::BN, sm);
}

template <class F>
int launch_form(const W8Args& a, hipStream_t s) {
    const int64_t tiles_n = (a.N + F::BN - 1) / F::BN;
    if (a.experts) {
        const int64_t most = std::min<int64_t>(a.M, a.M / F::BM + a.experts);     // row tiles
        const dim3 grid((unsigned)((most * tiles_n + 7) / 8 * 8));
        return a.rows ? launch(w8a8_tile_experts_kernel<F, true>, grid, dim3(kThreads), 0, s, a, (int)tiles_n)
                      : launch(w8a8_tile_experts_kernel<F, false>, grid, dim3(kThreads), 0, s, a, (int)tiles_n);
    }
    const int64_t tiles_m = (a.M + F::BM - 1) / F::BM;
    return launch(w8a8_tile_kernel<F>, dim3((unsigned)((tiles_m * tiles_n + 7) / 8 * 8)), dim3(kThreads), 0, s, a,
                  (int)tiles_m, (int)tiles_n);
}

}  // namespace

int launch_w8a8_tile(const W8Args& a, int form, hipStream_t s) {
    switch (form) {
        case 0: return launch_form<Form<16, 4, 4, 4, 1>>(a, s);
        case 1: return launch_form<Form<8, 4, 8, 8, 1>>(a, s);
        case 2: return launch_form<Form<8, 4, 4, 4, 2>>(a, s);
        case 3: return launch_form<Form<8, 2, 8, 8, 1>>(a, s);
        case 4: return launch_form<Form<4, 2, 8, 8, 2>>(a, s);
        default: return launch_form<Form<4, 1, 8, 8, 2>>(a, s);
    }
}

}  // namespace tf
