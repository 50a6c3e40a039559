// The 8-bit matrix product for many rows (dense, or of each expert): C tiles of
// 256 x 256 down to 64 x 64, K in steps of 64.
//
// Workgroups of four waves, each with all rows of the tile by a quarter of its columns;
// in the largest form one a compute unit, one wave a SIMD with the whole register file:
// 256 rows by 64 columns (256 accumulators) of v_mfma_i32_16x16x64_i8, 64 of them a step.
//  - A goes global -> LDS by direct loads, two steps (128 bytes of a row, whole cache
//    lines) at a time into one of four or eight buffers, all but one or two of them
//    ahead; 16-byte chunks are XOR-swizzled by row, so that fragment reads meet no bank
//    twice.
//  - A fragments are read a step ahead of their use, one beside every few matrix
//    instructions.
//  - Weights are stored in the order of the matrix instruction's operand: a wave
//    loads its own columns straight into a ring of registers, three or seven steps ahead.
//  - Workgroups are dealt to the XCDs so that the 32 tiles that one runs at a time
//    are about 8 by 4: each L2 then serves 12 operand tiles to 32.
//  - Outputs are scaled and stored from the accumulators, past the L2 (one tile of K = 512
//    16.4 us through it, 14.5 past it), after the next tile's first loads are issued.
//    Tiles with a scale that is not near take a second form of that (w8_scaled_far in
//    place of w8_scaled: two operations an output more, 256 of them in the largest tile).
// The matrix cores and their power bound the large tile: 8192 x 8192 x 8192 384 us (2.87
// POP/s; torch's library product of int8 524), 8192 x 4096 x 28672 737 to 790 us from
// card to card (2.44 to 2.61 POP/s at 1.95 GHz, matrix cores 68% busy; of zeros 621 us
// at 2.4).  A step of its 64 takes 0.53 us, 97% of it matrix instructions; a tile's beginning and
// end some 7 us.  The smaller forms' steps take what their operands take through L1.
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
    static constexpr bool kSplits = kSlots <= 4;             // the form that K is split for
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

// v as a value of its own, so that what is computed from it for one tile is computed
// again for the next and not held in registers between.
__device__ __forceinline__ int again(int v) {
    asm volatile("" : "+v"(v));
    return v;
}

constexpr uint32_t kNowhere = 0xFFFFFF00u;        // an offset that no buffer reaches: not stored
__device__ __forceinline__ void store16(__amdgpu_buffer_rsrc_t r, const u32x4& v, uint32_t voff) {
    __builtin_amdgcn_raw_buffer_store_b128(v, r, voff, 0, kSc1);
}
__device__ __forceinline__ void store8(__amdgpu_buffer_rsrc_t r, const uint2& v, uint32_t voff) {
    __builtin_amdgcn_raw_buffer_store_b64(u32x2{v.x, v.y}, r, voff, 0, kSc1);
}
// Rows of 16 lanes swapped: lanes of row 2 g get (x, x of row 2 g + 1), those of row
// 2 g + 1 (y of row 2 g, y).
__device__ __forceinline__ u32x4 rows_swapped(const uint2& x, const uint2& y) {
    const auto p = __builtin_amdgcn_permlane16_swap(x.x, y.x, false, false);
    const auto q = __builtin_amdgcn_permlane16_swap(x.y, y.y, false, false);
    return u32x4{p[0], q[0], p[1], q[1]};
}

// Accumulators are pinned to AGPRs; the loop begins and ends with the wait states that
// the matrix instructions need behind writes and before reads of them.
__device__ __forceinline__ void mfma_i8(i32x4& acc, const u32x4& a, const u32x4& b) {
    asm("v_mfma_i32_16x16x64_i8 %0, %1, %2, %0" : "+a"(acc) : "v"(a), "v"(b));
}

// Four accumulators as they are, taken apart only here (else the compiler moves and
// spills single ones, at the loop's end already).
__device__ __forceinline__ i32x4 whole(i32x4 acc) {
    asm volatile("" : "+a"(acc));
    return acc;
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
    float rows[2][F::BM], columns[2][F::BN];          // scales of this tile and the next
    int far[2][4];                                    // whether some of them are not near, as each wave saw
    int found[4];
};

// One tile of C: rows row0 .. row0 + rows - 1 (A's, or those that a.rows names) by
// columns col0 .. col0 + BN - 1 of `packed`.
struct Tile {
    const uint8_t* packed;
    int64_t row0, col0;
    int rows;
    int from, steps, part;   // where K is split: the part's steps
};

// Tile number `at` of row tiles x column tiles, rows in groups of kRowGroup.
template <class F>
__device__ __forceinline__ void tile_of(int at, int tiles_m, int tiles_n, int& tm, int& tn) {
    const int group = at / (F::kRowGroup * tiles_n), rest = at - group * F::kRowGroup * tiles_n;
    const int height = min(F::kRowGroup, tiles_m - group * F::kRowGroup);
    tn = rest / height;
    tm = group * F::kRowGroup + rest - tn * height;
}

// Tiles next(0), next(1), ... (false: no more).  The loads that a tile begins with are
// issued before the outputs of the one before are scaled and stored.
template <class F, bool GATHER, bool SPLIT, class Next>
__device__ __forceinline__ void tile_products(const W8Args& a, Next&& next_tile, TileShared<F>& sm) {
    constexpr int RB = F::RB, CB = F::CB, P = F::P, R = F::R, S = F::kSlots;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 15, kg = lane >> 4;
    const int pairs = a.na / 2;
    int from = 0, steps = a.na;                       // this tile's steps of K

    __amdgpu_buffer_rsrc_t ar, wr[CB];
    uint32_t avoff[RB / 2];
    float row_scale = 0.f, column_scale = 0.f;
    // Direct load r of wave w fills rows 4 RB w + 8 r .. + 7 of a buffer, eight lanes a row.
    auto dma_a = [&](int pair, int buf, int r) {
        dma16(ar, sm.a + buf * F::kPairBytes + (RB / 2 * wave + r) * 1024,
              avoff[r] + (uint32_t)min(from / 2 + pair, pairs - 1) * 128u);
    };
    u32x4 ring[R][CB];
    auto load_b = [&](int step, int t, u32x4& v) {
        v = load16(wr[t], (uint32_t)(lane * 16 + (from + step) * kW8AtomBytes));
    };

    constexpr int kOps = F::kDma + CB;                // vector-memory operations of a wave and step
    constexpr int kHalf0 = F::kOften ? 2 * P - 2 : 2 * P - 3;      // half of a pair that step 0 brings
    constexpr int kBefore = kHalf0 - (R - 1);
    static_assert(kBefore >= 2, "the first pair is among those waited for");
    // A tile's operands, and what is on its way when its loop begins: the loop's own loads
    // of the R - 1 steps before it, in its order (so that the same counts tell what has
    // landed), and before them the halves of pairs that earlier steps would have brought,
    // which are waited for.
    auto begin = [&](const Tile& t) {
        const int lane = again(threadIdx.x & 63), tid = 64 * wave + lane;
        // Rows of A are counted from `base`, of which `there` are; rows that are not there
        // repeat one that is, and are not stored or scaled by 0.
        const int64_t base = GATHER ? 0 : t.row0;
        const int there = GATHER ? (int)a.a_rows : (int)max(min(a.a_rows - t.row0, (int64_t)t.rows), (int64_t)0);
        const int64_t first = there > 0 ? base : 0;
        ar = make_rsrc(a.A + first * a.K, (uint32_t)min((a.a_rows - first) * a.K, (int64_t)0xFFFFFF00));
        auto row_of = [&](int r) { return GATHER ? a.rows[t.row0 + min(r, t.rows - 1)] : r; };
        auto in = [&](int at) { return (uint32_t)at < (uint32_t)there; };
#pragma unroll
        for (int r = 0; r < RB / 2; ++r) {
            const int row = 4 * RB * wave + 8 * r + (lane >> 3);
            const int at = row_of(row);
            avoff[r] = (uint32_t)(in(at) ? at : 0) * (uint32_t)a.K + (uint32_t)((lane & 7) ^ a_swz(row)) * 16u;
        }
        // this wave's panels; one past N is empty, and so is what follows K
#pragma unroll
        for (int u = 0; u < CB; ++u) {
            const int64_t panel = t.col0 / kW8Panel + CB * wave + u;
            const bool here = panel < a.np;
            wr[u] = make_rsrc(t.packed + (here ? panel : 0) * a.na * kW8AtomBytes,
                              here ? (uint32_t)a.na * kW8AtomBytes : 0u);
        }
        if (tid < F::BM) {
            const int at = row_of(tid);
            const float s = a.a_scale[in(at) ? base + at : 0];
            row_scale = in(at) ? s : 0.f;
        }
        if (tid < F::BN) {
            const int64_t n = t.col0 + tid;
            column_scale = reinterpret_cast<const float*>(t.packed + a.s_off)[n < a.np * 16 ? n : 0];
        }
        if constexpr (SPLIT) {
            from = t.from;
            steps = t.steps;
        }
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
            for (int u = 0; u < CB; ++u) load_b(j, u, ring[j][u]);
        }
        __builtin_amdgcn_sched_barrier(0);
    };

    const uint32_t lds = (uint32_t)reinterpret_cast<uintptr_t>(sm.a);
    uint32_t a_lane[2];
#pragma unroll
    for (int odd = 0; odd < 2; ++odd) a_lane[odd] = lds + (uint32_t)(c * 128 + ((kg + 4 * odd) ^ a_swz(c)) * 16);

    Tile tile;
    if (!next_tile(0, tile)) return;
    begin(tile);
    constexpr int kStores = SPLIT ? RB * CB : CB > 1 ? RB * CB / 2 : RB;      // of a wave and tile
    for (int turn = 0;; ++turn) {
        i32x4 acc[RB][CB];
#pragma unroll
        for (int i = 0; i < RB; ++i)
#pragma unroll
            for (int t = 0; t < CB; ++t) acc[i][t] = i32x4{0, 0, 0, 0};
        if (tid < F::BM) sm.rows[turn & 1][tid] = row_scale;
        if (tid < F::BN) sm.columns[turn & 1][tid] = column_scale;
        if constexpr (!SPLIT) {
            const uint64_t far = __ballot((tid < F::BM && !w8_near(row_scale)) || (tid < F::BN && !w8_near(column_scale)));
            if (lane == 0) sm.far[turn & 1][wave] = far != 0;
        }
        lds_wait();
        // (the outputs of the tile before were stored after these loads were issued)
        constexpr int kFirst = (R - 1) * kOps, kNext = kFirst + kStores;
        if (turn == 0) barrier_after_loads<kFirst < 63 ? kFirst : 63>();
        else barrier_after_loads<kNext < 63 ? kNext : 63>();
        u32x4 af[F::kAhead ? 2 : 1][RB];
#pragma unroll
        for (int i = 0; i < (F::kAhead ? RB : RB - 1); ++i) af[0][i] = lds_read_block(a_lane[0], i);
        lds_wait();

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
                if (j == 0) asm volatile("s_nop 1");     // (after the accumulators' zeros)
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
                        for (int r = q * RB / S; r < (q + 1) * RB / S; ++r)
                            nxt[r] = lds_read_block(a_lane[odd ^ 1] + next, r);
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
                // what follows the loop may read the accumulators at once
                if (j == R - 1) asm volatile("s_nop 7\n\ts_nop 7\n\ts_nop 1");
                if (!odd) barrier_after_loads<kLater < 63 ? kLater : 63>();
                else if (F::kOften) barrier_only();
            }
        }
        // The last step's reads, which nothing uses, keep their registers until they are done.
        lds_wait();
#pragma unroll
        for (int i = 0; i < RB; ++i) asm volatile("" ::"v"(af[0][i]), "v"(af[F::kAhead ? 1 : 0][i]));
        __builtin_amdgcn_s_waitcnt(0);       // the direct loads past the end have landed
        __syncthreads();                     // and no wave reads the buffers
        // (read here: after the next loads are issued the compiler would wait for them)
        bool far = false;
        if constexpr (!SPLIT) {
            const int4 seen = *reinterpret_cast<const int4*>(sm.far[turn & 1]);
            far = __builtin_amdgcn_readfirstlane(seen.x | seen.y | seen.z | seen.w);
        }
        const Tile done = tile;
        const bool more = next_tile(turn + 1, tile);
        if (more) begin(tile);

        // Outputs.  Lane (c, kg) holds row 16 i + c, columns 16 t + 4 kg + 0..3 of the wave's;
        // rows of 16 lanes swapped between blocks t and t + 1 make that eight columns a lane,
        // 64 bytes of a row of C a store.  Rows and columns past the end have offsets that the
        // buffer drops: the number of stores is the same for every tile.
        if constexpr (SPLIT) {
            const int lane = again(threadIdx.x & 63), c = lane & 15, kg = lane >> 4;
            const __amdgpu_buffer_rsrc_t pr = make_rsrc(a.parts + (done.part * a.M + done.row0) * a.N,
                                                        (uint32_t)done.rows * (uint32_t)a.N * 4u);
            const int64_t n0 = done.col0 + 16 * CB * wave + 4 * kg;
            uint32_t row = ((uint32_t)c * (uint32_t)a.N + (uint32_t)n0) * 4u, sixteen = 64u * (uint32_t)a.N;
            int left = done.rows;
#pragma unroll
            for (int i = 0; i < RB; ++i) {
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int t = 0; t < CB; ++t)
                    store16(pr, __builtin_bit_cast(u32x4, whole(acc[i][t])),
                            c < left && n0 + 16 * t < a.N ? row + 64u * t : kNowhere);
                row += sixteen;
                left -= 16;
            }
        } else {
            const int lane = again(threadIdx.x & 63), c = lane & 15, kg = lane >> 4;
            const __amdgpu_buffer_rsrc_t cr =
                make_rsrc(a.C + done.row0 * a.N, (uint32_t)done.rows * (uint32_t)a.N * 2u);
            const float* sr = sm.rows[turn & 1];
            const float* sc = sm.columns[turn & 1] + 16 * CB * wave + 4 * kg;
            float4_t sw[CB];
#pragma unroll
            for (int t = 0; t < CB; ++t) sw[t] = *reinterpret_cast<const float4_t*>(sc + 16 * t);
            uint32_t to[(CB + 1) / 2];
#pragma unroll
            for (int t = 0; t < CB; t += 2) {
                const int64_t n = done.col0 + 16 * CB * wave + (CB > 1 ? 16 * (t + (kg & 1)) + 8 * (kg >> 1) : 4 * kg);
                to[t / 2] = n < a.N ? (uint32_t)n * 2u : kNowhere;
            }
            uint32_t row = (uint32_t)c * (uint32_t)a.N * 2u, sixteen = 32u * (uint32_t)a.N;
            int left = done.rows;
            auto store_all = [&](auto is_bf, auto is_far) {
                constexpr bool bf = decltype(is_bf)::value;
#pragma unroll
                for (int i = 0; i < RB; ++i) {
                    __builtin_amdgcn_sched_barrier(0);
                    const float sa = sr[16 * i + c];
                    const bool here = c < left;
                    bool there = false;
                    if constexpr (decltype(is_far)::value) {
                        int64_t at = done.row0 + 16 * i + c;
                        if (GATHER && here) at = a.rows[at];
                        there = at >= 0 && at < a.a_rows;
                    }
                    auto scaled = [&](int t) {
                        if constexpr (decltype(is_far)::value) return w8_scaled_far(bf, whole(acc[i][t]), sa, sw[t], there);
                        else return w8_scaled(bf, whole(acc[i][t]), sa, sw[t]);
                    };
#pragma unroll
                    for (int t = 0; t < CB; t += 2) {
                        const uint32_t off = here && to[t / 2] != kNowhere ? row + to[t / 2] : kNowhere;
                        const uint2 x = scaled(t);
                        if constexpr (CB > 1) {
                            const uint2 y = scaled(t + 1);
                            store16(cr, rows_swapped(x, y), off);
                        } else {
                            store8(cr, x, off);
                        }
                    }
                    row += sixteen;
                    left -= 16;
                }
            };
            if (__builtin_expect(far, 0)) {
                if (a.bf) store_all(std::true_type{}, std::true_type{});
                else store_all(std::false_type{}, std::true_type{});
            } else {
                if (a.bf) store_all(std::true_type{}, std::false_type{});
                else store_all(std::false_type{}, std::false_type{});
            }
        }
        if (!more) return;
    }
}

// The place in the list of workgroup b's tile number k: each XCD (workgroups go to the
// eight in turn) has a contiguous part of the list and goes through it in order.  Past
// the end: -1.
__device__ __forceinline__ int place_of(int b, int grid, int k, int total) {
    const int per = total / kXcds, rem = total % kXcds, x = b % kXcds, i = b / kXcds + k * (grid / kXcds);
    return i < per + (x < rem ? 1 : 0) ? x * per + min(x, rem) + i : -1;
}

template <class F, bool SPLIT>
__global__ __launch_bounds__(kThreads, F::WGS) void w8a8_tile_kernel(W8Args a, int tiles_m, int tiles_n) {
    __shared__ __align__(16) TileShared<F> sm;
    auto next_tile = [&](int k, Tile& t) {
        int at = place_of(blockIdx.x, gridDim.x, k, tiles_m * tiles_n * (SPLIT ? a.splits : 1));
        if (at < 0) return false;
        if constexpr (SPLIT) {                        // parts of whole passes of the loop
            const int passes = (a.na + F::R - 1) / F::R;
            t.part = __builtin_amdgcn_readfirstlane(at % a.splits);
            t.from = passes * t.part / a.splits * F::R;
            t.steps = passes * (t.part + 1) / a.splits * F::R - t.from;
            at /= a.splits;
        }
        int tm, tn;
        tile_of<F>(at, tiles_m, tiles_n, tm, tn);
        t.packed = a.packed;
        t.row0 = (int64_t)__builtin_amdgcn_readfirstlane(tm) * F::BM;
        t.col0 = (int64_t)__builtin_amdgcn_readfirstlane(tn) * F::BN;
        t.rows = (int)min((int64_t)F::BM, a.M - t.row0);
        return true;
    };
    tile_products<F, false, SPLIT>(a, next_tile, sm);
}

// The parts' sums added, scaled and rounded: eight columns of a row a thread.
__global__ __launch_bounds__(256) void w8a8_join_kernel(W8Args a) {
    const int per_row = (int)(a.N / 8);
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= a.M * per_row) return;
    const int64_t m = i / per_row, n = (i - m * per_row) * 8;
    const float4_t* scales = reinterpret_cast<const float4_t*>(a.packed + a.s_off + n * 4);
    const float sa = a.a_scale[m];
    const float4_t sw[2] = {scales[0], scales[1]};
    const i32x4* p = reinterpret_cast<const i32x4*>(a.parts + m * a.N + n);
    i32x4 lo = p[0], hi = p[1];
    for (int s = 1; s < a.splits; ++s) {
        p += a.M * a.N / 4;
        lo += p[0];
        hi += p[1];
    }
    const uint2 x = w8_scaled_far(a.bf, lo, sa, sw[0], true), y = w8_scaled_far(a.bf, hi, sa, sw[1], true);
    *reinterpret_cast<u32x4*>(a.C + m * a.N + n) = u32x4{x.x, x.y, y.x, y.y};
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
    __syncthreads();                                  // the buffers take the place of these numbers
    auto next_tile = [&](int k, Tile& t) {
        const int at = place_of(blockIdx.x, gridDim.x, k, total * tiles_n);
        if (at < 0) return false;                     // (the whole workgroup)
        int tm, tn, f = from;
        tile_of<F>(at, total, tiles_n, tm, tn);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (tm >= f && tm < f + tiles[u]) {
                sm.found[0] = 4 * tid + u;
                sm.found[1] = start[u] + (tm - f) * F::BM;
                sm.found[2] = end[u];
            }
            f += tiles[u];
        }
        __syncthreads();
        t.packed = a.packed + __builtin_amdgcn_readfirstlane(sm.found[0]) * a.total;
        t.row0 = __builtin_amdgcn_readfirstlane(sm.found[1]);
        t.rows = min(F::BM, __builtin_amdgcn_readfirstlane(sm.found[2]) - (int)t.row0);
        t.col0 = (int64_t)__builtin_amdgcn_readfirstlane(tn) * F::BN;
        return true;                                  // (barriers follow before the next call)
    };
    tile_products<F, GATHER, false>(a, next_tile, sm);
}

template <class F>
int launch_form(const W8Args& a, hipStream_t s) {
    const int64_t tiles_n = (a.N + F::BN - 1) / F::BN;
    const int64_t tiles_m = a.experts ? std::min<int64_t>(a.M, a.M / F::BM + a.experts)      // at most
                                      : (a.M + F::BM - 1) / F::BM;
    // as many workgroups as run at a time, whole eights
    const int64_t most = (int64_t)device_cus(s) * F::WGS;
    const dim3 grid((unsigned)((std::min(tiles_m * tiles_n * a.splits, most) + kXcds - 1) / kXcds * kXcds));
    if constexpr (F::kSplits) {
        if (a.splits > 1) {
            const int rc = launch(w8a8_tile_kernel<F, true>, grid, dim3(kThreads), 0, s, a, (int)tiles_m, (int)tiles_n);
            if (rc) return rc;
            return launch(w8a8_join_kernel, dim3((unsigned)((a.M * (a.N / 8) + 255) / 256)), dim3(256), 0, s, a);
        }
    }
    if (!a.experts)
        return launch(w8a8_tile_kernel<F, false>, grid, dim3(kThreads), 0, s, a, (int)tiles_m, (int)tiles_n);
    return a.rows ? launch(w8a8_tile_experts_kernel<F, true>, grid, dim3(kThreads), 0, s, a, (int)tiles_n)
                  : launch(w8a8_tile_experts_kernel<F, false>, grid, dim3(kThreads), 0, s, a, (int)tiles_n);
}

}  // namespace

int launch_w8a8_tile(const W8Args& a, int form, hipStream_t s) {
    switch (form) {
        case 0: return launch_form<Form<16, 4, 4, 4, 1>>(a, s);
        case 1: return launch_form<Form<8, 4, 8, 8, 1>>(a, s);
        case 2: return launch_form<Form<8, 2, 8, 8, 1>>(a, s);
        case 3: return launch_form<Form<4, 2, 8, 8, 2>>(a, s);
        default: return launch_form<Form<4, 1, 8, 8, 2>>(a, s);
    }
}

}  // namespace tf
