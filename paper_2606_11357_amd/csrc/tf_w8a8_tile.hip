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

constexpr int kBM = 256, kBN = 256, kThreads = 256, kXcds = 8;
constexpr int kRB = kBM / 16;                    // 16-row blocks
constexpr int kPairBytes = kBM * 128;            // A of two steps: 32 KB
constexpr int kPairs = 4;                        // buffers
constexpr int kRowGroup = 8;                     // row tiles that share the columns' order

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

__device__ __forceinline__ u32x4 load16(__amdgpu_buffer_rsrc_t r, uint32_t voff) {
    return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, voff, 0, 0));
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

struct TileShared {
    uint8_t a[kPairs * kPairBytes];
    float scale[kBM];
};

// Tile number `at` of row tiles x column tiles, rows in groups of kRowGroup.
__device__ __forceinline__ void tile_of(int at, int tiles_m, int tiles_n, int& tm, int& tn) {
    const int group = at / (kRowGroup * tiles_n), rest = at - group * kRowGroup * tiles_n;
    const int height = min(kRowGroup, tiles_m - group * kRowGroup);
    tn = rest / height;
    tm = group * kRowGroup + rest - tn * height;
}

// Rows row0 .. row0 + rows - 1 of C (A's, or those that a.rows names) by columns
// col0 .. col0 + 255 of `packed`.
template <bool GATHER>
__device__ __forceinline__ void tile_product(const W8Args& a, const uint8_t* packed, int64_t row0, int rows,
                                             int64_t col0, TileShared& sm) {
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 15, kg = lane >> 4;
    const int steps = a.na, pairs = steps / 2, chunks = (steps + 3) / 4;

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
    // Direct load r of wave w fills rows 64 w + 8 r .. + 7 of a buffer, eight lanes a row.
    uint32_t avoff[8];
#pragma unroll
    for (int r = 0; r < 8; ++r) {
        const int row = 64 * wave + 8 * r + (lane >> 3);
        const int at = row_of(row);
        avoff[r] = (uint32_t)(in(at) ? at : 0) * (uint32_t)a.K + (uint32_t)((lane & 7) ^ a_swz(row)) * 16u;
    }
    auto dma_a = [&](int pair, uint32_t buf, int r) {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(
            ar, (__attribute__((address_space(3))) void*)(sm.a + buf + (8 * wave + r) * 1024), 16,
            avoff[r] + (uint32_t)min(pair, pairs - 1) * 128u, 0, 0, 0);
    };
    const uint32_t lds = (uint32_t)reinterpret_cast<uintptr_t>(sm.a);
    uint32_t a_lane[2];
#pragma unroll
    for (int odd = 0; odd < 2; ++odd) a_lane[odd] = lds + (uint32_t)(c * 128 + ((kg + 4 * odd) ^ a_swz(c)) * 16);

    // B: this wave's four panels; one past N is empty, and so is what follows K.
    __amdgpu_buffer_rsrc_t wr[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const int64_t panel = col0 / kW8Panel + 4 * wave + t;
        const bool here = panel < a.np;
        wr[t] = make_rsrc(packed + (here ? panel : 0) * a.na * kW8AtomBytes, here ? (uint32_t)a.na * kW8AtomBytes : 0u);
    }
    u32x4 ring[4][4];
    auto load_b = [&](int step, int t, u32x4& v) { v = load16(wr[t], (uint32_t)(lane * 16 + step * kW8AtomBytes)); };

    uint32_t b0 = 0, b1 = kPairBytes, b2 = 2 * kPairBytes, b3 = 3 * kPairBytes;
#pragma unroll
    for (int r = 0; r < 8; ++r) dma_a(0, b0, r);
#pragma unroll
    for (int r = 0; r < 8; ++r) dma_a(1, b1, r);
#pragma unroll
    for (int j = 0; j < 3; ++j)
#pragma unroll
        for (int t = 0; t < 4; ++t) load_b(j, t, ring[j][t]);
#pragma unroll
    for (int r = 0; r < 8; ++r) dma_a(2, b2, r);
    i32x4 acc[kRB][4];
#pragma unroll
    for (int i = 0; i < kRB; ++i)
#pragma unroll
        for (int t = 0; t < 4; ++t) acc[i][t] = i32x4{0, 0, 0, 0};
    {
        const int at = row_of(tid);
        const float s = a.a_scale[in(at) ? base + at : 0];
        sm.scale[tid] = in(at) ? s : 0.f;
    }
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    u32x4 af[kRB];
#pragma unroll
    for (int i = 0; i < kRB / 2; ++i) af[i] = lds_read_block(a_lane[0] + b0, i);
    lds_wait();
    mfma_hazard_gap();

    // Step s = 4 ch + j, 64 slots of one matrix instruction (row block q / 4, column
    // block q % 4), each followed by at most one other:
    //   0         wait for the fragments of row blocks 0..7
    //   0..7      fragments of blocks 8..15
    //   8..14     direct loads 4 (j % 2) .. + 3 of the pair three ahead
    //   16..28    weights of step s + 3
    //   32        wait for blocks 8..15
    //   32..39    fragments of blocks 0..7 of step s + 1
    // A pair is read from half a step before its first step on: at the end of the even
    // step before, its direct loads have to have landed, which leaves this wave's later
    // operations: the weights of the step of its last direct loads, and eight operations
    // in each of three steps since.  The barrier of odd steps frees the pair's buffer.
    for (int ch = 0; ch < chunks; ++ch) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int step = 4 * ch + j, odd = j & 1;
            const uint32_t bcur = j < 2 ? b0 : b1;
            const uint32_t bnxt = j == 0 ? b0 : (j == 3 ? b2 : b1);
            const uint32_t bdma = j < 2 ? b3 : b0;
            const int dpair = 2 * ch + 3 + (j >> 1);
#pragma unroll
            for (int q = 0; q < 64; ++q) {
                const int i = q / 4, t = q % 4;
                __builtin_amdgcn_sched_barrier(0);
                if (q == 0 || q == 32) lds_wait();
                mfma_i8(acc[i][t], ring[j][t], af[i]);
                if (q < 8) af[8 + q] = lds_read_block(a_lane[odd] + bcur, 8 + q);
                if (q >= 32 && q < 40) af[q - 32] = lds_read_block(a_lane[odd ^ 1] + bnxt, q - 32);
                if (q >= 8 && q < 16 && q % 2 == 0) dma_a(dpair, bdma, 4 * odd + (q - 8) / 2);
                if (q >= 16 && q < 32 && q % 4 == 0) load_b(step + 3, (q - 16) / 4, ring[(j + 3) % 4][(q - 16) / 4]);
            }
            if (odd) barrier_only();
            else barrier_after_loads<4 + 3 * 8>();
        }
        const uint32_t x0 = b0, x1 = b1;
        b0 = b2;
        b1 = b3;
        b2 = x0;
        b3 = x1;
    }
    mfma_hazard_gap();
    __builtin_amdgcn_s_waitcnt(0);       // the direct loads past the end have landed
    __syncthreads();                     // and no wave reads the buffers, which the output passes through

    // A row block at a time through LDS (rows of 144 bytes), stored as 16 bytes a
    // lane, eight whole 128-byte rows an instruction.
    const float* scales = reinterpret_cast<const float*>(packed + a.s_off);
    const int64_t wcol = col0 + 64 * wave;
    float4_t sw[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const int64_t n = wcol + 16 * t + 4 * kg;
        sw[t] = n < a.np * 16 ? *reinterpret_cast<const float4_t*>(scales + n) : float4_t{0.f, 0.f, 0.f, 0.f};
    }
    uint8_t* stage = sm.a + wave * 4096;
    constexpr int kStageRow = 144;
    const int rr = lane >> 3, cc = lane & 7;
#pragma unroll
    for (int i = 0; i < kRB; ++i) {
        __builtin_amdgcn_sched_barrier(0);
        const float sa = sm.scale[16 * i + c];
#pragma unroll
        for (int t = 0; t < 4; ++t)
            *reinterpret_cast<uint2*>(stage + c * kStageRow + 32 * t + 8 * kg) = w8_scaled(a.bf, acc[i][t], sa, sw[t]);
        __builtin_amdgcn_s_waitcnt(0xC07F);       // lgkmcnt(0): this wave's stores landed
        u32x4 v[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) v[h] = *reinterpret_cast<const u32x4*>(stage + (rr + 8 * h) * kStageRow + 16 * cc);
        __builtin_amdgcn_s_waitcnt(0xC07F);       // read before the area is written again
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int r = 16 * i + rr + 8 * h;
            const int64_t n = wcol + 8 * cc;
            if (r < rows && n < a.N) *reinterpret_cast<u32x4*>(a.C + (row0 + r) * a.N + n) = v[h];
        }
    }
}

// The place in the list of workgroup b's tile: each XCD (workgroups go to the eight in
// turn) has a contiguous part of the list.  Past the end: -1.
__device__ __forceinline__ int place_of(int b, int total) {
    const int per = total / kXcds, rem = total % kXcds, x = b % kXcds, i = b / kXcds;
    return i < per + (x < rem ? 1 : 0) ? x * per + min(x, rem) + i : -1;
}

__global__ __launch_bounds__(kThreads, 1) void w8a8_tile_kernel(W8Args a, int tiles_m, int tiles_n) {
    __shared__ __align__(16) TileShared sm;
    const int at = place_of(blockIdx.x, tiles_m * tiles_n);
    if (at < 0) return;
    int tm, tn;
    tile_of(at, tiles_m, tiles_n, tm, tn);
    tm = __builtin_amdgcn_readfirstlane(tm);
    tn = __builtin_amdgcn_readfirstlane(tn);
    const int64_t row0 = (int64_t)tm * kBM;
    tile_product<false>(a, a.packed, row0, (int)min((int64_t)kBM, a.M - row0), (int64_t)tn * kBN, sm);
}

// By expert: the row tiles of all experts in one list, found from the offsets by
// every workgroup (thread t has experts 4 t .. 4 t + 3).
template <bool GATHER>
__global__ __launch_bounds__(kThreads, 1) void w8a8_tile_experts_kernel(W8Args a, int tiles_n) {
    __shared__ __align__(16) TileShared sm;
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
        tiles[u] = (end[u] - start[u] + kBM - 1) / kBM;
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
    tile_of(at, total, tiles_n, tm, tn);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        if (tm >= from && tm < from + tiles[u]) {
            ints[16] = 4 * tid + u;
            ints[17] = start[u] + (tm - from) * kBM;
            ints[18] = end[u];
        }
        from += tiles[u];
    }
    __syncthreads();
    const int e = __builtin_amdgcn_readfirstlane(ints[16]), row0 = __builtin_amdgcn_readfirstlane(ints[17]);
    const int rows = min(kBM, __builtin_amdgcn_readfirstlane(ints[18]) - row0);
    tn = __builtin_amdgcn_readfirstlane(tn);
    __syncthreads();                                  // the buffers take this place
    tile_product<GATHER>(a, a.packed + e * a.total, row0, rows, (int64_t)tn * kBN, sm);
}

}  // namespace

int launch_w8a8_tile(const W8Args& a, hipStream_t s) {
    const int64_t tiles_n = (a.N + kBN - 1) / kBN;
    if (a.experts) {
        const int64_t most = std::min<int64_t>(a.M, a.M / kBM + a.experts);     // row tiles
        const dim3 grid((unsigned)((most * tiles_n + 7) / 8 * 8));
        return a.rows ? launch(w8a8_tile_experts_kernel<true>, grid, dim3(kThreads), 0, s, a, (int)tiles_n)
                      : launch(w8a8_tile_experts_kernel<false>, grid, dim3(kThreads), 0, s, a, (int)tiles_n);
    }
    const int64_t tiles_m = (a.M + kBM - 1) / kBM;
    return launch(w8a8_tile_kernel, dim3((unsigned)((tiles_m * tiles_n + 7) / 8 * 8)), dim3(kThreads), 0, s, a,
                  (int)tiles_m, (int)tiles_n);
}

}  // namespace tf
