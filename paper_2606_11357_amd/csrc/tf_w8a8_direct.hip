// Matrix product of int8 codes with a scale for each row and each column, for few
// rows (dense, or of each expert):
//   C[m, n] = s_a[m] s_w[n] sum_k qa[m, k] qw[k, n]
// Sums are int32 and exact (65536 products of at most 2^14), so the order in which
// they are added does not change them.  A workgroup owns 16 rows and 16 columns and
// deals K's atoms of 64 to its four waves in turn; each wave takes both operands
// straight into registers, a ring of eight atoms ahead, and the waves' sums are added
// in LDS.  Memory-bound: weights are read once for 16 rows, and every workgroup reads
// all of its rows.  16 columns and four waves a workgroup: N = 4096 is then one a compute
// unit.  One row, 4096 x 4096: 5.8 us (of which 3.3 are the memory's; with the outputs' scales
// loaded at the end 6.0, then 32 columns 6.6 and eight waves 6.0), 14336 x 4096: 13.6 us
// (4.3 TB/s; 32 columns 16.8); 16 rows 6.4 and 17.5 us.
#include "tf_w8a8.h"

namespace tf {
namespace {

__device__ __forceinline__ u32x4 load16(__amdgpu_buffer_rsrc_t r, uint32_t voff, uint32_t soff) {
    return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, voff, soff, 0));
}

constexpr uint32_t kNowhere = 0xFFFFFF00u;     // an offset that no buffer reaches: reads as zero
constexpr int kRows = 16, kWaves = 4, kThreads = 64 * kWaves, kRing = 8;

// Rows row0 .. row0 + rows - 1 by the columns of one panel.
__device__ __forceinline__ void direct_block(const W8Args& a, const uint8_t* packed, int panel, int64_t row0, int rows,
                                             i32x4* red) {
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 15, g = lane >> 4;
    // A: from its first row here on, or all of it where rows are gathered
    const int64_t base = a.rows ? 0 : row0;
    const int64_t a_bytes = max((a.a_rows - base) * a.K, (int64_t)0);        // (0: all of these rows are missing)
    const __amdgpu_buffer_rsrc_t ar = make_rsrc(a.A + base * a.K, (uint32_t)min(a_bytes, (int64_t)kNowhere));
    int64_t at = -1;
    if (c < rows) at = a.rows ? a.rows[row0 + c] : row0 + c;
    const bool there = at >= 0 && at < a.a_rows;
    const uint32_t a_off = there ? (uint32_t)((at - base) * a.K) + 16 * g : kNowhere;
    // The scales of the outputs, which the first wave stores: their loads go ahead.
    const int n = kW8Panel * panel + 4 * g;
    float sa = 0.f;
    float4_t sw{};
    if (wave == 0) {
        if (there) sa = a.a_scale[at];
        sw = *reinterpret_cast<const float4_t*>(packed + a.s_off + 4 * n);
    }
    const __amdgpu_buffer_rsrc_t br =
        make_rsrc(packed + (int64_t)panel * a.na * kW8AtomBytes, (uint32_t)a.na * kW8AtomBytes);

    u32x4 av[kRing], bv[kRing];
    // an atom past K is zeros in A, so whatever is there in B adds nothing
    auto load = [&](int d, int atom) {
        const bool in = atom < a.na;
        bv[d] = load16(br, 16 * lane, in ? (uint32_t)atom * kW8AtomBytes : 0);
        av[d] = load16(ar, in && a_off != kNowhere ? a_off + (uint32_t)atom * kW8AtomK : kNowhere, 0);
    };
    i32x4 acc{0, 0, 0, 0};
#pragma unroll
    for (int d = 0; d < kRing; ++d) load(d, wave + d * kWaves);
    for (int j = wave; j < a.na; j += kRing * kWaves) {
#pragma unroll
        for (int d = 0; d < kRing; ++d) {
            acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, bv[d]), __builtin_bit_cast(i32x4, av[d]),
                                                        acc, 0, 0, 0);
            load(d, j + (d + kRing) * kWaves);
        }
    }
    // Lane l of a wave has row l % 16, columns 4 (l / 16) + 0..3.
    red[tid] = acc;
    __syncthreads();
    if (tid >= 64) return;
    i32x4 sum = red[tid];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) sum += red[w * 64 + tid];
    if (c >= rows || n >= a.N) return;
    *reinterpret_cast<uint2*>(a.C + (row0 + c) * a.N + n) = w8_scaled_far(a.bf, sum, sa, sw, there);
}

// Dense: workgroup b has the columns of panel b % 8 + 8 (i / blocks) and the rows of
// block i % blocks, i = b / 8: blocks that share weights run on one XCD, one after
// the other.
__global__ __launch_bounds__(kThreads) void w8a8_direct_kernel(W8Args a, int blocks) {
    __shared__ i32x4 red[kThreads];
    const int i = blockIdx.x / 8, panel = blockIdx.x % 8 + 8 * (i / blocks);
    if (panel >= a.np) return;
    const int64_t row0 = (int64_t)(i % blocks) * kRows;
    direct_block(a, a.packed, panel, row0, (int)min(a.M - row0, (int64_t)kRows), red);
}

// By expert: a workgroup has a panel of one expert and goes through its rows.
__global__ __launch_bounds__(kThreads) void w8a8_direct_experts_kernel(W8Args a) {
    __shared__ i32x4 red[kThreads];
    const int e = blockIdx.y;
    int first, last;
    w8_slots(a, e, first, last);
    const uint8_t* packed = a.packed + e * a.total;
    for (int row0 = first; row0 < last; row0 += kRows) {
        if (row0 != first) __syncthreads();          // the sums of the rows before have been read
        direct_block(a, packed, blockIdx.x, row0, min(last - row0, kRows), red);
    }
}

}  // namespace

int launch_w8a8_direct(const W8Args& a, hipStream_t s) {
    if (a.experts)
        return launch(w8a8_direct_experts_kernel, dim3((unsigned)a.np, (unsigned)a.experts), dim3(kThreads), 0, s, a);
    const int64_t blocks = (a.M + kRows - 1) / kRows;
    const dim3 grid((unsigned)((a.np + 7) / 8 * 8 * blocks));
    return launch(w8a8_direct_kernel, grid, dim3(kThreads), 0, s, a, (int)blocks);
}

}  // namespace tf
