// Matrix product of int8 codes with a scale for each row and each column, for few
// rows (dense, or of each expert):
//   C[m, n] = s_a[m] s_w[n] sum_k qa[m, k] qw[k, n]
// Sums are int32 and exact (65536 products of at most 2^14), so the order in which
// they are added does not change them.  A workgroup owns 16 MB rows and 16 PN
// columns and deals K's atoms of 64 to its waves in turn; each wave takes both
// operands straight into registers, a ring of D atoms ahead, and the waves' sums
// are added in LDS.  Memory-bound: weights are read once, and every workgroup reads all
// of its rows.  16 columns and four waves a workgroup: N = 4096 is then one a compute
// unit.  One row, 4096 x 4096: 6.0 us (of which 3.3 are the memory's; 32 columns 6.6, eight
// waves 6.0), 14336 x 4096: 13.6 us (4.3 TB/s; 32 columns 16.8); 16 rows 6.4 and 17.3 us.
#include <algorithm>

#include "tf_w8a8.h"

namespace tf {
namespace {

__device__ __forceinline__ u32x4 load16(__amdgpu_buffer_rsrc_t r, uint32_t voff, uint32_t soff) {
    return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, voff, soff, 0));
}

constexpr uint32_t kNowhere = 0xFFFFFF00u;     // an offset that no buffer reaches: reads as zero

template <int MB, int PN, int WAVES, int D>
__device__ __forceinline__ void direct_block(const W8Args& a, const uint8_t* packed, int panel0, int64_t row0, int rows,
                                             i32x4* red) {
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 15, g = lane >> 4;
    // A: from its first row here on, or all of it where rows are gathered
    const int64_t base = a.rows ? 0 : row0;
    const int64_t a_bytes = max((a.a_rows - base) * a.K, (int64_t)0);        // (0: all of these rows are missing)
    const __amdgpu_buffer_rsrc_t ar = make_rsrc(a.A + base * a.K, (uint32_t)min(a_bytes, (int64_t)kNowhere));
    uint32_t a_off[MB];
    int64_t a_row[MB];
#pragma unroll
    for (int b = 0; b < MB; ++b) {
        const int r = 16 * b + c;
        int64_t at = -1;
        if (r < rows) at = a.rows ? a.rows[row0 + r] : row0 + r;
        const bool in = at >= 0 && at < a.a_rows;
        a_row[b] = in ? at : -1;
        a_off[b] = in ? (uint32_t)((at - base) * a.K) + 16 * g : kNowhere;
    }
    const int panels = min(PN, a.np - panel0);
    const __amdgpu_buffer_rsrc_t br =
        make_rsrc(packed + (int64_t)panel0 * a.na * kW8AtomBytes, (uint32_t)panels * a.na * kW8AtomBytes);
    uint32_t b_off[PN];
#pragma unroll
    for (int p = 0; p < PN; ++p) b_off[p] = (uint32_t)p * a.na * kW8AtomBytes + 16 * lane;

    u32x4 av[D][MB], bv[D][PN];
    // an atom past K is zeros in A, so whatever is there in B adds nothing
    auto load = [&](int d, int atom) {
        const bool in = atom < a.na;
#pragma unroll
        for (int p = 0; p < PN; ++p) bv[d][p] = load16(br, b_off[p], in ? (uint32_t)atom * kW8AtomBytes : 0);
#pragma unroll
        for (int b = 0; b < MB; ++b)
            av[d][b] = load16(ar, in && a_off[b] != kNowhere ? a_off[b] + (uint32_t)atom * kW8AtomK : kNowhere, 0);
    };
    i32x4 acc[PN][MB];
#pragma unroll
    for (int p = 0; p < PN; ++p)
#pragma unroll
        for (int b = 0; b < MB; ++b) acc[p][b] = i32x4{0, 0, 0, 0};
#pragma unroll
    for (int d = 0; d < D; ++d) load(d, wave + d * WAVES);
    for (int j = wave; j < a.na; j += D * WAVES) {
#pragma unroll
        for (int d = 0; d < D; ++d) {
#pragma unroll
            for (int p = 0; p < PN; ++p)
#pragma unroll
                for (int b = 0; b < MB; ++b)
                    acc[p][b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, bv[d][p]),
                                                                      __builtin_bit_cast(i32x4, av[d][b]), acc[p][b],
                                                                      0, 0, 0);
            load(d, j + (d + D) * WAVES);
        }
    }
    // Block (p, b) of a wave: lane l has row 16 b + l % 16, columns 16 p + 4 (l / 16) + 0..3.
#pragma unroll
    for (int p = 0; p < PN; ++p)
#pragma unroll
        for (int b = 0; b < MB; ++b) red[(wave * PN * MB + p * MB + b) * 64 + lane] = acc[p][b];
    __syncthreads();
    const float* scales = reinterpret_cast<const float*>(packed + a.s_off);
    for (int i = tid; i < PN * MB * 64; i += WAVES * 64) {
        i32x4 sum = red[i];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) sum += red[w * PN * MB * 64 + i];
        const int l = i & 63, b = (i >> 6) % MB, p = (i >> 6) / MB;
        const int r = 16 * b + (l & 15), n = 16 * (panel0 + p) + 4 * (l >> 4);
        if (r >= rows || n >= a.N) continue;
        const int64_t at = a.rows ? a.rows[row0 + r] : row0 + r;
        const float sa = at >= 0 && at < a.a_rows ? a.a_scale[at] : 0.f;
        const float4_t sw = *reinterpret_cast<const float4_t*>(scales + n);
        *reinterpret_cast<uint2*>(a.C + (row0 + r) * a.N + n) = w8_scaled(a.bf, sum, sa, sw);
    }
}

// Dense: workgroup b has the columns of group b % 8 + 8 (i / blocks) and the rows of
// block i % blocks, i = b / 8: blocks that share weights run on one XCD, one after
// the other.
template <int MB, int PN, int WAVES, int D>
__global__ __launch_bounds__(WAVES * 64) void w8a8_direct_kernel(W8Args a, int blocks, int groups) {
    __shared__ i32x4 red[WAVES * PN * MB * 64];
    const int i = blockIdx.x / 8, group = blockIdx.x % 8 + 8 * (i / blocks);
    if (group >= groups) return;
    const int64_t row0 = (int64_t)(i % blocks) * 16 * MB;
    direct_block<MB, PN, WAVES, D>(a, a.packed, group * PN, row0, (int)min(a.M - row0, (int64_t)16 * MB), red);
}

// By expert: a workgroup has PN panels of one expert and goes through its rows.
template <int MB, int PN, int WAVES, int D>
__global__ __launch_bounds__(WAVES * 64) void w8a8_direct_experts_kernel(W8Args a) {
    __shared__ i32x4 red[WAVES * PN * MB * 64];
    const int e = blockIdx.y;
    int first, last;
    w8_slots(a, e, first, last);
    const uint8_t* packed = a.packed + e * a.total;
    for (int row0 = first; row0 < last; row0 += 16 * MB) {
        if (row0 != first) __syncthreads();          // the sums of the rows before have been read
        direct_block<MB, PN, WAVES, D>(a, packed, blockIdx.x * PN, row0, min(last - row0, 16 * MB), red);
    }
}

template <int MB, int PN, int WAVES, int D>
int launch_direct(const W8Args& a, hipStream_t s) {
    const int groups = (a.np + PN - 1) / PN;
    if (a.experts) {
        const dim3 grid((unsigned)groups, (unsigned)a.experts);
        return launch(w8a8_direct_experts_kernel<MB, PN, WAVES, D>, grid, dim3(WAVES * 64), 0, s, a);
    }
    const int64_t blocks = (a.M + 16 * MB - 1) / (16 * MB);
    const dim3 grid((unsigned)((groups + 7) / 8 * 8 * blocks));
    return launch(w8a8_direct_kernel<MB, PN, WAVES, D>, grid, dim3(WAVES * 64), 0, s, a, (int)blocks, groups);
}

}  // namespace

int launch_w8a8_direct(const W8Args& a, hipStream_t s) { return launch_direct<1, 1, 4, 8>(a, s); }

}  // namespace tf
