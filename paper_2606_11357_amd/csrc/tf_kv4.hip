// The 4-bit paged key/value cache: append (with the rotation of queries and
// keys on the way) and read back.
#include "tf_kv4.h"

namespace tf {
namespace {

typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));

// Values (of keys, and as many of values) from which a read goes tile by tile.
// Measured, 8 heads of 128, us row by row and tile by tile: 2000 tokens (2 M
// values) 5.4 / 6.3, 4097 8.5 / 7.7, 8192 13.2 / 10.9.
constexpr int64_t kTileValues = 1 << 22;
// What a sequence has to have of them for that, and of tokens: each brings tiles of
// which part is read for nothing.  And the most sequences, in all and by the elements
// of a token: a workgroup for tiles looks through all of them.  Measured likewise,
// tokens x sequences: 8 heads of 128, 1 x 5120 14.5 / 619, 16 x 320 9.5 / 14.4, 64 x 80
// 8.5 / 8.3, 64 x 1024 91 / 81, 128 x 2048 578 / 464, 256 x 4000 2285 / 3767; 2 of 256,
// 64 x 512 24.8 / 20.9; 4 of 64, 64 x 512 18.0 / 19.8, 128 x 1024 65.7 / 63.8, 128 x
// 2048 139 / 178; 1 of 64, 512 x 128 7.8 / 9.4, 8192 x 64 42 / 45.
constexpr int64_t kTileValuesEach = 1 << 15, kTileTokensEach = 64, kTileLeastElements = 128, kTileMostBatch = 2048;
constexpr int kStagedBatch = 1024;     // up to this many sequences' offsets are searched in LDS

struct AppendArgs {
    Kv4 cache;
    const uint16_t *q, *k, *v;
    int64_t q_stride, k_stride, v_stride;
    const float *cos, *sin;
    int64_t positions;
    const int32_t *cu, *starts;
    int batch, q_heads;
    int64_t tokens;
    uint16_t *q_out, *k_out;
    Divisor by_rows;                  // q_heads + 2 kv_heads
};

// Offsets of up to kStagedBatch sequences in LDS (a search of log2(batch)
// dependent steps costs LDS latency there); more are searched where they are.
__device__ __forceinline__ const int32_t* stage_offsets(const int32_t* cu, int batch, int32_t* lds) {
    if (batch > kStagedBatch) return cu;
    for (int i = threadIdx.x; i <= batch; i += blockDim.x) lds[i] = cu[i];
    __syncthreads();
    return lds;
}

// max over the lanes of one row (LPR consecutive lanes, a power of two)
template <int LPR>
__device__ __forceinline__ float row_max(float v) {
#pragma unroll
    for (int d = 1; d < LPR; d <<= 1) v = fmaxf(v, __shfl_xor(v, d));
    return v;
}

// Scale and zero-point of a row from its least and largest value, as rounded
// to 16 bits, and the fp32 forms that the codes are made with.
struct RowQuant {
    uint16_t s16, z16;
    float inv, z;        // code = round(x * inv + z); inv = 0, z = 0 where all codes are 0
};

// Every step is a rounded fp32 operation of its own (no contraction), so the
// codes are those of the formula wherever it is computed in fp32.
template <bool BF>
__device__ __forceinline__ RowQuant row_quant(float lo, float hi) {
#pragma clang fp contract(off)
    RowQuant r;
    const float fifteenth = 1.0f / 15.0f;
    const float a = hi * fifteenth, b = lo * fifteenth;
    r.s16 = round_out<BF>(a - b);
    float s = scale_f32<BF>(r.s16);
    if (!(s < __builtin_inff())) {                    // a value that is not finite (hi = inf), or too large a range
        r.s16 = BF ? 0x7FC0 : 0x7E00;                 // NaN
        r.z16 = 0;
        r.inv = r.z = 0.f;
    } else if (s <= 0x1p-100f || fabsf(lo) > 32768.0f * s) {
        r.s16 = round_out<BF>(lo);                    // lo * (0 - (-1))
        r.z16 = round_out<BF>(-1.0f);
        r.inv = r.z = 0.f;
    } else {
        r.z16 = round_out<BF>(-lo / s);
        r.inv = 1.0f / s;
        r.z = scale_f32<BF>(r.z16);
    }
    return r;
}

__device__ __forceinline__ uint32_t code_of(float x, const RowQuant& r) {
#pragma clang fp contract(off)
    const float p = x * r.inv;
    const float t = fminf(fmaxf(rintf(p + r.z), 0.0f), 15.0f);
    return (uint32_t)t;
}

// A row of D values (a query, key or value of one token and head) on D / 16
// lanes: lane i holds dims 8 i .. + 7 and their partners D/2 + 8 i .. + 7, so the
// rotation needs no exchange and both operands come in 16-byte loads.
struct Row {
    u16x8 a, b;          // as loaded
    int kind, h;         // 0 query, 1 key, 2 value; head
    int64_t t;           // packed token
    uint32_t pos;        // its position, where known
    bool active, known;  // a row of the call; one with a position (and angles)
};

template <int D>
__device__ __forceinline__ void load_row(const AppendArgs& a, Row& r, int i) {
    const uint16_t* src = (r.kind == 0   ? a.q + r.t * a.q_stride
                           : r.kind == 1 ? a.k + r.t * a.k_stride
                                         : a.v + r.t * a.v_stride) +
                          (int64_t)r.h * D + 8 * i;
    r.a = r.b = u16x8{};
    if (r.active) {
        r.a = *reinterpret_cast<const u16x8*>(src);
        r.b = *reinterpret_cast<const u16x8*>(src + D / 2);
    }
}

// Rotates, writes the 16-bit outputs, and quantizes a key or value into its
// tile (null: nowhere).  All lanes of the wave; tile() is asked once per row.
template <bool BF, int D, typename TileOf>
__device__ __forceinline__ void append_row(const AppendArgs& a, const Row& r, int i, TileOf tile_of) {
    constexpr int LPR = D / 16;
    float lo[8], hi[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        lo[j] = scale_f32<BF>(r.a[j]);
        hi[j] = scale_f32<BF>(r.b[j]);
    }
    if (a.cos && r.kind < 2 && r.known) {
#pragma clang fp contract(off)
        const float* cp = a.cos + (int64_t)r.pos * (D / 2) + 8 * i;
        const float* sp = a.sin + (int64_t)r.pos * (D / 2) + 8 * i;
        float c[8], s[8];
#pragma unroll
        for (int j = 0; j < 8; j += 4) {
            const float4_t cv = *reinterpret_cast<const float4_t*>(cp + j);
            const float4_t sv = *reinterpret_cast<const float4_t*>(sp + j);
#pragma unroll
            for (int m = 0; m < 4; ++m) { c[j + m] = cv[m]; s[j + m] = sv[m]; }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float ac = lo[j] * c[j], bs = hi[j] * s[j];
            const float bc = hi[j] * c[j], as = lo[j] * s[j];
            lo[j] = ac - bs;
            hi[j] = bc + as;
        }
    }
    uint16_t* out = r.kind == 0 ? a.q_out : r.kind == 1 ? a.k_out : nullptr;
    if (r.active && out) {
        uint16_t* o = out + (r.t * (r.kind == 0 ? a.q_heads : a.cache.kv_heads) + r.h) * D + 8 * i;
        const uint16_t nan16 = BF ? 0x7FC0 : 0x7E00;
        u16x8 oa, ob;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            oa[j] = r.known ? round_out<BF>(lo[j]) : nan16;
            ob[j] = r.known ? round_out<BF>(hi[j]) : nan16;
        }
        store_past(reinterpret_cast<u16x8*>(o), oa);
        store_past(reinterpret_cast<u16x8*>(o + D / 2), ob);
    }
    if (!__any(r.active && r.kind != 0 && r.known)) return;       // queries only
    // the row's range over its lanes
    float least = lo[0], most = lo[0], total = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        least = fminf(least, fminf(lo[j], hi[j]));
        most = fmaxf(most, fmaxf(lo[j], hi[j]));
        total = fmaf(hi[j], 0.f, fmaf(lo[j], 0.f, total));    // 0, or NaN where one is not finite
    }
    if (!(total == 0.f)) most = __builtin_inff();
    least = -row_max<LPR>(-least);
    most = row_max<LPR>(most);
    if (!r.active || r.kind == 0 || !r.known) return;
    uint8_t* tile = tile_of();
    if (!tile) return;
    const RowQuant rq = row_quant<BF>(least, most);
    uint32_t qa[8], qb[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        qa[j] = code_of(lo[j], rq);
        qb[j] = code_of(hi[j], rq);
    }
    const int kk = (int)(r.pos % kKvTile), u = kk >> 4, c = kk & 15, g = c >> 2, jj = c & 3;
    if (r.kind == 1) {
        // two words of 8 codes: dims 8 i (lane group 8 i / (D/4)) and D/2 + 8 i
        uint32_t wa = 0, wb = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            wa |= qa[2 * e] << (4 * e) | qa[2 * e + 1] << (16 + 4 * e);
            wb |= qb[2 * e] << (4 * e) | qb[2 * e + 1] << (16 + 4 * e);
        }
        constexpr int WPL = D / 32;                     // words per lane
        const int gk = i / WPL, w = i % WPL;
        *reinterpret_cast<uint32_t*>(tile + kv4_word<D>(u, gk * 16 + c, w)) = wa;
        *reinterpret_cast<uint32_t*>(tile + kv4_word<D>(u, (gk + 2) * 16 + c, w)) = wb;
    } else {
        uint8_t* vt = tile + 16 * D;
        const uint32_t flip = jj & 1 ? 0xFFu : 0u;       // odd keys as 15 - q
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int d = 8 * i + j;                     // below D/2
            vt[kv4_word<D>(u, g * 16 + (d & 15), d >> 4) + kv4_byte(jj)] = (uint8_t)((qa[j] | qb[j] << 4) ^ flip);
        }
    }
    if (i == 0) {
        uint16_t* meta = reinterpret_cast<uint16_t*>(tile + 32 * D) + g * 32 + (r.kind == 1 ? 0 : 16) + 4 * u + jj;
        meta[0] = rq.s16;
        meta[8] = rq.z16;
    }
}

// The row at place `at` of (token, row of the token) pairs.
__device__ __forceinline__ void place_row(const AppendArgs& a, const int32_t* cu, uint32_t at, Row& r, int& sequence) {
    const uint32_t t = a.by_rows.of(at);      // (at is below 2^30: at least four lanes a row)
    r.active = t < a.tokens;
    r.t = r.active ? t : 0;
    const int row = r.active ? (int)(at - t * a.by_rows.d) : 0;
    r.kind = row < a.q_heads ? 0 : row < a.q_heads + a.cache.kv_heads ? 1 : 2;
    r.h = row - (r.kind == 0 ? 0 : r.kind == 1 ? a.q_heads : a.q_heads + a.cache.kv_heads);
    sequence = owner_of(cu, a.batch, r.t);
    const int64_t pos = sequence < 0 ? -1 : (int64_t)a.starts[sequence] + (r.t - cu[sequence]);
    r.known = pos >= 0 && pos <= INT32_MAX && (!a.cos || pos < a.positions);
    r.pos = (uint32_t)pos;
}

// Every row of every token in order, one row on D / 16 lanes.  Moves 2 bytes a
// value in, 2 out for rotated rows and D + 8 bytes a cached key and value; where
// tokens are many it is bound by the vector unit (91% busy: rotation, ranges,
// codes) and by these, else by a chain of four dependent loads (offsets, start,
// page, angles).  Two and four rows a lane group were no faster.  Measured (bf16,
// 32/8 heads of 128): 4 x 4096 tokens 88 us (93 with the rotated rows through the
// L2), one token each of 64 sequences 5.0.
template <bool BF, int D>
__global__ __launch_bounds__(256) void kv4_append_kernel(AppendArgs a) {
    constexpr int LPR = D / 16;
    __shared__ int32_t lds_cu[kStagedBatch + 1];
    const int32_t* cu = stage_offsets(a.cu, a.batch, lds_cu);
    const int i = threadIdx.x % LPR;
    Row r;
    int b;
    place_row(a, cu, blockIdx.x * (256 / LPR) + threadIdx.x / LPR, r, b);
    load_row<D>(a, r, i);
    append_row<BF, D>(a, r, i, [&] { return kv4_tile(a.cache, b, r.pos, r.h, kv4_tile_bytes(D)); });
}

// Tiles of the cache that the tokens of a call touch: sequence by sequence,
// with the tokens that no sequence owns, before cu[0] and from cu[batch] on, as
// two more.  slot -> its sequence, tile and the packed token of its key 0.
struct TileSlot {
    int sequence = -2;               // -1: unowned tokens; -2: no such slot
    int32_t tile;                    // may be negative (positions below 0)
    int64_t t0;                      // packed token of the tile's first position
    int64_t from, to;                // the sequence's packed tokens

    static __device__ __forceinline__ void range(const int32_t* cu, int batch, int64_t tokens, int i, int64_t& from,
                                                 int64_t& to) {
        from = i == 0 ? 0 : cu[i - 1];
        to = i > batch ? tokens : cu[i];
        from = from < 0 ? 0 : from;
        to = to > tokens ? tokens : to;
    }
    static __device__ __forceinline__ int32_t start_of(const int32_t* starts, int batch, int i) {
        return i == 0 || i > batch ? 0 : starts[i - 1];
    }
    static __device__ __forceinline__ uint32_t tiles_of(int64_t from, int64_t to, int32_t start) {
        if (to <= from) return 0;
        return (uint32_t)((((int64_t)start + (to - from) - 1) >> 5) - (start >> 5) + 1);
    }
    // All 256 threads; before: 257 words of LDS, scratch: 4.
    __device__ __forceinline__ TileSlot(const int32_t* cu, const int32_t* starts, int batch, int64_t tokens,
                                        uint32_t slot, uint32_t* before, uint32_t* scratch) {
        const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = batch + 2, seg = (n + 255) / 256;
        uint32_t sum = 0;
        for (int i = tid * seg; i < (tid + 1) * seg && i < n; ++i) {
            range(cu, batch, tokens, i, from, to);
            sum += tiles_of(from, to, start_of(starts, batch, i));
        }
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t o = __shfl_up(sum, d);
            if (lane >= d) sum += o;
        }
        if (lane == 63) scratch[wave] = sum;
        __syncthreads();
        for (int w = 0; w < wave; ++w) sum += scratch[w];
        before[tid + 1] = sum;
        if (tid == 0) before[0] = 0;
        __syncthreads();
        if (slot >= before[256]) return;
        int s0 = 0, s1 = 256;
        while (s1 - s0 > 1) {
            const int mid = (s0 + s1) >> 1;
            if (before[mid] <= slot) s0 = mid;
            else s1 = mid;
        }
        int i = s0 * seg;
        uint32_t done = before[s0];
        int32_t start;
        for (;; ++i) {
            range(cu, batch, tokens, i, from, to);
            start = start_of(starts, batch, i);
            const uint32_t k = tiles_of(from, to, start);
            if (slot < done + k) break;
            done += k;
        }
        sequence = i == 0 || i > batch ? -1 : __builtin_amdgcn_readfirstlane(i - 1);
        tile = (start >> 5) + (int32_t)(slot - done);
        t0 = from + ((int64_t)tile * kKvTile - start);
    }
};

struct ReadArgs {
    Kv4 cache;
    const int32_t *cu, *starts;
    int batch;
    int64_t tokens;
    uint16_t *k, *v;
};

// Few tokens of a sequence at a time: one row on D / 16 lanes, as in the append.
// Bound by the same chain of loads: 777 tokens of one head of 256 3.8 us.
template <bool BF, int D>
__global__ __launch_bounds__(256) void kv4_read_kernel(ReadArgs a) {
    constexpr int LPR = D / 16;
    __shared__ int32_t lds_cu[kStagedBatch + 1];
    const int32_t* cu = stage_offsets(a.cu, a.batch, lds_cu);
    const int rows = 2 * a.cache.kv_heads;
    const uint32_t at = blockIdx.x * (256 / LPR) + threadIdx.x / LPR;
    const int i = threadIdx.x % LPR;
    if (at >= a.tokens * rows) return;
    const int64_t t = at / (uint32_t)rows;
    const int row = (int)(at % (uint32_t)rows);
    const bool is_v = row >= a.cache.kv_heads;
    const int h = row - (is_v ? a.cache.kv_heads : 0);
    const int b = owner_of(cu, a.batch, t);
    const int64_t pos = b < 0 ? -1 : (int64_t)a.starts[b] + (t - cu[b]);
    constexpr int64_t TB = kv4_tile_bytes(D);
    const uint8_t* tile = pos < 0 || pos > INT32_MAX ? nullptr : kv4_tile(a.cache, b, (uint32_t)pos, h, TB);
    uint16_t* o = (is_v ? a.v : a.k) + (t * a.cache.kv_heads + h) * D + 8 * i;
    u16x8 oa, ob;
    if (!tile) {
#pragma unroll
        for (int j = 0; j < 8; ++j) oa[j] = ob[j] = BF ? 0x7FC0 : 0x7E00;
    } else {
        const int kk = (int)(pos % kKvTile), u = kk >> 4, c = kk & 15, g = c >> 2, jj = c & 3;
        const uint16_t* meta = reinterpret_cast<const uint16_t*>(tile + 32 * D) + g * 32 + (is_v ? 16 : 0) + 4 * u + jj;
        const float s = scale_f32<BF>(meta[0]), z = scale_f32<BF>(meta[8]);
        uint32_t qa[8], qb[8];
        if (!is_v) {
            constexpr int WPL = D / 32;
            const int gk = i / WPL, w = i % WPL;
            const uint32_t wa = *reinterpret_cast<const uint32_t*>(tile + kv4_word<D>(u, gk * 16 + c, w));
            const uint32_t wb = *reinterpret_cast<const uint32_t*>(tile + kv4_word<D>(u, (gk + 2) * 16 + c, w));
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int sh = 4 * (j >> 1) + 16 * (j & 1);
                qa[j] = wa >> sh & 15;
                qb[j] = wb >> sh & 15;
            }
        } else {
            const uint8_t* vt = tile + 16 * D;
            const uint32_t flip = jj & 1 ? 0xFFu : 0u;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int d = 8 * i + j;
                const uint32_t byte = vt[kv4_word<D>(u, g * 16 + (d & 15), d >> 4) + kv4_byte(jj)] ^ flip;
                qa[j] = byte & 15;
                qb[j] = byte >> 4;
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            oa[j] = round_out<BF>(((float)qa[j] - z) * s);
            ob[j] = round_out<BF>(((float)qb[j] - z) * s);
        }
    }
    store_past(reinterpret_cast<u16x8*>(o), oa);
    store_past(reinterpret_cast<u16x8*>(o + D / 2), ob);
}

// Many tokens of a sequence: a wave takes the keys (or values) of one head for
// one tile, whose lines it reads whole.  HBM-bound, by the 4 D bytes that it
// writes a token and head against D + 8 read: 4 sequences of up to 16384 tokens,
// 8 heads of 128, 32 us, 5.8 TB/s (46 with the outputs through the L2).
template <bool BF, int D>
__global__ __launch_bounds__(256) void kv4_read_tiles_kernel(ReadArgs a, uint32_t wgs_per_slot) {
    __shared__ uint32_t before[257], scratch[4];
    const TileSlot ts(a.cu, a.starts, a.batch, a.tokens, blockIdx.x / wgs_per_slot, before, scratch);
    const int item = (int)(blockIdx.x % wgs_per_slot) * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (ts.sequence == -2 || item >= 2 * a.cache.kv_heads) return;
    const bool is_v = item >= a.cache.kv_heads;
    const int h = item - (is_v ? a.cache.kv_heads : 0);
    const uint8_t* tile = nullptr;
    if (ts.sequence >= 0 && ts.tile >= 0 && ts.tile <= INT32_MAX / kKvTile)
        tile = kv4_tile(a.cache, ts.sequence, (uint32_t)ts.tile * kKvTile, h, kv4_tile_bytes(D));
    auto out = [&](int kk, int d) {
        return reinterpret_cast<u16x8*>((is_v ? a.v : a.k) + ((ts.t0 + kk) * a.cache.kv_heads + h) * (int64_t)D + d);
    };
    auto inside = [&](int kk) { return ts.t0 + kk >= ts.from && ts.t0 + kk < ts.to; };
    if (!tile) {
        u16x8 nan;
#pragma unroll
        for (int j = 0; j < 8; ++j) nan[j] = BF ? 0x7FC0 : 0x7E00;
        for (int x = lane; x < kKvTile * D / 8; x += 64)
            if (inside(x / (D / 8))) *out(x / (D / 8), x % (D / 8) * 8) = nan;
        return;
    }
    const uint16_t* meta = reinterpret_cast<const uint16_t*>(tile + 32 * D);
    if (!is_v) {
        // a word is 8 dims of one key
        constexpr int WPR = D / 8, ROUNDS = kKvTile * WPR / 64;
        uint32_t word[ROUNDS];
        float s[ROUNDS], z[ROUNDS];
#pragma unroll
        for (int n = 0; n < ROUNDS; ++n) {
            const int kk = (n * 64 + lane) / WPR, x = lane % WPR, g = x / (D / 32), w = x % (D / 32);
            word[n] = *reinterpret_cast<const uint32_t*>(tile + kv4_word<D>(kk >> 4, g * 16 + (kk & 15), w));
            const uint16_t* m = meta + (kk >> 2 & 3) * 32 + 4 * (kk >> 4) + (kk & 3);
            s[n] = scale_f32<BF>(m[0]);
            z[n] = scale_f32<BF>(m[8]);
        }
#pragma unroll
        for (int n = 0; n < ROUNDS; ++n) {
            const int kk = (n * 64 + lane) / WPR;
            u16x8 o;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                o[j] = round_out<BF>(((float)(word[n] >> (4 * (j >> 1) + 16 * (j & 1)) & 15) - z[n]) * s[n]);
            if (inside(kk)) store_past(out(kk, lane % WPR * 8), o);
        }
        return;
    }
    // eight words are 8 dims and their partners D/2 on of four keys
    constexpr int UNITS = kKvTile / 4 * (D / 16);
#pragma unroll
    for (int x = lane; x < UNITS; x += 64) {
        const int dims = x % (D / 16) * 8, ug = x / (D / 16), u = ug >> 2, g = ug & 3;
        uint32_t word[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            word[j] = *reinterpret_cast<const uint32_t*>(
                tile + 16 * D + kv4_word<D>(u, g * 16 + (dims & 15) + j, dims >> 4));
#pragma unroll
        for (int jj = 0; jj < 4; ++jj) {
            const int kk = 16 * u + 4 * g + jj;
            const uint16_t* m = meta + g * 32 + 16 + 4 * u + jj;
            const float s = scale_f32<BF>(m[0]), z = scale_f32<BF>(m[8]);
            u16x8 oa, ob;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t byte = (word[j] >> (8 * kv4_byte(jj)) & 0xFF) ^ (jj & 1 ? 0xFFu : 0u);
                oa[j] = round_out<BF>(((float)(byte & 15) - z) * s);
                ob[j] = round_out<BF>(((float)(byte >> 4) - z) * s);
            }
            if (inside(kk)) {
                store_past(out(kk, dims), oa);
                store_past(out(kk, dims + D / 2), ob);
            }
        }
    }
}

template <typename F>
int by_head_dim(int D, F&& f) {
    if (D == 64) return f(std::integral_constant<int, 64>{});
    if (D == 128) return f(std::integral_constant<int, 128>{});
    return f(std::integral_constant<int, 256>{});
}

// Tiles that the tokens of a call touch, at most: n tokens of a sequence (or of
// the two runs that none owns) touch no more than n / 32 + 2.
int64_t most_tiles(int64_t batch, int64_t tokens) {
    const int64_t runs = batch + 2 < tokens ? batch + 2 : tokens;
    return (tokens + 62 * runs) / kKvTile;
}

// Whether a read goes tile by tile; elements: of a token's keys.
bool by_tiles(int64_t batch, int64_t tokens, int64_t elements) {
    const int64_t values = tokens * elements, most = 4 * elements < kTileMostBatch ? 4 * elements : kTileMostBatch;
    return values >= kTileValues && values >= kTileValuesEach * batch && tokens >= kTileTokensEach * batch &&
           elements >= kTileLeastElements && batch <= most;
}

Kv4 device_view(const tf_kv4_cache& c) {
    Kv4 v;
    v.data = static_cast<uint8_t*>(c.data);
    v.pages = c.pages;
    v.page_bytes = (int64_t)c.kv_heads * (c.page_size / kKvTile) * kv4_tile_bytes(c.head_dim);
    v.page_size = c.page_size;
    v.tiles = c.page_size / kKvTile;
    v.kv_heads = c.kv_heads;
    v.table = c.table;
    v.table_stride = c.table_stride;
    v.max_pages = c.max_pages;
    return v;
}

}  // namespace

Kv4 kv4_view(const tf_kv4_cache& c) { return device_view(c); }

int launch_kv4_append(const tf_kv4_cache& c, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                      const void* v, int64_t v_stride, const float* cos, const float* sin, int64_t positions,
                      const int32_t* cu, const int32_t* starts, int64_t batch, int64_t tokens, int q_heads,
                      void* q_out, void* k_out, hipStream_t s) {
    auto in = [](const void* p) { return static_cast<const uint16_t*>(p); };
    const AppendArgs a{device_view(c), in(q), in(k), in(v), q_stride, k_stride, v_stride, cos, sin, positions, cu,
                       starts, (int)batch, q_heads, tokens, static_cast<uint16_t*>(q_out),
                       static_cast<uint16_t*>(k_out), Divisor((uint32_t)(q_heads + 2 * c.kv_heads))};
    return by_head_dim(c.head_dim, [&](auto d) {
        constexpr int D = decltype(d)::value;
        const bool bf = c.dtype == TF_BF16;
        const dim3 grid((unsigned)((tokens * (q_heads + 2 * c.kv_heads) * (D / 16) + 255) / 256));
        return bf ? launch(kv4_append_kernel<true, D>, grid, dim3(256), 0, s, a)
                  : launch(kv4_append_kernel<false, D>, grid, dim3(256), 0, s, a);
    });
}

int launch_kv4_read(const tf_kv4_cache& c, const int32_t* cu, const int32_t* starts, int64_t batch, int64_t tokens,
                    void* k, void* v, hipStream_t s) {
    const ReadArgs a{device_view(c), cu, starts, (int)batch, tokens, static_cast<uint16_t*>(k),
                     static_cast<uint16_t*>(v)};
    return by_head_dim(c.head_dim, [&](auto d) {
        constexpr int D = decltype(d)::value;
        const bool bf = c.dtype == TF_BF16;
        const int64_t per_slot = (2 * (int64_t)c.kv_heads + 3) / 4, wgs = most_tiles(batch, tokens) * per_slot;
        if (by_tiles(batch, tokens, c.kv_heads * D) && wgs * 256 <= UINT32_MAX) {
            const dim3 grid((unsigned)wgs);
            return bf ? launch(kv4_read_tiles_kernel<true, D>, grid, dim3(256), 0, s, a, (uint32_t)per_slot)
                      : launch(kv4_read_tiles_kernel<false, D>, grid, dim3(256), 0, s, a, (uint32_t)per_slot);
        }
        const dim3 grid((unsigned)((tokens * 2 * c.kv_heads * (D / 16) + 255) / 256));
        return bf ? launch(kv4_read_kernel<true, D>, grid, dim3(256), 0, s, a)
                  : launch(kv4_read_kernel<false, D>, grid, dim3(256), 0, s, a);
    });
}

}  // namespace tf
