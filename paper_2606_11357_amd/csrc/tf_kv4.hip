// The 4-bit paged key/value cache: append (with the rotation of queries and
// keys on the way) and read back.
#include "tf_kv4.h"

namespace tf {
namespace {

typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));

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
__device__ __forceinline__ RowQuant row_quant(float lo, float hi, bool finite) {
#pragma clang fp contract(off)
    RowQuant r;
    const float fifteenth = 1.0f / 15.0f;
    const float a = hi * fifteenth, b = lo * fifteenth;
    r.s16 = round_out<BF>(a - b);
    float s = scale_f32<BF>(r.s16);
    if (!finite || !(s < __builtin_inff())) {
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

// One row of D values (a query, key or value of one token and head) on D / 16
// lanes: lane i holds dims 8 i .. + 7 and their partners D/2 + 8 i .. + 7, so
// the rotation needs no exchange and both operands come in 16-byte loads.
// HBM-bound: every input is read once and every output written once.
template <bool BF, int D>
__global__ __launch_bounds__(256) void kv4_append_kernel(AppendArgs a) {
    constexpr int LPR = D / 16;
    __shared__ int32_t lds_cu[kStagedBatch + 1];
    const int32_t* cu = stage_offsets(a.cu, a.batch, lds_cu);
    const int rows = a.q_heads + 2 * a.cache.kv_heads;
    // (token, row) pairs: at most TF_MAX_M * 3 TF_MAX_HEADS, below 2^32
    const uint32_t at = blockIdx.x * (256 / LPR) + threadIdx.x / LPR;
    const int i = threadIdx.x % LPR;
    const bool active = at < a.tokens * rows;
    const int64_t t = active ? at / (uint32_t)rows : 0;
    const int row = active ? (int)(at % (uint32_t)rows) : 0;
    const int kind = row < a.q_heads ? 0 : row < a.q_heads + a.cache.kv_heads ? 1 : 2;
    const int h = row - (kind == 0 ? 0 : kind == 1 ? a.q_heads : a.q_heads + a.cache.kv_heads);
    const uint16_t* src = (kind == 0   ? a.q + t * a.q_stride
                           : kind == 1 ? a.k + t * a.k_stride
                                       : a.v + t * a.v_stride) +
                          (int64_t)h * D + 8 * i;
    u16x8 xa{}, xb{};
    if (active) {
        xa = *reinterpret_cast<const u16x8*>(src);
        xb = *reinterpret_cast<const u16x8*>(src + D / 2);
    }
    const int b = owner_of(cu, a.batch, t);
    const int64_t pos = b < 0 ? -1 : (int64_t)a.starts[b] + (t - cu[b]);
    bool known = pos >= 0 && pos <= INT32_MAX;
    float lo[8], hi[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        lo[j] = scale_f32<BF>(xa[j]);
        hi[j] = scale_f32<BF>(xb[j]);
    }
    if (a.cos) {
        known = known && pos < a.positions;
        if (kind < 2 && known) {
#pragma clang fp contract(off)
            const float* cp = a.cos + pos * (D / 2) + 8 * i;
            const float* sp = a.sin + pos * (D / 2) + 8 * i;
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
    }
    uint16_t* out = kind == 0 ? a.q_out : kind == 1 ? a.k_out : nullptr;
    if (active && out) {
        uint16_t* o = out + (t * (kind == 0 ? a.q_heads : a.cache.kv_heads) + h) * D + 8 * i;
        const uint16_t nan16 = BF ? 0x7FC0 : 0x7E00;
        u16x8 oa, ob;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            oa[j] = known ? round_out<BF>(lo[j]) : nan16;
            ob[j] = known ? round_out<BF>(hi[j]) : nan16;
        }
        *reinterpret_cast<u16x8*>(o) = oa;
        *reinterpret_cast<u16x8*>(o + D / 2) = ob;
    }
    // the row's range over its lanes
    float least = lo[0], most = lo[0], total = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        least = fminf(least, fminf(lo[j], hi[j]));
        most = fmaxf(most, fmaxf(lo[j], hi[j]));
        total += (lo[j] - lo[j]) + (hi[j] - hi[j]);    // 0, or NaN where one is not finite
    }
    least = -row_max<LPR>(-least);
    most = row_max<LPR>(most);
    const bool finite = row_max<LPR>(total == 0.f ? 0.f : 1.f) == 0.f;
    if (!active || kind == 0 || !known) return;
    constexpr int64_t TB = kv4_tile_bytes(D);
    uint8_t* tile = kv4_tile(a.cache, b, (uint32_t)pos, h, TB);
    if (!tile) return;
    const RowQuant rq = row_quant<BF>(least, most, finite);
    uint32_t qa[8], qb[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        qa[j] = code_of(lo[j], rq);
        qb[j] = code_of(hi[j], rq);
    }
    const int kk = (int)(pos % kKvTile), u = kk >> 4, c = kk & 15, g = c >> 2, jj = c & 3;
    if (kind == 1) {
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
        uint16_t* meta = reinterpret_cast<uint16_t*>(tile + 32 * D) + g * 32 + (kind == 1 ? 0 : 16) + 4 * u + jj;
        meta[0] = rq.s16;
        meta[8] = rq.z16;
    }
}

struct ReadArgs {
    Kv4 cache;
    const int32_t *cu, *starts;
    int batch;
    int64_t tokens;
    uint16_t *k, *v;
};

// One row on D / 16 lanes, as in the append.
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
    *reinterpret_cast<u16x8*>(o) = oa;
    *reinterpret_cast<u16x8*>(o + D / 2) = ob;
}

template <typename F>
int by_head_dim(int D, F&& f) {
    if (D == 64) return f(std::integral_constant<int, 64>{});
    if (D == 128) return f(std::integral_constant<int, 128>{});
    return f(std::integral_constant<int, 256>{});
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
                       static_cast<uint16_t*>(k_out)};
    return by_head_dim(c.head_dim, [&](auto d) {
        constexpr int D = decltype(d)::value;
        const int64_t threads = tokens * (q_heads + 2 * c.kv_heads) * (D / 16);
        const dim3 grid((unsigned)((threads + 255) / 256));
        if (c.dtype == TF_BF16) return launch(kv4_append_kernel<true, D>, grid, dim3(256), 0, s, a);
        return launch(kv4_append_kernel<false, D>, grid, dim3(256), 0, s, a);
    });
}

int launch_kv4_read(const tf_kv4_cache& c, const int32_t* cu, const int32_t* starts, int64_t batch, int64_t tokens,
                    void* k, void* v, hipStream_t s) {
    const ReadArgs a{device_view(c), cu, starts, (int)batch, tokens, static_cast<uint16_t*>(k),
                     static_cast<uint16_t*>(v)};
    return by_head_dim(c.head_dim, [&](auto d) {
        constexpr int D = decltype(d)::value;
        const int64_t threads = tokens * 2 * c.kv_heads * (D / 16);
        const dim3 grid((unsigned)((threads + 255) / 256));
        if (c.dtype == TF_BF16) return launch(kv4_read_kernel<true, D>, grid, dim3(256), 0, s, a);
        return launch(kv4_read_kernel<false, D>, grid, dim3(256), 0, s, a);
    });
}

}  // namespace tf
