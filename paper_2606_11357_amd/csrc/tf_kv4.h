// Layout of the 4-bit paged key/value cache and the device code that every
// kernel reading or writing it shares.
//
// A row is the key or the value of one token in one head: D codes q of 4 bits,
// a 16-bit scale s and a 16-bit zero-point z, standing for s * (q - z).
//
// Keys are grouped into tiles of 32 consecutive positions.  A page holds, for
// each key/value head, page_size / 32 tiles, one after the other:
//   page base + (head * (page_size / 32) + tile) * kv4_tile_bytes(D)
// A tile is K codes (16 D bytes), V codes (16 D bytes) and 256 bytes of scales
// and zero-points, laid out as the lanes of a 64-lane wavefront take them:
//
//   key kk of the tile: u = kk / 16, c = kk % 16 (K), g = (kk % 16) / 4,
//   jj = kk % 4 (V, metadata)
//   K: lane g * 16 + c holds dims g (D/4) .. + D/4 of key 16 u + c; word w of
//      its D/32 words holds dims g (D/4) + 8 w + 0..7: nibble e (bits 4e..)
//      is dim 2e, nibble e + 4 is dim 2e + 1, so that the bits
//      4e..4e+3 and 16+4e..16+4e+3 make one 16-bit pair of a matrix operand
//   V: lane g * 16 + c holds dims c + 16 t of keys 16 u + 4 g + jj; word w of
//      half u has one byte a key (jj = 0, 1, 2, 3 in bytes 0, 2, 1, 3), dim
//      c + 16 w in the low nibble and dim D/2 + c + 16 w in the high one; the
//      codes of keys with odd jj are stored as 15 - q (see tf_kv4_attn.hip)
//   metadata: 16-bit words [g][k scale, k zero, v scale, v zero][4 u + jj]
//
// Each lane so reads what it multiplies in whole 16-byte loads, no row shares
// a byte with another (an append only stores), and the 32 keys of a tile meet
// the matrix cores in the order in which the scores come out of them.
#pragma once

#include "tf_internal.h"

namespace tf {

constexpr int kKvTile = 32;

__host__ __device__ constexpr int64_t kv4_tile_bytes(int D) { return 32 * (int64_t)D + 256; }

// Byte offset of word w (0 .. D/32 - 1) of lane L for key half u inside the K
// or V codes of a tile: whole 16-byte pieces of each lane, 1 KiB apart.
template <int D>
__host__ __device__ constexpr int kv4_word(int u, int L, int w) {
    if constexpr (D == 64) return L * 16 + u * 8 + w * 4;
    else return ((u * (D / 128) + w / 4) * 64 + L) * 16 + (w % 4) * 4;
}
// Byte of key jj inside a V word.
__host__ __device__ constexpr int kv4_byte(int jj) { return jj == 1 ? 2 : jj == 2 ? 1 : jj; }

// Division by a number that the host knows, of numbers below 2^31: with
// 2^(s-1) < d <= 2^s and m = floor(2^(31+s) / d) + 1, n / d = n m >> 31 + s.
struct Divisor {
    uint32_t d = 1, m = 0, s = 0;
    Divisor() = default;
    explicit Divisor(uint32_t by) : d(by) {
        while (d > 1u << s) ++s;
        m = (uint32_t)(((uint64_t)1 << (31 + s)) / d + 1);
    }
    __device__ __forceinline__ uint32_t of(uint32_t n) const { return (uint32_t)((uint64_t)n * m >> (31 + s)); }
};

// A paged cache as the kernels take it.
struct Kv4 {
    uint8_t* data;
    int64_t pages;
    int64_t page_bytes;
    int page_size;
    int tiles;              // tiles per page and head
    int kv_heads;
    const int32_t* table;   // [batch, table_stride], the first max_pages of a row valid
    int64_t table_stride;
    int64_t max_pages;
};

// Tile of position pos (below 2^31) of sequence b in head h, or null where the sequence
// has no page there (past its table, or an entry outside the pool).
__device__ __forceinline__ uint8_t* kv4_tile(const Kv4& c, int64_t b, uint32_t pos, int h, int64_t tile_bytes) {
    const uint32_t p = pos / (uint32_t)c.page_size;
    if (p >= c.max_pages) return nullptr;
    const int32_t page = c.table[b * c.table_stride + p];
    if (page < 0 || page >= c.pages) return nullptr;
    const uint32_t t = (pos - p * (uint32_t)c.page_size) / kKvTile;
    return c.data + (int64_t)page * c.page_bytes + ((int64_t)h * c.tiles + t) * tile_bytes;
}

// The sequence that packed token t belongs to: the last b with cu[b] <= t, or
// -1 where there is none (cu: batch + 1 offsets).
__device__ __forceinline__ int owner_of(const int32_t* cu, int batch, int64_t t) {
    if (t < cu[0] || t >= cu[batch]) return -1;
    int lo = 0, hi = batch;                // cu[lo] <= t < cu[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (cu[mid] <= t) lo = mid;
        else hi = mid;
    }
    return lo;
}

}  // namespace tf
