// Where the paged key-value cache's elements stand and which of them a workgroup takes.  Integer arithmetic only, so that it
// compiles for the device and, without HIP, for a test on the host: whatever a page table, a length or a row start holds, no
// index that these functions give lies outside the cache, the table or the rows.
#pragma once
#include <cstdint>

#if !defined(BITNET_BOTH)
#if defined(__HIPCC__)
#define BITNET_BOTH __host__ __device__
#else
#define BITNET_BOTH
#endif
#endif

namespace bitnet {

constexpr int kKvBlock = 32;           // tokens of one cache block: two MFMA operand tiles of 16 keys, one K step of values

BITNET_BOTH constexpr int kv_padded_dim(int D) { return (D + 7) / 8 * 8; }
// Keys are two operand tiles of a 16 x 16 x 32 product whose result, keys down and queries across, is the operand of the next
// product as it stands, if lane group g's eight values (rows 4 g + i of both tiles) are eight consecutive tokens: so row
// 4 a + b of tile u is token 8 a + 4 u + b, and the block stores the rows of tile 0, then those of tile 1.
BITNET_BOTH constexpr int kv_key_slot(int t) { return 16 * ((t >> 2) & 1) + 4 * (t >> 3) + (t & 3); }
// elements within a block of 32 Dp: keys are [Dp / 8][32 slots][8 dims], values [4][Dp][8 tokens]
BITNET_BOTH constexpr int kv_key_at(int t, int d) { return ((d >> 3) * kKvBlock + kv_key_slot(t)) * 8 + (d & 7); }
BITNET_BOTH constexpr int kv_value_at(int t, int d, int Dp) { return ((t >> 3) * Dp + d) * 8 + (t & 7); }

// What the kernels take of a bitnet_kv (bitnet.h).
struct KvView {
    uint16_t *k, *v;
    const int32_t *table, *kv_len, *q_start;
    int64_t table_stride;
    int32_t pages, page_blocks /* of a page, for one head */, max_pages /* of a table row */, max_blocks /* ... times page_blocks */, kv_heads, D, B;

    // tokens of sequence b that can be in the cache
    BITNET_BOTH int length(int32_t len) const {
        const int64_t most = (int64_t)max_blocks * kKvBlock;
        return len < 0 ? 0 : len > most ? (int)most : len;
    }
    // block `in` of a page, as the table names it, for key-value head h: its number in the cache, or -1 where there is no such page
    BITNET_BOTH int block_on(int page, int in, int h) const {
        return page < 0 || page >= pages ? -1 : (page * kv_heads + h) * page_blocks + in;
    }
    // the same for block `blk` of a sequence, 0 <= blk < max_blocks
    BITNET_BOTH int block(const int32_t* row, int blk, int h) const {
        const int p = blk / page_blocks;
        return block_on(row[p], blk - p * page_blocks, h);
    }
};

// The rows [first, first + n) of one sequence's new tokens among T, and the position of the first (negative where kv_len is less
// than n: such tokens are in no cache and see nothing).
struct NewTokens {
    int first, n, pos0;
    BITNET_BOTH NewTokens(const KvView& kv, int b, int T) {
        const int s = kv.q_start[b], e = kv.q_start[b + 1];
        first = s < 0 ? 0 : s > T ? T : s;
        const int end = e < first ? first : e > T ? T : e;
        n = end - first;
        pos0 = kv.length(kv.kv_len[b]) - n;
    }
};

// Tiles of `size` units over sequences with ragged numbers of units (each q_start[b + 1] - q_start[b] new tokens of `each` units), dealt out
// without a pass over the lengths: sequence b's tiles start at q_start[b] * each / size + extra * b.  With extra = 1 that leaves room for
// ceil(units / size) of them, with 2 for one more (tiles that are aligned to positions and cut at both ends).  Gives the
// sequence that tile x may belong to, by bisection, 0 <= b < B for any contents of q_start; tile numbers without work are the caller's to see.
BITNET_BOTH inline int64_t first_tile(int32_t start, int b, int each, int size, int extra) {
    return (int64_t)(start < 0 ? 0 : start) * each / size + (int64_t)extra * b;
}
BITNET_BOTH inline int sequence_of_tile(const int32_t* q_start, int B, int64_t x, int each, int size, int extra) {
    int lo = 0, hi = B - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (first_tile(q_start[mid], mid, each, size, extra) <= x) lo = mid; else hi = mid - 1;
    }
    return lo;
}
BITNET_BOTH inline int64_t tiles_at_most(int64_t T, int64_t B, int each, int size, int extra) {
    return extra == 1 ? (T * each + size - 1) / size + B - 1 : T * each / size + extra * B;
}

}  // namespace bitnet
