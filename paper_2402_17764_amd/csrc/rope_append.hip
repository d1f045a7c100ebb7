// Rotary positions on the queries and keys of a merged Q | K | V product, keys and values into the paged cache.
//
// Per pair (a, b) of a head's dims and position p, with the angle p f_i of the pair: (a cos - b sin, b cos + a sin).  The angle is
// brought to a fraction of a turn in 64 bits (p f_i alone has up to 55 significant bits, and only the fraction counts),
// its sine and cosine and the products are 32 bits wide, and the result is rounded once, to the cache's bf16.
#include "rope_slots.hpp"

namespace bitnet {
namespace {

constexpr int kThreads = 256;

// n of eight elements into LDS, two at a time where p allows it
__device__ inline void stage_any(uint16_t* p, uint4 w, int n, bool words) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
    if (words) {
#pragma unroll
        for (int i = 0; i < 4; ++i) if (2 * i + 1 < n) *reinterpret_cast<uint32_t*>(p + 2 * i) = u[i];
        if (n & 1)
#pragma unroll
            for (int i = 0; i < 8; i += 2) if (i + 1 == n) p[i] = (uint16_t)u[i >> 1];
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) if (i < n) p[i] = (uint16_t)(u[i >> 1] >> (16 * (i & 1)));
}

// One new token for each sequence.  A thread takes eight dims of a head; what counts is the chain of loads (length, page, row),
// so the row is requested first and a workgroup holds few heads.
template <bool kBf16>
__global__ __launch_bounds__(kThreads) void rope_append_tokens(const void* __restrict__ qkv, const float* __restrict__ inv_freq, KvView kv,
                                                               RopeShape s, int quads, uint16_t* __restrict__ q) {
    __shared__ Turn turns[128];
    const int b = blockIdx.x, unit = (blockIdx.y * kThreads + threadIdx.x) / quads, j = (blockIdx.y * kThreads + threadIdx.x) % quads;
    const int units = s.heads + 2 * kv.kv_heads, D = kv.D, d0 = 8 * j;
    const bool mine = unit < units;
    const int64_t row = (int64_t)b * units * D, head = row + (int64_t)unit * D;
    const int pos = kv.length(kv.kv_len[b]) - 1;
    const bool turned = mine && unit < s.heads + kv.kv_heads;
    Slot<kBf16, Turned::Any> slot;
    if (mine) slot.load(qkv, head, (int64_t)(units - unit) * D, d0, D, turned && !s.pairs, s);
    for (int i = threadIdx.x; i < s.rotary >> 1; i += kThreads) turns[i] = turn_of(pos, inv_freq[i]);
    __syncthreads();
    float x[8], none[8];
    Turn by[8];
    if (turned)
#pragma unroll
        for (int e = 0; e < 8; ++e) by[e] = d0 + e < s.rotary ? turns[pair_of(d0 + e, s)] : Turn{1.0f, 0.0f};
    if (s.pairs) {
        const Slot<kBf16, Turned::Pairs> p{slot.own, {}, {}};
        p.turn(x, none, d0, turned, by, s);
    } else {
        slot.turn(x, none, d0, turned, by, s);
    }
    if (!mine) return;
    const uint4 w = pack8(x);
    if (unit < s.heads) {
        store_any(q + ((int64_t)b * s.heads + unit) * D + d0, w, D - d0);
        return;
    }
    if (pos < 0) return;
    const int h = unit < s.heads + kv.kv_heads ? unit - s.heads : unit - s.heads - kv.kv_heads;
    const int Dp = kv_padded_dim(D), t = pos & 31;
    const int block = kv.block(kv.table + b * kv.table_stride, pos >> 5, h);
    if (block < 0) return;
    const int64_t at = (int64_t)block * kKvBlock * Dp;
    if (unit < s.heads + kv.kv_heads) {
        *reinterpret_cast<uint4*>(kv.k + at + kv_key_at(t, d0)) = w;
    } else {
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (d0 + i < D) kv.v[at + kv_value_at(t, d0 + i, Dp)] = (uint16_t)(u[i >> 1] >> (16 * (i & 1)));
    }
}

// Runs of new tokens: a workgroup takes the new tokens of one cache block (32 positions) and `per` heads of their rows.  A thread keeps
// its token and dims over the heads, so that sines and cosines are computed once and stay in registers.  Values are turned
// over through LDS: the cache holds eight tokens of a dim together.
//
// What a thread takes of a head is a slot: eight dims, or where halves are turned together eight of the lower half and their eight partners,
// so that each is read and each angle computed once.  Where the halves do not begin at multiples of eight (Odd) the results
// come together in LDS first, as the cache takes eight dims at a time, or slots of all dims read their partners on both sides (Any); see
// launch_blocks.
template <bool kBf16, Turned kTurned, int kM /* slots a thread */>
__global__ __launch_bounds__(kThreads) void rope_append_blocks(const void* __restrict__ qkv, const float* __restrict__ inv_freq, KvView kv,
                                                               RopeShape s, int per, uint16_t* __restrict__ q) {
    constexpr int kPitch = 256 + 8;
    __shared__ uint4 tile4[kKvBlock * kPitch / 8];
    uint16_t* tile = reinterpret_cast<uint16_t*>(tile4);
    const int D = kv.D, Dp = kv_padded_dim(D), quads = Dp >> 3, units = s.heads + 2 * kv.kv_heads;
    const int b = sequence_of_tile(kv.q_start, kv.B, blockIdx.x, 1, kKvBlock, 2);
    const NewTokens nt(kv, b, s.T);
    const int64_t tile_in = (int64_t)blockIdx.x - first_tile(kv.q_start[b], b, 1, kKvBlock, 2);
    if (nt.n == 0 || tile_in < 0) return;
    const int64_t blk64 = (nt.pos0 >> 5) + tile_in;            // floor: positions may be negative
    if (blk64 * kKvBlock >= (int64_t)nt.pos0 + nt.n) return;
    const int blk = (int)blk64;
    const int t0 = max(nt.pos0 - blk * kKvBlock, 0), t1 = min(nt.pos0 + nt.n - blk * kKvBlock, kKvBlock);     // the block's new tokens
    const int row0 = nt.first + blk * kKvBlock - nt.pos0;      // of token 0 of the block
    const int u0 = blockIdx.y * per, u1 = min(u0 + per, units);
    // the page: its number is the same for all heads
    const int page_index = blk >= 0 ? blk / kv.page_blocks : 0, page = blk >= 0 ? kv.table[b * kv.table_stride + page_index] : -1;

    constexpr bool kTogether = kTurned == Turned::Split || kTurned == Turned::Odd;
    const int half = s.rotary >> 1, half8 = (half + 7) >> 3;   // slots of a half
    const int slots = slots_of<kTurned>(D, s), tiles = (slots + 7) >> 3;
    int tok[kM], d0[kM];
    Turn turn[kM][8];
#pragma unroll
    for (int m = 0; m < kM; ++m) {
        // eight slots of a row next to each other, then eight tokens: 128 bytes of a bf16 row at a time
        const int i = threadIdx.x + m * kThreads, j = (i & 7) + 8 * ((i >> 6) % tiles);
        tok[m] = ((i >> 3) & 7) + 8 * ((i >> 6) / tiles);
        if (j >= slots || tok[m] < t0 || tok[m] >= t1) tok[m] = -1;
        // the lower half's, then those that are not turned
        d0[m] = kTogether && j >= half8 ? s.rotary + 8 * (j - half8) : 8 * j;
        if (kTurned != Turned::Any && tok[m] >= 0 && u0 < s.heads + kv.kv_heads)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (kTurned == Turned::Pairs && (e & 1)) { turn[m][e] = turn[m][e - 1]; continue; }
                const bool angle = kTurned == Turned::Odd ? d0[m] + e < half : d0[m] + e < s.rotary;
                turn[m][e] = angle ? turn_of(blk * kKvBlock + tok[m], inv_freq[pair_of(d0[m] + e, s)]) : Turn{1.0f, 0.0f};
            }
    }
    if (kTurned == Turned::Any && u0 < s.heads + kv.kv_heads) {      // two dims have an angle: computed once, taken twice
        Turn* table = reinterpret_cast<Turn*>(tile4);          // [32][half]: heads of up to 64 dims
        for (int i = threadIdx.x; i < kKvBlock * half; i += kThreads) table[i] = turn_of(blk * kKvBlock + i / half, inv_freq[i % half]);
        __syncthreads();
#pragma unroll
        for (int m = 0; m < kM; ++m)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (tok[m] >= 0 && d0[m] + e < s.rotary) turn[m][e] = table[tok[m] * half + pair_of(d0[m] + e, s)];
        __syncthreads();
    }
    if (kTurned == Turned::Odd)                                // dims behind a head's end
        for (int i = threadIdx.x; i < kKvBlock * (Dp - D); i += kThreads) tile[i / (Dp - D) * kPitch + D + i % (Dp - D)] = 0;
    Slot<kBf16, kTurned> slot[kM], next[kM];
    auto request = [&](Slot<kBf16, kTurned> (&x)[kM], int u) {
#pragma unroll
        for (int m = 0; m < kM; ++m)
            if (tok[m] >= 0) x[m].load(qkv, ((int64_t)(row0 + tok[m]) * units + u) * D, (int64_t)(units - u) * D, d0[m], D, u < s.heads + kv.kv_heads, s);
    };
    request(next, u0);
#pragma unroll 1
    for (int u = u0; u < u1; ++u) {
#pragma unroll
        for (int m = 0; m < kM; ++m) slot[m] = next[m];
        if (u + 1 < u1) request(next, u + 1);
        const bool query = u < s.heads, key = !query && u < s.heads + kv.kv_heads;
        int block = -1;
        if (!query) block = kv.block_on(page, blk - page_index * kv.page_blocks, key ? u - s.heads : u - s.heads - kv.kv_heads);
        if (!query && block < 0) continue;                     // the same for the whole workgroup
        const int64_t at = (int64_t)block * kKvBlock * Dp;
#pragma unroll
        for (int m = 0; m < kM; ++m) {
            if (tok[m] < 0) continue;
            const int64_t out = ((int64_t)(row0 + tok[m]) * s.heads + u) * D;
            auto put = [&](int d, uint4 w) {
                if (kTurned == Turned::Odd) stage_any(&tile[tok[m] * kPitch + d], w, d0[m] < half ? min(half - d0[m], 8) : min(D - d0[m], 8), (half & 1) == 0 || d == d0[m]);
                else if (query) store_any(q + out + d, w, D - d);
                else if (key) *reinterpret_cast<uint4*>(kv.k + at + kv_key_at(tok[m], d)) = kTurned == Turned::Pairs ? first_of(w, D - d) : w;
                else *reinterpret_cast<uint4*>(&tile[tok[m] * kPitch + d]) = w;
            };
            float x[8], y[8];
            slot[m].turn(x, y, d0[m], query || key, turn[m], s);
            put(d0[m], pack8(x));
            if (kTogether && d0[m] < half) put(d0[m] + half, pack8(y));
        }
        if (kTurned != Turned::Odd && (query || key)) continue;
        __syncthreads();
        if (query || key) {
            // queries by rows, as in memory; keys by eight dims of 32 tokens, which stand next to each other in the cache
            const int across = query ? (quads + 7) >> 3 : 0;
            for (int i = threadIdx.x; i < 32 * (query ? 8 * across : quads); i += kThreads) {
                const int j = query ? (i & 7) + 8 * ((i >> 6) % across) : i >> 5, t = query ? ((i >> 3) & 7) + 8 * ((i >> 6) / across) : i & 31;
                if (j >= quads || t < t0 || t >= t1) continue;
                const uint4 w = *reinterpret_cast<const uint4*>(&tile[t * kPitch + 8 * j]);
                if (query) store_any(q + ((int64_t)(row0 + t) * s.heads + u) * D + 8 * j, w, D - 8 * j);
                else *reinterpret_cast<uint4*>(kv.k + at + kv_key_at(t, 8 * j)) = w;
            }
            __syncthreads();
            continue;
        }
        for (int i = threadIdx.x; i < 4 * D; i += kThreads) {
            const int g = i / D, d = i - g * D;
            if (8 * g + 8 <= t0 || 8 * g >= t1) continue;
            uint16_t e[8];
#pragma unroll
            for (int t = 0; t < 8; ++t) e[t] = tile[(8 * g + t) * kPitch + d];
            uint16_t* to = kv.v + at + (g * Dp + d) * 8;
            if (8 * g >= t0 && 8 * g + 8 <= t1) {
                uint4 w;
                __builtin_memcpy(&w, e, 16);
                *reinterpret_cast<uint4*>(to) = w;
            } else {                                           // tokens of earlier calls stay as they are
#pragma unroll
                for (int t = 0; t < 8; ++t) if (8 * g + t >= t0 && 8 * g + t < t1) to[t] = e[t];
            }
        }
        __syncthreads();
    }
}

template <bool kBf16, Turned kTurned>
hipError_t launch_blocks(const void* qkv, const float* inv_freq, const KvView& kv, const RopeShape& s, uint16_t* q, hipStream_t stream) {
    const int units = s.heads + 2 * kv.kv_heads, m = (slots_of<kTurned>(kv.D, s) + 7) / 8;
    const int64_t tiles = tiles_at_most(s.T, kv.B, 1, kKvBlock, 2);
    // Heads of a workgroup: four share a token's sines and cosines and the loads that say where its row and its page are, if that leaves
    // 704 workgroups, two and three quarters for each CU, of those that `tiles` counts (up to two a sequence have no token), and fewer
    // otherwise (us, one / two / three / four: 64 heads over 8, two prompts of 2048 tokens 65 / 48 / 43 / 43, one of 2048 23 / 18.6 / 18.1 /
    // 17.6, two of 512 14.7 / 12.6 / 12.7 / 12.7, one of 512 10.3 / 9.2 / 9.4 / 10.6, two of 256 10.0 / 9.6 / 10.1 / 10.7, one of 256 6.2 / 6.8 /
    // 7.1 / 7.4, of 77 5.1 / 5.5 / 6.3 / 7.0; with 768 the one of 512 has one).
    const int64_t all = tiles * units / 704;
    const int per = (int)(all < 1 ? 1 : all > 4 ? 4 : all);
    const dim3 grid((unsigned)tiles, (unsigned)ceil_div(units, per));
    if (m == 1) rope_append_blocks<kBf16, kTurned, 1><<<grid, kThreads, 0, stream>>>(qkv, inv_freq, kv, s, per, q);
    else if constexpr (kTurned == Turned::Any) return hipErrorInvalidValue;
    else if (m == 2) rope_append_blocks<kBf16, kTurned, 2><<<grid, kThreads, 0, stream>>>(qkv, inv_freq, kv, s, per, q);
    else if (kTurned != Turned::Odd || m <= 4) rope_append_blocks<kBf16, kTurned, 4><<<grid, kThreads, 0, stream>>>(qkv, inv_freq, kv, s, per, q);
    else rope_append_blocks<kBf16, Turned::Odd, 5><<<grid, kThreads, 0, stream>>>(qkv, inv_freq, kv, s, per, q);      // 33 slots
    return hipGetLastError();
}
template <bool kBf16>
hipError_t launch_blocks(const void* qkv, const float* inv_freq, const KvView& kv, const RopeShape& s, uint16_t* q, hipStream_t stream) {
    if (s.pairs) return launch_blocks<kBf16, Turned::Pairs>(qkv, inv_freq, kv, s, q, stream);
    if (s.rotary % 16 == 0) return launch_blocks<kBf16, Turned::Split>(qkv, inv_freq, kv, s, q, stream);
    // Halves that are no multiple of eight: turned together through LDS, whose barriers cost more than partners that are read on both sides
    // where a thread's one slot of eight is enough for that, a head of up to 64 dims (us, Odd / Any, 32 heads, 4096 tokens: of 24 dims bf16 25.4 / 21.4,
    // fp32 25.1 / 20.4, of 40 26.3 / 23.0 and 28.7 / 26.4, of 50 29.5 / 26.7 and 36.9 / 38.1; of 72 39 / 72 and 43 / 54, of 100 48 / 83 and
    // 59 / 73; 512 tokens of 40 dims 8.8 / 7.8 and 8.5 / 7.2, of 50 9.8 / 9.0 and 9.5 / 8.0, of 72 10.4 / 13.0 and 9.4 / 10.8).
    if (kv.D <= 64) return launch_blocks<kBf16, Turned::Any>(qkv, inv_freq, kv, s, q, stream);
    return launch_blocks<kBf16, Turned::Odd>(qkv, inv_freq, kv, s, q, stream);
}

}  // namespace

hipError_t launch_rope_append(const void* qkv, bool bf16, const float* inv_freq, int rotary, bool pairs, const KvView& kv, int64_t T, int heads,
                              void* q, hipStream_t stream) {
    const RopeShape s{heads, rotary, (int)T, pairs ? 1 : 0};
    const int units = heads + 2 * kv.kv_heads, quads = kv_padded_dim(kv.D) / 8;
    uint16_t* qo = static_cast<uint16_t*>(q);
    if (!kv.q_start) {
        const dim3 grid((unsigned)T, (unsigned)ceil_div((int64_t)units * quads, kThreads));
        if (bf16) rope_append_tokens<true><<<grid, kThreads, 0, stream>>>(qkv, inv_freq, kv, s, quads, qo);
        else rope_append_tokens<false><<<grid, kThreads, 0, stream>>>(qkv, inv_freq, kv, s, quads, qo);
        return hipGetLastError();
    }
    return bf16 ? launch_blocks<true>(qkv, inv_freq, kv, s, qo, stream) : launch_blocks<false>(qkv, inv_freq, kv, s, qo, stream);
}

}  // namespace bitnet
