// Rotary positions on the queries and keys of a merged Q | K | V product, keys and values into the paged cache.
//
// Per pair (a, b) of a head's dims and position p, with the angle p f_i of the pair: (a cos - b sin, b cos + a sin).  The angle is
// brought to a fraction of a turn in 64 bits (p f_i alone has up to 55 significant bits, and only the fraction counts),
// its sine and cosine and the products are 32 bits wide, and the result is rounded once, to the cache's bf16.
#include "bitnet_device.hpp"
#include "bitnet_internal.hpp"
#include "kv_layout.hpp"

namespace bitnet {
namespace {

constexpr int kThreads = 256;

struct RopeShape {
    int heads, rotary, T;              // query heads; dims that are turned, the first ones of a head
    int pairs;                         // 0: dim i with i + rotary / 2; 1: 2 i with 2 i + 1
};

struct Turn { float cos, sin; };

__device__ inline Turn turn_of(int pos, float freq) {
    double t = (double)pos * (double)freq * 0.15915494309189533577;
    t -= rint(t);
    Turn r;
    sincospif(2.0f * (float)t, &r.sin, &r.cos);
    return r;
}

// eight consecutive elements from an address of any alignment, `count` of them (the others are zero)
template <bool kBf16>
__device__ inline void load8(float (&x)[8], const void* base, int64_t at, int count) {
    if (kBf16) {
        const uint16_t* p = static_cast<const uint16_t*>(base) + at;
        uint16_t u[8] = {};
        if (count >= 8) __builtin_memcpy(u, p, 16);
        else
#pragma unroll
            for (int i = 0; i < 7; ++i) if (i < count) u[i] = p[i];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = bf16_to_f32(u[i]);
    } else {
        const float* p = static_cast<const float*>(base) + at;
        if (count >= 8) __builtin_memcpy(x, p, 32);
        else
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = i < count ? p[i] : 0.0f;
    }
}

__device__ inline uint4 pack8(const float (&x)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = (uint32_t)f32_to_bf16(x[2 * i]) | (uint32_t)f32_to_bf16(x[2 * i + 1]) << 16;
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// The partners of dims d0 ... d0 + 7: what the sine multiplies, with its sign.
template <bool kBf16>
__device__ inline void partners(float (&y)[8], const float (&x)[8], const void* base, int64_t head, int d0, const RopeShape& s) {
    if (s.pairs) {
#pragma unroll
        for (int i = 0; i < 8; i += 2) { y[i] = -x[i + 1]; y[i + 1] = x[i]; }
        return;
    }
    const int half = s.rotary >> 1;
    if (d0 + 8 <= half || (d0 >= half && d0 + 8 <= s.rotary)) {
        const bool low = d0 < half;
        load8<kBf16>(y, base, head + (low ? d0 + half : d0 - half), 8);
        if (low)
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = -y[i];
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {                  // across the middle, or past the dims that are turned
        const int d = d0 + i;
        float v[8];
        load8<kBf16>(v, base, head + (d < half ? d + half : d - half), d < s.rotary ? 1 : 0);
        y[i] = d < half ? -v[0] : v[0];
    }
}

__device__ inline int pair_of(int d, const RopeShape& s) { return s.pairs ? d >> 1 : d < (s.rotary >> 1) ? d : d - (s.rotary >> 1); }

__device__ inline void store_any(uint16_t* p, uint4 w, int count) {
    if (count >= 8) { __builtin_memcpy(p, &w, 16); return; }
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 7; ++i) if (i < count) p[i] = (uint16_t)(u[i >> 1] >> (16 * (i & 1)));
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
    float x[8], y[8];
    if (mine) load8<kBf16>(x, qkv, head + d0, D - d0);
    const bool turned = mine && unit < s.heads + kv.kv_heads;
    if (turned && d0 < s.rotary) partners<kBf16>(y, x, qkv, head, d0, s);
    for (int i = threadIdx.x; i < s.rotary >> 1; i += kThreads) turns[i] = turn_of(pos, inv_freq[i]);
    __syncthreads();
    if (turned) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (d0 + i < s.rotary) {
                const Turn t = turns[pair_of(d0 + i, s)];
                x[i] = x[i] * t.cos + y[i] * t.sin;
            }
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

// Runs of new tokens: a workgroup takes the new tokens of one cache block (32 positions) and `per` heads of their rows.  Its threads keep
// their token and dims over the heads, so that sines and cosines are computed once and stay in registers.  Values are turned
// over through LDS: the cache holds eight tokens of a dim together.
template <bool kBf16>
__global__ __launch_bounds__(kThreads) void rope_append_blocks(const void* __restrict__ qkv, const float* __restrict__ inv_freq, KvView kv,
                                                               RopeShape s, int per, uint16_t* __restrict__ q) {
    constexpr int kMost = 256 / 8 * kKvBlock / kThreads;       // pieces of eight dims a thread at most: four
    __shared__ uint16_t tile[kKvBlock * (256 + 2)];
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

    int tok[kMost], d0[kMost];
    Turn turn[kMost][8];
#pragma unroll
    for (int m = 0; m < kMost; ++m) {
        // eight pieces of a row next to each other, then eight tokens: 128 bytes of a bf16 row at a time
        const int i = threadIdx.x + m * kThreads, tiles = (quads + 7) >> 3;
        const int j = (i & 7) + 8 * ((i >> 6) % tiles);
        tok[m] = ((i >> 3) & 7) + 8 * ((i >> 6) / tiles);
        d0[m] = 8 * j;
        if (j >= quads || tok[m] < t0 || tok[m] >= t1) tok[m] = -1;
        if (tok[m] >= 0 && u0 < s.heads + kv.kv_heads)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (s.pairs && (e & 1)) { turn[m][e] = turn[m][e - 1]; continue; }
                turn[m][e] = d0[m] + e < s.rotary ? turn_of(blk * kKvBlock + tok[m], inv_freq[pair_of(d0[m] + e, s)]) : Turn{1.0f, 0.0f};
            }
    }
    for (int u = u0; u < u1; ++u) {
        const bool query = u < s.heads, key = !query && u < s.heads + kv.kv_heads;
        int block = -1;
        if (!query && blk >= 0) block = kv.block(kv.table + b * kv.table_stride, blk, key ? u - s.heads : u - s.heads - kv.kv_heads);
        if (!query && block < 0) continue;                     // the same for the whole workgroup
        const int64_t at = (int64_t)block * kKvBlock * Dp;
#pragma unroll
        for (int m = 0; m < kMost; ++m) {
            if (tok[m] < 0) continue;
            const int64_t r = row0 + tok[m], head = (r * units + u) * D;
            float x[8];
            load8<kBf16>(x, qkv, head + d0[m], D - d0[m]);
            if (query || key) {
                if (d0[m] < s.rotary) {
                    float y[8];
                    partners<kBf16>(y, x, qkv, head, d0[m], s);
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (d0[m] + e < s.rotary) x[e] = x[e] * turn[m][e].cos + y[e] * turn[m][e].sin;
                }
                const uint4 w = pack8(x);
                if (query) store_any(q + (r * s.heads + u) * D + d0[m], w, D - d0[m]);
                else *reinterpret_cast<uint4*>(kv.k + at + kv_key_at(tok[m], d0[m])) = w;
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) tile[tok[m] * (256 + 2) + d0[m] + e] = f32_to_bf16(x[e]);
            }
        }
        if (query || key) continue;
        __syncthreads();
        for (int i = threadIdx.x; i < 4 * D; i += kThreads) {
            const int g = i / D, d = i - g * D;
            if (8 * g + 8 <= t0 || 8 * g >= t1) continue;
            uint16_t e[8];
#pragma unroll
            for (int t = 0; t < 8; ++t) e[t] = tile[(8 * g + t) * (256 + 2) + d];
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
    const int64_t tiles = tiles_at_most(T, kv.B, 1, kKvBlock, 2);
    const int per = (int)(tiles * units <= 1024 ? 1 : tiles * units >= 8192 ? 8 : ceil_div(tiles * units, 1024));
    const dim3 grid((unsigned)tiles, (unsigned)ceil_div(units, per));
    if (bf16) rope_append_blocks<true><<<grid, kThreads, 0, stream>>>(qkv, inv_freq, kv, s, per, qo);
    else rope_append_blocks<false><<<grid, kThreads, 0, stream>>>(qkv, inv_freq, kv, s, per, qo);
    return hipGetLastError();
}

}  // namespace bitnet
