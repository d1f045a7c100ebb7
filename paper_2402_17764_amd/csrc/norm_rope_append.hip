// Norms of queries and keys head by head, rotary positions and the paged cache, in one pass over the rows of a merged Q | K | V product.
//
// A head x of D dims becomes y = x r gain, r = 1 / sqrt(mean(x^2) + eps), and y is turned by its position as in rope_append.hip; the position
// is the token's place in the cache plus its sequence's shift.  Squares are summed in 64 bits, which hold them whatever the head's size is; products and
// turns are 32 bits wide, and the result is rounded once, to the cache's bf16.
#include "rope_slots.hpp"

namespace bitnet {
namespace {

constexpr int kThreads = 256, kGains = 256;

struct NormShape {
    const float *q_gain, *k_gain;      // [D] or NULL
    const int32_t* shift;              // [B] or NULL
    float eps;
    int norm;                          // 0: heads are turned as they are
};

// 1 / sqrt(mean + eps): the 64-bit instruction's 2^-23 and one Newton step.  A head of zeros stays zeros, whatever eps is; of one with an infinity (its sum in
// 64 bits has no other way to be one) the finite dims become zeros and the others NaN.
struct HeadScale { float first, then; };   // two factors: of heads whose elements are near either end of fp32's range the one would not be a normal number
__device__ inline HeadScale head_scale(double sum, double inv_d, float eps) {
#if defined(__HIP_DEVICE_COMPILE__)
    const double a = __builtin_fma(sum, inv_d, (double)eps);
    const double y = __builtin_amdgcn_rsq(a), r = y * __builtin_fma(-0.5 * a, y * y, 1.5);
    if (r >= 0x1p-64 && r <= 0x1p64 && sum > 0.0) return {1.0f, (float)r};
    if (!(sum > 0.0)) return {1.0f, sum == 0.0 ? 0.0f : (float)sum};   // NaN stays
    if (sum == __builtin_inf()) return {1.0f, 0.0f};
    if (r > 1.0) return {0x1p64f, (float)(r * 0x1p-64)};                // elements below 2^-60: exact
    return {0x1p-64f, (float)(r * 0x1p64)};
#else
    return {};
#endif
}

template <bool kBf16>
__device__ inline double squares_of(const Eight<kBf16>& v, int count) {
    float x[8];
    floats_of<kBf16>(x, v);
    double s = 0.0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const double y = e < count ? (double)x[e] : 0.0;
        s = __builtin_fma(y, y, s);
    }
    return s;
}
// the sum over kLanes neighbouring lanes
template <int kLanes>
__device__ inline double lanes_sum(double v) {
    v += dpp_f64<0xB1>(v);
    v += dpp_f64<0x4E>(v);
    v += dpp_f64<0x141>(v);
    if (kLanes >= 16) v += dpp_f64<0x140>(v);
    if (kLanes >= 32) v += __shfl_xor(v, 16);
    return v;
}

// x[e] *= r gain[d + e], of the dims in front of `end`; gain NULL: ones
__device__ inline void gains_of(float (&g)[8], const float* gain, int d, int end) {
#pragma unroll
    for (int e = 0; e < 8; ++e) g[e] = gain && d + e >= 0 && d + e < end ? gain[d + e] : 1.0f;
}

// Eight dims from d0 on of a head, with their partners' raw values (Split: of the lower half; Any: those in front and behind) and all gains, turned.
template <bool kBf16, Turned kTurned>
__device__ inline void norm_and_turn(float (&x)[8], float (&y)[8], const Slot<kBf16, kTurned>& v, int d0, HeadScale r, const float (&g)[8], const float (&partner)[8],
                                     const Turn (&t)[8], const RopeShape& s) {
    const int half = s.rotary >> 1;
    auto scale = [&](float (&z)[8], const float (&gains)[8]) {
        if (__builtin_amdgcn_ballot_w64(r.first != 1.0f))
#pragma unroll
            for (int e = 0; e < 8; ++e) z[e] *= r.first;
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] = z[e] * r.then * gains[e];
    };
    floats_of<kBf16>(x, v.own);
    scale(x, g);
    if constexpr (kTurned == Turned::Split) {
        if (d0 >= half) return;
        floats_of<kBf16>(y, v.low);
        scale(y, partner);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float a = x[e] * t[e].cos - y[e] * t[e].sin;
            y[e] = y[e] * t[e].cos + x[e] * t[e].sin;
            x[e] = a;
        }
    } else if constexpr (kTurned == Turned::Pairs) {
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            if (d0 + e >= s.rotary) continue;
            const float a = x[e] * t[e].cos - x[e + 1] * t[e].sin;
            x[e + 1] = x[e + 1] * t[e].cos + x[e] * t[e].sin;
            x[e] = a;
        }
    } else {
        float l[8], h[8];
        floats_of<kBf16>(l, v.low);
        floats_of<kBf16>(h, v.high);
#pragma unroll
        for (int e = 0; e < 8; ++e) l[e] = d0 + e < half ? -l[e] : h[e];
        scale(l, partner);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (d0 + e < s.rotary) x[e] = x[e] * t[e].cos + l[e] * t[e].sin;
    }
}
// the gains of eight dims and of their partners
template <Turned kTurned>
__device__ inline void gains_for(float (&g)[8], float (&partner)[8], const float* gain, int d0, int D, const RopeShape& s) {
    const int half = s.rotary >> 1;
    gains_of(g, gain, d0, D);
    if (kTurned == Turned::Split) gains_of(partner, gain, d0 + half, d0 < half ? D : 0);
    if (kTurned == Turned::Any)
#pragma unroll
        for (int e = 0; e < 8; ++e) partner[e] = gain && d0 + e < s.rotary ? gain[d0 + e < half ? d0 + e + half : d0 + e - half] : 1.0f;
}

// One new token for each sequence.  A thread takes eight dims of a head, a workgroup whole heads, whose threads' sums of squares meet in LDS at the
// barrier that the sines and cosines need anyway.
template <bool kBf16>
__global__ __launch_bounds__(kThreads) void norm_rope_append_tokens(const void* __restrict__ qkv, const float* __restrict__ inv_freq, NormShape w, KvView kv,
                                                                    RopeShape s, int quads, uint16_t* __restrict__ q) {
    __shared__ Turn turns[128];
    __shared__ double squares[kThreads];
    const int b = blockIdx.x, per = kThreads / quads, in = threadIdx.x / quads, j = threadIdx.x - in * quads;
    const int unit = blockIdx.y * per + in, units = s.heads + 2 * kv.kv_heads, D = kv.D, d0 = 8 * j;
    const bool mine = in < per && unit < units;
    const int64_t row = (int64_t)b * units * D, head = row + (int64_t)unit * D;
    const int pos = kv.length(kv.kv_len[b]) - 1;
    const bool query = unit < s.heads, turned = mine && unit < s.heads + kv.kv_heads;
    Slot<kBf16, Turned::Any> slot;
    if (mine) slot.load(qkv, head, (int64_t)(units - unit) * D, d0, D, turned && !s.pairs, s);
    float g[8], partner[8];
    if (turned) {
        const float* gain = w.norm ? (query ? w.q_gain : w.k_gain) : nullptr;
        if (s.pairs) gains_for<Turned::Pairs>(g, partner, gain, d0, D, s);
        else gains_for<Turned::Any>(g, partner, gain, d0, D, s);
    }
    const double at = (double)pos + (double)(w.shift ? w.shift[b] : 0);
    for (int i = threadIdx.x; i < s.rotary >> 1; i += kThreads) turns[i] = turn_of(at, inv_freq[i]);
    if (w.norm && turned) squares[threadIdx.x] = squares_of<kBf16>(slot.own, D - d0);
    __syncthreads();
    if (!mine) return;
    float x[8], none[8];
    if (turned) {
        HeadScale r{1.0f, 1.0f};
        if (w.norm) {
            double sum = 0.0;
            for (int i = 0; i < quads; ++i) sum += squares[threadIdx.x - j + i];
            r = head_scale(sum, 1.0 / D, w.eps);
        }
        Turn by[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) by[e] = d0 + e < s.rotary ? turns[pair_of(d0 + e, s)] : Turn{1.0f, 0.0f};
        if (s.pairs) {
            const Slot<kBf16, Turned::Pairs> p{slot.own, {}, {}};
            norm_and_turn(x, none, p, d0, r, g, partner, by, s);
        } else {
            norm_and_turn(x, none, slot, d0, r, g, partner, by, s);
        }
    } else {
        floats_of<kBf16>(x, slot.own);
    }
    const uint4 out = pack8(x);
    if (query) {
        store_any(q + ((int64_t)b * s.heads + unit) * D + d0, out, D - d0);
        return;
    }
    if (pos < 0) return;
    const int h = turned ? unit - s.heads : unit - s.heads - kv.kv_heads;
    const int Dp = kv_padded_dim(D), t = pos & 31;
    const int block = kv.block(kv.table + b * kv.table_stride, pos >> 5, h);
    if (block < 0) return;
    const int64_t place = (int64_t)block * kKvBlock * Dp;
    if (turned) {
        *reinterpret_cast<uint4*>(kv.k + place + kv_key_at(t, d0)) = first_of(out, D - d0);
    } else {
        const uint32_t u[4] = {out.x, out.y, out.z, out.w};
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (d0 + i < D) kv.v[place + kv_value_at(t, d0 + i, Dp)] = (uint16_t)(u[i >> 1] >> (16 * (i & 1)));
    }
}

// Waves that have to fit on a SIMD: pairs of bf16 that miss one by two registers cost 10 %.
constexpr int norm_waves(bool bf16, Turned turned, int lanes) {
    return !bf16 || turned != Turned::Pairs ? 1 : lanes == 8 ? 8 : lanes == 16 ? 6 : 4;
}

// Runs of new tokens: a workgroup takes the new tokens of one cache block (32 positions) and `per` heads of their rows.  The slots of a head of a token
// stand in kLanes neighbouring lanes of a wave, which add up their squares without LDS; a thread keeps its tokens and dims over the heads, so that
// sines and cosines are computed once.  Values are turned over through LDS: the cache holds eight tokens of a dim together.
//
// Bound by memory: two prompts of 2000 tokens, 64 heads of 128 over 8, 47.8 us, 3.5 TB/s (the same without norms 42).  Gains come from LDS (in 16 registers more
// 62, as fewer waves fit).  Sums of squares in 32 bits, which lose what is small beside a large element: 46, and 16.4 instead of 17.7 on ragged prompts of
// 41 MB, 32 heads of 100.
template <bool kBf16, Turned kTurned, int kLanes>
__global__ __launch_bounds__(kThreads, norm_waves(kBf16, kTurned, kLanes)) void norm_rope_append_blocks(const void* __restrict__ qkv, const float* __restrict__ inv_freq, NormShape w, KvView kv,
                                                                    RopeShape s, int per, uint16_t* __restrict__ q) {
    constexpr int kM = kLanes / 8, kTokens = kThreads / kLanes, kPitch = 256 + 8;      // tokens of a workgroup at a time
    __shared__ uint4 tile4[kKvBlock * kPitch / 8];
    __shared__ __attribute__((aligned(16))) float gain_of[2 * kGains];                 // of queries, of keys: ones where there is none
    uint16_t* tile = reinterpret_cast<uint16_t*>(tile4);
    const int D = kv.D, Dp = kv_padded_dim(D), units = s.heads + 2 * kv.kv_heads, keys = s.heads + kv.kv_heads;
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
    const int page_index = blk >= 0 ? blk / kv.page_blocks : 0, page = blk >= 0 ? kv.table[b * kv.table_stride + page_index] : -1;
    const double shift = w.shift ? (double)w.shift[b] : 0.0;
    const double inv_d = 1.0 / D;
    const int half = s.rotary >> 1, half8 = (half + 7) >> 3, slots = slots_of<kTurned>(D, s);
    const int j = threadIdx.x & (kLanes - 1);
    const int d0 = kTurned == Turned::Split && j >= half8 ? s.rotary + 8 * (j - half8) : 8 * j;
    const bool both = kTurned == Turned::Split && d0 < half;   // eight dims of the lower half and their partners
    int tok[kM];
    Turn turn[kM][8];
#pragma unroll
    for (int m = 0; m < kM; ++m) {
        tok[m] = threadIdx.x / kLanes + m * kTokens;
        if (j >= slots || tok[m] < t0 || tok[m] >= t1) tok[m] = -1;
        if (tok[m] >= 0 && u0 < keys)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (kTurned == Turned::Pairs && (e & 1)) { turn[m][e] = turn[m][e - 1]; continue; }
                turn[m][e] = d0 + e < s.rotary ? turn_of((double)(blk * kKvBlock + tok[m]) + shift, inv_freq[pair_of(d0 + e, s)]) : Turn{1.0f, 0.0f};
            }
    }
    Slot<kBf16, kTurned> slot[kM], next[kM];
    auto request = [&](Slot<kBf16, kTurned> (&x)[kM], int u) {
#pragma unroll
        for (int m = 0; m < kM; ++m)
            if (tok[m] >= 0) x[m].load(qkv, ((int64_t)(row0 + tok[m]) * units + u) * D, (int64_t)(units - u) * D, d0, D, u < keys, s);
    };
    request(next, u0);
    for (int i = threadIdx.x; i < 2 * kGains; i += kThreads) {
        const float* gain = !w.norm ? nullptr : i < kGains ? w.q_gain : w.k_gain;
        const int d = i & (kGains - 1);
        gain_of[i] = gain && d < D ? gain[d] : 1.0f;
    }
    __syncthreads();
#pragma unroll 1
    for (int u = u0; u < u1; ++u) {
#pragma unroll
        for (int m = 0; m < kM; ++m) slot[m] = next[m];
        if (u + 1 < u1) request(next, u + 1);
        const bool query = u < s.heads, key = !query && u < keys;
        int block = -1;
        if (!query) block = kv.block_on(page, blk - page_index * kv.page_blocks, key ? u - s.heads : u - keys);
        if (!query && block < 0) continue;                     // the same for the whole workgroup
        const int64_t at = (int64_t)block * kKvBlock * Dp;
#pragma unroll
        for (int m = 0; m < kM; ++m) {
            HeadScale r{1.0f, 1.0f};
            if (w.norm && (query || key)) {                    // all lanes: the sum goes over neighbours
                double sum = 0.0;
                if (tok[m] >= 0) {
                    sum = squares_of<kBf16>(slot[m].own, D - d0);
                    if (both) sum += squares_of<kBf16>(slot[m].low, 8);
                }
                r = head_scale(lanes_sum<kLanes>(sum), inv_d, w.eps);
            }
            if (tok[m] < 0) continue;
            const int64_t out = ((int64_t)(row0 + tok[m]) * s.heads + u) * D;
            auto put = [&](int d, uint4 v) {
                if (query) store_any(q + out + d, v, D - d);
                else if (key) *reinterpret_cast<uint4*>(kv.k + at + kv_key_at(tok[m], d)) = first_of(v, D - d);
                else *reinterpret_cast<uint4*>(&tile[tok[m] * kPitch + d]) = v;
            };
            float x[8], y[8];
            if (query || key) {
                float g[8], partner[8];
                const float* gain = gain_of + (query ? 0 : kGains);
                __builtin_memcpy(g, __builtin_assume_aligned(gain + d0, 16), sizeof g);
                if (kTurned == Turned::Split) __builtin_memcpy(partner, __builtin_assume_aligned(gain + (both ? d0 + half : d0), 16), sizeof partner);
                if (kTurned == Turned::Any)
#pragma unroll
                    for (int e = 0; e < 8; ++e) partner[e] = gain[d0 + e < half ? d0 + e + half : max(d0 + e - half, 0)];
                norm_and_turn(x, y, slot[m], d0, r, g, partner, turn[m], s);
            } else {
                floats_of<kBf16>(x, slot[m].own);
                if (both) floats_of<kBf16>(y, slot[m].low);
            }
            put(d0, pack8(x));
            if (both) put(d0 + half, pack8(y));
        }
        if (query || key) continue;
        __syncthreads();
        for (int i = threadIdx.x; i < 4 * D; i += kThreads) {
            const int c = i / D, d = i - c * D;
            if (8 * c + 8 <= t0 || 8 * c >= t1) continue;
            uint16_t e[8];
#pragma unroll
            for (int t = 0; t < 8; ++t) e[t] = tile[(8 * c + t) * kPitch + d];
            uint16_t* to = kv.v + at + (c * Dp + d) * 8;
            if (8 * c >= t0 && 8 * c + 8 <= t1) {
                uint4 v;
                __builtin_memcpy(&v, e, 16);
                *reinterpret_cast<uint4*>(to) = v;
            } else {                                           // tokens of earlier calls stay as they are
#pragma unroll
                for (int t = 0; t < 8; ++t) if (8 * c + t >= t0 && 8 * c + t < t1) to[t] = e[t];
            }
        }
        __syncthreads();
    }
}

template <bool kBf16, Turned kTurned>
hipError_t launch_norm_blocks(const void* qkv, const float* inv_freq, const NormShape& w, const KvView& kv, const RopeShape& s, uint16_t* q, hipStream_t stream) {
    const int units = s.heads + 2 * kv.kv_heads, slots = slots_of<kTurned>(kv.D, s);
    const int64_t tiles = tiles_at_most(s.T, kv.B, 1, kKvBlock, 2);
    const int64_t all = tiles * units / 704;                   // heads of a workgroup: as in rope_append.hip
    const int per = (int)(all < 1 ? 1 : all > 4 ? 4 : all);
    const dim3 grid((unsigned)tiles, (unsigned)ceil_div(units, per));
    if (slots <= 8) norm_rope_append_blocks<kBf16, kTurned, 8><<<grid, kThreads, 0, stream>>>(qkv, inv_freq, w, kv, s, per, q);
    else if (slots <= 16) norm_rope_append_blocks<kBf16, kTurned, 16><<<grid, kThreads, 0, stream>>>(qkv, inv_freq, w, kv, s, per, q);
    else norm_rope_append_blocks<kBf16, kTurned, 32><<<grid, kThreads, 0, stream>>>(qkv, inv_freq, w, kv, s, per, q);
    return hipGetLastError();
}
template <bool kBf16>
hipError_t launch_norm_blocks(const void* qkv, const float* inv_freq, const NormShape& w, const KvView& kv, const RopeShape& s, uint16_t* q, hipStream_t stream) {
    // halves that are no multiple of eight have only the form that reads partners on both sides (4096 tokens, 32 heads of 100: bf16 80 us, pairs 38)
    if (s.pairs) return launch_norm_blocks<kBf16, Turned::Pairs>(qkv, inv_freq, w, kv, s, q, stream);
    if (s.rotary % 16 == 0) return launch_norm_blocks<kBf16, Turned::Split>(qkv, inv_freq, w, kv, s, q, stream);
    return launch_norm_blocks<kBf16, Turned::Any>(qkv, inv_freq, w, kv, s, q, stream);
}

}  // namespace

hipError_t launch_norm_rope_append(const void* qkv, bool bf16, bool norm, const float* q_gain, const float* k_gain, float eps, const float* inv_freq, int rotary,
                                   bool pairs, const int32_t* shift, const KvView& kv, int64_t T, int heads, void* q, hipStream_t stream) {
    const RopeShape s{heads, rotary, (int)T, pairs ? 1 : 0};
    const NormShape w{q_gain, k_gain, shift, eps, norm ? 1 : 0};
    uint16_t* qo = static_cast<uint16_t*>(q);
    if (!kv.q_start) {
        const int units = heads + 2 * kv.kv_heads, quads = kv_padded_dim(kv.D) / 8;
        const dim3 grid((unsigned)T, (unsigned)ceil_div(units, kThreads / quads));
        if (bf16) norm_rope_append_tokens<true><<<grid, kThreads, 0, stream>>>(qkv, inv_freq, w, kv, s, quads, qo);
        else norm_rope_append_tokens<false><<<grid, kThreads, 0, stream>>>(qkv, inv_freq, w, kv, s, quads, qo);
        return hipGetLastError();
    }
    return bf16 ? launch_norm_blocks<true>(qkv, inv_freq, w, kv, s, qo, stream) : launch_norm_blocks<false>(qkv, inv_freq, w, kv, s, qo, stream);
}

}  // namespace bitnet
