// Eviction: of each sequence and key-value head the `recent` last tokens stay and the keep - recent of the others that have had the most weight, ties to
// the lower position, in their order; keys, values and accumulated weights go to other pages.
//
// First launch: one workgroup for a sequence's head.  The weight of the last token that stays is found digit by digit (11, 11 and 10 bits of an
// unsigned image of the float that keeps the order), by counts in LDS; then the positions above it, and of those equal to it the first ones, are
// numbered by a running sum.  Second launch: the tokens of a block of the new pages to a workgroup.
//
// Measured on five sequences of 20000 to 40000 tokens, 8 heads of 128, cut to 8000: the choice 41 us, bound by one CU's instructions and LDS (a pass over 30000
// weights 6, numbering and writing 8000 positions 13); the move 145, bound by memory, as a token's dims share 128-byte lines with the tokens
// around it: 581 MB read for the 164 that stay, 5.1 TB/s.
#include "bitnet_device.hpp"
#include "bitnet_internal.hpp"
#include "kv_layout.hpp"

namespace bitnet {
namespace {

struct EvictArgs {
    const float* weights;              // [B][kv heads][stride]
    float* weights_out;                // [B][kv heads][stride_out]
    const int32_t* table_out;
    int32_t *len_out, *kept;           // [B], [B][kv heads][keep]
    int64_t stride, stride_out, table_stride;
    int keep, recent;
};

// unsigned integers in the order of the weights: -0 with 0, what is no number above all others
__device__ inline uint32_t rank_of(float w) {
    const uint32_t u = __float_as_uint(w + 0.0f);
    return w != w ? 0xFFFFFFFFu : u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ inline float weight_of(uint32_t rank) { return __uint_as_float(rank & 0x80000000u ? rank == 0xFFFFFFFFu ? 0x7FC00000u : rank & 0x7FFFFFFFu : ~rank); }

constexpr int kThreads = 1024, kWaves = kThreads / 64, kEach = 4, kTurn = kThreads * kEach;

// the sum over the lanes in front of this one
__device__ inline uint32_t wave_before(uint32_t v, uint32_t* all) {
    const int lane = threadIdx.x & 63;
    uint32_t s = v;
#pragma unroll
    for (int by = 1; by < 64; by *= 2) {
        const uint32_t o = __shfl_up(s, by);
        if (lane >= by) s += o;
    }
    *all = __shfl(s, 63);
    return s - v;
}
// n plus the number of lanes in front of this one whose bit is set
__device__ inline uint32_t lanes_before(uint64_t bits, uint32_t n) {
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(bits >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)bits, n));
}

// kTurns turns of kTurn tokens stay in registers, four consecutive ones a thread and turn, all of them requested at once; what a sequence has
// beyond them is read again in every pass.
template <int kTurns>
__global__ __launch_bounds__(kThreads) void evict_choose(EvictArgs a, KvView kv) {
    // of each digit, four times over, a quarter of the lanes each: lanes that meet on one word wait for each other (30000 weights of which a tenth are zero: 38 us
    // with one count, 36 with four)
    __shared__ uint4 counts[2048];
    __shared__ uint32_t sums[2][kWaves];
    __shared__ uint32_t found[2];                          // the digit, and how many of the tokens that have it are still to be taken
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int b = blockIdx.x / kv.kv_heads;
    const uint32_t len = kv.length(kv.kv_len[b]);
    const float* w = a.weights + (int64_t)blockIdx.x * a.stride;
    float* w_out = a.weights_out + (int64_t)blockIdx.x * a.stride_out;
    int32_t* kept = a.kept + (int64_t)blockIdx.x * a.keep;
    const uint32_t keep = a.keep, recent = a.recent;
    const uint32_t late = len <= keep ? 0 : len - recent;  // the first of the tokens that stay for being the last ones
    const bool some = late > 0 && keep > recent;
    struct Four { uint32_t rank[kEach]; };
    auto fetch = [&](uint32_t turn) {
        const uint32_t p = turn * kTurn + threadIdx.x * kEach;
        float x[kEach] = {};
        if (len >= kEach) {                                // one load without a condition, so that those of all turns go out together; behind the
            const uint32_t at = min(p, len - kEach);       // last token whatever stands in the last four
            __builtin_memcpy(x, w + at, sizeof x);
            if (p - at & 1) x[0] = x[1], x[1] = x[2], x[2] = x[3];
            if (p - at & 2) x[0] = x[2], x[1] = x[3];
        } else if (p == 0) {
#pragma unroll
            for (int e = 0; e < kEach - 1; ++e) if ((uint32_t)e < len) x[e] = w[e];
        }
        Four f;
#pragma unroll
        for (int e = 0; e < kEach; ++e) f.rank[e] = rank_of(x[e]);
        return f;
    };
    Four held[kTurns];
#pragma unroll
    for (int t = 0; t < kTurns; ++t) held[t] = fetch(t);
    const uint32_t turns = (len + kTurn - 1) / kTurn;
    // `go` for each turn in front of `end`, with its number and its tokens
    auto each_turn = [&](uint32_t end, auto go) {
#pragma unroll
        for (int t = 0; t < kTurns; ++t)
            if ((uint32_t)t < end) go((uint32_t)t, held[t]);
        for (uint32_t t = kTurns; t < end; ++t) go(t, fetch(t));
    };
    uint32_t least = 0, take = 0;                          // the rank of the last one of the others that stays, and how many of those that have it
    if (some) {
        uint32_t prefix = 0, mask = 0;
        take = keep - recent;
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
            for (int i = threadIdx.x; i < 2048; i += kThreads) counts[i] = uint4{0, 0, 0, 0};
            __syncthreads();
            each_turn((late + kTurn - 1) / kTurn, [&](uint32_t t, const Four& f) {
                const uint32_t first = t * kTurn + threadIdx.x * kEach;
#pragma unroll
                for (int e = 0; e < kEach; ++e) {
                    const uint32_t digit = (f.rank[e] >> shift) & ((1u << bits) - 1);
                    const bool counted = (f.rank[e] & mask) == prefix && first + e < late;
                    if (pass > 0) {                        // few, or many that are alike: lanes that all have one digit count it together
                        const uint64_t who = __builtin_amdgcn_ballot_w64(counted);
                        if (!who) continue;
                        const uint32_t one = __builtin_amdgcn_readlane(digit, __builtin_ctzll(who));
                        if (__builtin_amdgcn_ballot_w64(counted && digit == one) == who) {
                            if (lane == __builtin_ctzll(who)) atomicAdd(&counts[one].x, (uint32_t)__builtin_popcountll(who));
                            continue;
                        }
                    }
                    if (counted) atomicAdd(&counts[digit].x + (lane & 3), 1u);
                }
            });
            __syncthreads();
            // from the largest digit down: two a thread, counts of those above them
            const int d = 2047 - 2 * threadIdx.x;
            auto count_of = [&](int digit) { const uint4 c = counts[digit]; return (c.x + c.y) + (c.z + c.w); };
            const uint32_t high = count_of(d), own = high + count_of(d - 1);
            uint32_t all, above = wave_before(own, &all);
            if (lane == 0) sums[0][wave] = all;
            __syncthreads();
            for (int i = 0; i < wave; ++i) above += sums[0][i];
            if (above < take && above + high >= take) found[0] = d, found[1] = take - above;
            else if (above + high < take && above + own >= take) found[0] = d - 1, found[1] = take - above - high;
            __syncthreads();
            prefix |= found[0] << shift;
            mask |= ((1u << bits) - 1) << shift;
            take = found[1];
            least = prefix;
            const bool all_of_it = take == count_of(found[0]);
            __syncthreads();
            if (all_of_it && prefix) {                     // all that have the digit stay, and none needs to be told from another
                least = prefix - 1, take = 0;
                break;
            }
        }
    }
    // Positions in order: those above `least`, equal to it (as far as `take` goes), or late.  What has been counted in front of a turn is the same in all
    // threads.  A turn's tokens go to places in front of the next one's, and are all read in front of its barrier: the weights may stay where they are.
    uint32_t equal = 0, number = 0;
    each_turn(turns, [&](uint32_t t, const Four& f) {
        const uint32_t first = t * kTurn + threadIdx.x * kEach;
        uint32_t more = 0, same = 0, before_more = 0, before_same = 0, all_more = 0, all_same = 0;      // more, same: bits
        const bool inside = (t + 1) * kTurn <= late;       // no token of the turn stays for being late
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const uint32_t p = first + e, u = f.rank[e];
            const bool is_more = inside ? some && u > least : p < len && (p >= late || (some && u > least));
            const uint64_t m = __builtin_amdgcn_ballot_w64(is_more);
            before_more = lanes_before(m, before_more);
            all_more += __builtin_popcountll(m);
            more |= (uint32_t)is_more << e;
            if (take == 0) continue;
            const bool is_same = u == least && p < late;
            const uint64_t q = __builtin_amdgcn_ballot_w64(is_same);
            before_same = lanes_before(q, before_same);
            all_same += __builtin_popcountll(q);
            same |= (uint32_t)is_same << e;
        }
        if (lane == 0) sums[t & 1][wave] = all_more | all_same << 16;
        __syncthreads();
        const uint32_t each = sums[t & 1][lane & (kWaves - 1)];
        uint32_t total = 0, front = 0;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) {
            if (i == wave) front = total;
            total += __builtin_amdgcn_readlane(each, i);
        }
        uint32_t eq = equal + (front >> 16) + before_same, to = number + (front & 0xFFFFu) + before_more + min(eq, take);
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const bool tie = same >> e & 1 && eq < take;
            eq += same >> e & 1;
            if ((more >> e & 1) || tie) {
                kept[to] = (int32_t)(first + e);
                w_out[to] = weight_of(f.rank[e]);
                ++to;
            }
        }
        equal += total >> 16;
        number += total & 0xFFFFu;
    });
}

__global__ __launch_bounds__(256) void evict_move(EvictArgs a, KvView kv, int blocks_out, int64_t tasks) {
    __shared__ int64_t from[kKvBlock];                     // of each token of the block: its block's first element, or -1
    __shared__ int in[kKvBlock];                           // and its place there
    const int Dp = kv_padded_dim(kv.D), quads = Dp >> 3;
    for (int64_t task = blockIdx.x; task < tasks; task += gridDim.x) {
        const int64_t pair = task / blocks_out;
        const int blk = (int)(task - pair * blocks_out), b = (int)(pair / kv.kv_heads), h = (int)(pair - (int64_t)b * kv.kv_heads);
        const int len = min(kv.length(kv.kv_len[b]), a.keep), count = min(len - blk * kKvBlock, kKvBlock);
        if (blk == 0 && h == 0 && threadIdx.x == 0) a.len_out[b] = len;      // may be kv_len itself: `len` comes out the same
        if (count <= 0) continue;
        const int p = blk / kv.page_blocks, to_block = kv.block_on(a.table_out[b * a.table_stride + p], blk - p * kv.page_blocks, h);
        if (to_block < 0) continue;
        __syncthreads();
        if ((int)threadIdx.x < count) {
            const int pos = a.kept[pair * a.keep + blk * kKvBlock + threadIdx.x];
            const int number = kv.block(kv.table + b * kv.table_stride, pos >> 5, h);
            from[threadIdx.x] = number < 0 ? -1 : (int64_t)number * kKvBlock * Dp;
            in[threadIdx.x] = pos & 31;
        }
        __syncthreads();
        const int64_t to = (int64_t)to_block * kKvBlock * Dp;
        for (int i = threadIdx.x; i < kKvBlock * quads; i += 256) {
            const int place = i & 31, j = i >> 5, t = 8 * ((place >> 2) & 3) + 4 * (place >> 4) + (place & 3);      // the token at that place
            if (t >= count) continue;
            const int64_t f = from[t];
            *reinterpret_cast<uint4*>(kv.k + to + i * 8) = f < 0 ? uint4{0, 0, 0, 0} : *reinterpret_cast<const uint4*>(kv.k + f + kv_key_at(in[t], 8 * j));
        }
        for (int i = threadIdx.x; i < 4 * Dp; i += 256) {
            const int g = i / Dp, d = i - g * Dp;
            if (8 * g >= count) continue;
            uint16_t e[8];
#pragma unroll
            for (int t = 0; t < 8; ++t) {
                const int64_t f = 8 * g + t < count ? from[8 * g + t] : -1;
                e[t] = f < 0 ? (uint16_t)0 : kv.v[f + kv_value_at(in[8 * g + t], d, Dp)];
            }
            uint16_t* v = kv.v + to + i * 8;
            if (8 * g + 8 <= count) {
                uint4 w;
                __builtin_memcpy(&w, e, 16);
                *reinterpret_cast<uint4*>(v) = w;
            } else {
#pragma unroll
                for (int t = 0; t < 8; ++t) if (8 * g + t < count) v[t] = e[t];
            }
        }
    }
}

}  // namespace

hipError_t launch_kv_evict(const KvView& kv, const float* weights, int64_t stride, int keep, int recent, const int32_t* table_out, int64_t table_out_stride,
                           float* weights_out, int64_t stride_out, int32_t* len_out, int32_t* kept, hipStream_t stream) {
    const EvictArgs a{weights, weights_out, table_out, len_out, kept, stride, stride_out, table_out_stride, keep, recent};
    const unsigned pairs = (unsigned)((int64_t)kv.B * kv.kv_heads);
    const int64_t turns = ceil_div((int64_t)kv.max_blocks * kKvBlock, kTurn);
    if (turns <= 1) evict_choose<1><<<pairs, kThreads, 0, stream>>>(a, kv);
    else if (turns <= 4) evict_choose<4><<<pairs, kThreads, 0, stream>>>(a, kv);
    else evict_choose<10><<<pairs, kThreads, 0, stream>>>(a, kv);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int64_t most = (int64_t)kv.max_blocks * kKvBlock;
    const int blocks_out = (int)ceil_div(keep < most ? keep : most, kKvBlock);
    const int64_t tasks = (int64_t)kv.B * kv.kv_heads * blocks_out;
    evict_move<<<(unsigned)(tasks < kMaxLoopBlocks ? tasks : kMaxLoopBlocks), 256, 0, stream>>>(a, kv, blocks_out, tasks);
    return hipGetLastError();
}

}  // namespace bitnet
