// Eviction: of each sequence and key-value head the `recent` last tokens stay and the keep - recent of the others that have had the most weight, ties to
// the lower position, in their order; keys, values and accumulated weights go to other pages.
//
// First launch: one workgroup for a sequence's head.  The weight of the last token that stays is found digit by digit (11, 11 and 10 bits of an
// unsigned image of the float that keeps the order), by counts in LDS; then the positions above it, and of those equal to it the first ones, are
// numbered by a running sum.  Second launch: the tokens of a block of the new pages to a workgroup.
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

constexpr int kThreads = 1024, kWaves = kThreads / 64, kEach = 4;

// the sum over the lanes in front of this one, of two counts in one word
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

__global__ __launch_bounds__(kThreads) void evict_choose(EvictArgs a, KvView kv) {
    __shared__ uint32_t counts[2048], sums[2][kWaves];
    __shared__ uint32_t found[2];                          // the digit, and how many of the tokens that have it are still to be taken
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int b = blockIdx.x / kv.kv_heads;
    const int len = kv.length(kv.kv_len[b]);
    const float* w = a.weights + (int64_t)blockIdx.x * a.stride;
    float* w_out = a.weights_out + (int64_t)blockIdx.x * a.stride_out;
    int32_t* kept = a.kept + (int64_t)blockIdx.x * a.keep;
    const int late = len <= a.keep ? 0 : len - a.recent;   // the first of the tokens that stay for being the last ones
    uint32_t least = 0, take = 0;                          // the rank of the last one of the others that stays, and how many of those that have it
    if (late > 0 && a.keep > a.recent) {
        uint32_t prefix = 0, mask = 0;
        take = a.keep - a.recent;
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
            for (int i = threadIdx.x; i < 2048; i += kThreads) counts[i] = 0;
            __syncthreads();
            for (uint32_t i = threadIdx.x; i < (uint32_t)late; i += kThreads) {
                const uint32_t u = rank_of(w[i]);
                if ((u & mask) == prefix) atomicAdd(&counts[(u >> shift) & ((1u << bits) - 1)], 1u);
            }
            __syncthreads();
            // from the largest digit down: two a thread, counts of those above them
            const int d = 2047 - 2 * threadIdx.x;
            const uint32_t own = counts[d] + counts[d - 1];
            uint32_t all, above = wave_before(own, &all);
            if (lane == 0) sums[0][wave] = all;
            __syncthreads();
            for (int i = 0; i < wave; ++i) above += sums[0][i];
            if (above < take && above + counts[d] >= take) found[0] = d, found[1] = take - above;
            else if (above + counts[d] < take && above + own >= take) found[0] = d - 1, found[1] = take - above - counts[d];
            __syncthreads();
            prefix |= found[0] << shift;
            mask |= ((1u << bits) - 1) << shift;
            take = found[1];
            __syncthreads();
        }
        least = prefix;
    }
    // Positions in order, kEach a thread and turn: above `least`, equal to it (as far as `take` goes), or late.  What has been counted in front of
    // this turn is the same in all threads.
    uint32_t equal = 0, number = 0;
    const uint32_t end = len, last = late;
    const bool some = late > 0 && a.keep > a.recent;
    for (uint32_t i0 = 0; i0 < end; i0 += kThreads * kEach) {
        const uint32_t first = i0 + threadIdx.x * kEach;
        float x[kEach];
        uint32_t more = 0, same = 0;                       // bits
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const uint32_t p = first + e;
            x[e] = p < end ? w[p] : 0.0f;
            const uint32_t u = rank_of(x[e]);
            if (p < end && (p >= last || (some && u > least))) more |= 1u << e;
            else if (p < end && some && u == least) same |= 1u << e;
        }
        uint32_t all, before = wave_before(__popc(more) | (uint32_t)__popc(same) << 16, &all);
        if (lane == 0) sums[0][wave] = all;
        __syncthreads();                                   // all of this turn has been read: what follows may write where it was
        uint32_t total = 0;
        for (int i = 0; i < kWaves; ++i) {
            if (i == wave) before += total;
            total += sums[0][i];
        }
        uint32_t eq = equal + (before >> 16), to = number + (before & 0xFFFFu) + min(eq, take);
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const bool tie = same >> e & 1 && eq < take;
            eq += same >> e & 1;
            if ((more >> e & 1) || tie) {
                kept[to] = (int32_t)(first + e);
                w_out[to] = x[e];
                ++to;
            }
        }
        equal += total >> 16;
        number += total & 0xFFFFu;
        __syncthreads();
    }
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
    evict_choose<<<(unsigned)((int64_t)kv.B * kv.kv_heads), kThreads, 0, stream>>>(a, kv);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int64_t most = (int64_t)kv.max_blocks * kKvBlock;
    const int blocks_out = (int)ceil_div(keep < most ? keep : most, kKvBlock);
    const int64_t tasks = (int64_t)kv.B * kv.kv_heads * blocks_out;
    evict_move<<<(unsigned)(tasks < kMaxLoopBlocks ? tasks : kMaxLoopBlocks), 256, 0, stream>>>(a, kv, blocks_out, tasks);
    return hipGetLastError();
}

}  // namespace bitnet
