// Attention of one new token of each sequence over its cached keys and values:
//   s_j = scale q . k_j,  p = softmax(s),  o = sum_j p_j v_j,
// in one pass over the cache: a wave keeps, for each query of a key-value head, the running maximum m of the scores, the sum l
// of exp(s_j - m) and the values' sum under the same weights, in 32 bits; a new maximum rescales both.
//
// A wave takes 32 tokens at a time.  Scores are MFMA 16 x 16 x 32 products of keys (down) and the queries of the head's group (across,
// up to 16); the cache's order of keys makes their result the operand of the second product, values (dims down) times weights, as it
// stands, and values are stored as that product's other operand: nothing passes through LDS or other lanes but the maximum.
// Every byte of the cache goes from memory to the register that the MFMA reads it from, in 16-byte loads.
#pragma once
#include "attention_common.hpp"

#include <type_traits>

namespace bitnet {

struct DecodeArgs {
    const uint16_t* q;
    void* o;
    float scale;                       // of the softmax, times log2 e
    int heads, group;                  // query heads, and of them per key-value head
    int column_tiles;                  // of 16 query heads, per key-value head
};

// What a launch does: all of a row's attention; the part of it behind what its sequence shares with others (a row's splits stand behind `first` others,
// `pitch` in all); or all of it, leaving the row's scores and softmax state too, for the weights of the tokens.
enum class Single { All, Own, Scored };
struct SingleMore {
    Prefixes prefixes;
    int first, pitch;                  // Own
    float* scores;                     // Scored: [B][heads][max_blocks * 32], what q . k is, -inf for no key
    float* weights;                    // Scored, where a workgroup has all heads and keys of a row: what it adds the weights to itself, or NULL
    int64_t stride;
};

// A row is 16 query heads (or what a group has left) of one key-value head of one sequence.  Its blocks are dealt out to up to
// parts.splits workgroups (blockIdx.y).
template <int kC, int kV, bool kExact, bool kF32, int kW, Single kDo>
__global__ __launch_bounds__(64 * kW, kC <= 4 ? 2 : 1) void attention_decode_rows(DecodeArgs a, Parts parts, KvView kv, std::conditional_t<kDo == Single::All, char, SingleMore> more) {
    constexpr int kWholeChunks = whole_chunks(kC), kParts = kF32 || kDo == Single::Scored ? 3 : 2;      // bf16 operands of a weight
    constexpr int kRound = kV < 4 ? kV : 4;                // tiles that the waves add up at a time
    constexpr int kPitch = 16 * kRound + 4;
    __shared__ float sums[kW * 16 * kPitch], maxima[kW * 16], totals[kW * 16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, g = lane >> 4;
    const int D = kExact ? 32 * kC : kv.D, Dp = kv_padded_dim(D), quads = Dp >> 3;
    const int rows_a_sequence = kv.kv_heads * a.column_tiles, b = blockIdx.x / rows_a_sequence, rest = blockIdx.x - b * rows_a_sequence;
    const int h = rest / a.column_tiles, ct = rest - h * a.column_tiles;
    const int head0 = h * a.group + 16 * ct, columns = min(a.group - 16 * ct, 16);
    // What does not hang on the sequence's length is requested along with it: the queries, and of the page table the first 64
    // entries, one a lane, which are all of it more often than not.
    const int32_t* table = kv.table + b * kv.table_stride;
    const bool short_table = kv.max_pages <= 64;
    const int pages = short_table && lane < kv.max_pages ? table[lane] : -1;
    const int len = kv.length(kv.kv_len[b]), blocks = (len + kKvBlock - 1) / kKvBlock;
    int shared = 0;                                        // tokens that this launch leaves out, the first ones
    if constexpr (kDo == Single::Own) shared = shared_tokens(kv, more.prefixes, b, len);
    const int begin = kDo == Single::Own ? own_first(shared, kKvBlock) : 0, units = kDo == Single::Own ? own_units(len, shared, kKvBlock) : blocks;
    const int run = parts.run(units), blk0 = begin + (int)blockIdx.y * run, blk1 = min(blk0 + run, blocks);
    if (kDo == Single::Own ? blk0 - begin >= units : blk0 >= blocks && blockIdx.y > 0) return;

    v8bf qf[kC];
    load_query<kC, kExact>(qf, r < columns ? a.q + ((int64_t)b * a.heads + head0 + r) * D : nullptr, g, D);

    int koff[kC], voff[kV];                                // bytes within a block
#pragma unroll
    for (int c = 0; c < kC; ++c) koff[c] = (kExact || c < kWholeChunks ? 4 * c + g : min(4 * c + g, quads - 1)) * 512 + r * 16;
#pragma unroll
    for (int i = 0; i < kV; ++i) voff[i] = (g * Dp + (kExact || i < 2 * kWholeChunks ? 16 * i + r : min(16 * i + r, Dp - 1))) * 16;

    v4f acc[kV], l = {0, 0, 0, 0};                         // l: the sum of the weights, four times
#pragma unroll
    for (int i = 0; i < kV; ++i) acc[i] = (v4f){0, 0, 0, 0};
    float m = kMinusInf;
    const v8bf ones = ones_operand();

    struct Block { v4u k[kC][2], v[kV]; };
    // this wave's blocks are first, first + kW, ...; their numbers in the cache stand in the lanes, 64 at a time
    const int first = blk0 + wave, mine = blk1 > first ? (blk1 - first + kW - 1) / kW : 0;
    int numbers = -1;
    auto fetch_numbers = [&](int it) {
        const int blk = first + (it + lane) * kW, p = blk / kv.page_blocks;
        int page = short_table ? __shfl(pages, p) : -1;
        if (!short_table && blk < blk1) page = table[p];
        numbers = blk < blk1 ? kv.block_on(page, blk - p * kv.page_blocks, h) : -1;
    };
    const int64_t block_bytes = (int64_t)kKvBlock * Dp * 2;
    auto load = [&](Block& x, int it) {
        const int64_t at = max(__builtin_amdgcn_readlane(numbers, it & 63), 0) * block_bytes;
        const char *k = reinterpret_cast<const char*>(kv.k) + at, *v = reinterpret_cast<const char*>(kv.v) + at;
#pragma unroll
        for (int c = 0; c < kC; ++c)
#pragma unroll
            for (int t = 0; t < 2; ++t) x.k[c][t] = __builtin_nontemporal_load(reinterpret_cast<const v4u*>(k + koff[c] + 256 * t));
#pragma unroll
        for (int i = 0; i < kV; ++i) x.v[i] = __builtin_nontemporal_load(reinterpret_cast<const v4u*>(v + voff[i]));
    };
    auto take = [&](Block& x, int it, bool known /* whether the block's page exists */) {
        const int left = known ? len - kKvBlock * (first + it * kW) : 0;      // of the block's tokens, how many count
        v4f s[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
#pragma unroll
        for (int c = 0; c < kC; ++c)
#pragma unroll
            for (int t = 0; t < 2; ++t) s[t] = mfma_bf16(__builtin_bit_cast(v8bf, x.k[c][t]), qf[c], s[t]);
        float p[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) p[j] = s[j >> 2][j & 3];
        if (left < kKvBlock) {
#pragma unroll
            for (int j = 0; j < 8; ++j) if (8 * g + j >= left) p[j] = kMinusInf;
#pragma unroll
            for (int i = 0; i < kV; ++i) values_keep(x.v[i], left - 8 * g);
        }
        if constexpr (kDo == Single::Own) {
            const int skip = shared - kKvBlock * (first + it * kW);           // of the block's tokens, how many are shared ones
            if (skip > 0) {
#pragma unroll
                for (int j = 0; j < 8; ++j) if (8 * g + j < skip) p[j] = kMinusInf;
#pragma unroll
                for (int i = 0; i < kV; ++i) values_drop(x.v[i], skip - 8 * g);
            }
        }
        if constexpr (kDo == Single::Scored) {
            if (r < columns) {
                float* to = more.scores + ((int64_t)b * a.heads + head0 + r) * ((int64_t)kv.max_blocks * kKvBlock) + (int64_t)kKvBlock * (first + it * kW) + 8 * g;
                *reinterpret_cast<v4f*>(to) = (v4f){p[0], p[1], p[2], p[3]};
                *reinterpret_cast<v4f*>(to + 4) = (v4f){p[4], p[5], p[6], p[7]};
            }
        }
        float top = fmaxf(fmaxf(fmaxf(p[0], p[1]), fmaxf(p[2], p[3])), fmaxf(fmaxf(p[4], p[5]), fmaxf(p[6], p[7])));
        top = groups_max(top);
        if (__builtin_amdgcn_ballot_w64(top > m)) {
            const float now = fmaxf(m, top), by = now == kMinusInf ? 1.0f : exp2_fast((m - now) * a.scale);
            m = now;
            l *= by;
#pragma unroll
            for (int i = 0; i < kV; ++i) acc[i] *= by;
        }
        const float base = m == kMinusInf ? 0.0f : m * a.scale;
#pragma unroll
        for (int j = 0; j < 8; ++j) p[j] = exp2_fast(__builtin_fmaf(p[j], a.scale, -base));
        v8bf w[kParts];
#pragma unroll
        for (int j = 0; j < 8; j += 2) weights_pair<kParts>(w, j, p[j], p[j + 1]);
#pragma unroll
        for (int e = 0; e < kParts; ++e) l = mfma_bf16(ones, w[e], l);
#pragma unroll
        for (int e = 0; e < kParts; ++e)
#pragma unroll
            for (int i = 0; i < kV; ++i) acc[i] = mfma_bf16(__builtin_bit_cast(v8bf, x.v[i]), w[e], acc[i]);
    };
    Block x0, x1;
    if (mine > 0) {
        fetch_numbers(0);
        load(x0, 0);
    }
    settle_query<kC, kExact>(qf, g, D);
    for (int it = 0; it < mine; it += 2) {                 // two sets of registers that swap roles by name
        const bool known0 = __builtin_amdgcn_readlane(numbers, it & 63) >= 0;
        bool known1 = false;
        if (it + 1 < mine) {
            load(x1, it + 1);
            known1 = __builtin_amdgcn_readlane(numbers, (it + 1) & 63) >= 0;
        }
        if (((it + 2) & 63) == 0 && it + 2 < mine) fetch_numbers(it + 2);
        take(x0, it, known0);
        if (it + 1 < mine) {
            if (it + 2 < mine) load(x0, it + 2);
            take(x1, it + 1, known1);
        }
    }

    // The waves' states into one: weights exp(m_w - m), sums by rounds of 64 dims through LDS.
    if (g == 0) {
        maxima[wave * 16 + r] = m;
        totals[wave * 16 + r] = l[0];
    }
    __syncthreads();
    float all = kMinusInf;
#pragma unroll
    for (int w = 0; w < kW; ++w) all = fmaxf(all, maxima[w * 16 + r]);
    const float by = m == kMinusInf ? 0.0f : exp2_fast((m - all) * a.scale);
#pragma unroll
    for (int round = 0; round < (kV + kRound - 1) / kRound; ++round) {
        if (r < columns)
#pragma unroll
            for (int i = 0; i < kRound; ++i) {
                if (round * kRound + i >= kV) break;
                const v4f x = acc[round * kRound + i] * by;
                *reinterpret_cast<v4f*>(&sums[(wave * 16 + r) * kPitch + 16 * i + 4 * g]) = x;
            }
        __syncthreads();
        for (int i = threadIdx.x; i < columns * 4 * kRound; i += 64 * kW) {
            const int col = i / (4 * kRound), d = (i % (4 * kRound)) * 4, dim = 16 * kRound * round + d;
            if (dim >= D) continue;
            float top = kMinusInf, total = 0.0f;
#pragma unroll
            for (int w = 0; w < kW; ++w) top = fmaxf(top, maxima[w * 16 + col]);
            v4f x = {0, 0, 0, 0};
#pragma unroll
            for (int w = 0; w < kW; ++w) {
                const float mw = maxima[w * 16 + col];
                x += *reinterpret_cast<const v4f*>(&sums[(w * 16 + col) * kPitch + d]);
                total += mw == kMinusInf ? 0.0f : totals[w * 16 + col] * exp2_fast((mw - top) * a.scale);
            }
            const int64_t row = (int64_t)b * a.heads + head0 + col;
            int64_t place = row * parts.splits + blockIdx.y;
            if constexpr (kDo == Single::Own) place = row * more.pitch + more.first + blockIdx.y;
            const bool whole = kDo != Single::Own && run >= blocks;
            if (whole) {
                const float inv = total > 0.0f ? 1.0f / total : 0.0f;
                const float out[4] = {finite_or_nan(x[0], inv), finite_or_nan(x[1], inv), finite_or_nan(x[2], inv), finite_or_nan(x[3], inv)};
                store4<kF32>(a.o, row * D, dim, D, out);
            } else {
                const float out[4] = {x[0], x[1], x[2], x[3]};
                store4<true>(parts.sums, place * D, dim, D, out);
            }
            if ((!whole || kDo == Single::Scored) && dim == 0) {
                parts.state[2 * place] = top;
                parts.state[2 * place + 1] = total;
            }
        }
        __syncthreads();
    }
    // The row's scores, written by this workgroup in front of those barriers, into weights: four tokens a thread, all heads one behind the other.
    if constexpr (kDo == Single::Scored) {
        if (!more.weights) return;
        if (threadIdx.x < 16) {
            float top = kMinusInf, total = 0.0f;
#pragma unroll
            for (int w = 0; w < kW; ++w) top = fmaxf(top, maxima[w * 16 + threadIdx.x]);
#pragma unroll
            for (int w = 0; w < kW; ++w) {
                const float mw = maxima[w * 16 + threadIdx.x];
                total += mw == kMinusInf ? 0.0f : totals[w * 16 + threadIdx.x] * exp2_fast((mw - top) * a.scale);
            }
            sums[2 * threadIdx.x] = top == kMinusInf ? 0.0f : top * a.scale;
            sums[2 * threadIdx.x + 1] = total > 0.0f ? 1.0f / total : 0.0f;
        }
        __syncthreads();
        const int64_t capacity = (int64_t)kv.max_blocks * kKvBlock;
        const float* from = more.scores + ((int64_t)b * a.heads + head0) * capacity;
        float* to = more.weights + ((int64_t)b * kv.kv_heads + h) * more.stride;
        for (int64_t pos = 4 * threadIdx.x; pos < len; pos += 4 * 64 * kW) {
            v4f sum = {0, 0, 0, 0};
#pragma unroll 4
            for (int e = 0; e < columns; ++e) {
                const v4f s = *reinterpret_cast<const v4f*>(from + e * capacity + pos);
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[i] = __builtin_fmaf(exp2_fast(__builtin_fmaf(s[i], a.scale, -sums[2 * e])), sums[2 * e + 1], sum[i]);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (pos + i < len) to[pos + i] = (pos + i == len - 1 ? 0.0f : to[pos + i]) + sum[i];      // the call's own token begins with nothing
        }
    }
}

// How many workgroups share a row at most (attention_decode.hip)
struct Splits { int n, least; };
Splits decode_splits(const KvView& kv, int heads);

}  // namespace bitnet
