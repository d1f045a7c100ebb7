// Attention of one new token of each sequence over its cached keys and values:
//   s_j = scale q . k_j,  p = softmax(s),  o = sum_j p_j v_j,
// in one pass over the cache: a wave keeps, for each query of a key-value head, the running maximum m of the scores, the sum l
// of exp(s_j - m) and the values' sum under the same weights, in 32 bits; a new maximum rescales both.
//
// A wave takes 32 tokens at a time.  Scores are MFMA 16 x 16 x 32 products of keys (down) and the queries of the head's group (across,
// up to 16); the cache's order of keys makes their result the operand of the second product, values (dims down) times weights, as it
// stands, and values are stored as that product's other operand: nothing passes through LDS or other lanes but the maximum.
// Every byte of the cache goes from memory to the register that the MFMA reads it from, in 16-byte loads.
#include "attention_common.hpp"

namespace bitnet {
namespace {

struct DecodeArgs {
    const uint16_t* q;
    void* o;
    float scale;                       // of the softmax, times log2 e
    int heads, group;                  // query heads, and of them per key-value head
    int column_tiles;                  // of 16 query heads, per key-value head
};

// A row is 16 query heads (or what a group has left) of one key-value head of one sequence.  Its blocks are dealt out to up to
// parts.splits workgroups (blockIdx.y).
template <int kC, int kV, bool kExact, bool kF32, int kW>
__global__ __launch_bounds__(64 * kW, kC <= 4 ? 2 : 1) void attention_decode_rows(DecodeArgs a, Parts parts, KvView kv) {
    constexpr int kWholeChunks = whole_chunks(kC), kParts = kF32 ? 3 : 2;      // bf16 operands of a weight
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
    const int run = parts.run(blocks), blk0 = blockIdx.y * run, blk1 = min(blk0 + run, blocks);
    if (blk0 >= blocks && blockIdx.y > 0) return;

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
            if (run >= blocks) {
                const float inv = total > 0.0f ? 1.0f / total : 0.0f;
                const float out[4] = {finite_or_nan(x[0], inv), finite_or_nan(x[1], inv), finite_or_nan(x[2], inv), finite_or_nan(x[3], inv)};
                store4<kF32>(a.o, ((int64_t)b * a.heads + head0 + col) * D, dim, D, out);
            } else {
                const float out[4] = {x[0], x[1], x[2], x[3]};
                const int64_t place = ((int64_t)b * a.heads + head0 + col) * parts.splits + blockIdx.y;
                store4<true>(parts.sums, place * D, dim, D, out);
                if (dim == 0) {
                    parts.state[2 * place] = top;
                    parts.state[2 * place + 1] = total;
                }
            }
        }
        __syncthreads();
    }
}

template <int kC, int kV, bool kExact>
hipError_t launch_decode(const DecodeArgs& a, const Parts& parts, const KvView& kv, bool f32, hipStream_t stream) {
    const dim3 grid((unsigned)((int64_t)kv.B * kv.kv_heads * a.column_tiles), parts.splits);
    if (f32) attention_decode_rows<kC, kV, kExact, true, 4><<<grid, 256, 0, stream>>>(a, parts, kv);
    else attention_decode_rows<kC, kV, kExact, false, 4><<<grid, 256, 0, stream>>>(a, parts, kv);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || parts.splits < 2) return e;
    return launch_attention_join({a.o, a.scale, a.heads, a.group, kv.B, 0}, parts, kv, f32, stream);
}

// How many workgroups share a row at most, by the length that the page tables have room for.  A CU draws 25 to 45 bytes a cycle,
// whatever number of waves asks, and a second launch costs 4 us in a chain of launches: so rows are shared where there are fewer
// than 256 and more than 1023 tokens (one token, 32 heads of 128, a key-value head each, 1000 tokens: 13.4 us in one launch, 10.0 shared;
// 64 heads over 8, 500 tokens 7.5 / 9.5, 1000 tokens 9.4 / 9.4), until there are as many as the CUs hold at a time: two each (three
// sequences of 23000 to 41000 tokens, 64 heads over 8: 512 workgroups 74.7 us, 1024 79.1, 2048 79.2, none shared 359), of heads of more than 128
// dims, whose registers leave room for one, one each (one sequence of 32000 tokens, 32 heads of 160 over 8, 256 / 512 workgroups 35.0 /
// 42.4, of 256 dims 47.3 / 53.4; three of 3000, 16 heads of 160 21.9 / 26.8).  More rows are shared only at every 8192 tokens,
// so that one long sequence among short ones is not what the call waits for.
struct Splits { int n, least; };
Splits decode_splits(const KvView& kv, int heads) {
    const int64_t rows = (int64_t)kv.B * kv.kv_heads * ceil_div(heads / kv.kv_heads, 16);
    constexpr int kShort = 8, kLong = 256;                 // blocks: two for each wave of a workgroup; 8192 tokens
    if (kv.max_blocks < 32) return {1, 1};
    const int64_t fill = rows < 256 ? (kv.D <= 128 ? 512 : 256) / rows : 1, long_ones = ceil_div(kv.max_blocks, kLong), room = 8192 / rows;
    const int least = fill > 1 ? kShort : kLong / 2;
    int64_t n = fill > long_ones ? fill : long_ones < room ? long_ones : room;
    const int64_t most = ceil_div(kv.max_blocks, least);
    n = n < most ? n : most;
    return {(int)(n < 1 ? 1 : n > kMostSplits ? kMostSplits : n), least};
}

}  // namespace

size_t attention_decode_workspace_bytes(const KvView& kv, int heads) {
    return Parts::bytes((int64_t)kv.B * heads, decode_splits(kv, heads).n, kv.D);
}

hipError_t launch_attention_decode(const void* q, const KvView& kv, int heads, float scale, void* o, bool f32, void* workspace,
                                   size_t workspace_bytes, hipStream_t stream) {
    const int group = heads / kv.kv_heads;
    const DecodeArgs a{static_cast<const uint16_t*>(q), o, scale * 1.44269504f, heads, group, (int)ceil_div(group, 16)};
    Parts parts;
    const Splits s = decode_splits(kv, heads);
    if (s.n > 1 && workspace_bytes >= attention_decode_workspace_bytes(kv, heads)) parts = Parts(workspace, (int64_t)kv.B * heads, s.n, s.least, kv.D);
    const int chunks = (int)ceil_div(kv.D, 32);
    const bool exact = kv.D % 32 == 0, one_tile = kv.D % 32 != 0 && kv.D % 32 <= 16;
#define DECODE(kC_, kV_, kE_) return launch_decode<kC_, kV_, kE_>(a, parts, kv, f32, stream)
    switch (chunks) {
        case 1: if (exact) DECODE(1, 2, true); if (one_tile) DECODE(1, 1, false); DECODE(1, 2, false);
        case 2: if (exact) DECODE(2, 4, true); if (one_tile) DECODE(2, 3, false); DECODE(2, 4, false);
        case 3: if (exact) DECODE(3, 6, true); if (one_tile) DECODE(3, 5, false); DECODE(3, 6, false);
        case 4: if (exact) DECODE(4, 8, true); if (one_tile) DECODE(4, 7, false); DECODE(4, 8, false);
        case 5: case 6: if (exact && chunks == 6) DECODE(6, 12, true); DECODE(6, 12, false);
        default: if (exact && chunks == 8) DECODE(8, 16, true); DECODE(8, 16, false);
    }
#undef DECODE
}

}  // namespace bitnet
