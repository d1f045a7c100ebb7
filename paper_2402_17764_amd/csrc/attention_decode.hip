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
    float* part;                       // partial sums, or NULL
    float scale;                       // of the softmax, times log2 e
    int heads, group;                  // query heads, and of them per key-value head
    int column_tiles;                  // of 16 query heads, per key-value head
};

template <int kC, bool kExact, bool kF32, int kW>
__global__ __launch_bounds__(64 * kW) void attention_decode_rows(DecodeArgs a, KvView kv) {
    constexpr int kV = 2 * kC;                             // tiles of 16 dims
    constexpr int kRound = kV < 4 ? kV : 4;                // ... that the waves add up at a time
    constexpr int kPitch = 16 * kRound + 4;
    __shared__ float sums[kW * 16 * kPitch], maxima[kW * 16], totals[kW * 16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, g = lane >> 4;
    const int D = kExact ? 32 * kC : kv.D, Dp = kv_padded_dim(D), quads = Dp >> 3;
    int row = blockIdx.x;
    const int ct = row % a.column_tiles;
    row /= a.column_tiles;
    const int h = row % kv.kv_heads, b = row / kv.kv_heads;
    const int head0 = h * a.group + 16 * ct, columns = min(a.group - 16 * ct, 16);
    const int len = kv.length(kv.kv_len[b]), blocks = (len + kKvBlock - 1) / kKvBlock;

    v8bf qf[kC];
    load_query<kC>(qf, r < columns ? a.q + ((int64_t)b * a.heads + head0 + r) * D : nullptr, g, D);

    int koff[kC], voff[kV];                                // bytes within a block
#pragma unroll
    for (int c = 0; c < kC; ++c) koff[c] = (kExact ? 4 * c + g : min(4 * c + g, quads - 1)) * 512 + r * 16;
#pragma unroll
    for (int i = 0; i < kV; ++i) voff[i] = (g * Dp + (kExact ? 16 * i + r : min(16 * i + r, Dp - 1))) * 16;

    v4f acc[kV];
#pragma unroll
    for (int i = 0; i < kV; ++i) acc[i] = (v4f){0, 0, 0, 0};
    float m = kMinusInf, l = 0.0f;                         // l: of this lane's tokens

    struct Block { v4u k[kC][2], v[kV]; };
    // this wave's blocks are wave, wave + kW, ...; their numbers in the cache stand in the lanes, 64 at a time
    const int mine = blocks > wave ? (blocks - wave + kW - 1) / kW : 0;
    const int32_t* table = kv.table + b * kv.table_stride;
    int numbers = -1;
    auto fetch_numbers = [&](int it) {
        const int blk = wave + (it + lane) * kW;
        numbers = blk < blocks ? kv.block(table, blk, h) : -1;
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
        const int left = known ? len - kKvBlock * (wave + it * kW) : 0;      // of the block's tokens, how many count
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
        for (int j = 0; j < 8; ++j) {
            p[j] = exp2_fast(__builtin_fmaf(p[j], a.scale, -base));
            l += p[j];
        }
        const v8bf w = weights_operand(p);
#pragma unroll
        for (int i = 0; i < kV; ++i) acc[i] = mfma_bf16(__builtin_bit_cast(v8bf, x.v[i]), w, acc[i]);
        if (kF32) {
            const v8bf rest = weights_rest(p, w);
#pragma unroll
            for (int i = 0; i < kV; ++i) acc[i] = mfma_bf16(__builtin_bit_cast(v8bf, x.v[i]), rest, acc[i]);
        }
    };
    Block x0, x1;
    if (mine > 0) {
        fetch_numbers(0);
        load(x0, 0);
    }
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
    l = groups_sum(l);
    if (g == 0) {
        maxima[wave * 16 + r] = m;
        totals[wave * 16 + r] = l;
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
            const int col = i / (4 * kRound), d = (i % (4 * kRound)) * 4;
            float top = kMinusInf, total = 0.0f;
#pragma unroll
            for (int w = 0; w < kW; ++w) top = fmaxf(top, maxima[w * 16 + col]);
            v4f x = {0, 0, 0, 0};
#pragma unroll
            for (int w = 0; w < kW; ++w) {
                x += *reinterpret_cast<const v4f*>(&sums[(w * 16 + col) * kPitch + d]);
                total += maxima[w * 16 + col] == kMinusInf ? 0.0f : totals[w * 16 + col] * exp2_fast((maxima[w * 16 + col] - top) * a.scale);
            }
            const float inv = total > 0.0f ? 1.0f / total : 0.0f;
            const float out[4] = {x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv};
            const int dim = 16 * kRound * round + d;
            if (dim < D) store4<kF32>(a.o, ((int64_t)b * a.heads + head0 + col) * D, dim, D, out);
        }
        __syncthreads();
    }
}

template <int kC, bool kExact>
hipError_t launch_rows(const DecodeArgs& a, const KvView& kv, bool f32, hipStream_t stream) {
    const int64_t rows = (int64_t)kv.B * kv.kv_heads * a.column_tiles;
    if (f32) attention_decode_rows<kC, kExact, true, 4><<<(unsigned)rows, 256, 0, stream>>>(a, kv);
    else attention_decode_rows<kC, kExact, false, 4><<<(unsigned)rows, 256, 0, stream>>>(a, kv);
    return hipGetLastError();
}

}  // namespace

size_t attention_decode_workspace_bytes(const KvView&, int) { return 0; }

hipError_t launch_attention_decode(const void* q, const KvView& kv, int heads, float scale, void* o, bool f32, void* workspace,
                                   size_t workspace_bytes, hipStream_t stream) {
    DecodeArgs a{static_cast<const uint16_t*>(q), o, nullptr, scale * 1.44269504f, heads, heads / kv.kv_heads, 0};
    a.column_tiles = (int)ceil_div(a.group, 16);
    const int chunks = (int)ceil_div(kv.D, 32);
    const bool exact = kv.D % 32 == 0;
#define ROWS(kC_) return exact ? launch_rows<kC_, true>(a, kv, f32, stream) : launch_rows<kC_, false>(a, kv, f32, stream)
    switch (chunks) {
        case 1: ROWS(1);
        case 2: ROWS(2);
        case 3: ROWS(3);
        case 4: ROWS(4);
        case 5: case 6: return chunks == 6 && exact ? launch_rows<6, true>(a, kv, f32, stream) : launch_rows<6, false>(a, kv, f32, stream);
        default: return chunks == 8 && exact ? launch_rows<8, true>(a, kv, f32, stream) : launch_rows<8, false>(a, kv, f32, stream);
    }
#undef ROWS
}

}  // namespace bitnet
