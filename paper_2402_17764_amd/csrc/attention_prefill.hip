// Attention of runs of new tokens over their sequences' caches, causal: the token at position p sees the keys of positions 0 ... p.
//   s_j = scale q . k_j (j <= p),  p = softmax(s),  o = sum_j p_j v_j,
// with the running maximum and sum of a softmax in 32 bits, one pass over the keys.
//
// A workgroup takes a tile of rows of one sequence and one key-value head -- a row is one query head of one new token, the heads of a
// group next to each other, so that grouped heads share what they read -- and walks the cache 64 tokens at a time.  Both cache
// blocks come through LDS (copied as they stand, by loads that go to LDS directly; the cache's order is already that of the MFMA
// operands), double-buffered: the next blocks are requested right behind the barrier that publishes the current ones.  Scores are products
// keys (down) times queries (across), which leaves a lane with eight consecutive tokens of its query: the operand of the second product.
#include "attention_common.hpp"

namespace bitnet {
namespace {

struct PrefillArgs {
    const uint16_t* q;
    void* o;
    float scale;                       // of the softmax, times log2 e
    int heads, group, T;               // query heads, and of them per key-value head; rows of q
    int tiles;                         // of the launch, per key-value head
};

constexpr int kStageBlocks = 2;        // cache blocks of a stage

constexpr int prefill_piece(int Dp) { return (Dp * 64 + 1023) / 1024 * 1024; }     // a block's keys (or values) in LDS: whole wave loads

template <int kC, bool kExact, int kNT, int kW, bool kF32>
__global__ __launch_bounds__(64 * kW) void attention_prefill_tiles(PrefillArgs a, KvView kv) {
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int kV = 2 * kC, kRows = 16 * kNT * kW;
    extern __shared__ uint4 smem[];
    char* lds = reinterpret_cast<char*>(smem);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, g = lane >> 4;
    const int D = kExact ? 32 * kC : kv.D, Dp = kv_padded_dim(D), quads = Dp >> 3;
    const int piece = kExact ? prefill_piece(32 * kC) : prefill_piece(Dp), stage_bytes = 2 * kStageBlocks * piece;

    const int h = blockIdx.x % kv.kv_heads;
    const int64_t x = a.tiles - 1 - (int)(blockIdx.x / kv.kv_heads);       // late tiles, which see most, first
    const int b = sequence_of_tile(kv.q_start, kv.B, x, a.group, kRows, 1);
    const NewTokens nt(kv, b, a.T);
    const int64_t tile = x - first_tile(kv.q_start[b], b, a.group, kRows, 1);
    const int64_t rows = (int64_t)nt.n * a.group;
    if (tile < 0 || tile * kRows >= rows) return;
    const int64_t row0 = tile * kRows;                                     // of the sequence's rows for this head
    const int64_t row_last = min(row0 + kRows, rows) - 1;
    const int seen = nt.pos0 + (int)(row_last / a.group) + 1;              // keys that the tile's last token sees
    const int blocks = seen > 0 ? (seen + kKvBlock - 1) / kKvBlock : 0;
    const int stages = (blocks + kStageBlocks - 1) / kStageBlocks;

    v8bf qf[kNT][kC];
    int pos[kNT];                                                          // of the lane's queries; -1: none
    int64_t out_at[kNT];
    const int64_t wave_row = row0 + wave * 16 * kNT;
#pragma unroll
    for (int n = 0; n < kNT; ++n) {
        const int64_t R = wave_row + 16 * n + r;
        const int tok = (int)(R / a.group), hh = (int)(R - (int64_t)tok * a.group);
        out_at[n] = ((int64_t)(nt.first + tok) * a.heads + h * a.group + hh) * D;
        pos[n] = R < rows ? nt.pos0 + tok : -1;
        if (R >= rows) out_at[n] = -1;
        load_query<kC>(qf[n], R < rows ? a.q + out_at[n] : nullptr, g, D);
    }
    const int pos_first = nt.pos0 + (int)(wave_row / a.group);             // the wave's first and last token's
    const int pos_last = wave_row < rows ? nt.pos0 + (int)((min(wave_row + 16 * kNT, rows) - 1) / a.group) : -1;

    const int32_t* table = kv.table + b * kv.table_stride;
    int numbers = -1;                                                      // of 64 blocks, one a lane
    auto fetch_numbers = [&](int blk0) {
        const int blk = blk0 + lane;
        numbers = blk < blocks ? kv.block(table, blk, h) : -1;
    };
    const int64_t block_bytes = (int64_t)kKvBlock * Dp * 2;
    auto copy = [&](int stage) {                                           // both blocks' keys, then both blocks' values
        char* to = lds + (stage & 1) * stage_bytes;
        const int loads = piece >> 10;
#pragma unroll
        for (int u = 0; u < kStageBlocks; ++u) {
            const int64_t at = max(__builtin_amdgcn_readlane(numbers, (stage * kStageBlocks + u) & 63), 0) * block_bytes;
#pragma unroll
            for (int kv_ = 0; kv_ < 2; ++kv_) {
                const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<char*>(kv_ ? kv.v : kv.k) + at, 0, (int)block_bytes, 0x00020000);
                char* dst = to + (kv_ * kStageBlocks + u) * piece;
                for (int i = wave; i < loads; i += kW)
                    __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void*)(dst + i * 1024), 16, i * 1024 + lane * 16, 0, 0, 0);
            }
        }
    };
    int koff[kC], voff[kV];
#pragma unroll
    for (int c = 0; c < kC; ++c) koff[c] = (kExact ? 4 * c + g : min(4 * c + g, quads - 1)) * 512 + r * 16;
#pragma unroll
    for (int i = 0; i < kV; ++i) voff[i] = (g * Dp + (kExact ? 16 * i + r : min(16 * i + r, Dp - 1))) * 16;

    v4f acc[kNT][kV];
    float m[kNT], l[kNT];
#pragma unroll
    for (int n = 0; n < kNT; ++n) {
        m[n] = kMinusInf;
        l[n] = 0.0f;
#pragma unroll
        for (int i = 0; i < kV; ++i) acc[n][i] = (v4f){0, 0, 0, 0};
    }
    if (stages > 0) {
        fetch_numbers(0);
        copy(0);
    }
    for (int s = 0; s < stages; ++s) {
        const int current = numbers;                                       // holds this stage's blocks
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();
        if (s + 1 < stages) {
            if ((((s + 1) * kStageBlocks) & 63) == 0) fetch_numbers((s + 1) * kStageBlocks);
            copy(s + 1);
        }
        const int j0 = s * kStageBlocks * kKvBlock;                        // position of the stage's first token
        if (j0 > pos_last) continue;                                       // nothing that this wave's rows see
        const char* keys = lds + (s & 1) * stage_bytes;
        const char* values = keys + kStageBlocks * piece;
        v4f sc[kStageBlocks][2][kNT];
#pragma unroll
        for (int u = 0; u < kStageBlocks; ++u)
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int n = 0; n < kNT; ++n) sc[u][t][n] = (v4f){0, 0, 0, 0};
#pragma unroll
        for (int u = 0; u < kStageBlocks; ++u)
#pragma unroll
            for (int c = 0; c < kC; ++c)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const v8bf k = *reinterpret_cast<const v8bf*>(keys + u * piece + koff[c] + 256 * t);
#pragma unroll
                    for (int n = 0; n < kNT; ++n) sc[u][t][n] = mfma_bf16(k, qf[n][c], sc[u][t][n]);
                }
        bool known[kStageBlocks];
#pragma unroll
        for (int u = 0; u < kStageBlocks; ++u) known[u] = __builtin_amdgcn_readlane(current, (s * kStageBlocks + u) & 63) >= 0;
        const bool masked = j0 + kStageBlocks * kKvBlock - 1 > pos_first || !known[0] || !known[kStageBlocks - 1] || pos_last < 0;
        v8bf w[kStageBlocks][kNT], rest[kStageBlocks][kNT];
#pragma unroll
        for (int n = 0; n < kNT; ++n) {
            if (masked)
#pragma unroll
                for (int u = 0; u < kStageBlocks; ++u)
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (!known[u] || j0 + u * kKvBlock + 8 * g + j > pos[n]) sc[u][j >> 2][n][j & 3] = kMinusInf;
            float top = kMinusInf;
#pragma unroll
            for (int u = 0; u < kStageBlocks; ++u)
#pragma unroll
                for (int j = 0; j < 8; ++j) top = fmaxf(top, sc[u][j >> 2][n][j & 3]);
            top = groups_max(top);
            if (__builtin_amdgcn_ballot_w64(top > m[n])) {
                const float now = fmaxf(m[n], top), by = now == kMinusInf ? 1.0f : exp2_fast((m[n] - now) * a.scale);
                m[n] = now;
                l[n] *= by;
#pragma unroll
                for (int i = 0; i < kV; ++i) acc[n][i] *= by;
            }
            const float base = m[n] == kMinusInf ? 0.0f : m[n] * a.scale;
#pragma unroll
            for (int u = 0; u < kStageBlocks; ++u) {
                float p[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    p[j] = exp2_fast(__builtin_fmaf(sc[u][j >> 2][n][j & 3], a.scale, -base));
                    l[n] += p[j];
                }
                w[u][n] = weights_operand(p);
                if (kF32) rest[u][n] = weights_rest(p, w[u][n]);
            }
        }
#pragma unroll
        for (int u = 0; u < kStageBlocks; ++u) {
            if (masked) {
                // The blocks that some row does not see to their end.  A weight of zero does not make an infinity nothing: tokens that no row
                // sees are cleared, and if a value of one that some rows see is not finite, the tokens go through the product one by
                // one, each added to the rows that see it.
                const int block0 = j0 + u * kKvBlock;
                const int some = known[u] ? min(max(pos_last + 1 - block0, 0), kKvBlock) : 0;     // tokens that some row of the wave sees
                unsigned bad = 0;
#pragma unroll
                for (int i = 0; i < kV; ++i) {
                    v4u v = *reinterpret_cast<const v4u*>(values + u * piece + voff[i]);
                    values_keep(v, some - 8 * g);
#pragma unroll
                    for (int e = 0; e < 4; ++e) bad |= (unsigned)((v[e] & 0x7F80u) == 0x7F80u) | (unsigned)((v[e] & 0x7F800000u) == 0x7F800000u);
                }
                if (__builtin_amdgcn_ballot_w64(bad != 0)) {
                    for (int t = 0; t < some; ++t) {
#pragma unroll
                        for (int i = 0; i < kV; ++i) {
                            v4u v = *reinterpret_cast<const v4u*>(values + u * piece + voff[i]), v1 = v;
                            values_keep(v, t + 1 - 8 * g);
                            values_keep(v1, t - 8 * g);
                            v ^= v1;                                       // token t alone
#pragma unroll
                            for (int n = 0; n < kNT; ++n) {
                                v4f one = mfma_bf16(__builtin_bit_cast(v8bf, v), w[u][n], (v4f){0, 0, 0, 0});
                                if (kF32) one = mfma_bf16(__builtin_bit_cast(v8bf, v), rest[u][n], one);
                                if (block0 + t <= pos[n]) acc[n][i] += one;
                            }
                        }
                    }
                    continue;
                }
#pragma unroll
                for (int i = 0; i < kV; ++i) {
                    v4u v = *reinterpret_cast<const v4u*>(values + u * piece + voff[i]);
                    values_keep(v, some - 8 * g);
#pragma unroll
                    for (int n = 0; n < kNT; ++n) {
                        acc[n][i] = mfma_bf16(__builtin_bit_cast(v8bf, v), w[u][n], acc[n][i]);
                        if (kF32) acc[n][i] = mfma_bf16(__builtin_bit_cast(v8bf, v), rest[u][n], acc[n][i]);
                    }
                }
                continue;
            }
#pragma unroll
            for (int i = 0; i < kV; ++i) {
                const v8bf v = *reinterpret_cast<const v8bf*>(values + u * piece + voff[i]);
#pragma unroll
                for (int n = 0; n < kNT; ++n) {
                    acc[n][i] = mfma_bf16(v, w[u][n], acc[n][i]);
                    if (kF32) acc[n][i] = mfma_bf16(v, rest[u][n], acc[n][i]);
                }
            }
        }
    }
#pragma unroll
    for (int n = 0; n < kNT; ++n) {
        const float total = groups_sum(l[n]), inv = total > 0.0f ? 1.0f / total : 0.0f;
        if (out_at[n] < 0) continue;
#pragma unroll
        for (int i = 0; i < kV; ++i) {
            const int d = 16 * i + 4 * g;
            const float out[4] = {acc[n][i][0] * inv, acc[n][i][1] * inv, acc[n][i][2] * inv, acc[n][i][3] * inv};
            if (d < D) store4<kF32>(a.o, out_at[n], d, D, out);
        }
    }
#endif
}

template <int kC, bool kExact, int kNT, int kW, bool kF32>
hipError_t launch_tiles(PrefillArgs a, const KvView& kv, hipStream_t stream) {
    static RaisedFlags raised;
    const auto kernel = attention_prefill_tiles<kC, kExact, kNT, kW, kF32>;
    const int lds = 2 * 2 * kStageBlocks * prefill_piece(kv_padded_dim(kv.D));
    if (lds > 65536) {
        const hipError_t e = raise_dynamic_lds(reinterpret_cast<const void*>(kernel), 2 * 2 * kStageBlocks * prefill_piece(32 * kC), raised);
        if (e != hipSuccess) return e;
    }
    a.tiles = (int)tiles_at_most(a.T, kv.B, a.group, 16 * kNT * kW, 1);
    kernel<<<(unsigned)((int64_t)a.tiles * kv.kv_heads), 64 * kW, lds, stream>>>(a, kv);
    return hipGetLastError();
}

}  // namespace

size_t attention_prefill_workspace_bytes(const KvView&, int64_t, int) { return 0; }

hipError_t launch_attention_prefill(const void* q, const KvView& kv, int64_t T, int heads, float scale, void* o, bool f32, void* workspace,
                                    size_t workspace_bytes, hipStream_t stream) {
    const PrefillArgs a{static_cast<const uint16_t*>(q), o, scale * 1.44269504f, heads, heads / kv.kv_heads, (int)T, 0};
    const int chunks = (int)ceil_div(kv.D, 32);
    const bool exact = kv.D % 32 == 0;
#define TILES(kC_, kE_, kNT_) return f32 ? launch_tiles<kC_, kE_, kNT_, 4, true>(a, kv, stream) : launch_tiles<kC_, kE_, kNT_, 4, false>(a, kv, stream)
    switch (chunks) {
        case 1: if (exact) TILES(1, true, 2); TILES(1, false, 2);
        case 2: if (exact) TILES(2, true, 2); TILES(2, false, 2);
        case 3: if (exact) TILES(3, true, 2); TILES(3, false, 2);
        case 4: if (exact) TILES(4, true, 2); TILES(4, false, 2);
        case 5: case 6: if (chunks == 6 && exact) TILES(6, true, 2); TILES(6, false, 2);
        default: if (chunks == 8 && exact) TILES(8, true, 1); TILES(8, false, 1);
    }
#undef TILES
}

}  // namespace bitnet
