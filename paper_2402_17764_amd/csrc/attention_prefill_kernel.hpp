// Attention of runs of new tokens over their sequences' caches, causal: the token at position p sees the keys of positions 0 ... p.
//   s_j = scale q . k_j (j <= p),  p = softmax(s),  o = sum_j p_j v_j,
// with the running maximum and sum of a softmax in 32 bits, one pass over the keys.
//
// A workgroup takes a tile of rows of one sequence and one key-value head -- a row is one query head of one new token, the heads of a
// group next to each other, so that grouped heads share what they read -- and walks the cache a stage of one or two blocks
// of 32 tokens at a time.  Keys and values come through LDS (copied as they stand, by loads that go to LDS directly; the cache's order is
// already that of the MFMA operands), double-buffered: the next stage is requested right behind the barrier that publishes the current
// one.  Scores are products keys (down) times queries (across), which leaves a lane with eight consecutive tokens of its query: the
// operand of the second product.
#pragma once
#include "attention_common.hpp"

#include <type_traits>

namespace bitnet {

struct PrefillArgs {
    const uint16_t* q;
    void* o;
    float scale;                       // of the softmax, times log2 e
    float slack;                       // kSlack in units of a score; finite, so that the first score of all passes
    int heads, group, T;               // query heads, and of them per key-value head; rows of q
    int tiles;                         // of the launch, per key-value head
};

// Whose rows a launch takes: runs of new tokens, causal; the same, leaving each row's softmax state for the weights of the keys; or the single new tokens of sequences that share their first tokens, as parts of rows: over those of a group alone, its
// sequences in place of new tokens, or over what each sequence has behind them as well.
enum class Rows { Causal, Kept, Prefix, Shared };
constexpr bool of_groups(Rows r) { return r == Rows::Prefix || r == Rows::Shared; }
struct SharedLaunch {
    Prefixes prefixes;
    uint32_t near_blocks, far_blocks;  // workgroups of a key-value head over what is shared (tiles of rows times splits), and over what is not
    uint32_t far_ratio;                // far_blocks 2^32 / (near_blocks + far_blocks), rounded up
    int near, far;                     // splits of a row over either; their parts stand behind one another
    int least_near, least_far;         // units of tokens that a split has at least
    int far_tiles;                     // of a sequence's rows, per key-value head
    int far_unit;                      // tokens: a stage's, or a block's if another launch takes what is not shared
};
struct RowsMore {
    KeptRows keep;                     // Kept
    SharedLaunch shared;
};

// The shapes of a workgroup: four waves of one or two times 16 rows each (heads of more than 128 dims: four or eight waves of 16, as a wave's
// sums take its registers), and stages of LDS of one cache block, or two where a block is small.  Both leave room for three or
// four workgroups on a CU, which is what hides a stage's barrier and the chain of loads that a workgroup begins with (us, one prompt of
// 2048 tokens and 40 heads of 128 / sixteen of 100 to 400 and 64 heads over 8 / one of 1024 behind 15000, 64 over 8: 64 rows and
// one block 60 / 58 / 539, two blocks 66 / 80 / 579; 128 rows and one block 61 / 54 / 466, two blocks 58 / 66 / 466; 256 rows in
// eight waves, two blocks 67 / 74 / 456; 256 rows in four waves, whose sums move to and from the accumulation registers, 100 / - / 591).
enum class PrefillTile { Rows64, Rows128 };
constexpr int prefill_rows(PrefillTile t) { return t == PrefillTile::Rows64 ? 64 : 128; }
constexpr float kSlack = 8.0f;         // in the exponent of 2

// LDS of a cache block: the keys' 4 kC quads of 512 bytes, then the values, 16 kV dims of each of the four groups of eight tokens.  Where a head has
// fewer, its last eight dims of the same token, and a group's last dim, stand again, so that the groups are multiples of 256
// bytes apart (in the cache's own steps of 16 Dp, heads of 100, reads met in LDS banks on 28 % of the cycles).  Queries have zeros
// there, and results of such dims are not stored.
constexpr int prefill_lds(int kC, int kV, int blocks) { return 2 * blocks * (2 * kC + kV) * 1024; }

template <int kC, int kV, bool kExact, int kNT, int kStageBlocks, int kW, int kOcc, bool kF32, Rows kOf>
__global__ __launch_bounds__(64 * kW, kOcc) void attention_prefill_tiles(PrefillArgs a, Parts parts, KvView kv, std::conditional_t<kOf == Rows::Causal, char, RowsMore> more) {
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int kRows = 16 * kNT * kW, kU = kStageBlocks;   // cache blocks of a stage
    constexpr int kPerUnit = kStageTokens / (kKvBlock * kStageBlocks);
    extern __shared__ uint4 smem[];
    __shared__ int bad_at[256 + 4];                                        // of each dim: the first position whose value is not finite
    for (int i = threadIdx.x; i < 256 + 4; i += 64 * kW) bad_at[i] = 0x7FFFFFFF;
    char* lds = reinterpret_cast<char*>(smem);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, g = lane >> 4;
    const int D = kExact ? 32 * kC : kv.D, Dp = kv_padded_dim(D);
    constexpr int kKeyPiece = 2 * kC * 1024, kValuePiece = kV * 1024, kStage = kStageBlocks * (kKeyPiece + kValuePiece);
    // where this lane's share of a wave's pieces of a stage comes from, bytes within a block
    constexpr int kKeyLoads = kStageBlocks * 2 * kC, kAll = kKeyLoads + kStageBlocks * kV, kPieces = (kAll + kW - 1) / kW;
    int piece_from[kPieces];
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
        const int p = j * kW + wave, key = p % (2 * kC) * 64 + lane, value = (p - kKeyLoads) % kV * 64 + lane;
        piece_from[j] = 16 * (p < kKeyLoads ? min(key >> 5, (Dp >> 3) - 1) * 32 + (key & 31) : value / (16 * kV) * Dp + min(value % (16 * kV), Dp - 1));
    }

    int h, row0, rows, row_last, seen; [[maybe_unused]] int front = 0;       // front, seen: the first key that the tile's rows see, and the end of the last row's
    int blocks, all_stages, run, split, stage0, stages;
    const int32_t* table = kv.table;
    int first_row, pos0;                                                   // the rows' first token among all, and its position
    if constexpr (of_groups(kOf)) {
        const SharedLaunch& l = more.shared;
        // The two kinds of workgroups mixed evenly: those over shared tokens are bound by their matrix instructions, the others by memory.
        // Heads side by side, so that with a multiple of eight of them a head's tiles meet on one XCD.
        const uint32_t x = blockIdx.x / (uint32_t)kv.kv_heads, far_before = kOf == Rows::Shared ? (uint32_t)((uint64_t)x * l.far_ratio >> 32) : 0;
        const bool far = kOf == Rows::Shared && (uint32_t)((uint64_t)(x + 1) * l.far_ratio >> 32) > far_before;
        const uint32_t i = far ? far_before : x - far_before;
        h = (int)(blockIdx.x - x * (uint32_t)kv.kv_heads);
        int first_unit = 0;
        if (far) {
            const uint32_t each = i / l.far_tiles;
            const int tile = (int)(i - each * l.far_tiles), b = (int)(each % kv.B);
            split = (int)(each / kv.B);
            rows = a.group;
            row0 = tile * kRows;
            seen = kv.length(kv.kv_len[b]);
            front = shared_tokens(kv, l.prefixes, b, seen);
            first_row = b;
            first_unit = own_first(front, kStageTokens);
            all_stages = own_units(seen, front, kStageTokens);
            run = max((all_stages + l.far - 1) / l.far, l.least_far);
        } else {
            split = (int)(i / a.tiles);
            const int64_t t = i - (uint32_t)split * a.tiles;
            const int b = sequence_of_tile(l.prefixes.start, l.prefixes.groups, t, a.group, kRows, 1);
            const SharedRows r(kv, l.prefixes, b);
            const int64_t tile = t - first_tile(l.prefixes.start[b], b, a.group, kRows, 1);
            rows = r.n * a.group;
            if (tile < 0 || tile * kRows >= rows) return;
            row0 = (int)tile * kRows;
            seen = r.len;
            first_row = r.first;
            all_stages = stages_of(seen);
            run = max((all_stages + l.near - 1) / l.near, l.least_near);
        }
        if (split * run >= all_stages) return;
        row_last = min(row0 + kRows, rows) - 1;
        blocks = (seen + kKvBlock - 1) / kKvBlock;
        stage0 = (first_unit + split * run) * kPerUnit;
        stages = min(stage0 + run * kPerUnit, (blocks + kStageBlocks - 1) / kStageBlocks);
        table += first_row * kv.table_stride;
        split += far ? l.near : 0;
        pos0 = 0;
    } else {
        // Heads side by side: with a multiple of eight of them a head's tiles meet on one XCD, whose L2 then holds its keys and values once.
        h = blockIdx.x % kv.kv_heads;
        const int64_t x = a.tiles - 1 - (int)(blockIdx.x / kv.kv_heads);       // late tiles, which see most, first
        const int b = sequence_of_tile(kv.q_start, kv.B, x, a.group, kRows, 1);
        const NewTokens nt(kv, b, a.T);
        // tokens times heads are below 2^28, so rows have 32 bits: 64-bit quotients are a hundred instructions each in front of the first load
        const int64_t tile = x - first_tile(kv.q_start[b], b, a.group, kRows, 1);
        rows = nt.n * a.group;                                                 // of the sequence, for this head
        if (tile < 0 || tile * kRows >= rows) return;
        row0 = (int)tile * kRows;
        row_last = min(row0 + kRows, rows) - 1;
        seen = tile_sees(nt, row_last, a.group);                               // keys that the tile's last token sees
        blocks = seen > 0 ? (seen + kKvBlock - 1) / kKvBlock : 0, all_stages = stages_of(seen);
        // this workgroup's stages
        run = parts.run(all_stages), stage0 = blockIdx.y * run * kPerUnit;
        stages = min(stage0 + run * kPerUnit, (blocks + kStageBlocks - 1) / kStageBlocks);
        if (blockIdx.y > 0 && stage0 >= stages) return;
        split = blockIdx.y;
        table += b * kv.table_stride;
        first_row = nt.first;
        pos0 = nt.pos0;
    }

    v8bf qf[kNT][kC];
    int pos[kNT];                                                          // of the lane's queries; -1: none
    int out_row[kNT];                                                      // row of q times heads, plus head; -1: none
    const int wave_row = row0 + wave * 16 * kNT;
#pragma unroll
    for (int n = 0; n < kNT; ++n) {
        const int R = wave_row + 16 * n + r, tok = token_of(R, a.group), hh = R - tok * a.group;
        out_row[n] = R < rows ? (first_row + tok) * a.heads + h * a.group + hh : -1;
        if constexpr (of_groups(kOf)) pos[n] = R < rows ? min(kv.length(kv.kv_len[first_row + tok]), seen) - 1 : -1;
        else pos[n] = R < rows ? pos0 + tok : -1;
        load_query<kC, kExact>(qf[n], R < rows ? a.q + (int64_t)out_row[n] * D : nullptr, g, D);
    }
    int tile_pos, pos_last;                                                 // of the tile's first token, and of the wave's last
    if constexpr (of_groups(kOf)) {                                         // the least of the tile, and the most
        const int tok0 = token_of(row0, a.group), toks = token_of(row_last, a.group) - tok0 + 1;
        int least = 0x7FFFFFFF, most = 0;
        for (int i = lane; i < toks; i += 64) {
            const int n = min(kv.length(kv.kv_len[first_row + tok0 + i]), seen);
            least = min(least, n);
            most = max(most, n);
        }
#pragma unroll
        for (int by = 1; by < 64; by *= 2) {
            least = min(least, __shfl_xor(least, by));
            most = max(most, __shfl_xor(most, by));
        }
        tile_pos = __builtin_amdgcn_readfirstlane(least) - 1;
        pos_last = wave_row < rows ? __builtin_amdgcn_readfirstlane(most) - 1 : -1;
    } else {
        tile_pos = pos0 + token_of(row0, a.group);
        pos_last = wave_row < rows ? pos0 + token_of(min(wave_row + 16 * kNT, rows) - 1, a.group) : -1;
    }
    int numbers = -1;                                                      // of 64 blocks, one a lane
    auto fetch_numbers = [&](int blk0) {
        const int blk = blk0 + lane;
        numbers = blk < blocks ? kv.block(table, blk, h) : -1;
    };
    const int64_t block_bytes = (int64_t)kKvBlock * Dp * 2;
    // 1 KiB at a time, the keys of the stage's blocks, then their values, dealt out to the waves
    auto copy = [&](int stage) {
        char* to = lds + (stage & 1) * kStage;
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
            const int p = j * kW + wave;
            if (kAll % kW && p >= kAll) break;
            const bool key = kKeyLoads % kW == 0 ? j * kW < kKeyLoads : p < kKeyLoads;
            const int at_kind = key ? p : p - kKeyLoads, of = key ? 2 * kC : kV, u = kStageBlocks == 1 ? 0 : at_kind / of, i = at_kind - u * of;
            const int64_t at = max(__builtin_amdgcn_readlane(numbers, (stage * kStageBlocks + u) & 63), 0) * block_bytes;
            const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<char*>(key ? kv.k : kv.v) + at, 0, (int)block_bytes, 0x00020000);
            const int from = kExact ? (i * 64 + lane) * 16 : piece_from[j];
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void*)(to + p * 1024), 16, from, 0, 0, 0);
        }
    };
    const int koff = g * 512 + r * 16, voff = (g * (16 * kV) + r) * 16;

    v4f acc[kNT][kV];
    float m[kNT], base[kNT], l[kNT];                                       // base: m times scale, or 0; l: of this lane's tokens
#pragma unroll
    for (int n = 0; n < kNT; ++n) {
        m[n] = kMinusInf;
        base[n] = l[n] = 0.0f;
#pragma unroll
        for (int i = 0; i < kV; ++i) acc[n][i] = (v4f){0, 0, 0, 0};
    }
    // A stage's blocks, in LDS from `keys` and `values` on, the first token at position j0.  Masked: some row does not see all of them.
    //
    // A wave's matrix instructions run beside its exponentials where the source puts them so, a slice at a time with a fence behind each: in a
    // stage of two blocks the scores of the second with the weights of the first, the values of the first with the weights of the second (with
    // one block, the other waves' matrix instructions fill that time).  Operands are read from LDS kAhead fragments ahead of their products,
    // keys and values in one sequence.
    constexpr int kParts = kF32 ? 3 : kOf == Rows::Causal ? 1 : 2, kAhead = 3, kKeys = 2 * kC;       // kKeys: fragments of a block's keys; it has kV of values
    auto take = [&](auto masked_, const char* keys, const char* values, int j0, const bool (&known)[kU]) {
        constexpr bool kMasked = decltype(masked_)::value;
        v4f sc[kU][2][kNT];
        v8bf w[kU][kNT][kParts], frag[kAhead];
        auto read = [&](int f) {
            if (f < kKeys * kU) frag[f % kAhead] = *reinterpret_cast<const v8bf*>(keys + f / kKeys * kKeyPiece + koff + 2048 * (f / 2 % kC) + 256 * (f & 1));
            else if (f < (kKeys + kV) * kU)
                frag[f % kAhead] = *reinterpret_cast<const v8bf*>(values + (f - kKeys * kU) / kV * kValuePiece + voff + 256 * ((f - kKeys * kU) % kV));
        };
        // the i-th of `slices` shares of block u's weights, two at a time
        auto weights = [&](int u, int i, int slices) {
#pragma unroll
            for (int q = i * (4 * kNT) / slices; q < (i + 1) * (4 * kNT) / slices; ++q) {
                const int n = q / 4, j = q % 4 * 2;
                const float p0 = exp2_fast(__builtin_fmaf(sc[u][j >> 2][n][j & 3], a.scale, -base[n]));
                const float p1 = exp2_fast(__builtin_fmaf(sc[u][j >> 2][n][(j & 3) + 1], a.scale, -base[n]));
                weights_pair<kParts>(w[u][n], j, p0, p1);
                l[n] = kParts > 1 ? l[n] + p0 + p1 : add_rounded(l[n], w[u][n][0], j);
            }
        };
        auto scores = [&](int u, int with) {
#pragma unroll
            for (int i = 0; i < kKeys; ++i) {
                const int f = u * kKeys + i, c = i / 2, t = i & 1;
#pragma unroll
                for (int n = 0; n < kNT; ++n) sc[u][t][n] = mfma_bf16(frag[f % kAhead], qf[n][c], c ? sc[u][t][n] : (v4f){0, 0, 0, 0});
                read(f + kAhead);
                if (with >= 0) weights(with, i, kKeys);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        auto product = [&](int u, int with) {
#pragma unroll
            for (int i = 0; i < kV; ++i) {
                const int f = kU * kKeys + u * kV + i;
#pragma unroll
                for (int n = 0; n < kNT; ++n)
#pragma unroll
                    for (int e = 0; e < kParts; ++e) acc[n][i] = mfma_bf16(frag[f % kAhead], w[u][n][e], acc[n][i]);
                read(f + kAhead);
                if (with >= 0) weights(with, i, kV);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        // The maximum so far against block u's scores.  One that is passed by less than kSlack stays: weights up to 2^kSlack lose nothing in
        // 32-bit sums nor, being floating-point numbers, in bf16.  Otherwise what has been summed is rescaled, together with the values of
        // the block in front of u, whose weights went by the old maximum.
        auto check = [&](int u) {
            bool passed = false;
            float tops[kNT];
#pragma unroll
            for (int n = 0; n < kNT; ++n) {
                if (kMasked)
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (!known[u] || j0 + u * kKvBlock + 8 * g + j > pos[n] || (kOf == Rows::Shared && j0 + u * kKvBlock + 8 * g + j < front)) sc[u][j >> 2][n][j & 3] = kMinusInf;
                float top = sc[u][0][n][0];
#pragma unroll
                for (int j = 1; j < 8; ++j) top = fmaxf(top, sc[u][j >> 2][n][j & 3]);
                tops[n] = top;
                passed = passed || top > m[n] + a.slack;
            }
            if (__builtin_amdgcn_ballot_w64(passed)) {
                if (u > 0) {
#pragma unroll
                    for (int i = 0; i < kV; ++i) {
                        const v8bf v = *reinterpret_cast<const v8bf*>(values + (u - 1) * kValuePiece + voff + 256 * i);
#pragma unroll
                        for (int n = 0; n < kNT; ++n)
#pragma unroll
                            for (int e = 0; e < kParts; ++e) acc[n][i] = mfma_bf16(v, w[u - 1][n][e], acc[n][i]);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
#pragma unroll
                for (int n = 0; n < kNT; ++n) {
                    const float now = fmaxf(m[n], groups_max(tops[n])), by = now == kMinusInf ? 1.0f : exp2_fast((m[n] - now) * a.scale);
                    m[n] = now;
                    base[n] = now == kMinusInf ? 0.0f : now * a.scale;
                    l[n] *= by;
#pragma unroll
                    for (int i = 0; i < kV; ++i) acc[n][i] *= by;
                    if (u > 0)
#pragma unroll
                        for (int e = 0; e < kParts; ++e) w[u - 1][n][e] = v8bf{};
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        };
#pragma unroll
        for (int i = 0; i < kAhead; ++i) read(i);
        scores(0, -1);
        check(0);
        if (kU == 2) {
            scores(kU - 1, 0);
            check(kU - 1);
            product(0, kU - 1);
        } else {
            weights(0, 0, 1);
        }
        product(kU - 1, -1);
    };
    auto stage_there = [&](int s) {                                        // publishes stage s, requests the next
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();
        if (s + 1 < stages) {
            if ((((s + 1) * kStageBlocks) & 63) == 0) fetch_numbers((s + 1) * kStageBlocks);
            copy(s + 1);
        }
    };
    __syncthreads();
    if (stage0 < stages) {
        fetch_numbers((stage0 * kStageBlocks) & ~63);
        copy(stage0);
    }
#pragma unroll
    for (int n = 0; n < kNT; ++n) settle_query<kC, kExact>(qf[n], g, D);
    // The values of a stage that some row does not see to its end.  A weight of zero does not make an infinity nothing: tokens that no row sees
    // are cleared in LDS, and of the others what is not finite, which is noted: rows that see it get NaN in its dim at the end, the rows in
    // front of it their sums.
    auto clean = [&](char* values, int j0, const bool (&known)[kStageBlocks]) {
        for (int i = threadIdx.x; i < kStageBlocks * 64 * kV; i += 64 * kW) {
            const int u = i / (64 * kV), at = i % (64 * kV), first = j0 + u * kKvBlock + at / (16 * kV) * 8, d = at % (16 * kV);
            const int some = known[u] ? min(max(seen - first, 0), 8) : 0;
            uint4* place = reinterpret_cast<uint4*>(values + i * 16);
            v4u v = __builtin_bit_cast(v4u, *place);
            values_keep(v, some);
            if (kOf == Rows::Shared && first < front) values_drop(v, front - first);
            unsigned bad = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) bad |= (unsigned)((v[e] & 0x7F80u) == 0x7F80u) | (unsigned)((v[e] & 0x7F800000u) == 0x7F800000u);
            if (bad) {
                for (int e = 7; e >= 0; --e) {
                    const unsigned half = 0xFFFFu << (16 * (e & 1)), exponent = 0x7F80u << (16 * (e & 1));
                    if ((v[e >> 1] & exponent) != exponent) continue;
                    v[e >> 1] &= ~half;
                    atomicMin(&bad_at[d], first + e);
                }
            }
            if (bad || some < 8 || (kOf == Rows::Shared && first < front)) *place = __builtin_bit_cast(uint4, v);
        }
    };
    int s = stage0;
    auto whole_stage = [&](int s) {                                        // that all rows of the tile see, and all of whose pages exist
        const int j0 = s * kStageBlocks * kKvBlock, at = (s * kStageBlocks) & 63;
        return (kOf != Rows::Shared || j0 >= front) && j0 + kStageBlocks * kKvBlock - 1 <= tile_pos && __builtin_amdgcn_readlane(numbers, at) >= 0 &&
               __builtin_amdgcn_readlane(numbers, at + kStageBlocks - 1) >= 0;
    };
    auto plain_stage = [&](int s) {
        stage_there(s);
        const char* keys = lds + (s & 1) * kStage;
        const char* values = keys + kStageBlocks * kKeyPiece;
        const bool known[kU] = {};
        if (kOf != Rows::Shared || wave_row < rows) take(std::false_type(), keys, values, s * kStageBlocks * kKvBlock, known);
    };
    auto masked_stage = [&](int s) {
        const int j0 = s * kStageBlocks * kKvBlock;
        bool known[kStageBlocks];
#pragma unroll
        for (int u = 0; u < kStageBlocks; ++u) known[u] = __builtin_amdgcn_readlane(numbers, (s * kStageBlocks + u) & 63) >= 0;
        stage_there(s);
        char* keys = lds + (s & 1) * kStage;
        char* values = keys + kStageBlocks * kKeyPiece;
        clean(values, j0, known);
        __syncthreads();
        if (j0 > pos_last) return;                                         // nothing that this wave's rows see
        take(std::true_type(), keys, values, j0, known);
    };
    if constexpr (kOf == Rows::Shared) {                                   // the first stage may begin with shared tokens
        for (; s < stages; ++s)
            if (whole_stage(s)) plain_stage(s);
            else masked_stage(s);
    } else {
        for (; s < stages && whole_stage(s); ++s) plain_stage(s);
        for (; s < stages; ++s) masked_stage(s);
    }
#pragma unroll
    for (int n = 0; n < kNT; ++n) {
        const float total = groups_sum(l[n]), inv = total > 0.0f ? 1.0f / total : 0.0f;
        if (out_row[n] < 0) continue;
        const int64_t place = (int64_t)out_row[n] * parts.splits + split;
        const bool whole = !of_groups(kOf) && run >= all_stages;
        const float by = whole ? inv : 1.0f;
#pragma unroll
        for (int i = 0; i < kV; ++i) {
            const int d = 16 * i + 4 * g, end = kExact || i < 2 * whole_chunks(kC) ? d + 4 : D;
            if (d >= end) continue;
            float out[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) out[e] = pos[n] >= bad_at[d + e] ? __builtin_nanf("") : finite_or_nan(acc[n][i][e], by);
            if (whole) store4<kF32>(a.o, (int64_t)out_row[n] * D, d, end, out);
            else store4<true>(parts.sums, place * D, d, end, out);
        }
        if (!whole && g == 0) {
            parts.state[2 * place] = m[n];
            parts.state[2 * place + 1] = total;
        }
        if constexpr (kOf == Rows::Kept)
            if (whole && g == 0) {
                more.keep.state[2 * (int64_t)out_row[n]] = m[n];
                more.keep.state[2 * (int64_t)out_row[n] + 1] = total;
            }
    }
#endif
}

template <int kC, int kV, bool kExact, int kNT, int kStageBlocks, int kW, int kOcc, bool kF32, Rows kOf, typename More>
hipError_t launch_prefill_tiles(PrefillArgs a, const Parts& parts, const KvView& kv, More more, hipStream_t stream) {
    static RaisedFlags raised;
    const auto kernel = attention_prefill_tiles<kC, kV, kExact, kNT, kStageBlocks, kW, kOcc, kF32, kOf>;
    constexpr int kLds = prefill_lds(kC, kV, kStageBlocks);
    if (kLds > 65536 - 2048) {                             // with the static part
        const hipError_t e = raise_dynamic_lds(reinterpret_cast<const void*>(kernel), kLds, raised);
        if (e != hipSuccess) return e;
    }
    if constexpr (of_groups(kOf)) {
        kernel<<<(more.shared.near_blocks + more.shared.far_blocks) * kv.kv_heads, 64 * kW, kLds, stream>>>(a, parts, kv, more);
    } else {
        a.tiles = (int)tiles_at_most(a.T, kv.B, a.group, 16 * kNT * kW, 1);
        kernel<<<dim3((unsigned)((int64_t)a.tiles * kv.kv_heads), parts.splits), 64 * kW, kLds, stream>>>(a, parts, kv, more);
    }
    return hipGetLastError();
}
template <int kC, int kV, bool kExact, bool kF32, Rows kOf, typename More>
hipError_t launch_prefill_form(PrefillTile tile, const PrefillArgs& a, const Parts& parts, const KvView& kv, More more, hipStream_t stream) {
    constexpr int kStageBlocks = kC <= 2 ? 2 : 1;
    if (tile == PrefillTile::Rows64) return launch_prefill_tiles<kC, kV, kExact, 1, kStageBlocks, 4, kC <= 4 ? 4 : 2, kF32, kOf>(a, parts, kv, more, stream);
    return launch_prefill_tiles<kC, kV, kExact, kC <= 4 ? 2 : 1, kStageBlocks, kC <= 4 ? 4 : 8, kC <= 4 && !kF32 ? 3 : 2, kF32, kOf>(a, parts, kv, more, stream);
}
// compiled in translation units of their own
template <int kC, int kV, bool kExact>
hipError_t launch_prefill(PrefillTile tile, const PrefillArgs& a, const Parts& parts, const KvView& kv, bool f32, hipStream_t stream) {
    return f32 ? launch_prefill_form<kC, kV, kExact, true, Rows::Causal>(tile, a, parts, kv, (char)0, stream)
               : launch_prefill_form<kC, kV, kExact, false, Rows::Causal>(tile, a, parts, kv, (char)0, stream);
}
template <int kC, int kV, bool kExact>
hipError_t launch_prefill_kept(PrefillTile tile, const PrefillArgs& a, const Parts& parts, const KvView& kv, bool f32, const RowsMore& more, hipStream_t stream) {
    return f32 ? launch_prefill_form<kC, kV, kExact, true, Rows::Kept>(tile, a, parts, kv, more, stream)
               : launch_prefill_form<kC, kV, kExact, false, Rows::Kept>(tile, a, parts, kv, more, stream);
}
template <int kC, int kV, bool kExact>
hipError_t launch_prefill_shared(PrefillTile tile, const PrefillArgs& a, const Parts& parts, const KvView& kv, bool f32, const RowsMore& more, hipStream_t stream) {
    constexpr int kStageBlocks = kC <= 2 ? 2 : 1, kOcc = kC <= 4 ? 4 : 2, kLess = kC <= 4 ? 3 : 2;
    if (more.shared.far_blocks) {
        if (f32) return launch_prefill_tiles<kC, kV, kExact, 1, kStageBlocks, 4, kLess, true, Rows::Shared>(a, parts, kv, more, stream);
        return launch_prefill_tiles<kC, kV, kExact, 1, kStageBlocks, 4, kLess, false, Rows::Shared>(a, parts, kv, more, stream);
    }
    if (f32) return launch_prefill_tiles<kC, kV, kExact, 1, kStageBlocks, 4, kOcc, true, Rows::Prefix>(a, parts, kv, more, stream);
    if constexpr (kC <= 4) {                               // of larger heads there is no tile of 128 rows that shares its operands
        if (tile == PrefillTile::Rows128) return launch_prefill_tiles<kC, kV, kExact, 2, kStageBlocks, 4, 3, false, Rows::Prefix>(a, parts, kv, more, stream);
    }
    return launch_prefill_tiles<kC, kV, kExact, 1, kStageBlocks, 4, kOcc, false, Rows::Prefix>(a, parts, kv, more, stream);
}

// The sizes that those units build, and the one for a head of D dims: `go` is called with it as types.
#define BITNET_PREFILL_SIZES(X) \
    X(1, 2, true) X(2, 4, true) X(3, 6, true) X(4, 8, true) X(6, 12, true) X(8, 16, true) X(1, 1, false) X(2, 3, false) X(3, 5, false) X(4, 7, false) \
    X(1, 2, false) X(2, 4, false) X(3, 6, false) X(4, 8, false) X(6, 12, false) X(8, 16, false)
#define BITNET_PREFILL_UNIT(kC_, kV_, kE_)                                                                                                          \
    template hipError_t launch_prefill<kC_, kV_, kE_>(PrefillTile, const PrefillArgs&, const Parts&, const KvView&, bool, hipStream_t);                \
    template hipError_t launch_prefill_kept<kC_, kV_, kE_>(PrefillTile, const PrefillArgs&, const Parts&, const KvView&, bool, const RowsMore&, hipStream_t); \
    template hipError_t launch_prefill_shared<kC_, kV_, kE_>(PrefillTile, const PrefillArgs&, const Parts&, const KvView&, bool, const RowsMore&, hipStream_t);

// Runs of rows whose softmax states are kept; the workspace is that of runs.
hipError_t launch_attention_prefill_kept(const void* q, const KvView& kv, int64_t T, int heads, float scale, void* o, bool f32, const KeptRows& keep, void* workspace,
                                         size_t workspace_bytes, hipStream_t stream);

}  // namespace bitnet
