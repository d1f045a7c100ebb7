// Attention that also adds up what weight each cached token has had, over rows and over the heads of its key-value head:
//   acc[b][h][j] += sum over the call's rows i of sequence b and the heads of h of exp(scale q_i . k_j - m_i) / l_i.
// A row's m and l are known when its attention is: single tokens leave their scores (4 bytes for a key and head beside the 4 D that a key and its
// value are read in) and a second launch turns them into weights; for runs of tokens scores would be as many as there are pairs, so the second
// launch works them out again, a tile of keys against all rows that see it.
#include "attention_decode_kernel.hpp"
#include "attention_join.hpp"
#include "attention_prefill_kernel.hpp"

namespace bitnet {
namespace {

struct WeightsArgs {
    const float* scores;               // [B][heads][max_blocks * 32]
    float* weights;                    // [B][kv heads][stride]
    int64_t stride, tasks;             // of the weights: sequences times kv heads times chunks
    float scale;
    int heads, group, chunks, joins;   // chunks of kChunk tokens for which the tables have room; rows to join in front
};
constexpr int kChunk = 1024;

// Joins the rows that several workgroups shared, one to a workgroup, then turns chunks of scores into weights, four tokens a thread.  Bound by memory: three
// sequences of 20000 to 49152 tokens, 64 heads over 8, 31 MB of scores in 9.7 us.  What scores cost more is that they are written beside the stream of the
// cache (there 83 us with them, 66 without; with streaming stores 87).
template <bool kF32>
__global__ __launch_bounds__(256) void attention_weights_of_tokens(void* o, WeightsArgs a, Parts parts, KvView kv) {
    __shared__ JoinRoom room;
    __shared__ float base[64], inv[64];
    if ((int)blockIdx.x < a.joins) {
        const int b = blockIdx.x / a.heads, blocks = blocks_of(kv, b), run = parts.run(blocks), n = (blocks + run - 1) / run;
        if (n < 2) return;                                  // stored by the workgroup that had all of it
        join_row<kF32>(room, parts, (int64_t)blockIdx.x * parts.splits, n, a.scale, kv.D, o, blockIdx.x);
        return;
    }
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t capacity = (int64_t)kv.max_blocks * kKvBlock;
    for (int64_t task = blockIdx.x - a.joins; task < a.tasks; task += gridDim.x - a.joins) {
        const int64_t pair = task / a.chunks;
        const int chunk = (int)(task - pair * a.chunks), b = (int)(pair / kv.kv_heads), h = (int)(pair - (int64_t)b * kv.kv_heads);
        const int len = kv.length(kv.kv_len[b]);
        const int64_t pos = (int64_t)chunk * kChunk + 4 * threadIdx.x;
        if ((int64_t)chunk * kChunk >= len) continue;       // the same for all threads
        const int blocks = (len + kKvBlock - 1) / kKvBlock, run = parts.run(blocks), n = (blocks + run - 1) / run;
        v4f sum = {0, 0, 0, 0};
        for (int e0 = 0; e0 < a.group; e0 += 64) {
            const int some = min(a.group - e0, 64);
            __syncthreads();
            for (int e = wave; e < some; e += 4) {
                const int64_t place0 = ((int64_t)b * a.heads + h * a.group + e0 + e) * parts.splits;
                float m = kMinusInf, l = 0.0f;
                for (int s = lane; s < n; s += 64) m = fmaxf(m, parts.state[(place0 + s) * 2]);
                m = wave_max(m);
                for (int s = lane; s < n; s += 64) {
                    const float ms = parts.state[(place0 + s) * 2];
                    l += ms == kMinusInf ? 0.0f : parts.state[(place0 + s) * 2 + 1] * exp2_fast((ms - m) * a.scale);
                }
                l = wave_sum(l);
                if (lane == 0) {
                    base[e] = m == kMinusInf ? 0.0f : m * a.scale;
                    inv[e] = l > 0.0f ? 1.0f / l : 0.0f;
                }
            }
            __syncthreads();
            if (pos < len) {
                const float* from = a.scores + ((int64_t)b * a.heads + h * a.group + e0) * capacity + pos;
#pragma unroll 4
                for (int e = 0; e < some; ++e) {
                    const v4f s = *reinterpret_cast<const v4f*>(from + e * capacity);
#pragma unroll
                    for (int i = 0; i < 4; ++i) sum[i] = __builtin_fmaf(exp2_fast(__builtin_fmaf(s[i], a.scale, -base[e])), inv[e], sum[i]);
                }
            }
        }
        if (pos < len) {
            float* to = a.weights + pair * a.stride + pos;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (pos + i < len) to[i] = (pos + i == len - 1 ? 0.0f : to[i]) + sum[i];      // the call's own token begins with nothing
        }
    }
}

// ---- runs of tokens -------------------------------------------------------------------------------------------------------------------
struct ColumnArgs {
    const uint16_t* q;
    const float* state;                // [T][heads][2]: m, l
    float* weights;                    // [B][kv heads][stride]
    float* parts;                      // [shares][sequences times kv heads][keys of a tile]
    int64_t stride, tasks;             // of the weights: tiles of keys, or shares of them, times sequences times kv heads
    float scale;
    int heads, group, T;
    uint32_t shares, most;             // of a sequence's tiles for one head, together, that the parts have room for; workgroups that share a tile's rows, at most
    int least;                         // stages that one has at least
    uint32_t magic, shift;             // of the division by `group`: the quotient of n is (high word of n magic + n) >> shift, n below 2^31
    __device__ int token(int row) const { return (int)((__umulhi((uint32_t)row, magic) + (uint32_t)row) >> shift); }
};

// The shape of a workgroup: four waves of 32 kKB keys each, in registers, and stages of 16 kTiles rows in LDS.
template <int kC> struct Columns {
    static constexpr int kKB = kC <= 4 ? 2 : 1, kKeys = 128 * kKB, kTiles = kC <= 4 ? 4 : 2, kRows = 16 * kTiles;
};

// What a tile of keys is: its sequence and head, the rows that see any of it, and how they are shared out, in stages.
template <int kC>
struct ColumnTile {
    int h, b, share, tile, blocks, blk, j0, rows, first, stages, run;
    NewTokens nt;
    // Heads side by side, so that with a multiple of eight of them a head's tiles meet on one XCD, whose L2 holds its queries; the first tiles, which most
    // rows see, first with all their shares, so that what comes last is short.
    // 64-bit quotients are a hundred instructions each in front of the first load
    __device__ static uint32_t each_of(int64_t task, uint32_t pairs) { return task >> 32 ? (uint32_t)(task / pairs) : (uint32_t)task / pairs; }
    __device__ ColumnTile(const ColumnArgs& a, const KvView& kv, int64_t task)
        : ColumnTile(a, kv, task, (uint32_t)(kv.B * kv.kv_heads), each_of(task, (uint32_t)(kv.B * kv.kv_heads))) {}
    __device__ ColumnTile(const ColumnArgs& a, const KvView& kv, int64_t task, uint32_t pairs, uint32_t each)
        : h((int)((uint32_t)(task - (int64_t)each * pairs) % (uint32_t)kv.kv_heads)), b((int)((uint32_t)(task - (int64_t)each * pairs) / (uint32_t)kv.kv_heads)),
          nt(kv, b, a.T) {
        blocks = blocks_of(kv, b);
        // as many shares of a tile as the sequence's tiles leave, whatever its table has room for
        const uint32_t tiles = ((uint32_t)blocks + 4 * Columns<kC>::kKB - 1) / (4 * Columns<kC>::kKB), splits = min(max(a.shares / max(tiles, 1u), 1u), a.most);
        tile = (int)(each / splits);
        share = (int)(each - (uint32_t)tile * splits);
        blk = tile * (4 * Columns<kC>::kKB);
        j0 = blk * kKvBlock;
        rows = nt.n * a.group;
        if (nt.n == 0 || blk >= blocks) { stages = 0, run = 1, first = 0; return; }
        first = max(j0 - nt.pos0, 0) * a.group / 16 * 16;
        stages = (rows - first + Columns<kC>::kRows - 1) / Columns<kC>::kRows;
        run = max((stages + (int)splits - 1) / (int)splits, a.least);
    }
};

// dims d0 ... d0 + 7 of a row, zeros behind its end; settle_dims once they are there
__device__ inline v4u load_dims(const uint16_t* row, int d0, int D) {
    v4u w = {0, 0, 0, 0};
    if (D >= 8) {
        __builtin_memcpy(&w, row + min(d0, D - 8), 16);
    } else {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (d0 + 2 * i < D) {
                uint32_t two;
                __builtin_memcpy(&two, row + d0 + 2 * i, 4);
                w[i] = two;
            }
    }
    return w;
}
__device__ inline v4u settle_dims(v4u w, int d0, int D) {
    if (D < 8) return w;
    const int over = max(d0 + 8 - D, 0) >> 1;
    if (over & 1) w = (v4u){w[1], w[2], w[3], 0};
    if (over & 2) w = (v4u){w[2], w[3], 0, 0};
    if (over >= 4) w = (v4u){0, 0, 0, 0};
    return w;
}

// A workgroup takes a tile of keys and a run of the rows that see any of it, which come through LDS a stage at a time for its four waves, the next
// stage requested while one is worked on.  Scores are products of keys (down) and queries (across), so that a lane sums up eight tokens of a block for
// its queries; the lanes of a group meet at the end.
//
// Bound by exponentials and matrix instructions in turn (counters on a chunk of 1024 tokens behind 15000, 64 heads over 8: the matrix pipe 37 % busy, the vector
// pipe 59 %; 285 us, 0.91 PFLOP/s), of short runs by what a workgroup begins with and by its rows' way from memory, one stage ahead (a prompt of 2048 tokens, 40
// heads: 39 us, 0.55 PFLOP/s).  Rows straight from memory to each wave's registers, without LDS, took 64 us there: four times as many bytes through the L2.
template <int kC, bool kExact>
__global__ __launch_bounds__(256, 2) void attention_weights_of_runs(ColumnArgs a, KvView kv) {
    using Shape = Columns<kC>;
    constexpr int kKB = Shape::kKB, kTiles = Shape::kTiles, kRows = Shape::kRows, kPieces = kTiles * kC / 4;
    __shared__ uint4 queries[2][kTiles * kC * 64];
    __shared__ float2 stats[2][kRows];                      // m times scale, or 0, and 1 / l, or 0
    __shared__ int positions[2][kRows];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int D = kExact ? 32 * kC : kv.D, Dp = kv_padded_dim(D), quads = Dp >> 3;
    // this wave's share of a stage: kPieces chunks of 32 dims, from c0 on, of the rows of one tile
    const int my_tile = wave * kTiles / 4, c0 = kTiles == 4 ? 0 : (wave & 1) * (kC / 2);
    for (int64_t task = blockIdx.x; task < a.tasks; task += gridDim.x) {
        const ColumnTile<kC> t(a, kv, task);
        const int s0 = t.share * t.run, s1 = min(s0 + t.run, t.stages);
        if (s0 >= s1) continue;                             // the same for all waves
        struct { v4u w[kPieces]; float m, l; int pos; bool there; } next;
        auto load = [&](int s) {
            const int R = t.first + s * kRows + my_tile * 16 + r, tok = a.token(R), row = (t.nt.first + tok) * a.heads + t.h * a.group + R - tok * a.group;
            const bool there = R < t.rows;
            const uint16_t* from = a.q + (int64_t)(there ? row : 0) * D;
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                const int d0 = 32 * (c0 + i) + 8 * g;
                if (kExact) __builtin_memcpy(&next.w[i], from + d0, 16);
                else next.w[i] = load_dims(from, d0, D);
            }
            next.m = kMinusInf, next.l = 0.0f;
            if (there) {
                next.m = a.state[2 * (int64_t)row];
                next.l = a.state[2 * (int64_t)row + 1];
            }
            next.pos = there ? t.nt.pos0 + tok : -1;
            next.there = there;
        };
        auto publish = [&](int s) {                         // rows that there are not are zeros, and their l is 0
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                v4u w = kExact ? next.w[i] : settle_dims(next.w[i], 32 * (c0 + i) + 8 * g, D);
                if (!next.there) w = (v4u){0, 0, 0, 0};
                queries[s & 1][(my_tile * kC + c0 + i) * 64 + lane] = __builtin_bit_cast(uint4, w);
            }
            if (c0 == 0 && g == 0) {
                stats[s & 1][my_tile * 16 + r] = {next.m == kMinusInf ? 0.0f : next.m * a.scale, next.l > 0.0f ? 1.0f / next.l : 0.0f};
                positions[s & 1][my_tile * 16 + r] = next.pos;
            }
        };
        load(s0);
        const int blk = t.blk + wave * kKB, j0 = blk * kKvBlock;
        v8bf k[kKB][kC][2];
        bool known[kKB];
#pragma unroll
        for (int u = 0; u < kKB; ++u) {
            const int number = blk + u < t.blocks ? kv.block(kv.table + t.b * kv.table_stride, blk + u, t.h) : -1;
            known[u] = number >= 0;
            const char* from = reinterpret_cast<const char*>(kv.k) + (int64_t)max(number, 0) * kKvBlock * Dp * 2;
#pragma unroll
            for (int c = 0; c < kC; ++c)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int off = (kExact || c < whole_chunks(kC) ? 4 * c + g : min(4 * c + g, quads - 1)) * 512 + r * 16 + 256 * i;
                    k[u][c][i] = __builtin_bit_cast(v8bf, *reinterpret_cast<const v4u*>(from + off));
                }
        }
        float acc[kKB][8] = {};
        // Scores of 16 rows against the wave's keys, and what becomes of them.  The matrix instructions of a tile of rows run beside the exponentials of
        // the one in front of it, where the source puts them so: one after each, with a fence behind.
        struct Scores { v4f x[kKB][2]; float2 st; int pos; };
        // adds token j of block u; masked: rows in front of it have no weight for it
        auto add = [&](auto masked, const Scores& y, int u, int j) {
            float p = exp2_fast(__builtin_fmaf(y.x[u][j >> 2][j & 3], a.scale, -y.st.x));
            if (decltype(masked)::value) p = j0 + u * kKvBlock + 8 * g + j <= y.pos ? p : 0.0f;
            acc[u][j] = __builtin_fmaf(p, y.st.y, acc[u][j]);
        };
        auto scores = [&](auto masked, auto with, Scores& x, const v8bf (&q)[kC], const Scores& old) {
#pragma unroll
            for (int i = 0; i < 2 * kC * kKB; ++i) {
                const int c = i / (2 * kKB), u = i / 2 % kKB, e = i % 2;
                x.x[u][e] = mfma_bf16(k[u][c][e], q[c], c ? x.x[u][e] : (v4f){0, 0, 0, 0});
#pragma unroll
                for (int w = 0; w < 8 * kKB; ++w)
                    if (decltype(with)::value && w * kC / 4 == i) add(masked, old, w / 8, w % 8);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        auto stage = [&](auto masked, int s) {
            v8bf q[2][kC];
            Scores x[2];
            auto read = [&](int i) {
#pragma unroll
                for (int c = 0; c < kC; ++c) q[i & 1][c] = __builtin_bit_cast(v8bf, queries[s & 1][(i * kC + c) * 64 + lane]);
                x[i & 1].st = stats[s & 1][i * 16 + r];
                if (decltype(masked)::value) x[i & 1].pos = positions[s & 1][i * 16 + r];
            };
            read(0);
#pragma unroll
            for (int i = 0; i < kTiles; ++i) {
                if (i == 0) scores(masked, std::false_type(), x[0], q[0], x[0]);
                else scores(masked, std::true_type(), x[i & 1], q[i & 1], x[1 - (i & 1)]);
                if (i + 1 < kTiles) read(i + 1);
            }
#pragma unroll
            for (int u = 0; u < kKB; ++u)
#pragma unroll
                for (int j = 0; j < 8; ++j) add(masked, x[(kTiles - 1) & 1], u, j);
        };
        publish(s0);
        __builtin_amdgcn_s_waitcnt(0);                      // the keys: waited for in the loop, they would be the next stage's loads too
        for (int s = s0; s < s1; ++s) {
            __syncthreads();
            if (s + 1 < s1) load(s + 1);
            // positions do not fall, and rows that there are not have -1: the first row's says whether all see all of the wave's keys
            const int pos = positions[s & 1][lane & (kRows - 1)];
            if (__builtin_amdgcn_readfirstlane(pos) >= j0 + kKvBlock * kKB - 1) stage(std::false_type(), s);
            else if (__builtin_amdgcn_ballot_w64(pos >= j0)) stage(std::true_type(), s);
            if (s + 1 < s1) publish(s + 1);                 // the other half, which all waves left at the barrier
        }
        const bool whole = t.run >= t.stages;
        const int len = kv.length(kv.kv_len[t.b]);
        float* to = a.weights + ((int64_t)t.b * kv.kv_heads + t.h) * a.stride;
        float* part = a.parts + task * Shape::kKeys - t.j0;
#pragma unroll
        for (int u = 0; u < kKB; ++u)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float v = acc[u][j];
                v += dpp_f32<0xB1>(v);
                v += dpp_f32<0x4E>(v);
                v += dpp_f32<0x141>(v);
                v += dpp_f32<0x140>(v);
                v = known[u] ? v : 0.0f;
                const int at = j0 + u * kKvBlock + 8 * g + j;
                if (r != j || at >= len) continue;
                if (whole) to[at] = (at >= t.nt.pos0 ? 0.0f : to[at]) + v;       // the call's own tokens begin with nothing
                else part[at] = v;
            }
        __syncthreads();
    }
}

// The parts of tiles whose rows several workgroups shared, added up.
template <int kC>
__global__ __launch_bounds__(Columns<kC>::kKeys) void attention_weights_join(ColumnArgs a, KvView kv) {
    for (int64_t task = blockIdx.x; task < a.tasks; task += gridDim.x) {
        const ColumnTile<kC> t(a, kv, task);
        const int at = t.j0 + (int)threadIdx.x;
        if (t.share > 0 || t.run >= t.stages || at >= kv.length(kv.kv_len[t.b])) continue;
        const int64_t pitch = (int64_t)kv.B * kv.kv_heads * Columns<kC>::kKeys;
        const float* part = a.parts + task * Columns<kC>::kKeys + threadIdx.x;
        float sum = 0.0f;
        for (int s = 0; s * t.run < t.stages; ++s) sum += part[s * pitch];
        float* to = a.weights + ((int64_t)t.b * kv.kv_heads + t.h) * a.stride + at;
        *to = (at >= t.nt.pos0 ? 0.0f : *to) + sum;
    }
}

// How many workgroups share the rows of a tile of keys: as many as make 1024 of them, two rounds of what the chip holds, with two stages or more each;
// their sums go through the workspace and another launch (us without that launch, 1 / 2 / 4 / 8 / 16 / 32: 64 heads over 8, 512 tokens 110 / 70 / 37 / 21 / 13 /
// 8.8, 2048 tokens 351 / 192 / 112 / 81 / 73 / -; 40 heads, 2048 tokens 57 / 46 / 49 / 50 / 57 / -; six of 450 behind 250, 32 heads of 100 36 / 38 / 42 / 54 / 66 / -).
// A sequence's tiles are counted where its length is known, on the device, and not by the room in the tables (64 heads over 8 in a table of 32768 tokens, whole
// calls: 512 tokens 31.5 us, by the room 110); here stands what all of them may be together.  Where tables have more than four
// times the call's tokens the other launch, 4 us, is there whether tiles are shared or not; where they have less, only if they are by the room.
struct ColumnsPlan {
    int64_t tasks;
    int shares, most;                  // as in ColumnArgs
    size_t bytes;
};
constexpr int kLeastStages = 2;
template <int kC>
ColumnsPlan columns_plan(const KvView& kv, int64_t T, int group) {
    using Shape = Columns<kC>;
    const int64_t pairs = (int64_t)kv.B * kv.kv_heads, room = ceil_div(kv.max_blocks, 4 * Shape::kKB), most = ceil_div(T * group, Shape::kRows * kLeastStages);
    const bool roomy = (int64_t)kv.max_blocks * kKvBlock > 4 * (T / kv.B);
    int64_t shares = 1024 / pairs;
    if (most < 2 || shares < 2 || (!roomy && shares / room < 2)) return {pairs * room, 1, 1, 0};
    if (shares / most >= room) shares = room * most;
    return {pairs * (room > shares ? room : shares), (int)shares, (int)(most < shares ? most : shares), (size_t)(pairs * shares * Shape::kKeys) * 4};
}

// Splits of single tokens' rows and the workspace: parts, then scores.
struct TokensPlan {
    Splits splits;
    size_t parts, scores;
};
TokensPlan tokens_plan(const KvView& kv, int heads) {
    const Splits s = decode_splits(kv, heads);
    const int64_t rows = (int64_t)kv.B * heads;
    return {s, ((size_t)(rows * s.n) * (kv.D + 2) * 4 + 15) / 16 * 16, (size_t)rows * kv.max_blocks * kKvBlock * 4};
}
constexpr int64_t kMostBlocks = 1 << 20;                   // of a launch that loops over its tasks

}  // namespace

// Of runs: the rows' states, the parts of tiles of keys, and what the attention takes.
struct RunsPlan { size_t states, parts, attention; };
static RunsPlan runs_plan(const KvView& kv, int64_t T, int heads) {
    RunsPlan p{((size_t)(T * heads) * 8 + 15) / 16 * 16, 0, attention_prefill_workspace_bytes(kv, T, heads)};
    (void)for_head_size(kv.D, [&](auto c, auto, auto) {
        p.parts = columns_plan<c.value>(kv, T, heads / kv.kv_heads).bytes;
        return hipSuccess;
    });
    return p;
}

size_t attention_weights_workspace_bytes(const KvView& kv, int64_t T, int heads, bool prefill) {
    if (prefill) {
        const RunsPlan p = runs_plan(kv, T, heads);
        return p.states + p.parts + p.attention;
    }
    const TokensPlan p = tokens_plan(kv, heads);
    return p.parts + p.scores;
}

hipError_t launch_attention_decode_weights(const void* q, const KvView& kv, int heads, float scale, void* o, bool f32, float* weights, int64_t stride,
                                           void* workspace, hipStream_t stream) {
    const int group = heads / kv.kv_heads;
    const float by = scale * 1.44269504f;
    const TokensPlan plan = tokens_plan(kv, heads);
    const int64_t rows = (int64_t)kv.B * heads;
    const Parts parts(workspace, rows, plan.splits.n, plan.splits.least, kv.D);
    const DecodeArgs a{static_cast<const uint16_t*>(q), o, by, heads, group, (int)ceil_div(group, 16)};
    float* scores = reinterpret_cast<float*>(static_cast<char*>(workspace) + plan.parts);
    // Rows that one workgroup has are weighed by it, in the one launch (us, two launches / one: a sequence of 700 tokens, 24 heads of 64 10.8 / 8.5; 29 of up to
    // 500, 32 heads 31.4 / 28.6, of up to 4000 190 / 194; 40 of up to 2000, 64 heads over 8 58 / 53).
    const bool alone = plan.splits.n == 1 && a.column_tiles == 1;
    const SingleMore more{{}, 0, 0, scores, alone ? weights : nullptr, stride};
    const hipError_t e = for_head_size(kv.D, [&](auto c, auto v, auto exact) {
        const dim3 grid((unsigned)((int64_t)kv.B * kv.kv_heads * a.column_tiles), parts.splits);
        if (f32) attention_decode_rows<c.value, v.value, exact.value, true, 4, Single::Scored><<<grid, 256, 0, stream>>>(a, parts, kv, more);
        else attention_decode_rows<c.value, v.value, exact.value, false, 4, Single::Scored><<<grid, 256, 0, stream>>>(a, parts, kv, more);
        return hipGetLastError();
    });
    if (e != hipSuccess || alone) return e;
    const int chunks = (int)ceil_div((int64_t)kv.max_blocks * kKvBlock, kChunk), joins = parts.splits > 1 ? (int)rows : 0;
    const int64_t tasks = (int64_t)kv.B * kv.kv_heads * chunks;
    const WeightsArgs w{scores, weights, stride, tasks, by, heads, group, chunks, joins};
    const unsigned blocks = (unsigned)(joins + (tasks < kMostBlocks ? tasks : kMostBlocks));
    if (f32) attention_weights_of_tokens<true><<<blocks, 256, 0, stream>>>(o, w, parts, kv);
    else attention_weights_of_tokens<false><<<blocks, 256, 0, stream>>>(o, w, parts, kv);
    return hipGetLastError();
}

hipError_t launch_attention_prefill_weights(const void* q, const KvView& kv, int64_t T, int heads, float scale, void* o, bool f32, float* weights, int64_t stride,
                                            void* workspace, size_t workspace_bytes, hipStream_t stream) {
    const RunsPlan plan = runs_plan(kv, T, heads);
    char* at = static_cast<char*>(workspace);
    KeptRows keep;
    keep.state = reinterpret_cast<float*>(at);
    const hipError_t e = launch_attention_prefill_kept(q, kv, T, heads, scale, o, f32, keep, at + plan.states + plan.parts, workspace_bytes - plan.states - plan.parts, stream);
    if (e != hipSuccess) return e;
    return for_head_size(kv.D, [&](auto c, auto, auto exact) {
        const int group = heads / kv.kv_heads;
        const ColumnsPlan p = columns_plan<c.value>(kv, T, group);
        int shift = 0;
        while ((1 << shift) < group) ++shift;
        const ColumnArgs a{static_cast<const uint16_t*>(q), keep.state, weights, reinterpret_cast<float*>(at + plan.states), stride, p.tasks, scale * 1.44269504f,
                           heads, group, (int)T, (uint32_t)p.shares, (uint32_t)p.most, kLeastStages, (uint32_t)((((uint64_t)1 << 32) * (((uint64_t)1 << shift) - group)) / group + 1), (uint32_t)shift};
        const unsigned blocks = (unsigned)(p.tasks < kMostBlocks ? p.tasks : kMostBlocks);
        attention_weights_of_runs<c.value, exact.value><<<blocks, 256, 0, stream>>>(a, kv);
        const hipError_t ran = hipGetLastError();
        if (ran != hipSuccess || p.bytes == 0) return ran;
        ColumnArgs join = a;
        join.tasks = (int64_t)kv.B * kv.kv_heads * p.shares;             // at most 1024
        attention_weights_join<c.value><<<(unsigned)join.tasks, Columns<c.value>::kKeys, 0, stream>>>(join, kv);
        return hipGetLastError();
    });
}

}  // namespace bitnet
