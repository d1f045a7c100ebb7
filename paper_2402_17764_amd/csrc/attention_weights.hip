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

// Joins the rows that several workgroups shared, one to a workgroup, then turns chunks of scores into weights, four tokens a thread.
template <bool kF32>
__global__ __launch_bounds__(256) void attention_weights_of_tokens(void* o, WeightsArgs a, Parts parts, KvView kv) {
    __shared__ JoinRoom room;
    __shared__ float base[64], inv[64];
    if ((int)blockIdx.x < a.joins) {
        const int b = blockIdx.x / a.heads, blocks = blocks_of(kv, b), run = parts.run(blocks), n = (blocks + run - 1) / run;
        if (n < 2) return;                                  // stored by the workgroup that had all of it
        join_row<kF32>(room, parts, (int64_t)blockIdx.x * parts.splits, n, n, 0, a.scale, kv.D, o, blockIdx.x);
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
    int64_t stride, tasks;             // of the weights: sequences times kv heads times tiles of keys
    float scale;
    int heads, group, T, tiles;
};

// A workgroup takes a tile of keys of one sequence and key-value head, 32 kKB for each of its four waves, in registers, and goes through the rows that
// see any of them, 16 at a time: scores are products of keys (down) and queries (across), so that a lane sums up eight tokens for its
// queries, and the 16 lanes of a group meet at the end.
template <int kC, bool kExact, int kKB>
__global__ __launch_bounds__(256, 2) void attention_weights_of_runs(ColumnArgs a, KvView kv) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int D = kExact ? 32 * kC : kv.D, Dp = kv_padded_dim(D), quads = Dp >> 3;
    for (int64_t task = blockIdx.x; task < a.tasks; task += gridDim.x) {
        // heads side by side, so that with a multiple of eight of them a head's tiles meet on one XCD, whose L2 holds its queries
        const int h = (int)(task % kv.kv_heads);
        const int64_t rest = task / kv.kv_heads;
        const int tile = (int)(rest % a.tiles), b = (int)(rest / a.tiles);
        const NewTokens nt(kv, b, a.T);
        const int len = kv.length(kv.kv_len[b]), blocks = (len + kKvBlock - 1) / kKvBlock, blk = (tile * 4 + wave) * kKB, j0 = blk * kKvBlock;
        if (nt.n == 0 || blk >= blocks) continue;
        v8bf k[kKB][kC][2];
        bool known[kKB];
#pragma unroll
        for (int u = 0; u < kKB; ++u) {
            const int number = blk + u < blocks ? kv.block(kv.table + b * kv.table_stride, blk + u, h) : -1;
            known[u] = number >= 0;
            const char* from = reinterpret_cast<const char*>(kv.k) + (int64_t)max(number, 0) * kKvBlock * Dp * 2;
#pragma unroll
            for (int c = 0; c < kC; ++c)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const int off = (kExact || c < whole_chunks(kC) ? 4 * c + g : min(4 * c + g, quads - 1)) * 512 + r * 16 + 256 * t;
                    k[u][c][t] = __builtin_bit_cast(v8bf, *reinterpret_cast<const v4u*>(from + off));
                }
        }
        float acc[kKB][8] = {};
        const int rows = nt.n * a.group, tok0 = max(j0 - nt.pos0, 0);
        for (int R0 = tok0 * a.group / 16 * 16; R0 < rows; R0 += 16) {
            const int R = R0 + r, tok = token_of(R, a.group), row = R < rows ? (nt.first + tok) * a.heads + h * a.group + R - tok * a.group : -1;
            const int pos = row >= 0 ? nt.pos0 + tok : -1;
            v8bf qf[kC];
            load_query<kC, kExact>(qf, row >= 0 ? a.q + (int64_t)row * D : nullptr, g, D);
            float m = kMinusInf, l = 0.0f;
            if (row >= 0) {
                m = a.state[2 * (int64_t)row];
                l = a.state[2 * (int64_t)row + 1];
            }
            settle_query<kC, kExact>(qf, g, D);
            const float base = m == kMinusInf ? 0.0f : m * a.scale, inv = l > 0.0f ? 1.0f / l : 0.0f;
            v4f s[kKB][2] = {};
#pragma unroll
            for (int u = 0; u < kKB; ++u)
#pragma unroll
                for (int c = 0; c < kC; ++c)
#pragma unroll
                    for (int t = 0; t < 2; ++t) s[u][t] = mfma_bf16(k[u][c][t], qf[c], s[u][t]);
#pragma unroll
            for (int u = 0; u < kKB; ++u)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float p = exp2_fast(__builtin_fmaf(s[u][j >> 2][j & 3], a.scale, -base));
                    if (known[u] && j0 + u * kKvBlock + 8 * g + j <= pos) acc[u][j] = __builtin_fmaf(p, inv, acc[u][j]);
                }
        }
#pragma unroll
        for (int u = 0; u < kKB; ++u)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float v = acc[u][j];
                v += dpp_f32<0xB1>(v);
                v += dpp_f32<0x4E>(v);
                v += dpp_f32<0x141>(v);
                v += dpp_f32<0x140>(v);
                const int at = j0 + u * kKvBlock + 8 * g + j;
                if (r == j && at < len) {
                    float* to = a.weights + ((int64_t)b * kv.kv_heads + h) * a.stride + at;
                    *to = (at >= nt.pos0 ? 0.0f : *to) + v;           // the call's own tokens begin with nothing
                }
            }
    }
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

size_t attention_weights_workspace_bytes(const KvView& kv, int64_t T, int heads, bool prefill, bool f32) {
    if (prefill) return ((size_t)(T * heads) * 8 + 15) / 16 * 16 + attention_prefill_kept_bytes(kv, T, heads, f32);
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
    const SingleMore more{{}, 0, 0, scores};
    const hipError_t e = for_head_size(kv.D, [&](auto c, auto v, auto exact) {
        const dim3 grid((unsigned)((int64_t)kv.B * kv.kv_heads * a.column_tiles), parts.splits);
        if (f32) attention_decode_rows<c.value, v.value, exact.value, true, 4, Single::Scored><<<grid, 256, 0, stream>>>(a, parts, kv, more);
        else attention_decode_rows<c.value, v.value, exact.value, false, 4, Single::Scored><<<grid, 256, 0, stream>>>(a, parts, kv, more);
        return hipGetLastError();
    });
    if (e != hipSuccess) return e;
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
    const size_t states = ((size_t)(T * heads) * 8 + 15) / 16 * 16;
    KeptRows keep;
    keep.state = static_cast<float*>(workspace);
    const hipError_t e = launch_attention_prefill_kept(q, kv, T, heads, scale, o, f32, keep, static_cast<char*>(workspace) + states, workspace_bytes - states, stream);
    if (e != hipSuccess) return e;
    return for_head_size(kv.D, [&](auto c, auto, auto exact) {
        constexpr int kKB = c.value <= 4 ? 2 : 1;
        const int tiles = (int)ceil_div(kv.max_blocks, 4 * kKB);
        const int64_t tasks = (int64_t)kv.B * kv.kv_heads * tiles;
        const ColumnArgs a{static_cast<const uint16_t*>(q), keep.state, weights, stride, tasks, scale * 1.44269504f, heads, heads / kv.kv_heads, (int)T, tiles};
        attention_weights_of_runs<c.value, exact.value, kKB><<<(unsigned)(tasks < kMostBlocks ? tasks : kMostBlocks), 256, 0, stream>>>(a, kv);
        return hipGetLastError();
    });
}

}  // namespace bitnet
