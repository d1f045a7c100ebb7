// Attention of one new token of each sequence where runs of sequences have their first tokens in common:
//   o_b = softmax(scale q_b [K_shared | K_b]) [V_shared | V_b].
// The shared tokens are gone through once for all rows of a group (its sequences' query heads of one key-value head), in tiles of rows as for
// runs of tokens; the tokens that a sequence has to itself by other workgroups of the same launch, or of another one as for single tokens.  All leave
// parts of the rows, m, l and sums over the values, which the last launch joins: softmax over two sets of keys is the sum of theirs, weighted by exp(m_s - m).
#include "attention_decode_kernel.hpp"
#include "attention_join.hpp"
#include "attention_prefill_kernel.hpp"

namespace bitnet {

#define EXTERN(kC_, kV_, kE_) \
    extern template hipError_t launch_prefill_shared<kC_, kV_, kE_>(PrefillTile, const PrefillArgs&, const Parts&, const KvView&, bool, const RowsMore&, hipStream_t);
BITNET_PREFILL_SIZES(EXTERN)
#undef EXTERN

namespace {

// How a row's keys are split: `near` of the shared tokens, `far` of its own.
struct SharedPlan {
    bool apart;                        // two launches
    PrefillTile tile;                  // of rows over the shared tokens
    int64_t near_tiles, far_tiles;     // of all groups, and of one sequence
    int near, least_near, far, least_far;
};
// Groups of up to 128 rows (of a key-value head, on average) take one launch for both: a few rows leave its matrix instructions to spare, and what counts
// are launches (us, one launch / two: 13 sequences behind 1500 tokens, 32 heads 20.1 / 25.5; 6 behind 8000, 64 heads over 8 22.5 / 24.7; 16 behind 16000
// 37.2 / 38.7, 20 45.2 / 40.5; 30 behind 16000, 28 over 4 42.5 / 41.0; 48 behind 24000, 64 over 8 135 / 115).  Two launches, and 256 rows: tiles of 128, which halve what comes
// through LDS (the last one 110; 30 behind 16000, which has 210, 44.8).  The shared keys are split until there are two workgroups for each CU, a sequence's own until there
// are four or five, with 256 tokens each or more (48 behind 24000, own ones in a workgroup each: 46 us for them, split 39; shared ones to three workgroups a CU 116 instead of 110).
SharedPlan shared_plan(const KvView& kv, int groups, int heads, bool f32) {
    const int group = heads / kv.kv_heads;
    const int64_t capacity = (int64_t)kv.max_blocks * kKvBlock, rows = ceil_div((int64_t)kv.B * group, groups), most = ceil_div(capacity, 256);
    SharedPlan p;
    p.apart = rows > 128;
    p.tile = rows >= 256 && kv.D <= 128 && !f32 ? PrefillTile::Rows128 : PrefillTile::Rows64;
    p.near_tiles = tiles_at_most(kv.B, groups, group, prefill_rows(p.tile), 1);
    p.far_tiles = ceil_div(group, p.apart ? 16 : 64);
    auto splits = [&](int64_t workgroups, int64_t fill) {
        const int64_t n = fill / workgroups < most ? fill / workgroups : most;
        return (int)(n < 1 ? 1 : n > kMostSplits / 2 ? kMostSplits / 2 : n);
    };
    p.near = splits(p.near_tiles * kv.kv_heads, 512);
    p.far = splits((int64_t)kv.B * kv.kv_heads * p.far_tiles, p.apart ? 1280 : 1024);
    p.least_near = 256 / kStageTokens;
    p.least_far = 256 / (p.apart ? kKvBlock : kStageTokens);
    return p;
}

// One row to a wave: its splits' weights stand in the lanes, 64 at a time, and each half of the wave (each wave, of heads of more than 128 dims) takes
// every other split's sums, four dims a lane.
template <bool kF32>
__global__ __launch_bounds__(256) void attention_join_shared(void* o, float scale, int heads, int64_t rows, Parts parts, SharedLaunch l, KvView kv) {
    __shared__ float weights[4][kMostSplits];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), D = kv.D;
    const int64_t row = (int64_t)blockIdx.x * 4 + wave;
    if (row >= rows) return;
    const int b = (int)(row / heads);
    const int len = kv.length(kv.kv_len[b]), shared = shared_tokens(kv, l.prefixes, b, len);
    int n1 = 0;
    if (shared > 0) {                                      // of the group's, as the workgroups that wrote them found it
        const SharedRows r(kv, l.prefixes, sequence_of_tile(l.prefixes.start, l.prefixes.groups, b, 1, 1, 0));
        const int stages = stages_of(r.len), run = max((stages + l.near - 1) / l.near, l.least_near);
        n1 = (stages + run - 1) / run;
    }
    const int own = own_units(len, shared, l.far_unit), run = max((own + l.far - 1) / l.far, l.least_far), n = n1 + (own + run - 1) / run;
    auto place = [&](int s) { return row * parts.splits + (s < n1 ? s : l.near + (s - n1)); };
    float m[4], sum[4], top = kMinusInf;                     // of splits lane, lane + 64, ... (up to 256)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        m[i] = kMinusInf, sum[i] = 0.0f;
        if (lane + 64 * i < n) {
            const float2 x = *reinterpret_cast<const float2*>(parts.state + 2 * place(lane + 64 * i));
            m[i] = x.x, sum[i] = x.y;
        }
        top = fmaxf(top, m[i]);
    }
    top = wave_max(top);
    float total = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        m[i] = m[i] == kMinusInf ? 0.0f : exp2_fast((m[i] - top) * scale);       // now the split's weight; of one that saw no token: 0
        total += sum[i] * m[i];
    }
    total = wave_sum(total);
#pragma unroll
    for (int i = 0; i < 4; ++i) weights[wave][lane + 64 * i] = m[i];          // read by this wave alone
    const bool halves = D <= 128;
    const int dim = 4 * (halves ? lane & 31 : lane), half = halves ? lane >> 5 : 0, by = halves ? 2 : 1;
    v4f x = {0, 0, 0, 0};
    for (int s0 = half; s0 - half < n; s0 += 8 * by) {
        v4f y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {                      // behind the last one the last one, times zero
            const float* p = parts.sums + place(min(s0 + e * by, n - 1)) * D + dim;
            y[e] = (v4f){0, 0, 0, 0};
            if (dim + 4 <= D) __builtin_memcpy(&y[e], p, 16);
            else if (dim < D) { y[e][0] = p[0]; y[e][1] = p[1]; }            // heads have an even number of dims
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) x += y[e] * (s0 + e * by < n ? weights[wave][s0 + e * by] : 0.0f);
    }
    if (halves)
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] += __shfl_xor(x[e], 32);
    if (dim >= D || (halves && lane >= 32)) return;
    const float inv = total > 0.0f ? 1.0f / total : 0.0f;
    const float y[4] = {finite_or_nan(x[0], inv), finite_or_nan(x[1], inv), finite_or_nan(x[2], inv), finite_or_nan(x[3], inv)};
    store4<kF32>(o, row * D, dim, D, y);
}

size_t shared_bytes(const SharedPlan& p, const KvView& kv, int heads) {
    return ((size_t)((int64_t)kv.B * heads * (p.near + p.far)) * (kv.D + 2) * 4 + 15) / 16 * 16;
}

}  // namespace

size_t attention_shared_workspace_bytes(const KvView& kv, int groups, int heads, bool f32) { return shared_bytes(shared_plan(kv, groups, heads, f32), kv, heads); }

hipError_t launch_attention_shared(const void* q, const KvView& kv, const int32_t* prefix_start, const int32_t* prefix_len, int groups, int heads, float scale,
                                   void* o, bool f32, void* workspace, hipStream_t stream) {
    const int group = heads / kv.kv_heads;
    const float by = scale * 1.44269504f;
    const SharedPlan plan = shared_plan(kv, groups, heads, f32);
    const int64_t rows = (int64_t)kv.B * heads;
    const Parts parts(workspace, rows, plan.near + plan.far, 1, kv.D);
    const uint64_t near = (uint64_t)(plan.near_tiles * plan.near), far = plan.apart ? 0 : (uint64_t)(kv.B * plan.far_tiles * plan.far);
    const SharedLaunch l{{prefix_start, prefix_len, groups}, (uint32_t)near, (uint32_t)far, (uint32_t)(((far << 32) + near + far - 1) / (near + far)), plan.near, plan.far,
                         plan.least_near, plan.least_far, (int)plan.far_tiles, plan.apart ? kKvBlock : kStageTokens};
    const PrefillArgs a{static_cast<const uint16_t*>(q), nullptr, by, fminf(kSlack / by, 3e38f), heads, group, 0, (int)plan.near_tiles};
    hipError_t e = for_head_size(kv.D, [&](auto c, auto v, auto exact) {
        return launch_prefill_shared<c.value, v.value, exact.value>(plan.tile, a, parts, kv, f32, RowsMore{{}, l}, stream);
    });
    if (e != hipSuccess) return e;
    if (plan.apart) {
        const DecodeArgs da{a.q, nullptr, by, heads, group, (int)plan.far_tiles};
        const SingleMore more{l.prefixes, plan.near, plan.near + plan.far, nullptr, nullptr, 0};
        Parts own = parts;
        own.splits = plan.far;
        own.least = plan.least_far;
        e = for_head_size(kv.D, [&](auto c, auto v, auto exact) {
            const dim3 grid((unsigned)((int64_t)kv.B * kv.kv_heads * da.column_tiles), own.splits);
            if (f32) attention_decode_rows<c.value, v.value, exact.value, true, 4, Single::Own><<<grid, 256, 0, stream>>>(da, own, kv, more);
            else attention_decode_rows<c.value, v.value, exact.value, false, 4, Single::Own><<<grid, 256, 0, stream>>>(da, own, kv, more);
            return hipGetLastError();
        });
        if (e != hipSuccess) return e;
    }
    const unsigned blocks = (unsigned)ceil_div(rows, 4);
    if (f32) attention_join_shared<true><<<blocks, 256, 0, stream>>>(o, by, heads, rows, parts, l, kv);
    else attention_join_shared<false><<<blocks, 256, 0, stream>>>(o, by, heads, rows, parts, l, kv);
    return hipGetLastError();
}

}  // namespace bitnet
