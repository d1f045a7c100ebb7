// Attention of one new token of each sequence where runs of sequences have their first tokens in common:
//   o_b = softmax(scale q_b [K_shared | K_b]) [V_shared | V_b].
// The shared tokens are gone through once for all rows of a group (its sequences' query heads of one key-value head), in tiles of rows as for
// runs of tokens; the tokens that a sequence has to itself as for single tokens.  Both leave parts of the rows, m, l and sums over the values,
// which a third launch joins: softmax over two sets of keys is the sum of theirs, weighted by exp(m_s - m).
#include "attention_decode_kernel.hpp"
#include "attention_join.hpp"
#include "attention_prefill_kernel.hpp"

namespace bitnet {

#define EXTERN(kC_, kV_, kE_) \
    extern template hipError_t launch_prefill_shared<kC_, kV_, kE_>(PrefillTile, const PrefillArgs&, const Parts&, const KvView&, bool, const RowsMore&, hipStream_t);
BITNET_PREFILL_SIZES(EXTERN)
#undef EXTERN

namespace {

// How a row's shares are split: `near` of the shared tokens, `far` of its own.
struct SharedPlan {
    PrefillTile tile;
    int near, least_near, far, least_far;
};
SharedPlan shared_plan(const KvView& kv, int groups, int heads) {
    const int group = heads / kv.kv_heads;
    const int64_t capacity = (int64_t)kv.max_blocks * kKvBlock;
    const int64_t tiles = tiles_at_most(kv.B, groups, group, 64, 1) * kv.kv_heads;
    constexpr int kLeast = 4;                              // times 64 tokens
    const int64_t most = ceil_div(capacity, kLeast * kStageTokens), fill = 512 / tiles, n = fill < most ? fill : most;
    const Splits own = decode_splits(kv, heads);
    return {PrefillTile::Rows64, (int)(n < 1 ? 1 : n > kMostSplits / 2 ? kMostSplits / 2 : n), kLeast, own.n > kMostSplits / 2 ? kMostSplits / 2 : own.n, own.least};
}

template <bool kF32>
__global__ __launch_bounds__(256) void attention_join_shared(void* o, float scale, int heads, Parts near, Parts far, KvView kv, Prefixes prefixes) {
    __shared__ JoinRoom room;
    const int b = blockIdx.x / heads, pitch = near.splits + far.splits;
    const int len = kv.length(kv.kv_len[b]), shared = shared_tokens(kv, prefixes, b, len);
    int n1 = 0;
    if (shared > 0) {                                      // of the group's, as the workgroups that wrote them found it
        const SharedRows r(kv, prefixes, sequence_of_tile(prefixes.start, prefixes.groups, b, 1, 1, 0));
        const int stages = stages_of(r.len), run = near.run(stages);
        n1 = (stages + run - 1) / run;
    }
    const int own = own_blocks(len, shared), run = far.run(own), n2 = (own + run - 1) / run;
    join_row<kF32>(room, near, (int64_t)blockIdx.x * pitch, n1 + n2, n1, near.splits, scale, kv.D, o, blockIdx.x);
}

size_t shared_bytes(const SharedPlan& p, const KvView& kv, int heads) {
    return ((size_t)((int64_t)kv.B * heads * (p.near + p.far)) * (kv.D + 2) * 4 + 15) / 16 * 16;
}

}  // namespace

size_t attention_shared_workspace_bytes(const KvView& kv, int groups, int heads) { return shared_bytes(shared_plan(kv, groups, heads), kv, heads); }

hipError_t launch_attention_shared(const void* q, const KvView& kv, const int32_t* prefix_start, const int32_t* prefix_len, int groups, int heads, float scale,
                                   void* o, bool f32, void* workspace, hipStream_t stream) {
    const int group = heads / kv.kv_heads;
    const float by = scale * 1.44269504f;
    const SharedPlan plan = shared_plan(kv, groups, heads);
    const Prefixes prefixes{prefix_start, prefix_len, groups};
    const int64_t rows = (int64_t)kv.B * heads;
    // one array of parts of both kinds, near.splits + far.splits to a row
    Parts near(workspace, rows, plan.near + plan.far, plan.least_near, kv.D), far = near;
    near.splits = plan.near;
    far.splits = plan.far;
    far.least = plan.least_far;
    const PrefillArgs pa{static_cast<const uint16_t*>(q), nullptr, by, fminf(kSlack / by, 3e38f), heads, group, 0, 0};
    const DecodeArgs da{static_cast<const uint16_t*>(q), nullptr, by, heads, group, (int)ceil_div(group, 16)};
    const RowsMore rows_more{{}, prefixes, plan.near + plan.far};
    const SingleMore single_more{prefixes, plan.near, plan.near + plan.far, nullptr};
    hipError_t e = for_head_size(kv.D, [&](auto c, auto v, auto exact) {
        return launch_prefill_shared<c.value, v.value, exact.value>(plan.tile, pa, near, kv, f32, rows_more, stream);
    });
    if (e != hipSuccess) return e;
    e = for_head_size(kv.D, [&](auto c, auto v, auto exact) {
        const dim3 grid((unsigned)((int64_t)kv.B * kv.kv_heads * da.column_tiles), far.splits);
        if (f32) attention_decode_rows<c.value, v.value, exact.value, true, 4, Single::Own><<<grid, 256, 0, stream>>>(da, far, kv, single_more);
        else attention_decode_rows<c.value, v.value, exact.value, false, 4, Single::Own><<<grid, 256, 0, stream>>>(da, far, kv, single_more);
        return hipGetLastError();
    });
    if (e != hipSuccess) return e;
    if (f32) attention_join_shared<true><<<(unsigned)rows, 256, 0, stream>>>(o, by, heads, near, far, kv, prefixes);
    else attention_join_shared<false><<<(unsigned)rows, 256, 0, stream>>>(o, by, heads, near, far, kv, prefixes);
    return hipGetLastError();
}

}  // namespace bitnet
