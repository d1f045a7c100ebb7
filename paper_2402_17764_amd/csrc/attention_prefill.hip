// Which launch shape the attention of runs of new tokens takes.
#include "attention_prefill_kernel.hpp"

namespace bitnet {

#define EXTERN(kC_, kV_, kE_) extern template hipError_t launch_prefill<kC_, kV_, kE_>(PrefillTile, const PrefillArgs&, const Parts&, const KvView&, bool, hipStream_t)
EXTERN(1, 2, true); EXTERN(2, 4, true); EXTERN(3, 6, true); EXTERN(4, 8, true); EXTERN(6, 12, true); EXTERN(8, 16, true);
EXTERN(1, 1, false); EXTERN(2, 3, false); EXTERN(3, 5, false); EXTERN(4, 7, false);
EXTERN(1, 2, false); EXTERN(2, 4, false); EXTERN(3, 6, false); EXTERN(4, 8, false); EXTERN(6, 12, false); EXTERN(8, 16, false);
#undef EXTERN

struct PrefillPlan { PrefillTile tile; int splits, least; };

// Tiles of 128 rows where there are two for each CU even so and the sequences have rows to fill them -- four for each CU if what a tile
// walks grows along the sequence, as in a prompt from its beginning, because the longest tile then ends last; what counts for that is
// how much more the page tables hold than the call's own tokens.  (us, 64 / 128 rows: 32 heads, 2048 tokens 49 / 56, 4096 tokens
// 162 / 141; 64 heads over 8, 1024 tokens 30 / 32, 2048 tokens 84 / 77, 1024 tokens behind 15000 539 / 466; 32 heads, sixteen prompts of
// 100 to 400 42 / 45.)
// Rows are shared by several workgroups where there are not two for each CU and sequences can have 1024 tokens, until there are two
// (16 tokens behind 8000, 32 heads: 136 us, shared by eight 32, by sixteen 32; 128 tokens behind 32000, 64 heads over 8: 506, by four 196).
static PrefillPlan prefill_plan(const KvView& kv, int64_t T, int heads) {
    const int group = heads / kv.kv_heads;
    const int64_t capacity = (int64_t)kv.max_blocks * kKvBlock, rows_a_sequence = T * group / kv.B;
    const int64_t large = tiles_at_most(T, kv.B, group, 128, 1) * kv.kv_heads;
    const bool behind_others = capacity >= 4 * (T / kv.B);
    if (rows_a_sequence >= 1024 && large >= (behind_others ? 512 : 1024)) return {PrefillTile::Rows128, 1, 1};
    const int64_t small = tiles_at_most(T, kv.B, group, 64, 1) * kv.kv_heads, n = capacity >= 1024 ? 512 / small : 1;
    constexpr int kLeast = 4;                              // times 64 tokens
    int64_t most = ceil_div(capacity, kLeast * kStageTokens);
    most = most < kMostSplits ? most : kMostSplits;
    return {PrefillTile::Rows64, (int)(n < 2 ? 1 : n < most ? n : most), kLeast};
}

size_t attention_prefill_workspace_bytes(const KvView& kv, int64_t T, int heads) {
    return Parts::bytes(T * heads, prefill_plan(kv, T, heads).splits, kv.D);
}

hipError_t launch_attention_prefill(const void* q, const KvView& kv, int64_t T, int heads, float scale, void* o, bool f32, void* workspace,
                                    size_t workspace_bytes, hipStream_t stream) {
    const float by = scale * 1.44269504f;
    const PrefillArgs a{static_cast<const uint16_t*>(q), o, by, fminf(kSlack / by, 3e38f), heads, heads / kv.kv_heads, (int)T, 0};
    const PrefillPlan plan = prefill_plan(kv, T, heads);
    Parts parts;
    if (plan.splits > 1 && workspace_bytes >= Parts::bytes(T * heads, plan.splits, kv.D)) parts = Parts(workspace, T * heads, plan.splits, plan.least, kv.D);
    const int chunks = (int)ceil_div(kv.D, 32);
    const bool exact = kv.D % 32 == 0, one_tile = !exact && kv.D % 32 <= 16;
    hipError_t e = hipErrorInvalidValue;
#define PREFILL(kC_, kV_, kE_) e = launch_prefill<kC_, kV_, kE_>(plan.tile, a, parts, kv, f32, stream)
#define SIZES(kC_) if (exact) PREFILL(kC_, 2 * kC_, true); else if (one_tile) PREFILL(kC_, 2 * kC_ - 1, false); else PREFILL(kC_, 2 * kC_, false); break
    switch (chunks) {
        case 1: SIZES(1);
        case 2: SIZES(2);
        case 3: SIZES(3);
        case 4: SIZES(4);
        case 5: case 6: if (exact && chunks == 6) PREFILL(6, 12, true); else PREFILL(6, 12, false); break;
        default: if (exact && chunks == 8) PREFILL(8, 16, true); else PREFILL(8, 16, false); break;
    }
#undef SIZES
#undef PREFILL
    if (e != hipSuccess || parts.splits < 2) return e;
    return launch_attention_join({o, a.scale, heads, a.group, (int)T, prefill_rows(plan.tile)}, parts, kv, f32, stream);
}

}  // namespace bitnet
