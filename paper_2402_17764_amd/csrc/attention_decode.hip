// Attention of single tokens, each row's blocks in one workgroup or shared by several.
#include "attention_decode_kernel.hpp"

namespace bitnet {
namespace {

template <int kC, int kV, bool kExact>
hipError_t launch_decode(const DecodeArgs& a, const Parts& parts, const KvView& kv, bool f32, hipStream_t stream) {
    const dim3 grid((unsigned)((int64_t)kv.B * kv.kv_heads * a.column_tiles), parts.splits);
    if (f32) attention_decode_rows<kC, kV, kExact, true, 4, Single::All><<<grid, 256, 0, stream>>>(a, parts, kv, 0);
    else attention_decode_rows<kC, kV, kExact, false, 4, Single::All><<<grid, 256, 0, stream>>>(a, parts, kv, 0);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || parts.splits < 2) return e;
    return launch_attention_join({a.o, a.scale, a.heads, a.group, kv.B, 0}, parts, kv, f32, stream);
}

}  // namespace

// How many workgroups share a row at most, by the length that the page tables have room for.  A CU draws 25 to 45 bytes a cycle,
// whatever number of waves asks, and a second launch costs 4 us in a chain of launches: so rows are shared where there are fewer
// than 256 and more than 1023 tokens (one token, 32 heads of 128, a key-value head each, 1000 tokens: 13.4 us in one launch, 10.0 shared;
// 64 heads over 8, 500 tokens 7.5 / 9.5, 1000 tokens 9.4 / 9.4), until there are as many as the CUs hold at a time: two each (three
// sequences of 23000 to 41000 tokens, 64 heads over 8: 512 workgroups 74.7 us, 1024 79.1, 2048 79.2, none shared 359), of heads of more than 128
// dims, whose registers leave room for one, one each (one sequence of 32000 tokens, 32 heads of 160 over 8, 256 / 512 workgroups 35.0 /
// 42.4, of 256 dims 47.3 / 53.4; three of 3000, 16 heads of 160 21.9 / 26.8).  More rows are shared only at every 8192 tokens,
// so that one long sequence among short ones is not what the call waits for.
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
    return for_head_size(kv.D, [&](auto c, auto v, auto exact) { return launch_decode<c.value, v.value, exact.value>(a, parts, kv, f32, stream); });
}

}  // namespace bitnet
