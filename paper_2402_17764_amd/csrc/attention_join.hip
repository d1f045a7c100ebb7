// The second launch of attention whose rows were shared by several workgroups: one query head of one row to a workgroup.
#include "attention_join.hpp"

#include <type_traits>

namespace bitnet {
namespace {

// how many splits of a row have been written: as the workgroups that wrote them found it
__device__ inline int splits_of(const JoinArgs& a, const Parts& parts, const KvView& kv, int t, int head) {
    int units;
    if (a.rows_a_tile == 0) {
        units = blocks_of(kv, t);
    } else {
        const int b = sequence_of_tile(kv.q_start, kv.B, t, 1, 1, 0);
        const NewTokens nt(kv, b, a.T);
        if (t < nt.first || t >= nt.first + nt.n) return 0;
        const int row = (t - nt.first) * a.group + head % a.group;
        const int behind = (row / a.rows_a_tile + 1) * a.rows_a_tile;
        units = stages_of(tile_sees(nt, min(behind, nt.n * a.group) - 1, a.group));
    }
    const int run = parts.run(units);
    return (units + run - 1) / run;
}

template <bool kF32, bool kKeep>
__global__ __launch_bounds__(256) void attention_join(JoinArgs a, Parts parts, KvView kv, std::conditional_t<kKeep, KeptRows, char> keep) {
    __shared__ JoinRoom room;
    const int t = blockIdx.x / a.heads, head = blockIdx.x - t * a.heads;
    const int n = splits_of(a, parts, kv, t, head);
    if (n < 2) return;                                      // stored by the workgroup that had all of it
    if constexpr (kKeep) {
        const JoinState all = join_row<kF32>(room, parts, (int64_t)blockIdx.x * parts.splits, n, a.scale, kv.D, a.o, blockIdx.x);
        if (threadIdx.x == 0) {
            keep.state[2 * (int64_t)blockIdx.x] = all.top;
            keep.state[2 * (int64_t)blockIdx.x + 1] = all.total;
        }
    } else {
        join_row<kF32>(room, parts, (int64_t)blockIdx.x * parts.splits, n, a.scale, kv.D, a.o, blockIdx.x);
    }
}

}  // namespace

hipError_t launch_attention_join(const JoinArgs& a, const Parts& parts, const KvView& kv, bool f32, hipStream_t stream, const KeptRows& keep) {
    const unsigned rows = (unsigned)((int64_t)a.T * a.heads);
    if (f32 && keep.state) attention_join<true, true><<<rows, 256, 0, stream>>>(a, parts, kv, keep);
    else if (f32) attention_join<true, false><<<rows, 256, 0, stream>>>(a, parts, kv, 0);
    else if (keep.state) attention_join<false, true><<<rows, 256, 0, stream>>>(a, parts, kv, keep);
    else attention_join<false, false><<<rows, 256, 0, stream>>>(a, parts, kv, 0);
    return hipGetLastError();
}

}  // namespace bitnet
