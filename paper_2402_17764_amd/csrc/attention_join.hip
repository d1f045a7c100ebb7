// The second launch of attention whose rows were shared by several workgroups: one query head of one row to a workgroup.
#include "attention_common.hpp"

namespace bitnet {
namespace {

__device__ inline float wave_max(float v) {
    v = fmaxf(v, dpp_f32<0xB1>(v));
    v = fmaxf(v, dpp_f32<0x4E>(v));
    v = fmaxf(v, dpp_f32<0x141>(v));
    v = fmaxf(v, dpp_f32<0x140>(v));
    return groups_max(v);
}
__device__ inline float wave_sum(float v) {
    v += dpp_f32<0xB1>(v);
    v += dpp_f32<0x4E>(v);
    v += dpp_f32<0x141>(v);
    v += dpp_f32<0x140>(v);
    return groups_sum(v);
}

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

template <bool kF32>
__global__ __launch_bounds__(256) void attention_join(JoinArgs a, Parts parts, KvView kv) {
    __shared__ float weights[kMostSplits], totals[4], tops[4];
    __shared__ v4f sums[4][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), D = kv.D, dim = 4 * lane;
    const int t = blockIdx.x / a.heads, head = blockIdx.x - t * a.heads;
    const int64_t place0 = (int64_t)blockIdx.x * parts.splits;
    auto sums_of = [&](int s) {
        v4f y = {0, 0, 0, 0};
        const float* p = parts.sums + (place0 + s) * D + dim;
        if (dim + 4 <= D) __builtin_memcpy(&y, p, 16);
        else if (dim < D) { y[0] = p[0]; y[1] = p[1]; }     // heads have an even number of dims
        return y;
    };
    const int n = splits_of(a, parts, kv, t, head);
    if (n < 2) return;                                      // stored by the workgroup that had all of it
    float m = kMinusInf, l = 0.0f;                          // one split a thread: its weight, exp(m_s - m), and its share of l
    if ((int)threadIdx.x < n) {
        m = parts.state[(place0 + threadIdx.x) * 2];
        l = parts.state[(place0 + threadIdx.x) * 2 + 1];
    }
    float top = wave_max(m);
    if (lane == 0) tops[wave] = top;
    __syncthreads();
    top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
    const float w = m == kMinusInf ? 0.0f : exp2_fast((m - top) * a.scale);      // of a split that saw no token: 0
    weights[threadIdx.x] = w;
    l = wave_sum(l * w);
    if (lane == 0) totals[wave] = l;
    __syncthreads();
    v4f x = {0, 0, 0, 0};
#pragma unroll 4
    for (int s = wave; s < n; s += 4) x += sums_of(s) * weights[s];
    sums[wave][lane] = x;
    __syncthreads();
    if (wave != 0 || dim >= D) return;
    x = (sums[0][lane] + sums[1][lane]) + (sums[2][lane] + sums[3][lane]);
    const float total = (totals[0] + totals[1]) + (totals[2] + totals[3]), inv = total > 0.0f ? 1.0f / total : 0.0f;
    const float y[4] = {finite_or_nan(x[0], inv), finite_or_nan(x[1], inv), finite_or_nan(x[2], inv), finite_or_nan(x[3], inv)};
    store4<kF32>(a.o, (int64_t)blockIdx.x * D, dim, D, y);
}

}  // namespace

hipError_t launch_attention_join(const JoinArgs& a, const Parts& parts, const KvView& kv, bool f32, hipStream_t stream) {
    const unsigned rows = (unsigned)((int64_t)a.T * a.heads);
    if (f32) attention_join<true><<<rows, 256, 0, stream>>>(a, parts, kv);
    else attention_join<false><<<rows, 256, 0, stream>>>(a, parts, kv);
    return hipGetLastError();
}

}  // namespace bitnet
