// How the splits of a row come together: one query head of one row to a workgroup of 256 threads.
#pragma once
#include "attention_common.hpp"

namespace bitnet {

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

// LDS of a workgroup that joins a row
struct JoinRoom {
    float weights[kMostSplits], totals[4], tops[4];
    v4f sums[4][64];
};
struct JoinState { float top, total; };                    // m and l of the row

// Joins the `n` splits of row `row`, which stand at places place0, place0 + 1, ...
template <bool kF32>
__device__ inline JoinState join_row(JoinRoom& room, const Parts& parts, int64_t place0, int n, float scale, int D, void* o, int64_t row) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), dim = 4 * lane;
    auto sums_of = [&](int s) {
        v4f y = {0, 0, 0, 0};
        const float* p = parts.sums + (place0 + s) * D + dim;
        if (dim + 4 <= D) __builtin_memcpy(&y, p, 16);
        else if (dim < D) { y[0] = p[0]; y[1] = p[1]; }     // heads have an even number of dims
        return y;
    };
    float m = kMinusInf, l = 0.0f;                          // one split a thread: its weight, exp(m_s - m), and its share of l
    if ((int)threadIdx.x < n) {
        m = parts.state[(place0 + threadIdx.x) * 2];
        l = parts.state[(place0 + threadIdx.x) * 2 + 1];
    }
    float top = wave_max(m);
    if (lane == 0) room.tops[wave] = top;
    __syncthreads();
    top = fmaxf(fmaxf(room.tops[0], room.tops[1]), fmaxf(room.tops[2], room.tops[3]));
    const float w = m == kMinusInf ? 0.0f : exp2_fast((m - top) * scale);      // of a split that saw no token: 0
    room.weights[threadIdx.x] = w;
    l = wave_sum(l * w);
    if (lane == 0) room.totals[wave] = l;
    __syncthreads();
    v4f x = {0, 0, 0, 0};
#pragma unroll 4
    for (int s = wave; s < n; s += 4) x += sums_of(s) * room.weights[s];
    room.sums[wave][lane] = x;
    __syncthreads();
    const float total = (room.totals[0] + room.totals[1]) + (room.totals[2] + room.totals[3]);
    if (wave != 0 || dim >= D) return {top, total};
    x = (room.sums[0][lane] + room.sums[1][lane]) + (room.sums[2][lane] + room.sums[3][lane]);
    const float inv = total > 0.0f ? 1.0f / total : 0.0f;
    const float y[4] = {finite_or_nan(x[0], inv), finite_or_nan(x[1], inv), finite_or_nan(x[2], inv), finite_or_nan(x[3], inv)};
    store4<kF32>(o, row * D, dim, D, y);
    return {top, total};
}

}  // namespace bitnet
