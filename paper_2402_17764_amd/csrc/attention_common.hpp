// What the two attention kernels share: operand fragments, the softmax's running state across lane groups, partial results and their join.
#pragma once
#include "bitnet_device.hpp"
#include "bitnet_internal.hpp"
#include "kv_layout.hpp"

namespace bitnet {

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef unsigned v4u __attribute__((ext_vector_type(4)));

constexpr float kMinusInf = -__builtin_inff();

__device__ inline v4f mfma_bf16(v8bf a, v8bf b, v4f c) {
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
#else
    return c;
#endif
}

// The reduction over the four lane groups of 16 that share a query; every lane gets the result.
__device__ inline float groups_max(float v) {
#if defined(__HIP_DEVICE_COMPILE__)
    auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
#endif
    return v;
}
__device__ inline float groups_sum(float v) {
#if defined(__HIP_DEVICE_COMPILE__)
    auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(b[0]) + __uint_as_float(b[1]);
#endif
    return v;
}

__device__ inline float exp2_fast(float x) {
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_exp2f(x);              // one unit in the last place; -inf gives 0, results below 2^-126 are 0
#else
    return x;
#endif
}

// A query row's operand: dims 32 c + 8 g ... + 7 (zeros behind the head's end, so that what lies behind the keys' dims counts
// for nothing).  `row` NULL: no such query.
template <int kC>
__device__ inline void load_query(v8bf (&f)[kC], const uint16_t* row, int g, int D) {
#pragma unroll
    for (int c = 0; c < kC; ++c) {
        const int d0 = 32 * c + 8 * g;
        uint16_t u[8] = {};
        if (row) {
            if (d0 + 8 <= D) __builtin_memcpy(u, row + d0, 16);
            else
#pragma unroll
                for (int i = 0; i < 7; ++i) if (d0 + i < D) u[i] = row[d0 + i];
        }
        __builtin_memcpy(&f[c], u, 16);
    }
}

// Eight weights as an operand.  bf16 keeps 8 bits of each: the sums of products then carry a relative error of about 2^-9 / sqrt(keys), which
// a bf16 result hides.  For a 32-bit result what that rounding left over goes through the product as a second operand.
__device__ inline v8bf weights_operand(const float (&p)[8]) {
    v8bf w;
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = (__bf16)p[i];
    return w;
}
__device__ inline v8bf weights_rest(const float (&p)[8], v8bf w) {
    v8bf r;
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = (__bf16)(p[i] - (float)w[i]);
    return r;
}

// Which of a lane's eight consecutive values of a dim belong to a token in front of `count`: the others are whatever the memory
// held, and a weight of zero does not make a NaN nothing.
__device__ inline void values_keep(v4u& v, int count) {
#pragma unroll
    for (int w = 0; w < 4; ++w) v[w] &= count >= 2 * w + 2 ? 0xFFFFFFFFu : count == 2 * w + 1 ? 0x0000FFFFu : 0u;
}

// four consecutive outputs of a row of D, from dim d on
template <bool kF32>
__device__ inline void store4(void* o, int64_t at, int d, int D, const float (&x)[4]) {
    if (kF32) {
        float* p = static_cast<float*>(o) + at + d;
        if (d + 4 <= D) __builtin_memcpy(p, x, 16);
        else
#pragma unroll
            for (int i = 0; i < 3; ++i) if (d + i < D) p[i] = x[i];
    } else {
        uint16_t* p = static_cast<uint16_t*>(o) + at + d;
        uint16_t u[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] = f32_to_bf16(x[i]);
        if (d + 4 <= D) __builtin_memcpy(p, u, 8);
        else
#pragma unroll
            for (int i = 0; i < 3; ++i) if (d + i < D) p[i] = u[i];
    }
}

}  // namespace bitnet
