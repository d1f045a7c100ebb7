// What the two attention kernels share: operand fragments, the softmax's running state across lane groups, partial results and their join.
#pragma once
#include "bitnet_device.hpp"
#include "bitnet_internal.hpp"
#include "kv_layout.hpp"

#include <type_traits>

namespace bitnet {

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef unsigned v4u __attribute__((ext_vector_type(4)));

// The sizes of heads that the kernels are built for: kC chunks of 32 dims for the scores, kV tiles of 16 for the values.  Exact: all of them are
// whole.  Otherwise whole_chunks(kC) are, those behind may be filled in part, and up to 128 dims the last chunk has one tile or two.
constexpr int whole_chunks(int kC) { return kC <= 4 ? kC - 1 : kC - 2; }

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
// for nothing -- once settle_query is through).  `row` NULL: no such query.
template <int kC, bool kExact>
__device__ inline void load_query(v8bf (&f)[kC], const uint16_t* row, int g, int D) {
#pragma unroll
    for (int c = 0; c < kC; ++c) {
        const int d0 = 32 * c + 8 * g;
        v4u w = {0, 0, 0, 0};
        if (row) {
            if (kExact || c < whole_chunks(kC)) {
                __builtin_memcpy(&w, row + d0, 16);
            } else if (kC > 1 || D >= 8) {                 // the last eight dims: one load, whatever is left
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
        }
        f[c] = __builtin_bit_cast(v8bf, w);
    }
}

// The last dims that load_query read, to their places.  A call of its own, as it waits for them: other loads go out in between (one prompt
// of 64 tokens and 32 heads of 126: 0.5 us).
template <int kC, bool kExact>
__device__ inline void settle_query(v8bf (&f)[kC], int g, int D) {
    if (kExact || (kC == 1 && D < 8)) return;
#pragma unroll
    for (int c = whole_chunks(kC); c < kC; ++c) {
        const int over = max(32 * c + 8 * g + 8 - D, 0) >> 1;
        v4u w = __builtin_bit_cast(v4u, f[c]);
        if (over & 1) w = (v4u){w[1], w[2], w[3], 0};
        if (over & 2) w = (v4u){w[2], w[3], 0, 0};
        if (over >= 4) w = (v4u){0, 0, 0, 0};
        f[c] = __builtin_bit_cast(v8bf, w);
    }
}

// Weights as operands, the pair j, j + 1 of eight, in kParts bf16 each: what the rounding of one leaves goes through the product too.  One keeps 8
// bits of a weight, which puts an error of the size of a bf16 result's own rounding on it; two leave 2^-17 of a weight, which such a
// result hides; three hold all 24 bits, for a 32-bit result (measured 1.3e-6 of the result with two, 2e-7 with three).  What they
// cost is a product of values each: of single tokens, which wait for memory, next to nothing (us, one / two / three: 29 sequences of up to 4096
// tokens, 32 heads of 128 160 / 164 / 162, 64 heads over 8, 20000 to 49000 tokens 73.6 / 74.2 / 74.5, 1000 tokens 8.4 / 8.6 / 8.8), of
// runs a quarter of the time or more (40 heads of 128, 2048 tokens 57 / 73, 64 heads over 8, 1024 behind 15000 445 / 666).  So
// decode takes two for a bf16 result and prefill one, and both take three for fp32.  Over shared prefixes, and where weights of tokens are added up, whose
// state of a row is that of weights as they are, runs take two as well (one would be 98 us instead of 111 for 48 sequences behind 24000 tokens, 101 instead of 113
// for a prompt of 2048 tokens, 40 heads).
template <int kParts>
__device__ inline void weights_pair(v8bf* w, int j, float p0, float p1) {
#pragma unroll
    for (int e = 0; e < kParts; ++e) {
        w[e][j] = (__bf16)p0;
        w[e][j + 1] = (__bf16)p1;
        p0 -= (float)w[e][j];
        p1 -= (float)w[e][j + 1];
    }
}

// The sum of a row's weights takes them as the values' product does, rounded, so that the rounding of a weight that outweighs the
// others is in both and goes out of their quotient: values that are all alike come back as they are.  The decode kernel does it as a product with
// ones, which every lane of a query's four groups gets, in all four places.  The prefill kernel, whose tiles of 128 rows have not the ten
// registers for that, adds a lane's weights two at a time (the weights as they were before the rounding: results off by another half step;
// us, those / these: 40 heads of 128, 2048 tokens 58.1 / 57.2, 64 heads over 8, 1024 behind 15000 463 / 445, 32 heads, 4096 tokens 138 / 142, of 64 dims 92 / 95).
__device__ inline v8bf ones_operand() {
    v8bf w;
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = (__bf16)1.0f;
    return w;
}

// l + w[j] + w[j + 1], in 32 bits
__device__ inline float add_rounded(float l, const v8bf& w, int j) {
#if defined(__HIP_DEVICE_COMPILE__)
    typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
    return __builtin_amdgcn_fdot2_f32_bf16((v2bf){w[j], w[j + 1]}, (v2bf){(__bf16)1.0f, (__bf16)1.0f}, l, false);
#else
    return l;
#endif
}

// Which of a lane's eight consecutive values of a dim belong to a token in front of `count`: the others are whatever the memory
// held, and a weight of zero does not make a NaN nothing.
__device__ inline void values_keep(v4u& v, int count) {
#pragma unroll
    for (int w = 0; w < 4; ++w) v[w] &= count >= 2 * w + 2 ? 0xFFFFFFFFu : count == 2 * w + 1 ? 0x0000FFFFu : 0u;
}

// ... and which of them do not: the first `count`, which are read elsewhere
__device__ inline void values_drop(v4u& v, int count) {
#pragma unroll
    for (int w = 0; w < 4; ++w) v[w] &= count >= 2 * w + 2 ? 0u : count == 2 * w + 1 ? 0xFFFF0000u : 0xFFFFFFFFu;
}

// A sum over values times `by`: NaN where the sum is an infinity.  An infinite value that a row sees meets weights of zero and factors of zero (0 inf) in some
// tiles, splits and types and in others not, and what is noted of it where a tile ends (prefill) is NaN: so all of them say NaN.
__device__ inline float finite_or_nan(float sum, float by) { return __builtin_fmaf(sum, 0.0f, sum * by); }

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

// ---- parts ------------------------------------------------------------------------------------------------------------------------
// Where few rows meet long sequences, several workgroups share a row's keys.  Each leaves its sums over the values and its m and l (all
// 32 bits) in the workspace, split s of row `row` (row of q times heads, plus head) at place row * splits + s, and a second launch joins them:
//   m = max m_s,  o = sum_s exp(m_s - m) sums_s / sum_s exp(m_s - m) l_s.
struct Parts {
    float* sums;                       // [rows][splits][D]
    float* state;                      // [rows][splits][2]: m, l
    int splits, least;                 // workgroups for a row, and blocks (of 32 tokens, or stages of 64) that one has at least
    Parts() : sums(nullptr), state(nullptr), splits(1), least(1) {}
    Parts(void* workspace, int64_t rows, int splits_, int least_, int D)
        : sums(static_cast<float*>(workspace)), state(sums + rows * splits_ * D), splits(splits_), least(least_) {}
    static size_t bytes(int64_t rows, int splits, int D) { return splits < 2 ? 0 : ((size_t)(rows * splits) * (D + 2) * 4 + 15) / 16 * 16; }
    __device__ int run(int units) const { const int n = (units + splits - 1) / splits; return n < least ? least : n; }
};
constexpr int kMostSplits = 256;       // of a row: one to a thread of the join

// Joins the splits of each row; `rows_a_tile` 0: rows of single tokens, dealt out by blocks; otherwise the prefill kernel's tile.
struct JoinArgs {
    void* o;
    float scale;                       // of the softmax, times log2 e
    int heads, group, T, rows_a_tile;
};
// Where rows leave their softmax states, m and l.
struct KeptRows {
    float* state = nullptr;            // [rows][2]
};
hipError_t launch_attention_join(const JoinArgs& a, const Parts& parts, const KvView& kv, bool f32, hipStream_t stream, const KeptRows& keep = KeptRows());

// The prefill kernel's tile of a sequence's rows for one head: the keys that its last token sees, and how many 64 tokens of them (the unit in
// which they are shared out).
constexpr int kStageTokens = 64;
__device__ inline int token_of(int row, int group) { return (int)((unsigned)row / (unsigned)group); }
__device__ inline int tile_sees(const NewTokens& nt, int row_last, int group) { return nt.pos0 + token_of(row_last, group) + 1; }
__device__ inline int stages_of(int seen) { return seen > 0 ? (seen + kStageTokens - 1) / kStageTokens : 0; }

// `unit` tokens at a time, those that hold some of a sequence's own, behind `shared` ones: the first, and how many
__device__ inline int own_first(int shared, int unit) { return shared / unit; }
__device__ inline int own_units(int len, int shared, int unit) { return shared >= len ? 0 : (len + unit - 1) / unit - own_first(shared, unit); }

__device__ inline int blocks_of(const KvView& kv, int b) { return (kv.length(kv.kv_len[b]) + kKvBlock - 1) / kKvBlock; }

// The kernel for a head's size: `go` is called with the sizes that it is built for, kC chunks of 32 dims and kV tiles of 16, as types
template <typename Go>
hipError_t for_head_size(int D, Go go) {
    const int chunks = (D + 31) / 32;
    const bool exact = D % 32 == 0, one_tile = D % 32 != 0 && D % 32 <= 16;
#define SIZE(kC_, kV_, kE_) return go(std::integral_constant<int, kC_>(), std::integral_constant<int, kV_>(), std::integral_constant<bool, kE_>())
    switch (chunks) {
        case 1: if (exact) SIZE(1, 2, true); if (one_tile) SIZE(1, 1, false); SIZE(1, 2, false);
        case 2: if (exact) SIZE(2, 4, true); if (one_tile) SIZE(2, 3, false); SIZE(2, 4, false);
        case 3: if (exact) SIZE(3, 6, true); if (one_tile) SIZE(3, 5, false); SIZE(3, 6, false);
        case 4: if (exact) SIZE(4, 8, true); if (one_tile) SIZE(4, 7, false); SIZE(4, 8, false);
        case 5: case 6: if (exact && chunks == 6) SIZE(6, 12, true); SIZE(6, 12, false);
        default: if (exact && chunks == 8) SIZE(8, 16, true); SIZE(8, 16, false);
    }
#undef SIZE
}

}  // namespace bitnet
