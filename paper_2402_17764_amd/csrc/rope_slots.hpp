// What the kernels that turn queries and keys by their positions share: sines and cosines, slots of eight dims with their partners.
#pragma once
#include "bitnet_device.hpp"
#include "bitnet_internal.hpp"
#include "kv_layout.hpp"

#include <type_traits>

namespace bitnet {

struct RopeShape {
    int heads, rotary, T;              // query heads; dims that are turned, the first ones of a head
    int pairs;                         // 0: dim i with i + rotary / 2; 1: 2 i with 2 i + 1
};

struct Turn { float cos, sin; };

// cos and sin of pos * freq.  The fraction of a turn is taken in 64 bits and brought to within an eighth of the nearest quarter;
// there the Taylor polynomials of degree 9 and 8 are within 2^-25 (their next terms, (pi / 4)^11 / 11! and (pi / 4)^10 / 10!, are below 2.5e-8),
// and the quarter says which of the two is which and with what sign.
__device__ inline Turn turn_of(double pos, float freq) {
    double t = pos * ((double)freq * 0.15915494309189533577);
    t -= rint(t);
    const double k = rint(4.0 * t);                        // -2 ... 2
    const float x = (float)(t - 0.25 * k) * 6.28318530718f, z = x * x;
    float s = __builtin_fmaf(z, 1.0f / 362880.0f, -1.0f / 5040.0f), c = __builtin_fmaf(z, 1.0f / 40320.0f, -1.0f / 720.0f);
    s = __builtin_fmaf(z, s, 1.0f / 120.0f);
    c = __builtin_fmaf(z, c, 1.0f / 24.0f);
    s = __builtin_fmaf(z, s, -1.0f / 6.0f);
    c = __builtin_fmaf(z, c, -0.5f);
    s = __builtin_fmaf(x * z, s, x);
    c = __builtin_fmaf(z, c, 1.0f);
    const int q = (int)k;
    const float a = q & 1 ? s : c, b = q & 1 ? c : s;      // of quarter 1: cos -> -sin, sin -> cos
    return {(q + 1) & 2 ? -a : a, q & 2 ? -b : b};
}

// Eight consecutive elements as they stand in memory, from an address of any alignment; `count` of them exist (the others are zero).
template <bool kBf16> struct Eight { uint4 w[kBf16 ? 1 : 2]; };
template <bool kBf16>
__device__ inline Eight<kBf16> load8(const void* base, int64_t at, int count) {
    using E = std::conditional_t<kBf16, uint16_t, uint32_t>;
    const E* p = static_cast<const E*>(base) + at;
    E u[8] = {};
    if (count >= 8) __builtin_memcpy(u, p, sizeof u);
    else
#pragma unroll
        for (int i = 0; i < 7; ++i) if (i < count) u[i] = p[i];
    Eight<kBf16> r;
    __builtin_memcpy(&r, u, sizeof u);
    return r;
}
template <bool kBf16>
__device__ inline void floats_of(float (&x)[8], const Eight<kBf16>& r) {
    if constexpr (kBf16) {
        const uint32_t w[4] = {r.w[0].x, r.w[0].y, r.w[0].z, r.w[0].w};
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(i & 1 ? w[i >> 1] & 0xFFFF0000u : w[i >> 1] << 16);
    } else {
        __builtin_memcpy(x, &r, sizeof x);
    }
}

__device__ inline uint4 pack8(const float (&x)[8]) {
    typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
    v8bf w;
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = (__bf16)x[i];       // to the nearest, ties to even
    return __builtin_bit_cast(uint4, w);
}

// A slot: dims d0 ... d0 + 7 of a head with what they are turned with, requested before any of it is used.  Split and Odd: slots of the lower
// half are turned together with their partners, whose slots there are none of; Odd is for halves that are no multiple of eight
// (of a half's last slot some dims may be the other half's and are not used).  Any: slots of all dims, each turned alone; such
// as cross the middle have partners in both directions.  Reads may reach behind a head, to the row's end and not further.
enum class Turned { Split, Odd, Pairs, Any };
template <bool kBf16, Turned kTurned>
struct Slot {
    static constexpr bool kTogether = kTurned == Turned::Split || kTurned == Turned::Odd;
    Eight<kBf16> own, low, high;       // low: partners of the dims of the lower half; Split, Odd: those alone
    // head: the head's first element among all, left: elements from there to the row's end
    __device__ void load(const void* base, int64_t head, int64_t left, int d0, int D, bool turned, const RopeShape& s) {
        own = load8<kBf16>(base, head + d0, kTurned == Turned::Odd || kTurned == Turned::Pairs ? (int)min(left - d0, (int64_t)8) : D - d0);
        const int half = s.rotary >> 1;
        if (kTogether) {
            if (d0 < half) low = load8<kBf16>(base, head + d0 + half, kTurned == Turned::Odd ? (int)min(left - d0 - half, (int64_t)8) : 8);
        } else if (kTurned == Turned::Any && turned && d0 < s.rotary) {
            if (d0 < half) low = load8<kBf16>(base, head + d0 + half, (int)min(left - d0 - half, (int64_t)8));
            if (d0 + 8 > half) {
                // in front of the tensor there is nothing: eight elements from its first one on, moved up
                const int64_t at = head + d0 - half;
                high = load8<kBf16>(base, at < 0 ? 0 : at, (int)min(head + left - (at < 0 ? 0 : at), (int64_t)8));
                if (at < 0) {
                    using E = std::conditional_t<kBf16, uint16_t, uint32_t>;
                    E u[8], v[8];
                    __builtin_memcpy(u, &high, sizeof u);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        v[i] = 0;
#pragma unroll
                        for (int k = 0; k < 8; ++k) if (i + at == k) v[i] = u[k];
                    }
                    __builtin_memcpy(&high, v, sizeof v);
                }
            }
        }
    }
    // x: own dims turned; y (Split, Odd): the partners, turned
    __device__ void turn(float (&x)[8], float (&y)[8], int d0, bool turned, const Turn (&t)[8], const RopeShape& s) const {
        floats_of<kBf16>(x, own);
        const int half = s.rotary >> 1;
        if (kTogether) {
            if (d0 < half) floats_of<kBf16>(y, low);
            if (!turned || d0 >= half) return;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float a = x[e] * t[e].cos - y[e] * t[e].sin;
                y[e] = y[e] * t[e].cos + x[e] * t[e].sin;
                x[e] = a;
            }
            return;
        }
        if (!turned || d0 >= s.rotary) return;
        if (kTurned == Turned::Pairs) {
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                if (d0 + e >= s.rotary) continue;
                const float a = x[e] * t[e].cos - x[e + 1] * t[e].sin;
                x[e + 1] = x[e + 1] * t[e].cos + x[e] * t[e].sin;
                x[e] = a;
            }
            return;
        }
        float l[8], h[8];
        floats_of<kBf16>(l, low);
        floats_of<kBf16>(h, high);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (d0 + e < s.rotary) x[e] = x[e] * t[e].cos + (d0 + e < half ? -l[e] : h[e]) * t[e].sin;
    }
};

__device__ inline int pair_of(int d, const RopeShape& s) { return s.pairs ? d >> 1 : d < (s.rotary >> 1) ? d : d - (s.rotary >> 1); }

// A head's last dims, `count` even: what stands behind them cleared, or left out.  (A last slot that is read past its head and written in one or
// two pieces, as against element by element: 4096 tokens, 32 heads of 100, pairs 55 -> 48 us.)
__device__ inline uint4 first_of(uint4 w, int count) { return {w.x, count > 2 ? w.y : 0, count > 4 ? w.z : 0, count > 6 ? w.w : 0}; }
__device__ inline void store_any(uint16_t* p, uint4 w, int count) {
    if (count >= 8) { __builtin_memcpy(p, &w, 16); return; }
    if (count & 4) __builtin_memcpy(p, &w, 8);
    const uint32_t two = count & 4 ? w.z : w.x;
    if (count & 2) __builtin_memcpy(p + (count & 4), &two, 4);
}

// The slots of a head: those of the lower half, and those of the dims that are not turned; or all.
template <Turned kTurned>
constexpr int slots_of(int D, const RopeShape& s) {
    if (kTurned == Turned::Pairs || kTurned == Turned::Any) return (D + 7) / 8;
    return (s.rotary / 2 + 7) / 8 + (D - s.rotary + 7) / 8;
}

}  // namespace bitnet
