// Rows of heads (one head of one token, D elements) as the norm and rotation kernels hold them: D / 16 consecutive lanes share a
// row, every lane with two units of eight consecutive elements, chosen so that whatever the rotation mixes stands in one lane.
#pragma once
#include "gfwa_device.h"
#include <type_traits>

namespace gfwa {

// Eight consecutive elements as they travel from and to memory.
template <typename T>
struct Unit8;
template <>
struct Unit8<bf16_t> {
    bf16x8 v;
    __device__ __forceinline__ void load(const bf16_t* p) { v = *reinterpret_cast<const bf16x8*>(p); }
    __device__ __forceinline__ void store(bf16_t* p) const { *reinterpret_cast<bf16x8*>(p) = v; }
    __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = (float)v[e];
    }
    __device__ __forceinline__ void set(const float (&x)[8]) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (bf16_t)x[e];
    }
};
template <>
struct Unit8<float> {
    f32x4 a, b;
    __device__ __forceinline__ void load(const float* p) {
        a = reinterpret_cast<const f32x4*>(p)[0];
        b = reinterpret_cast<const f32x4*>(p)[1];
    }
    __device__ __forceinline__ void store(float* p) const {
        reinterpret_cast<f32x4*>(p)[0] = a;
        reinterpret_cast<f32x4*>(p)[1] = b;
    }
    __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = e < 4 ? a[e] : b[e - 4];
    }
    __device__ __forceinline__ void set(const float (&x)[8]) {
        a = f32x4{x[0], x[1], x[2], x[3]};
        b = f32x4{x[4], x[5], x[6], x[7]};
    }
};

// Which elements of a row lane j (of D / 16) holds, and the rotation of them.
//   rotation of (m, m + rot/2): the first rot / 16 lanes hold the units at 8 j and rot/2 + 8 j, the others two neighbouring units
//   behind the rotated part;  rotation of (2m, 2m + 1): the units at 8 j and D/2 + 8 j, each rotated if it stands in front of rot.
// Either way a lane has at most eight angles.
template <int D>
struct LaneOfRow {
    static constexpr int LPR = D / 16;  // lanes of a row
    int a, b;                           // first elements of the two units
    int m;                              // first frequency of unit a's angles (and of unit b's four, paired)
    int mb;
    bool turn_a, turn_b;
    __device__ __forceinline__ LaneOfRow(int j, int rot, bool paired) {
        if (paired) {
            a = 8 * j;
            b = D / 2 + 8 * j;
            m = a / 2;
            mb = b / 2;
            turn_a = a < rot;
            turn_b = b < rot;
        } else {
            turn_a = turn_b = 16 * j < rot;
            a = turn_a ? 8 * j : 16 * j;
            b = turn_a ? rot / 2 + 8 * j : 16 * j + 8;
            m = 8 * j;
            mb = m + 4;
        }
    }
};

// cos and sin of p * freq.  The angle in half turns, fp64, is brought into one turn before it becomes fp32: to 2^-25 half turns,
// wherever p stands, plus the fp64 product's own rounding (2^-53 of the whole angle).
__device__ __forceinline__ void cos_sin_of(int p, double freq, float& c, float& s) {
    constexpr double kInvPi = 0.31830988618379067154;
    double t = (double)p * (freq * kInvPi);
    t = fma(-2.0, rint(0.5 * t), t);
    sincospif((float)t, &s, &c);
}

// The eight angles of a lane at position p.
struct Angles {
    float c[8], s[8];
    template <int D>
    __device__ __forceinline__ void at(const LaneOfRow<D>& l, int p, const double* freq) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const bool turn = e < 4 ? l.turn_a : l.turn_b;
            c[e] = 1.f;
            s[e] = 0.f;
            if (turn) cos_sin_of(p, freq[e < 4 ? l.m + e : l.mb + e - 4], c[e], s[e]);
        }
    }
    // The two units of a row turned by the angles (BACK: by their negatives).  Elements that are not rotated are left alone, not multiplied by
    // one and zero: an infinity next to them stays where it is.
    template <int D, bool BACK>
    __device__ __forceinline__ void turn(const LaneOfRow<D>& l, bool paired, float (&x)[8], float (&y)[8]) const {
        if (paired) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                pair<BACK>(l.turn_a, c[e], s[e], x[2 * e], x[2 * e + 1]);
                pair<BACK>(l.turn_b, c[4 + e], s[4 + e], y[2 * e], y[2 * e + 1]);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) pair<BACK>(l.turn_a, c[e], s[e], x[e], y[e]);
        }
    }

private:
    template <bool BACK>
    static __device__ __forceinline__ void pair(bool turn, float c, float s, float& x, float& y) {
        const float q = BACK ? -s : s;
        const float u = fmaf(x, c, -(y * q)), v = fmaf(x, q, y * c);
        x = turn ? u : x;
        y = turn ? v : y;
    }
};

// Sum over the LPR (8 or 4) consecutive lanes of a row, the same bits in all of them: DPP exchanges inside rows of 16 lanes.
template <int LPR>
__device__ __forceinline__ float sum_over_row(float x) {
    static_assert(LPR == 8 || LPR == 4, "eight or four lanes to a row");
    auto from = [](float v, auto ctrl) __attribute__((always_inline)) {
        return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), decltype(ctrl)::value, 0xF, 0xF, true));
    };
    x += from(x, std::integral_constant<int, (1 | 0 << 2 | 3 << 4 | 2 << 6)>{});  // lane ^ 1
    x += from(x, std::integral_constant<int, (2 | 3 << 2 | 0 << 4 | 1 << 6)>{});  // lane ^ 2
    if (LPR == 8) x += from(x, std::integral_constant<int, 0x141>{});             // half-row mirror: 7 - lane, the other quad
    return x;
}

// 1 / sqrt(mean(x^2) + eps) of the row whose two units this lane holds in x and y.
template <int D>
__device__ __forceinline__ float row_rstd(const float (&x)[8], const float (&y)[8], float eps) {
    float ss = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = fmaf(x[e], x[e], fmaf(y[e], y[e], ss));
    const float mean = sum_over_row<D / 16>(ss) * (1.f / D) + eps;
    return 1.f / sqrtf(mean);
}

// A lane's sixteen weights of the norm, ones where there are none.
struct LaneWeights {
    float a[8], b[8];
    template <int D>
    __device__ __forceinline__ void load(const float* w, const LaneOfRow<D>& l) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            a[e] = w != nullptr ? w[l.a + e] : 1.f;
            b[e] = w != nullptr ? w[l.b + e] : 1.f;
        }
    }
};

}  // namespace gfwa
