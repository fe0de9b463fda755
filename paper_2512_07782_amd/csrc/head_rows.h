// Rows of heads (one head of one token, D elements) as the norm and rotation kernels hold them: D / 16 consecutive lanes share a
// row, every lane with two units of eight consecutive elements, chosen so that whatever the rotation mixes stands in one lane.
#pragma once
#include "gfwa_device.h"
#include "gfwa_internal.h"
#include <type_traits>

namespace gfwa {

// Eight consecutive elements as they travel from and to memory.
template <typename T>
struct Unit8;
template <>
struct Unit8<bf16_t> {
    bf16x8 v;
    template <bool ONCE = false>
    __device__ __forceinline__ void load(const bf16_t* p) {
        const bf16x8* const from = reinterpret_cast<const bf16x8*>(p);
        if constexpr (ONCE) v = __builtin_nontemporal_load(from);
        else v = *from;
    }
    template <bool PAST = false>
    __device__ __forceinline__ void store(bf16_t* p) const {
        bf16x8* const to = reinterpret_cast<bf16x8*>(p);
        if constexpr (PAST) __builtin_nontemporal_store(v, to);
        else *to = v;
    }
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
    template <bool ONCE = false>
    __device__ __forceinline__ void load(const float* p) {
        a = reinterpret_cast<const f32x4*>(p)[0];
        b = reinterpret_cast<const f32x4*>(p)[1];
    }
    template <bool PAST = false>
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
//   rotation of (m, m + rot/2): the first rot / 16 lanes hold the units at 8 j and rot/2 + 8 j, the others those at the same place in the two
//   halves of what lies behind the rotated part, rot/2 + 8 j and D/2 + 8 j;  rotation of (2m, 2m + 1): the units at 8 j and D/2 + 8 j, each rotated if it stands in front of rot.
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
            a = turn_a ? 8 * j : 8 * j + rot / 2;
            b = turn_a ? rot / 2 + 8 * j : 8 * j + D / 2;
            m = 8 * j;
            mb = m + 4;
        }
    }
};

// cos and sin of p * freq.  The angle in half turns, fp64, is brought into one turn before it becomes fp32: to 2^-25 half turns,
// wherever p stands, plus what three roundings in fp64 (1/pi, freq / pi and its product with p) leave of the whole angle, 3 * 2^-53 of it.
__device__ __forceinline__ void cos_sin_of(double p, double freq, float& c, float& s) {
    constexpr double kInvPi = 0.31830988618379067154;
    double t = p * (freq * kInvPi);
    t = fma(-2.0, rint(0.5 * t), t);
    sincospif((float)t, &s, &c);
}

// A lane's eight frequencies.
struct Frequencies {
    double x[8];
    template <int D>
    __device__ __forceinline__ void load(const LaneOfRow<D>& l, const double* freq) {
        typedef double f64x2 __attribute__((ext_vector_type(2), aligned(8)));
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            f64x2 v = {0.0, 0.0};
            if (e < 4 ? l.turn_a : l.turn_b) v = *reinterpret_cast<const f64x2*>(freq + (e < 4 ? l.m + e : l.mb + e - 4));
            x[e] = v[0];
            x[e + 1] = v[1];
        }
    }
};

// The eight angles of a lane at position p (a whole number; new tokens of a cache may stand past 2^31).
struct Angles {
    float c[8], s[8];
    template <int D>
    __device__ __forceinline__ void at(const LaneOfRow<D>& l, double p, const Frequencies& f) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const bool turn = e < 4 ? l.turn_a : l.turn_b;
            c[e] = 1.f;
            s[e] = 0.f;
            if (turn) cos_sin_of(p, f.x[e], c[e], s[e]);
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

// A lane's sixteen values of a vector of D: weights of the norm, ones where there are none.
template <int D>
struct LaneVector {
    float a[8], b[8];
    __device__ __forceinline__ void load(const float* w, const LaneOfRow<D>& l) {
        typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
#pragma unroll
        for (int e = 0; e < 8; e += 4) {
            f32x4_any x = {1.f, 1.f, 1.f, 1.f}, y = x;
            if (w != nullptr) {
                x = *reinterpret_cast<const f32x4_any*>(w + l.a + e);
                y = *reinterpret_cast<const f32x4_any*>(w + l.b + e);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                a[e + i] = x[i];
                b[e + i] = y[i];
            }
        }
    }
};

// The two units of a lane's row.
// ONCE: loaded past the caches (bf16, where a load takes whole lines).  Large inputs are read faster (us, through / past the caches: forward of H 32, Hkv 8,
// d 128, N 4096, 50 MB, 21.2 / 20.4, of B 4, H 16, Hkv 4, N 4096, d 64 22.5 / 21.8, append of 16 prompts 103.6 / 96.4, backward of H 32, Hkv 8, N 16384
// 120.5 / 118.0), those that are small enough to be held from their making more slowly (forward of N 2600, 32 MB, 13.1 / 14.9; backward of H 16, Hkv 4,
// N 4100, 25 MB, 18.8 / 21.5).
// Forward and append count what they read (through / past the caches: append without queries, H 32, Hkv 8, d 128, 8100 tokens, 33 MB, 15.1 / 19.0,
// forward without values, H 16, Hkv 16, N 4100, 34 MB, 14.7 / 16.7).
constexpr long long kOnceBytes = 40 << 20;  // inputs of more than this are loaded past the caches: the L2s hold 32 MiB
template <typename T, int D, bool ONCE = false, bool PAIR = true>
struct LaneRow {
    static constexpr bool kPair = sizeof(T) == 2 && D == 64 && PAIR;
    Unit8<T> a, b;
    // row(s): the row of the lanes with the same place in their rows and side s.
    // kPair: rows of 128 bytes, of which a load of one unit by a row's four lanes takes half a line.  So the rows of sides 2 i and 2 i + 1 are loaded and stored
    // one after the other, each by the lanes of both, unit a by the even side's and b by the odd one's, and arrive() gives every lane its own row's (us, halves /
    // whole lines: forward of B 4, H 16, Hkv 4, d 64, N 4200 30.9 / 23.8, of H 32, Hkv 4, N 16384 37.8 / 31.2, gradients of N 4200 42.2 / 37.3, append of 40000
    // tokens 65.8 / 58.8; N 2048, 25 MB, forward 11.5 / 12.0).  PAIR false: not worth it, for the derivative's inputs through the caches.
    template <typename Row>
    __device__ __forceinline__ void load(Row&& row, int side, const LaneOfRow<D>& l) {
        if constexpr (kPair) {
            const int at = l.a + (side & 1) * (l.b - l.a);
            a.template load<ONCE>(row(side & ~1) + at);
            b.template load<ONCE>(row(side | 1) + at);
        } else {
            const T* const own = row(side);
            a.template load<ONCE>(own + l.a);
            b.template load<ONCE>(own + l.b);
        }
    }
    __device__ __forceinline__ void arrive() {
        if constexpr (kPair) exchange();
    }
    // PAST: stored past the caches, for what nothing reads soon.  (The cache's new rows: 16 prompts 105.7 -> 95.9 us.  The results of norm and rotation would
    // cost less themselves, us, H 32, Hkv 8, N 16384: forward 77.9 -> 74.0, backward 119 -> 116, and the kernel that reads them right after more: rope
    // and attention in a row (w 1024) 217 -> 225, at B 4, H 16, Hkv 4, N 4096, d 64 (w 512) 75.6 -> 76.4, the backward and a matrix product with its result
    // 419 -> 423.)
    // there(s): whether side s's row is to be written.  Called once a row; arrived: after arrive()
    template <bool PAST, typename Row, typename There>
    __device__ __forceinline__ void store(Row&& row, There&& there, int side, const LaneOfRow<D>& l, bool arrived = true) {
        if constexpr (kPair) {
            if (arrived) exchange();
            const int at = l.a + (side & 1) * (l.b - l.a);
            if (there(side & ~1)) a.template store<PAST>(row(side & ~1) + at);
            if (there(side | 1)) b.template store<PAST>(row(side | 1) + at);
        } else if (there(side)) {
            T* const own = row(side);
            a.template store<PAST>(own + l.a);
            b.template store<PAST>(own + l.b);
        }
    }
    // unit a of the odd side's lanes with unit b of the even one's, four lanes away
    __device__ __forceinline__ void exchange() {
        typedef int i32x4 __attribute__((ext_vector_type(4)));
        const i32x4 x = __builtin_bit_cast(i32x4, a.v), y = __builtin_bit_cast(i32x4, b.v);
        i32x4 u, v;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            u[e] = __builtin_amdgcn_update_dpp(x[e], y[e], 0x114, 0xf, 0xa, false);  // row_shr:4, into lanes 4..7 and 12..15
            v[e] = __builtin_amdgcn_update_dpp(y[e], x[e], 0x104, 0xf, 0x5, false);  // row_shl:4, into lanes 0..3 and 8..11
        }
        a.v = __builtin_bit_cast(bf16x8, u);
        b.v = __builtin_bit_cast(bf16x8, v);
    }
    // norm (with weights w) and rotation
    __device__ __forceinline__ void norm_and_turn(const LaneOfRow<D>& l, bool norm, float eps, const LaneVector<D>& w, bool rotated, bool paired,
                                                  const Angles& angles) {
        float x[8], y[8];
        a.get(x);
        b.get(y);
        if (norm) {
            const float r = row_rstd<D>(x, y, eps);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[e] *= r * w.a[e];
                y[e] *= r * w.b[e];
            }
        }
        if (rotated) angles.template turn<D, false>(l, paired, x, y);
        a.set(x);
        b.set(y);
    }
};

// Heads of a token that a wave takes side by side: what it reads of a token-major tensor comes in runs of kSide rows, what it writes of a head-major one in
// runs of its tokens.  (us, rows of 8 lanes, one / two / four / eight heads: forward of H 32, Hkv 8, N 16640, d 128 100 / 97 / 89 / 83, backward 152 / 140 / 126 /
// 119, of N 16384 131 / 124 / 118 / 118, of H 16, Hkv 4, N 4100 19.6 / 18.7 / 18.9 / 25.4, append of 16 prompts 123 / 113 / 96 / 98; rows of 4 lanes, two / four
// heads, B 4, H 16, Hkv 4, d 64: forward of N 4096 22.2 / 20.3, of N 4200 23.6 / 25.7, of N 2048 11.8 / 12.5, backward of N 4096 32.3 / 34.8, of N 4200
// 37.2 / 40.8.)
template <int D>
constexpr int kSide = D == 128 ? 4 : 2;

// Calls work(row, h) for the heads h0 <= h < h1; the next head's row is on its way meanwhile.  The first
// one is asked for at once, so that something else can be waited for in between.
template <typename R, typename Load>
struct HeadWalk {
    R row[2];
    Load load;  // load(row, h)
    int h0, h1;
    __device__ __forceinline__ HeadWalk(int from, int to, Load l) : load(l), h0(from), h1(to) { load(row[0], h0); }
    template <typename Work>
    __device__ __forceinline__ void run(Work&& work) {
        for (int h = h0; h < h1; h += 2) {
            if (h + 1 < h1) load(row[1], h + 1);
            work(row[0], h);
            if (h + 1 >= h1) break;
            if (h + 2 < h1) load(row[0], h + 2);
            work(row[1], h + 1);
        }
    }
};

// The heads of a token in one row of numbers: queries, then keys, then values.  A wave takes a range of them.
enum HeadKind { kQueries = 0, kKeys = 1, kValues = 2 };
struct HeadRange {
    int x0, x1;
    // the heads h0 <= h < h1 of a kind whose `count` heads begin at number `first`
    __device__ __forceinline__ bool part(int first, int count, int& h0, int& h1) const {
        h0 = max(x0 - first, 0);
        h1 = min(x1 - first, count);
        return h0 < h1;
    }
};
// How `tiles` tiles of tokens and `heads` heads are shared out over the waves: ranges of heads as long as still leave every SIMD two waves
// (what a wave finds out about a token serves all heads of its range).
struct Shares {
    int ranges, heads;  // ranges, and heads of one
    int items;          // tiles x ranges: more than one range only where there are few tiles
    Shares() = default;
    Shares(int tiles, int all, int side) {  // ranges are multiples of `side` heads
        int want = tiles < 8 * device_cu_count() ? (8 * device_cu_count() + tiles - 1) / tiles : 1;
        if (want > all) want = all;
        heads = (all + want - 1) / want;
        heads = (heads + side - 1) / side * side;
        ranges = (all + heads - 1) / heads;
        items = tiles * ranges;
    }
    __device__ __forceinline__ HeadRange range(int item, int& tile) const {
        tile = item / ranges;
        const int x0 = (item - tile * ranges) * heads;
        return {x0, x0 + heads};
    }
};

}  // namespace gfwa
