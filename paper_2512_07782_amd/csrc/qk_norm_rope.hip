// Norm and rotation of queries and keys, and its derivative, on gfx950 (paper Sec. 3.3: the layer norms its queries and
// keys per head).  Both are bound by memory: every row is read once from the projection's token-major layout and written once to
// the attention's head-major layout (or back).
//   * a row of D elements is held by D / 16 lanes (head_rows.h), so that the norm's sum takes two or three DPP exchanges, the rotation
//     none, and every access is whole 16-byte pieces;
//   * a wave takes two (D = 128) or eight (D = 64) consecutive tokens, four or two heads of each at a time (kSide; kManySide), and walks over a range of
//     heads: a token's angles are formed once for all of them, and both layouts are met in runs;
//   * the weights' gradients are summed in registers over the heads that a lane meets, over the waves through LDS and over the workgroups by
//     a second small launch, in an order that does not change from run to run.
#include "gfwa_internal.h"
#include "head_rows.h"

namespace gfwa {

namespace {

constexpr int kRopeWaves = 4;  // waves of a workgroup, each on its own

// Forward: eight heads side by side where the queries and the keys have a multiple of eight and the projection has more than 128 MiB; what a wave reads is then
// one token's (us, kSide / eight: H 32, Hkv 8, d 128, N 32768 175 / 148, 16384 84.0 / 78.0, 12000 63.3 / 60.8, 8192 37.1 / 38.9, 4096 20.3 / 21.4; B 8, H 16,
// Hkv 16, N 8192, d 64 150 / 151; fp32, B 2, H 16, Hkv 16, N 4400 97 / 90).  Without a multiple of eight, H 32, Hkv 4, d 128: N 13500 59.1 / 60.5, 16384
// 72.8 / 69.7, 32768 140 / 132; H 12, Hkv 4, N 27000 56.8 / 66.4; H 14, Hkv 2, N 30000 59.7 / 71.6.  Without values the projection counts all the same (H 16,
// Hkv 16, d 128, N 12000, 98 MB read, 39.0 / 37.9; d 64, B 4, N 5700 34.6 / 35.7).
constexpr int kManySide = 8;
constexpr long long kManyBytes = 128 << 20;

struct RopeArgs {
    HeadsView q, k, v;     // token-major, strided (backward: dq, dk, dv are written)
    HeadsView x_q, x_k;    // backward: the inputs
    const float *wq, *wk;
    float eps;
    const double* freq;
    int rot;
    const int* pos;
    bool norm, paired;
    void *Q, *K, *V;       // head-major, dense (backward: dQ, dK, dV are read)
    float* part;           // backward: the workgroups' sums of the weights' gradients, [workgroups][2][D], or nullptr
    int H, Hkv, N;
    int tokens;            // B * N
    Shares shares;         // of tiles of 1024 / D tokens
};

// A lane's token: where its rows stand in the token-major and the head-major layout.
struct LaneToken {
    bool there;
    int b, n, flat;
    __device__ __forceinline__ LaneToken(long long t, const RopeArgs& a) {
        there = t < a.tokens;
        flat = there ? (int)t : a.tokens - 1;
        b = flat / a.N;
        n = flat - b * a.N;
    }
    __device__ __forceinline__ long long in(const HeadsView& x) const { return b * x.batch + n * x.token; }
    __device__ __forceinline__ long long dense(int heads, int N) const { return (long long)b * heads * N + n; }  // row of the first head
};

template <typename T, int D, bool ONCE, int HG>
__global__ __launch_bounds__(64 * kRopeWaves) void qk_norm_rope_kernel(const RopeArgs a) {
    constexpr int LPR = D / 16, RPW = 64 / LPR / HG;
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const LaneOfRow<D> l(lane % LPR, a.rot, a.paired);
    Frequencies freq;
    if (a.rot > 0) freq.load(l, a.freq);
    for (int item = blockIdx.x * kRopeWaves + wv; item < a.shares.items; item += gridDim.x * kRopeWaves) {
        int tile;
        const HeadRange range = a.shares.range(item, tile);
        const int side = lane / LPR % HG;  // this lane's head of the HG next to each other
        const LaneToken t((long long)tile * RPW + lane / (LPR * HG), a);
        Angles angles;
        if (range.x0 < a.H + a.Hkv && a.rot > 0) angles.at(l, a.pos != nullptr ? a.pos[t.flat] : t.n, freq);
#pragma unroll 1
        for (int kind = kQueries; kind <= kKeys; ++kind) {
            const bool keys = kind == kKeys;
            const int count = keys ? a.Hkv : a.H;
            int h0, h1;
            if (!range.part(keys ? a.H : 0, count, h0, h1)) continue;
            const HeadsView in = keys ? a.k : a.q;
            const T* const from = (const T*)in.data + t.in(in);
            T* const to = (T*)(keys ? a.K : a.Q) + t.dense(count, a.N) * D;
            auto load = [&](LaneRow<T, D, ONCE>& r, int i) __attribute__((always_inline)) {
                r.load([&](int x) __attribute__((always_inline)) { return from + min(h0 + i * HG + x, h1 - 1) * in.head; }, side, l);
            };
            HeadWalk<LaneRow<T, D, ONCE>, decltype(load)> walk(0, (h1 - h0 + HG - 1) / HG, load);
            LaneVector<D> w;
            if (a.norm) w.load(keys ? a.wk : a.wq, l);
            walk.run([&](LaneRow<T, D, ONCE>& r, int i) __attribute__((always_inline)) {
                r.arrive();
                r.norm_and_turn(l, a.norm, a.eps, w, a.rot > 0, a.paired, angles);
                r.template store<false>([&](int x) __attribute__((always_inline)) { return to + (size_t)(h0 + i * HG + x) * a.N * D; },
                                        [&](int x) __attribute__((always_inline)) { return t.there && h0 + i * HG + x < h1; }, side, l);
            });
        }
        int h0, h1;
        if (a.V != nullptr && range.part(a.H + a.Hkv, a.Hkv, h0, h1)) {
            const T* const from = (const T*)a.v.data + t.in(a.v);
            T* const to = (T*)a.V + t.dense(a.Hkv, a.N) * D;
            auto load = [&](LaneRow<T, D, ONCE>& r, int i) __attribute__((always_inline)) {
                r.load([&](int x) __attribute__((always_inline)) { return from + min(h0 + i * HG + x, h1 - 1) * a.v.head; }, side, l);
            };
            HeadWalk<LaneRow<T, D, ONCE>, decltype(load)> walk(0, (h1 - h0 + HG - 1) / HG, load);
            walk.run([&](LaneRow<T, D, ONCE>& r, int i) __attribute__((always_inline)) {
                r.template store<false>([&](int x) __attribute__((always_inline)) { return to + (size_t)(h0 + i * HG + x) * a.N * D; },
                                        [&](int x) __attribute__((always_inline)) { return t.there && h0 + i * HG + x < h1; }, side, l, false);
            });
        }
    }
}

// By the size of the projection (bf16): of more than kOnceBytes gradients are read past the caches; between kInputsBytes and kManyBytes the inputs too (three
// tensors of that size pass the memory-side cache); of more than kManyBytes rows of four lanes are taken four side by side.  (us, inputs through / past the
// caches, calls on three sets of tensors in turn: H 32, Hkv 8, d 128, N 4096 31.4 / 31.1, 6000, 74 MB, 50.7 / 43.5, 6500 55.5 / 50.8, 8192 62.9 / 61.6, 12000, that
// no cache holds, 89.2 / 89.3, 16384 118 / 123; d 64, H 32, Hkv 4, N 16384, 84 MB, 55.9 / 48.2, B 4, H 16, Hkv 4, N 4096 31.7 / 33.1, 5500, 68 MB, 47.3 / 41.1;
// results in the same memory each time: N 6000 42.3 / 44.0, 6500 49.4 / 50.6, 8192 55.0 / 55.2, d 64, N 5500 40.1 / 40.8.  Four side by side instead of two:
// B 8, H 16, Hkv 16, N 8192 216 -> 208, B 4, H 16, Hkv 4, N 4096 31.7 -> 35.1.)
// The values' heads count, given or not: by what is read alone, H 16, Hkv 16, d 128, N 8192 without dV would take 48.0 instead of 42.6, H 32, Hkv 8, N 12000 84.5
// instead of 82.2.
enum BwdSize { kSmall = 0, kMiddle = 1, kSpread = 2, kLarge = 3 };
constexpr long long kInputsBytes = 72 << 20;
template <int D, int SIZE>
constexpr int kBwdSide = D == 64 && SIZE == kLarge ? 4 : kSide<D>;

template <typename T, int D, int SIZE>
__global__ __launch_bounds__(64 * kRopeWaves) void qk_norm_rope_bwd_kernel(const RopeArgs a) {
    constexpr bool ONCE = SIZE != kSmall;
    constexpr int LPR = D / 16, HG = kBwdSide<D, SIZE>, RPW = 64 / LPR / HG;
    __shared__ float sums[kRopeWaves][2][16][64 + LPR];  // of each lane's elements, for the queries' and the keys' weights (LPR: rows do not meet in a bank)
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const LaneOfRow<D> l(lane % LPR, a.rot, a.paired);
#pragma unroll
    for (int i = 0; i < 32; ++i) sums[wv][i >> 4][i & 15][lane] = 0.f;
    struct Rows {
        LaneRow<T, D, ONCE> g;
        LaneRow<T, D, SIZE == kSpread, SIZE == kSpread> x;
    };
    Frequencies freq;
    if (a.rot > 0) freq.load(l, a.freq);
    for (int item = blockIdx.x * kRopeWaves + wv; item < a.shares.items; item += gridDim.x * kRopeWaves) {
        int tile;
        const HeadRange range = a.shares.range(item, tile);
        const int side = lane / LPR % HG;  // this lane's head of the HG next to each other
        const LaneToken t((long long)tile * RPW + lane / (LPR * HG), a);
        Angles angles;
        if (range.x0 < a.H + a.Hkv && a.rot > 0) angles.at(l, a.pos != nullptr ? a.pos[t.flat] : t.n, freq);
#pragma unroll 1
        for (int kind = kQueries; kind <= kKeys; ++kind) {
            const bool keys = kind == kKeys;
            const int count = keys ? a.Hkv : a.H;
            int h0, h1;
            if (!range.part(keys ? a.H : 0, count, h0, h1)) continue;
            const HeadsView out = keys ? a.k : a.q, in = keys ? a.x_k : a.x_q;
            const T* const from = (const T*)(keys ? a.K : a.Q) + t.dense(count, a.N) * D;
            T* const to = (T*)out.data + t.in(out);
            const T* const xs = a.norm ? (const T*)in.data + t.in(in) : nullptr;
            auto load = [&](Rows& r, int i) __attribute__((always_inline)) {
                r.g.load([&](int x) __attribute__((always_inline)) { return from + (size_t)min(h0 + i * HG + x, h1 - 1) * a.N * D; }, side, l);
                if (a.norm) r.x.load([&](int x) __attribute__((always_inline)) { return xs + min(h0 + i * HG + x, h1 - 1) * in.head; }, side, l);
            };
            HeadWalk<Rows, decltype(load)> walk(0, (h1 - h0 + HG - 1) / HG, load);
            LaneVector<D> w, dw;
            if (a.norm) w.load(keys ? a.wk : a.wq, l);
#pragma unroll
            for (int e = 0; e < 8; ++e) dw.a[e] = dw.b[e] = 0.f;
            walk.run([&](Rows& r, int i) __attribute__((always_inline)) {
                const int h = h0 + i * HG + side;
                const bool there = t.there && h < h1;
                float g[8], f[8];
                r.g.arrive();
                r.g.a.get(g);
                r.g.b.get(f);
                if (a.rot > 0) angles.turn<D, true>(l, a.paired, g, f);
                if (a.norm) {
                    float x[8], y[8];
                    r.x.arrive();
                    r.x.a.get(x);
                    r.x.b.get(y);
                    const float rstd = row_rstd<D>(x, y, a.eps);
                    float dot = 0.f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        x[e] *= rstd;
                        y[e] *= rstd;
                        dw.a[e] = fmaf(there ? g[e] : 0.f, x[e], dw.a[e]);
                        dw.b[e] = fmaf(there ? f[e] : 0.f, y[e], dw.b[e]);
                        g[e] *= w.a[e];
                        f[e] *= w.b[e];
                        dot = fmaf(g[e], x[e], fmaf(f[e], y[e], dot));
                    }
                    dot = sum_over_row<LPR>(dot) * (1.f / D);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        g[e] = rstd * fmaf(-dot, x[e], g[e]);
                        f[e] = rstd * fmaf(-dot, y[e], f[e]);
                    }
                }
                r.g.a.set(g);
                r.g.b.set(f);
                r.g.template store<false>([&](int x) __attribute__((always_inline)) { return to + (h0 + i * HG + x) * out.head; },
                                          [&](int x) __attribute__((always_inline)) { return t.there && h0 + i * HG + x < h1; }, side, l);
            });
            if (a.part != nullptr) {  // the lane's own cells
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    sums[wv][kind][e][lane] += dw.a[e];
                    sums[wv][kind][8 + e][lane] += dw.b[e];
                }
            }
        }
        int h0, h1;
        if (a.V != nullptr && range.part(a.H + a.Hkv, a.Hkv, h0, h1)) {
            const T* const from = (const T*)a.V + t.dense(a.Hkv, a.N) * D;
            T* const to = (T*)a.v.data + t.in(a.v);
            auto load = [&](LaneRow<T, D, ONCE>& r, int i) __attribute__((always_inline)) {
                r.load([&](int x) __attribute__((always_inline)) { return from + (size_t)min(h0 + i * HG + x, h1 - 1) * a.N * D; }, side, l);
            };
            HeadWalk<LaneRow<T, D, ONCE>, decltype(load)> walk(0, (h1 - h0 + HG - 1) / HG, load);
            walk.run([&](LaneRow<T, D, ONCE>& r, int i) __attribute__((always_inline)) {
                r.template store<false>([&](int x) __attribute__((always_inline)) { return to + (h0 + i * HG + x) * a.v.head; },
                                        [&](int x) __attribute__((always_inline)) { return t.there && h0 + i * HG + x < h1; }, side, l, false);
            });
        }
    }
    if (a.part == nullptr) return;  // uniform over the launch
    __syncthreads();
    // over the tokens of a wave (lanes j, j + LPR, ..) and over the waves
    for (int i = threadIdx.x; i < 2 * D; i += 64 * kRopeWaves) {
        const int kind = i / D, j = i % LPR, e = i % D / LPR;  // element e of lane j
        double s = 0.0;
        for (int k = 0; k < kRopeWaves; ++k)
#pragma unroll
            for (int row = 0; row < 64 / LPR; ++row) s += sums[k][kind][e][row * LPR + j];
        const LaneOfRow<D> of(j, a.rot, a.paired);
        a.part[(size_t)blockIdx.x * 2 * D + kind * D + (e < 8 ? of.a + e : of.b + e - 8)] = (float)s;
    }
}

// dw[i] = sum over the workgroups of part[., i]: one workgroup for 16 of the 2 D sums, 64 partial rows at a time.  (Sums over lanes, waves and workgroups
// in fp64: as fast, and a gradient of 8000 to 300000 rows is off by 7e-8 of its norm instead of 2.4e-7.)
__global__ __launch_bounds__(1024) void weight_grad_sum_kernel(const float* __restrict__ part, float* dwq, float* dwk, int blocks, int D) {
    __shared__ double sums[64][17];
    const int col = threadIdx.x & 15, row = threadIdx.x >> 4;
    const int i = blockIdx.x * 16 + col;
    float* const dw = i < D ? dwq : dwk;
    double s = 0.0;
#pragma unroll 8
    for (int k = row; k < blocks; k += 64) s += part[(size_t)k * 2 * D + i];
    sums[row][col] = s;
    __syncthreads();
    if (row == 0 && dw != nullptr) {
        s = 0.0;
        for (int k = 0; k < 64; ++k) s += sums[k][col];
        dw[i % D] = (float)s;
    }
}

// Workgroups that leave sums of the weights' gradients.  In bf16 three waves a SIMD are there at a time, and what fits in them goes at once; more goes through
// two waves a SIMD, which meet memory in longer runs (us, 512 / 768 / 2048 workgroups: H 32, Hkv 8, N 16384, d 128 118 / 119 / 122, B 4, H 16, Hkv 16, N 8192
// 207 / 211 / 219; 513 workgroups' worth, H 16, Hkv 4, N 4100, 22.7 / 18.7 / 18.7).  In fp32 two waves a SIMD are all there are (512 / 768 workgroups,
// d 128: H 8, Hkv 2, N 5000 25.7 / 28.3, H 16, Hkv 4, N 6100 51.5 / 57.2, N 4200 44.5 / 44.6, H 32, Hkv 8, N 5000 83.0 / 82.2).
constexpr int kMostSums = 768, kManySums = 512;

long long share_out(RopeArgs& a, int D, int side, bool bf16) {
    a.shares = Shares((int)(((long long)a.tokens * side + 1024 / D - 1) / (1024 / D)), a.H + (a.V != nullptr ? 2 : 1) * a.Hkv, side);
    const long long blocks = ((long long)a.shares.items + kRopeWaves - 1) / kRopeWaves;
    if (a.part != nullptr) return blocks <= (bf16 ? kMostSums : kManySums) ? blocks : kManySums;
    return blocks < 1 << 20 ? blocks : 1 << 20;
}

}  // namespace

size_t qk_norm_rope_backward_workspace_bytes(int d) { return (size_t)kMostSums * 2 * d * sizeof(float); }

static RopeArgs rope_args(const HeadRotation& how, void* Q, void* K, void* V, int B, int H, int Hkv, int N) {
    RopeArgs a{};
    a.wq = how.wq;
    a.wk = how.wk;
    a.eps = how.eps;
    a.freq = how.freq;
    a.rot = how.rot;
    a.pos = how.pos;
    a.norm = how.norm;
    a.paired = how.paired;
    a.Q = Q;
    a.K = K;
    a.V = V;
    a.H = H;
    a.Hkv = Hkv;
    a.N = N;
    a.tokens = B * N;
    return a;
}

hipError_t qk_norm_rope(bool bf16, const HeadsView& q, const HeadsView& k, const HeadsView& v, const HeadRotation& how, void* Q, void* K, void* V,
                        int B, int H, int Hkv, int N, int d, hipStream_t s) {
    RopeArgs a = rope_args(how, Q, K, V, B, H, Hkv, N);
    a.q = q;
    a.k = k;
    a.v = v;
    const long long row = (long long)a.tokens * d * (bf16 ? 2 : 4);  // of one head
    const bool many = H % kManySide == 0 && Hkv % kManySide == 0 && row * (H + 2LL * Hkv) > kManyBytes;
    const bool once = row * (H + (V != nullptr ? 2LL : 1LL) * Hkv) > kOnceBytes;  // of what is read
    const long long blocks = share_out(a, d, many ? kManySide : d == 128 ? kSide<128> : kSide<64>, bf16);
    ProfScope prof(kKernNormRope, s);
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(64 * kRopeWaves), 0, s, a); };
    auto of_side = [&](auto side) {
        constexpr bool eight = decltype(side)::value;  // (then always ONCE: without values two thirds of kManyBytes are read at least)
        constexpr int HG128 = eight ? kManySide : kSide<128>, HG64 = eight ? kManySide : kSide<64>;
        if (!bf16) d == 128 ? launch(qk_norm_rope_kernel<float, 128, false, HG128>) : launch(qk_norm_rope_kernel<float, 64, false, HG64>);
        else if (d == 128) once ? launch(qk_norm_rope_kernel<bf16_t, 128, true, HG128>) : launch(qk_norm_rope_kernel<bf16_t, 128, eight, HG128>);
        else once ? launch(qk_norm_rope_kernel<bf16_t, 64, true, HG64>) : launch(qk_norm_rope_kernel<bf16_t, 64, eight, HG64>);
    };
    many ? of_side(std::true_type{}) : of_side(std::false_type{});
    return hipGetLastError();
}

hipError_t qk_norm_rope_backward(bool bf16, const HeadsView& q, const HeadsView& k, const HeadRotation& how, const void* dQ, const void* dK,
                                 const void* dV, const HeadsView& dq, const HeadsView& dk, const HeadsView& dv, float* dwq, float* dwk, float* part,
                                 int B, int H, int Hkv, int N, int d, hipStream_t s) {
    RopeArgs a = rope_args(how, const_cast<void*>(dQ), const_cast<void*>(dK), const_cast<void*>(dV), B, H, Hkv, N);
    a.q = dq;
    a.k = dk;
    a.v = dv;
    a.x_q = q;
    a.x_k = k;
    a.part = dwq != nullptr || dwk != nullptr ? part : nullptr;
    const long long bytes = (long long)a.tokens * (H + 2LL * Hkv) * d * 2;
    const int size = !bf16 || bytes <= kOnceBytes ? kSmall : bytes <= kInputsBytes ? kMiddle : bytes <= kManyBytes ? kSpread : kLarge;
    const long long blocks = share_out(a, d, d == 128 ? kSide<128> : size == kLarge ? kBwdSide<64, kLarge> : kSide<64>, bf16);
    {
        ProfScope prof(kKernNormRopeBwd, s);
        auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(64 * kRopeWaves), 0, s, a); };
        auto of_size = [&](auto D) {
            constexpr int d = decltype(D)::value;
            if (!bf16) launch(qk_norm_rope_bwd_kernel<float, d, kSmall>);
            else if (size == kSmall) launch(qk_norm_rope_bwd_kernel<bf16_t, d, kSmall>);
            else if (size == kMiddle) launch(qk_norm_rope_bwd_kernel<bf16_t, d, kMiddle>);
            else if (size == kSpread) launch(qk_norm_rope_bwd_kernel<bf16_t, d, kSpread>);
            else launch(qk_norm_rope_bwd_kernel<bf16_t, d, kLarge>);
        };
        d == 128 ? of_size(std::integral_constant<int, 128>{}) : of_size(std::integral_constant<int, 64>{});
    }
    if (a.part != nullptr) {
        ProfScope prof(kKernNormWeightSum, s);
        hipLaunchKernelGGL(weight_grad_sum_kernel, dim3(2 * d / 16), dim3(1024), 0, s, part, dwq, dwk, (int)blocks, d);
    }
    return hipGetLastError();
}

}  // namespace gfwa
