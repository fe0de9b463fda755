// Norm and rotation of queries and keys, and its derivative, on gfx950 (paper Sec. 3.3: the layer norms its queries and
// keys per head).  Both are bound by memory: every row is read once from the projection's token-major layout and written once to
// the attention's head-major layout (or back).
//   * a row of D elements is held by D / 16 lanes (head_rows.h), so that the norm's sum takes two or three DPP exchanges, the rotation
//     none, and every access is whole 16-byte pieces;
//   * a wave takes 1024 / D consecutive tokens and walks over a range of heads: a token's angles are formed once for all of them, and
//     what it writes for a head is one run of 2048 elements or less of the head-major layout;
//   * the weights' gradients are summed in registers over all rows of a wave, over the waves through LDS and over the workgroups by
//     a second small launch, in an order that does not change from run to run.
#include "gfwa_internal.h"
#include "head_rows.h"

namespace gfwa {

namespace {

constexpr int kRopeWaves = 4;  // waves of a workgroup, each on its own

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
    long long tokens;      // B * N
    long long items;       // token tiles x head ranges
    int ranges, heads;     // head ranges and heads of one
};

// A lane's token: where its rows stand in the token-major and the head-major layout.
struct LaneToken {
    bool there;
    long long b, n, flat;
    __device__ __forceinline__ LaneToken(long long t, const RopeArgs& a) {
        there = t < a.tokens;
        flat = there ? t : a.tokens - 1;
        b = flat / a.N;
        n = flat - b * a.N;
    }
};

template <typename T, int D>
__global__ __launch_bounds__(64 * kRopeWaves) void qk_norm_rope_kernel(const RopeArgs a) {
    constexpr int LPR = D / 16, RPW = 64 / LPR;
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    const LaneOfRow<D> l(lane % LPR, a.rot, a.paired);
    for (long long item = (long long)blockIdx.x * kRopeWaves + wv; item < a.items; item += (long long)gridDim.x * kRopeWaves) {
        const long long tile = item / a.ranges;
        const int x0 = (int)(item - tile * a.ranges) * a.heads, x1 = min(x0 + a.heads, a.H + 2 * a.Hkv);
        const LaneToken t(tile * RPW + lane / LPR, a);
        Angles angles;
        if (x0 < a.H + a.Hkv && a.rot > 0) angles.at(l, a.pos != nullptr ? a.pos[t.flat] : (int)t.n, a.freq);
        auto heads_of = [&](const HeadsView& in, const float* weight, void* out, int first, int count, bool plain) __attribute__((always_inline)) {
            const int h0 = max(x0 - first, 0), h1 = min(x1 - first, count);
            if (h0 >= h1) return;
            const T* from = (const T*)in.data + t.b * in.batch + t.n * in.token;
            T* to = (T*)out + (t.b * count * a.N + t.n) * D;
            LaneWeights w;
            if (!plain && a.norm) w.load(weight, l);
            for (int h = h0; h < h1; ++h) {
                Unit8<T> ua, ub;
                ua.load(from + h * in.head + l.a);
                ub.load(from + h * in.head + l.b);
                if (!plain) {
                    float x[8], y[8];
                    ua.get(x);
                    ub.get(y);
                    if (a.norm) {
                        const float r = row_rstd<D>(x, y, a.eps);
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            x[e] *= r * w.a[e];
                            y[e] *= r * w.b[e];
                        }
                    }
                    if (a.rot > 0) angles.turn<D, false>(l, a.paired, x, y);
                    ua.set(x);
                    ub.set(y);
                }
                if (t.there) {
                    ua.store(to + (size_t)h * a.N * D + l.a);
                    ub.store(to + (size_t)h * a.N * D + l.b);
                }
            }
        };
        heads_of(a.q, a.wq, a.Q, 0, a.H, false);
        heads_of(a.k, a.wk, a.K, a.H, a.Hkv, false);
        if (a.V != nullptr) heads_of(a.v, nullptr, a.V, a.H + a.Hkv, a.Hkv, true);
    }
}

template <typename T, int D>
__global__ __launch_bounds__(64 * kRopeWaves) void qk_norm_rope_bwd_kernel(const RopeArgs a) {
    constexpr int LPR = D / 16, RPW = 64 / LPR;
    __shared__ float sums[kRopeWaves][2][D];
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    const LaneOfRow<D> l(lane % LPR, a.rot, a.paired);
    LaneWeights dwq, dwk;
#pragma unroll
    for (int e = 0; e < 8; ++e) dwq.a[e] = dwq.b[e] = dwk.a[e] = dwk.b[e] = 0.f;
    for (long long item = (long long)blockIdx.x * kRopeWaves + wv; item < a.items; item += (long long)gridDim.x * kRopeWaves) {
        const long long tile = item / a.ranges;
        const int x0 = (int)(item - tile * a.ranges) * a.heads, x1 = min(x0 + a.heads, a.H + 2 * a.Hkv);
        const LaneToken t(tile * RPW + lane / LPR, a);
        Angles angles;
        if (x0 < a.H + a.Hkv && a.rot > 0) angles.at(l, a.pos != nullptr ? a.pos[t.flat] : (int)t.n, a.freq);
        auto heads_of = [&](const HeadsView& out, const HeadsView& in, const float* weight, const void* dy, LaneWeights& dw, int first, int count,
                            bool plain) __attribute__((always_inline)) {
            const int h0 = max(x0 - first, 0), h1 = min(x1 - first, count);
            if (h0 >= h1) return;
            const T* from = (const T*)dy + (t.b * count * a.N + t.n) * D;
            T* to = (T*)out.data + t.b * out.batch + t.n * out.token;
            const bool normed = !plain && a.norm;
            const T* xs = normed ? (const T*)in.data + t.b * in.batch + t.n * in.token : nullptr;
            LaneWeights w;
            if (normed) w.load(weight, l);
            for (int h = h0; h < h1; ++h) {
                Unit8<T> ga, gb, xa, xb;
                ga.load(from + (size_t)h * a.N * D + l.a);
                gb.load(from + (size_t)h * a.N * D + l.b);
                if (normed) {
                    xa.load(xs + h * in.head + l.a);
                    xb.load(xs + h * in.head + l.b);
                }
                if (!plain) {
                    float g[8], f[8];
                    ga.get(g);
                    gb.get(f);
                    if (a.rot > 0) angles.turn<D, true>(l, a.paired, g, f);
                    if (normed) {
                        float x[8], y[8];
                        xa.get(x);
                        xb.get(y);
                        const float r = row_rstd<D>(x, y, a.eps);
                        float dot = 0.f;
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            x[e] *= r;
                            y[e] *= r;
                            dw.a[e] += t.there ? g[e] * x[e] : 0.f;
                            dw.b[e] += t.there ? f[e] * y[e] : 0.f;
                            g[e] *= w.a[e];
                            f[e] *= w.b[e];
                            dot = fmaf(g[e], x[e], fmaf(f[e], y[e], dot));
                        }
                        dot = sum_over_row<LPR>(dot) * (1.f / D);
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            g[e] = r * fmaf(-dot, x[e], g[e]);
                            f[e] = r * fmaf(-dot, y[e], f[e]);
                        }
                    }
                    ga.set(g);
                    gb.set(f);
                }
                if (t.there) {
                    ga.store(to + h * out.head + l.a);
                    gb.store(to + h * out.head + l.b);
                }
            }
        };
        heads_of(a.q, a.x_q, a.wq, a.Q, dwq, 0, a.H, false);
        heads_of(a.k, a.x_k, a.wk, a.K, dwk, a.H, a.Hkv, false);
        if (a.V != nullptr) heads_of(a.v, a.x_k, nullptr, a.V, dwk, a.H + a.Hkv, a.Hkv, true);
    }
    if (a.part == nullptr) return;  // uniform over the launch
    // over the tokens of the wave, then over the waves
    auto over_tokens = [&](LaneWeights& dw, int which) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
#pragma unroll
            for (int off = LPR; off < 64; off <<= 1) {
                dw.a[e] += __shfl_xor(dw.a[e], off, 64);
                dw.b[e] += __shfl_xor(dw.b[e], off, 64);
            }
            if (lane < LPR) {
                sums[wv][which][l.a + e] = dw.a[e];
                sums[wv][which][l.b + e] = dw.b[e];
            }
        }
    };
    over_tokens(dwq, 0);
    over_tokens(dwk, 1);
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * D; i += 64 * kRopeWaves) {
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < kRopeWaves; ++k) s += sums[k][i / D][i % D];
        a.part[(size_t)blockIdx.x * 2 * D + i] = s;
    }
}

// dw[i] = sum over the workgroups of part[., i]: one workgroup for 32 sums, 32 partial rows at a time.
__global__ __launch_bounds__(1024) void weight_grad_sum_kernel(const float* __restrict__ part, float* dwq, float* dwk, int blocks, int D) {
    __shared__ float sums[32][33];
    const int col = threadIdx.x & 31, row = threadIdx.x >> 5;
    const int i = blockIdx.x * 32 + col;  // 2 D is a multiple of 32
    float s = 0.f;
    for (int k = row; k < blocks; k += 32) s += part[(size_t)k * 2 * D + i];
    sums[row][col] = s;
    __syncthreads();
    if (row == 0) {
        s = 0.f;
        for (int k = 0; k < 32; ++k) s += sums[k][col];
        float* dw = i < D ? dwq : dwk;
        if (dw != nullptr) dw[i % D] = s;
    }
}

// How the work is cut up: head ranges as long as still leave every SIMD its waves.
void cut(RopeArgs& a, int D, long long& blocks, long long most_blocks) {
    const int heads = a.H + (a.V != nullptr ? 2 : 1) * a.Hkv;
    const long long tiles = (a.tokens + 1024 / D - 1) / (1024 / D);
    const long long waves = 16LL * device_cu_count();
    long long ranges = (waves + tiles - 1) / tiles;
    if (ranges > heads) ranges = heads;
    a.heads = (int)((heads + ranges - 1) / ranges);
    a.ranges = (heads + a.heads - 1) / a.heads;
    a.items = tiles * a.ranges;
    blocks = (a.items + kRopeWaves - 1) / kRopeWaves;
    if (blocks > most_blocks) blocks = most_blocks;
}

long long most_bwd_blocks() { return 8LL * 256; }

}  // namespace

size_t qk_norm_rope_backward_workspace_bytes(int d) { return (size_t)most_bwd_blocks() * 2 * d * sizeof(float); }

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
    a.tokens = (long long)B * N;
    return a;
}

hipError_t qk_norm_rope(bool bf16, const HeadsView& q, const HeadsView& k, const HeadsView& v, const HeadRotation& how, void* Q, void* K, void* V,
                        int B, int H, int Hkv, int N, int d, hipStream_t s) {
    RopeArgs a = rope_args(how, Q, K, V, B, H, Hkv, N);
    a.q = q;
    a.k = k;
    a.v = v;
    long long blocks;
    cut(a, d, blocks, 1 << 20);
    ProfScope prof(kKernNormRope, s);
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(64 * kRopeWaves), 0, s, a); };
    if (bf16) d == 128 ? launch(qk_norm_rope_kernel<bf16_t, 128>) : launch(qk_norm_rope_kernel<bf16_t, 64>);
    else d == 128 ? launch(qk_norm_rope_kernel<float, 128>) : launch(qk_norm_rope_kernel<float, 64>);
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
    long long blocks;
    cut(a, d, blocks, most_bwd_blocks());
    {
        ProfScope prof(kKernNormRopeBwd, s);
        auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(64 * kRopeWaves), 0, s, a); };
        if (bf16) d == 128 ? launch(qk_norm_rope_bwd_kernel<bf16_t, 128>) : launch(qk_norm_rope_bwd_kernel<bf16_t, 64>);
        else d == 128 ? launch(qk_norm_rope_bwd_kernel<float, 128>) : launch(qk_norm_rope_bwd_kernel<float, 64>);
    }
    if (a.part != nullptr) {
        ProfScope prof(kKernNormWeightSum, s);
        hipLaunchKernelGGL(weight_grad_sum_kernel, dim3(2 * d / 32), dim3(1024), 0, s, part, dwq, dwk, (int)blocks, d);
    }
    return hipGetLastError();
}

}  // namespace gfwa
