// GatedFWA decoding step on gfx950 against a paged cache: one query per (sequence, head), the keys and values of its last w positions
// looked up page by page.  Row `pos` of the forward (paper Sec. 3.2 / Alg. 2) over the positions whose page is there.
//
// The step is bound by reading the window once (2 w d elements per key/value head).  Keys are taken in units of 16 consecutive positions,
// which lie in one page.
#include "gfwa_internal.h"
#include "head_rows.h"

namespace gfwa {

namespace {

constexpr int kUnit = 16;       // positions of a unit; pages are multiples of it
constexpr int kChunkUnits = 16; // a chunk of the window is a multiple of this many units
constexpr float kNone = -1.0e30f;

// Partial result of one (query head, chunk): D output columns (not yet divided by the sum), the exponent they are scaled
// by (log2 domain) and the sum.
__host__ __device__ constexpr int record(int D) { return D + 2; }

struct PagedArgs {
    const void *q, *Kp, *Vp;
    const float* cp;
    const int *table, *pos;
    void* o;
    float *L, *part;
    int H, Hkv, pages, page, max_pages, w;
    float scale;
    int splits, chunk;  // chunks of the window and units of one
};

// A sequence's query position and what of its prefix and window is there.
struct Query {
    int p, lo, page, row;  // page -1: no token
    __device__ __forceinline__ Query(const PagedArgs& a, int b) {
        p = min(a.pos[b], a.max_pages * a.page - 1);
        page = -1;
        row = lo = 0;
        if (p < 0) return;
        const int i = p / a.page;
        row = p - i * a.page;
        const int id = a.table[(size_t)b * a.max_pages + i];
        if (id >= 0 && id < a.pages) page = id;
        lo = max(0, p - a.w + 1);
    }
};

// One workgroup of four waves: GT query heads of one key/value head, one chunk of the window, every wave each fourth unit of it.  D / 8 lanes
// hold a row; every group of such lanes keeps its own running maximum and sum.
template <typename T, int D, int GT>
__global__ __launch_bounds__(256) void decode_paged_kernel(const PagedArgs a) {
    constexpr int LPR = D / 8, RPI = 64 / LPR, NW = 4;
    __shared__ __align__(16) float sm_acc[NW][GT][D];
    __shared__ float sm_m[NW][GT], sm_l[NW][GT];
    int idx = blockIdx.x;
    const int s = idx % a.splits;
    idx /= a.splits;
    const int G = a.H / a.Hkv, gchunks = G / GT, gc = idx % gchunks;
    idx /= gchunks;
    const int kvh = idx % a.Hkv, b = idx / a.Hkv;
    const int h0 = kvh * G + gc * GT;
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, r = lane / LPR, j = lane % LPR;
    const Query me(a, b);

    float acc[GT][8], m[GT], l[GT];
#pragma unroll
    for (int g = 0; g < GT; ++g) {
        m[g] = kNone;
        l[g] = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[g][e] = 0.f;
    }
    if (me.page >= 0) {
        float q[GT][8], c0[GT];
#pragma unroll
        for (int g = 0; g < GT; ++g) {
            Unit8<T> u;
            u.load((const T*)a.q + ((size_t)b * a.H + h0 + g) * D + 8 * j);
            u.get(q[g]);
            c0[g] = a.cp[((size_t)me.page * a.H + h0 + g) * a.page + me.row];
        }
        const int u0 = me.lo / kUnit + s * a.chunk, u1 = min(u0 + a.chunk, me.p / kUnit + 1);
        for (int u = u0 + wv; u < u1; u += NW) {
            const int i = u * kUnit / a.page, row0 = u * kUnit - i * a.page;
            const int id = a.table[(size_t)b * a.max_pages + i];
            if (id < 0 || id >= a.pages) continue;
            for (int k = r; k < kUnit; k += RPI) {
                const int key = u * kUnit + k;
                if (key < me.lo || key > me.p) continue;  // nothing of a row outside the window is read
                const size_t at = (((size_t)id * a.Hkv + kvh) * a.page + row0 + k) * D + 8 * j;
                Unit8<T> ku, vu;
                ku.load((const T*)a.Kp + at);
                vu.load((const T*)a.Vp + at);
                float x[8], v[8];
                ku.get(x);
                vu.get(v);
#pragma unroll
                for (int g = 0; g < GT; ++g) {
                    float dot = 0.f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) dot = fmaf(q[g][e], x[e], dot);
#pragma unroll
                    for (int off = 1; off < LPR; off <<= 1) dot += __shfl_xor(dot, off, 64);
                    const float c = a.cp[((size_t)id * a.H + h0 + g) * a.page + row0 + k];
                    const float sc = (dot * a.scale + (c - c0[g])) * kLog2e;
                    const float mn = fmaxf(m[g], sc), f = fast_exp2(m[g] - mn), e2 = fast_exp2(sc - mn);
                    l[g] = fmaf(l[g], f, e2);
#pragma unroll
                    for (int e = 0; e < 8; ++e) acc[g][e] = fmaf(acc[g][e], f, e2 * v[e]);
                    m[g] = mn;
                }
            }
        }
    }
    // over the lane groups of the wave, then over the waves
#pragma unroll
    for (int g = 0; g < GT; ++g) {
#pragma unroll
        for (int off = LPR; off < 64; off <<= 1) {
            const float mo = __shfl_xor(m[g], off, 64), lo = __shfl_xor(l[g], off, 64), mn = fmaxf(m[g], mo);
            const float f = fast_exp2(m[g] - mn), fo = fast_exp2(mo - mn);
            l[g] = l[g] * f + lo * fo;
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[g][e] = acc[g][e] * f + __shfl_xor(acc[g][e], off, 64) * fo;
            m[g] = mn;
        }
        if (r == 0) {
#pragma unroll
            for (int e = 0; e < 8; ++e) sm_acc[wv][g][8 * j + e] = acc[g][e];
            if (j == 0) {
                sm_m[wv][g] = m[g];
                sm_l[wv][g] = l[g];
            }
        }
    }
    __syncthreads();
    for (int x = threadIdx.x; x < GT * D; x += 64 * NW) {
        const int g = x / D, col = x % D;
        float mm = kNone, ll = 0.f, oo = 0.f;
#pragma unroll
        for (int k = 0; k < NW; ++k) mm = fmaxf(mm, sm_m[k][g]);
#pragma unroll
        for (int k = 0; k < NW; ++k) {
            const float f = fast_exp2(sm_m[k][g] - mm);
            ll = fmaf(sm_l[k][g], f, ll);
            oo = fmaf(sm_acc[k][g][col], f, oo);
        }
        const size_t bh = (size_t)b * a.H + h0 + g;
        if (a.splits == 1) {
            ((T*)a.o)[bh * D + col] = (T)(ll == 0.f ? 0.f : oo / ll);
            if (a.L != nullptr && col == 0) a.L[bh] = ll == 0.f ? -INFINITY : (mm + log2f(ll)) * kLn2;
        } else {
            float* rec = a.part + (bh * a.splits + s) * record(D);
            rec[col] = oo;
            if (col == 0) {
                rec[D] = mm;
                rec[D + 1] = ll;
            }
        }
    }
}

// o = sum_s acc_s 2^(m_s - M) / sum_s l_s 2^(m_s - M),  L = (M + log2 of that sum) ln 2
template <typename T, int D>
__global__ __launch_bounds__(D) void decode_paged_combine_kernel(const float* __restrict__ part, T* __restrict__ o, float* __restrict__ L, int S) {
    const size_t bh = blockIdx.x;
    const int col = threadIdx.x;
    const float* rec = part + bh * S * record(D);
    float mm = kNone, ll = 0.f, oo = 0.f;
    for (int s = 0; s < S; ++s) {
        const float* x = rec + (size_t)s * record(D);
        const float mn = fmaxf(mm, x[D]), f0 = fast_exp2(mm - mn), f = fast_exp2(x[D] - mn);
        ll = ll * f0 + x[D + 1] * f;
        oo = oo * f0 + x[col] * f;
        mm = mn;
    }
    o[bh * D + col] = (T)(ll == 0.f ? 0.f : oo / ll);
    if (L != nullptr && col == 0) L[bh] = ll == 0.f ? -INFINITY : (mm + log2f(ll)) * kLn2;
}

// Units a window may touch, and the most chunks it is cut into.
int most_units(int page, int max_pages, int w) {
    const long long keys = (long long)max_pages * page;
    const long long span = w < keys ? w : keys;
    return (int)((span + kUnit - 2) / kUnit + 1);  // a window may begin inside a unit
}

// How a step is cut up; follows from the sizes alone, as the workspace does.
struct Plan {
    int GT, chunk, splits;  // query heads of a workgroup, units of a chunk, chunks
    long long items;        // workgroups of one chunk
    Plan(int B, int H, int Hkv, int page, int max_pages, int w) {
        const int G = H / Hkv, units = most_units(page, max_pages, w);
        GT = G % 4 == 0 ? 4 : (G % 2 == 0 ? 2 : 1);
        items = (long long)B * Hkv * (G / GT);
        const long long want = 4LL * 256, S = (want + items - 1) / items;
        chunk = (int)(((units + S - 1) / S + kChunkUnits - 1) / kChunkUnits * kChunkUnits);
        splits = (units + chunk - 1) / chunk;
    }
};

}  // namespace

size_t decode_paged_workspace_bytes(int B, int H, int Hkv, int d, int page, int max_pages, int w) {
    return (size_t)B * H * Plan(B, H, Hkv, page, max_pages, w).splits * record(d) * sizeof(float);
}

template <typename T, int D>
static hipError_t launch(const PagedArgs& given, int B, hipStream_t s) {
    PagedArgs a = given;
    const Plan plan(B, a.H, a.Hkv, a.page, a.max_pages, a.w);
    a.chunk = plan.chunk;
    a.splits = plan.splits;
    {
        ProfScope prof(kKernDecodePaged, s);
        auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)(plan.items * a.splits)), dim3(256), 0, s, a); };
        plan.GT == 4 ? go(decode_paged_kernel<T, D, 4>) : plan.GT == 2 ? go(decode_paged_kernel<T, D, 2>) : go(decode_paged_kernel<T, D, 1>);
    }
    if (a.splits > 1) {
        ProfScope prof(kKernDecodePagedCombine, s);
        hipLaunchKernelGGL((decode_paged_combine_kernel<T, D>), dim3(B * a.H), dim3(D), 0, s, a.part, (T*)a.o, a.L, a.splits);
    }
    return hipGetLastError();
}

hipError_t decode_paged(bool bf16, const void* q, const PagedCache& cache, const int* pos, void* o, float* L, float* part, int B, int H, int Hkv,
                        int d, int w, float scale, hipStream_t s) {
    PagedArgs a{};
    a.q = q;
    a.Kp = cache.Kp;
    a.Vp = cache.Vp;
    a.cp = cache.cp;
    a.table = cache.table;
    a.pos = pos;
    a.o = o;
    a.L = L;
    a.part = part;
    a.H = H;
    a.Hkv = Hkv;
    a.pages = cache.pages;
    a.page = cache.page;
    a.max_pages = cache.max_pages;
    a.w = w;
    a.scale = scale;
    if (bf16) return d == 128 ? launch<bf16_t, 128>(a, B, s) : launch<bf16_t, 64>(a, B, s);
    return d == 128 ? launch<float, 128>(a, B, s) : launch<float, 64>(a, B, s);
}

}  // namespace gfwa
