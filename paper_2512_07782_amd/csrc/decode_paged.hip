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
constexpr int kTileWaves = 4;   // waves of a workgroup on the matrix cores
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
    int splits, chunk;  // chunks of the window and units (bf16: tiles) of one
    int units_shift;    // log2 of the units of a page, -1: no power of two
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

// ---- bf16: both products on the matrix cores
//
// A wave takes tiles of two units (32 keys), newest first, for up to 16 query heads of one key/value head:
//   S  [16 keys x 16 heads] = K [16 x D] Q^T          for each unit; K straight from memory in the A operand's layout (row: lane % 16)
//   O^T[D x 16 heads]      += V^T [D x 32 keys] P^T   P as it leaves S: lane (head, g) has the keys 4 g + 0..3 of both units, which is
//                                                     a B operand for a contraction over the keys in that order; V^T through LDS, which
//                                                     hands out transposed pieces in the same order
// Weights are rounded to bf16 on their way into the second product (half a step, 2^-8 of each, is what an output is rounded by too); their sum is
// that of the unrounded ones.  Heads past the group's are computed along on zeros; the matrix cores take 256 of the about 1700 cycles that
// a compute unit's share of the memory's rate gives the tile's 16 KiB (D = 128).
// A head's weights are taken against a reference that is raised, and sums rescaled, only when a score exceeds it by 2^16.
// Loads of the next tile are on their way while a tile is worked on.
template <int D>
struct VTile {  // 32 keys of V in LDS, 16-byte chunks permuted so that neither the row-wise writes nor the transposed reads meet in a bank
    static constexpr int kBytes = 32 * D * 2;
    static __device__ __forceinline__ int off(int row, int chunk) {
        const int f = D == 128 ? ((row & 3) << 2 | ((row >> 2) & 1) << 1 | ((row >> 3) & 1))
                               : (((row >> 1) & 1) << 2 | ((row >> 2) & 1) << 1 | ((row >> 3) & 1));  // two rows share the banks' width
        return row * (D * 2) + ((chunk ^ f) << 4);
    }
};

typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));

template <int D, int NW>
__global__ __launch_bounds__(64 * NW, 2) void decode_paged_mfma_kernel(const PagedArgs a) {
    constexpr int KS = D / 32, DT = D / 16, CPR = D / 8, RPI = 64 / CPR, VL = 32 / RPI;  // VL: loads of a lane for 32 rows of V
    constexpr int kHeads = 16, kPitch = D + 4;  // floats between the heads' sums when the waves merge
    constexpr int kWave = VTile<D>::kBytes > kHeads * kPitch * 4 ? VTile<D>::kBytes : kHeads * kPitch * 4;
    __shared__ __align__(16) char lds[NW * kWave];
    __shared__ float sm_m[NW][kHeads], sm_l[NW][kHeads];
    int idx = blockIdx.x;
    const int s = idx % a.splits;
    idx /= a.splits;
    const int G = a.H / a.Hkv, gchunks = (G + kHeads - 1) / kHeads, gc = idx % gchunks;
    idx /= gchunks;
    const int kvh = idx % a.Hkv, b = idx / a.Hkv;
    const int GT = min(kHeads, G - gc * kHeads), h0 = kvh * G + gc * kHeads;
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int hd = lane & 15, g = lane >> 4, head = h0 + min(hd, GT - 1);
    const Query me(a, b);

    f32x4 acc[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = kNone, sum = 0.f;  // reference of the lane's head; its weights' sum over the lane's keys
    char* const mine = lds + wv * kWave;

    // the tiles of this chunk, counted from the newest unit back
    const int u_hi = me.p / kUnit, u_lo = me.lo / kUnit;
    const int t1 = me.page < 0 ? 0 : min((s + 1) * a.chunk, (u_hi - u_lo) / 2 + 1);
    int t = s * a.chunk + wv;
    if (t < t1) {
        const bf16_t* const K = (const bf16_t*)a.Kp + (size_t)kvh * a.page * D;
        const bf16_t* const V = (const bf16_t*)a.Vp + (size_t)kvh * a.page * D;
        const float* const C = a.cp + (size_t)head * a.page;
        const int* const table = a.table + (size_t)b * a.max_pages;
        const float c0 = C[(size_t)me.page * a.H * a.page + me.row], to_log2 = a.scale * kLog2e;
        bf16x8 q[KS];
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            q[k] = *reinterpret_cast<const bf16x8*>((const bf16_t*)a.q + ((size_t)b * a.H + head) * D + 32 * k + 8 * g);
            if (hd >= GT) q[k] = bf16x8{};
        }
        // page and first row of a unit; one in front of the window, or whose page is not there: the query's own page, masked
        struct Unit {
            int page, row;
            bool there;
        };
        auto unit = [&](int u) __attribute__((always_inline)) {
            Unit x{me.page, 0, false};
            if (u < u_lo) return x;
            const int i = a.units_shift >= 0 ? u >> a.units_shift : u / (a.page / kUnit);
            const int id = __builtin_amdgcn_readfirstlane(table[i]);
            if (id >= 0 && id < a.pages) x = Unit{id, u * kUnit - i * a.page, true};
            return x;
        };
        bf16x8 kf[2][KS], vf[VL];
        f32x4_any cf[2];
        bool there[2];
        const int vrow = lane / CPR, vcol = lane % CPR;
        auto issue = [&](const Unit (&x)[2]) __attribute__((always_inline)) {
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                there[n] = x[n].there;
                const size_t at = ((size_t)x[n].page * a.Hkv * a.page + x[n].row) * D;
#pragma unroll
                for (int k = 0; k < KS; ++k) kf[n][k] = *reinterpret_cast<const bf16x8*>(K + at + hd * D + 32 * k + 8 * g);
                cf[n] = *reinterpret_cast<const f32x4_any*>(C + (size_t)x[n].page * a.H * a.page + x[n].row + 4 * g);
#pragma unroll
                for (int i = 0; i < VL / 2; ++i)
                    vf[n * (VL / 2) + i] = *reinterpret_cast<const bf16x8*>(V + at + (i * RPI + vrow) * D + 8 * vcol);
            }
        };
        Unit next[2] = {unit(u_hi - 2 * t), unit(u_hi - 2 * t - 1)};
        issue(next);
        if (t + NW < t1) {
            next[0] = unit(u_hi - 2 * (t + NW));
            next[1] = unit(u_hi - 2 * (t + NW) - 1);
        }
        for (; t < t1; t += NW) {
            const int key0 = (u_hi - 2 * t) * kUnit, key1 = key0 - kUnit;  // first keys of the two units
            const bool whole = there[0] && there[1] && key1 >= me.lo && key0 + kUnit - 1 <= me.p;
            if (!whole) {  // values of masked keys do not enter the product, whatever they are
#pragma unroll
                for (int i = 0; i < VL; ++i) {
                    const int n = i / (VL / 2), key = (n ? key1 : key0) + (i % (VL / 2)) * RPI + vrow;
                    if (!(there[n] && key >= me.lo && key <= me.p)) vf[i] = bf16x8{};
                }
            }
#pragma unroll
            for (int i = 0; i < VL; ++i) *reinterpret_cast<bf16x8*>(mine + VTile<D>::off(i * RPI + vrow, vcol)) = vf[i];
            f32x4 sc[2];
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                sc[n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = 0; k < KS; ++k) sc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[n][k], q[k], sc[n], 0, 0, 0);
            }
            float bias[2][4];
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) bias[n][e] = (cf[n][e] - c0) * kLog2e;
            const bool was[2] = {there[0], there[1]};
            if (t + NW < t1) {
                issue(next);
                if (t + 2 * NW < t1) {
                    next[0] = unit(u_hi - 2 * (t + 2 * NW));
                    next[1] = unit(u_hi - 2 * (t + 2 * NW) - 1);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            float top = -INFINITY;
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float x = fmaf(sc[n][e], to_log2, bias[n][e]);
                    const int key = (n ? key1 : key0) + 4 * g + e;
                    if (!whole) x = was[n] && key >= me.lo && key <= me.p ? x : -INFINITY;
                    sc[n][e] = x;
                    top = fmaxf(top, x);
                }
            if (__any(top > m + 16.f)) {
                auto r32 = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
                top = fmaxf(__uint_as_float(r32[0]), __uint_as_float(r32[1]));
                auto r16 = __builtin_amdgcn_permlane16_swap(__float_as_uint(top), __float_as_uint(top), false, false);
                top = fmaxf(__uint_as_float(r16[0]), __uint_as_float(r16[1]));
                const float mn = fmaxf(m, top), f = fast_exp2(m - mn);
                m = mn;
#pragma unroll
                for (int i = 0; i < DT; ++i) acc[i] *= f;
                sum *= f;
            }
            bf16x8 pr;
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float x = fast_exp2(sc[n][e] - m);
                    sum += x;
                    pr[4 * n + e] = (bf16_t)x;
                }
            asm volatile("" ::: "memory");
#pragma unroll
            for (int i = 0; i < DT; ++i) {
                const int row = 4 * g + (hd >> 2), col = 16 * i + 4 * (hd & 3);
                const char* const at = mine + (col & 7) * 2;
                const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + VTile<D>::off(row, col >> 3)));
                const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + VTile<D>::off(16 + row, col >> 3)));
                typedef short s16x8 __attribute__((ext_vector_type(8)));
                const s16x8 v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v), pr, acc[i], 0, 0, 0);
            }
            asm volatile("" ::: "memory");
        }
    }
    // over the waves, through the space of their tiles
    float* const out = reinterpret_cast<float*>(mine);
#pragma unroll
    for (int i = 0; i < DT; ++i) *reinterpret_cast<f32x4*>(out + hd * kPitch + 16 * i + 4 * g) = acc[i];
    {
        auto r32 = __builtin_amdgcn_permlane32_swap(__float_as_uint(sum), __float_as_uint(sum), false, false);
        sum = __uint_as_float(r32[0]) + __uint_as_float(r32[1]);
        auto r16 = __builtin_amdgcn_permlane16_swap(__float_as_uint(sum), __float_as_uint(sum), false, false);
        sum = __uint_as_float(r16[0]) + __uint_as_float(r16[1]);
    }
    if (g == 0) {
        sm_m[wv][hd] = m;
        sm_l[wv][hd] = sum;
    }
    __syncthreads();
    for (int x = threadIdx.x; x < GT * D; x += 64 * NW) {
        const int h = x / D, col = x % D;
        float mm = kNone, ll = 0.f, oo = 0.f;
#pragma unroll
        for (int k = 0; k < NW; ++k) mm = fmaxf(mm, sm_m[k][h]);
#pragma unroll
        for (int k = 0; k < NW; ++k) {
            const float f = fast_exp2(sm_m[k][h] - mm);
            ll = fmaf(sm_l[k][h], f, ll);
            oo = fmaf(reinterpret_cast<const float*>(lds + k * kWave)[h * kPitch + col], f, oo);
        }
        const size_t bh = (size_t)b * a.H + h0 + h;
        if (a.splits == 1) {
            ((bf16_t*)a.o)[bh * D + col] = (bf16_t)(ll == 0.f ? 0.f : oo / ll);
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

// ---- fp32

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
    int GT, chunk, splits;  // query heads of a workgroup, units (bf16: tiles) of a chunk, chunks
    long long items;        // workgroups of one chunk
    Plan(bool bf16, int B, int H, int Hkv, int page, int max_pages, int w) {
        const int G = H / Hkv, units = most_units(page, max_pages, w);
        if (bf16) {
            const int tiles = units / 2 + 1;
            GT = 16;
            items = (long long)B * Hkv * ((G + 15) / 16);
            long long S = (512 + items - 1) / items;  // two workgroups of four waves for each compute unit
            if (S > (tiles + kTileWaves - 1) / kTileWaves) S = (tiles + kTileWaves - 1) / kTileWaves;
            chunk = (int)(((tiles + S - 1) / S + kTileWaves - 1) / kTileWaves * kTileWaves);
            splits = (tiles + chunk - 1) / chunk;
            return;
        }
        GT = G % 4 == 0 ? 4 : (G % 2 == 0 ? 2 : 1);
        items = (long long)B * Hkv * (G / GT);
        const long long want = 4LL * 256, S = (want + items - 1) / items;
        chunk = (int)(((units + S - 1) / S + kChunkUnits - 1) / kChunkUnits * kChunkUnits);
        splits = (units + chunk - 1) / chunk;
    }
};

}  // namespace

size_t decode_paged_workspace_bytes(int B, int H, int Hkv, int d, int page, int max_pages, int w) {
    const int f32 = Plan(false, B, H, Hkv, page, max_pages, w).splits, bf16 = Plan(true, B, H, Hkv, page, max_pages, w).splits;
    return (size_t)B * H * (f32 > bf16 ? f32 : bf16) * record(d) * sizeof(float);
}

template <typename T, int D>
static hipError_t launch(const PagedArgs& given, int B, hipStream_t s) {
    PagedArgs a = given;
    constexpr bool kShort = sizeof(T) == 2;
    const Plan plan(kShort, B, a.H, a.Hkv, a.page, a.max_pages, a.w);
    a.chunk = plan.chunk;
    a.splits = plan.splits;
    {
        ProfScope prof(kKernDecodePaged, s);
        auto go = [&](auto kernel, int threads) { hipLaunchKernelGGL(kernel, dim3((unsigned)(plan.items * a.splits)), dim3(threads), 0, s, a); };
        if constexpr (kShort) go(decode_paged_mfma_kernel<D, kTileWaves>, 64 * kTileWaves);
        else plan.GT == 4 ? go(decode_paged_kernel<T, D, 4>, 256) : plan.GT == 2 ? go(decode_paged_kernel<T, D, 2>, 256) : go(decode_paged_kernel<T, D, 1>, 256);
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
    const int units = cache.page / kUnit;
    a.units_shift = (units & (units - 1)) == 0 ? __builtin_ctz(units) : -1;
    if (bf16) return d == 128 ? launch<bf16_t, 128>(a, B, s) : launch<bf16_t, 64>(a, B, s);
    return d == 128 ? launch<float, 128>(a, B, s) : launch<float, 64>(a, B, s);
}

}  // namespace gfwa
