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
constexpr int kTileUnits = 2;  // bf16: units of a tile
constexpr long long kOnceBytes = 24 << 20;  // windows of more than this are loaded past the caches: the L2s hold 32 MiB
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
    int items;          // workgroups of one chunk
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
//   O^T[D x 16 heads]      += V^T [D x 32 keys] P^T   P as it leaves S: lane (head, g) has the keys 4 g + 0..3 of two units, which is
//                                                     a B operand for a contraction over the keys in that order; V^T through LDS, which
//                                                     hands out transposed pieces in the same order
// Weights are rounded to bf16 on their way into the second product (half a step, 2^-8 of each, is what an output is rounded by too); their sum is
// that of the unrounded ones.  Heads past the group's are computed along on zeros; the matrix cores take 256 of the about 1700 cycles that
// a compute unit's share of the memory's rate gives the tile's 16 KiB (D = 128).
// A head's weights are taken against a reference that is raised, and sums rescaled, only when a score exceeds it by 2^16.
// Loads of the next tile are on their way while a tile is worked on.
template <int D>
struct VTile {  // 32 keys of V in LDS, 16-byte chunks permuted so that neither the row-wise writes nor the transposed reads meet in a bank
    static constexpr int kBytes = kTileUnits * kUnit * D * 2;
    static __device__ __forceinline__ int off(int row, int chunk) {
        const int f = D == 128 ? ((row & 3) << 2 | ((row >> 2) & 1) << 1 | ((row >> 3) & 1))
                               : (((row >> 1) & 1) << 2 | ((row >> 2) & 1) << 1 | ((row >> 3) & 1));  // two rows share the banks' width
        return row * (D * 2) + ((chunk ^ f) << 4);
    }
};

typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));

// ONCE: V is loaded past the caches.  No other workgroup reads it, and a window that the L2s do not hold is read faster (us, H 32, Hkv 8, d 128,
// w 1024: 64 sequences 49.4 -> 46.0, 32 26.1 -> 22.8; H 32, Hkv 4, d 64, whole sequences of up to 16384 40.7 -> 33.8), one that they do hold more
// slowly (2 sequences of H 16, d 64, w 512, 4 MB, 6.7 -> 7.2).  K's lines are asked for by two loads each: past the caches 47.6 for the first.
template <int D, int NW, bool ONCE>
__global__ __launch_bounds__(64 * NW, 2) void decode_paged_mfma_kernel(const PagedArgs a) {
    constexpr int KS = D / 32, DT = D / 16, CPR = D / 8, RPI = 64 / CPR, NU = kTileUnits, VU = kUnit / RPI;  // VU: loads of a lane for a unit of V
    constexpr int kHeads = 16, kPitch = D + 4;  // floats between the heads' sums when the waves merge
    constexpr int kWave = kHeads * kPitch * 4 > VTile<D>::kBytes ? kHeads * kPitch * 4 : VTile<D>::kBytes;
    __shared__ __align__(16) char lds[NW * kWave];
    __shared__ float sm_m[NW][kHeads], sm_l[NW][kHeads];
    const int s = blockIdx.x / a.items;  // the newest chunks of all come first, those that short sequences do not have last
    int idx = (blockIdx.x - s * a.items + s) % a.items;  // a sequence's chunks on other XCDs
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
    const int t1 = me.page < 0 ? 0 : min((s + 1) * a.chunk, (u_hi - u_lo) / NU + 1);
    if (a.splits > 1 && s * a.chunk >= t1) return;  // the merge knows
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
        bf16x8 kf[NU][KS], vf[NU][VU];
        f32x4_any cf[NU];
        bool there[NU];
        Unit next[NU];
        const int vrow = lane / CPR, vcol = lane % CPR;
        auto look_up = [&](int tile) __attribute__((always_inline)) {
#pragma unroll
            for (int n = 0; n < NU; ++n) next[n] = unit(u_hi - NU * tile - n);
        };
        auto issue = [&]() __attribute__((always_inline)) {
#pragma unroll
            for (int n = 0; n < NU; ++n) {
                there[n] = next[n].there;
                const size_t at = ((size_t)next[n].page * a.Hkv * a.page + next[n].row) * D;
#pragma unroll
                for (int k = 0; k < KS; ++k) kf[n][k] = *reinterpret_cast<const bf16x8*>(K + at + hd * D + 32 * k + 8 * g);
                cf[n] = *reinterpret_cast<const f32x4_any*>(C + (size_t)next[n].page * a.H * a.page + next[n].row + 4 * g);
#pragma unroll
                for (int i = 0; i < VU; ++i) {
                    const bf16x8* const from = reinterpret_cast<const bf16x8*>(V + at + (i * RPI + vrow) * D + 8 * vcol);
                    if constexpr (ONCE) vf[n][i] = __builtin_nontemporal_load(from);
                    else vf[n][i] = *from;
                }
            }
        };
        look_up(t);
        issue();
        if (t + NW < t1) look_up(t + NW);
        for (; t < t1; t += NW) {
            const int key0 = (u_hi - NU * t) * kUnit;  // first key of the newest unit
            bool whole = key0 - (NU - 1) * kUnit >= me.lo && key0 + kUnit - 1 <= me.p, was[NU];
#pragma unroll
            for (int n = 0; n < NU; ++n) {
                was[n] = there[n];
                whole = whole && there[n];
            }
            if (!whole) {  // values of masked keys do not enter the product, whatever they are
#pragma unroll
                for (int n = 0; n < NU; ++n)
#pragma unroll
                    for (int i = 0; i < VU; ++i) {
                        const int key = key0 - n * kUnit + i * RPI + vrow;
                        if (!(there[n] && key >= me.lo && key <= me.p)) vf[n][i] = bf16x8{};
                    }
            }
#pragma unroll
            for (int n = 0; n < NU; ++n)
#pragma unroll
                for (int i = 0; i < VU; ++i) *reinterpret_cast<bf16x8*>(mine + VTile<D>::off(n * kUnit + i * RPI + vrow, vcol)) = vf[n][i];
            f32x4 sc[NU];
            float bias[NU][4];
#pragma unroll
            for (int n = 0; n < NU; ++n) {
                sc[n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = 0; k < KS; ++k) sc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[n][k], q[k], sc[n], 0, 0, 0);
#pragma unroll
                for (int e = 0; e < 4; ++e) bias[n][e] = (cf[n][e] - c0) * kLog2e;
            }
            if (t + NW < t1) {
                issue();
                if (t + 2 * NW < t1) look_up(t + 2 * NW);
            }
            __builtin_amdgcn_sched_barrier(0);
            float top = -INFINITY;
#pragma unroll
            for (int n = 0; n < NU; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float x = fmaf(sc[n][e], to_log2, bias[n][e]);
                    const int key = key0 - n * kUnit + 4 * g + e;
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
            asm volatile("" ::: "memory");
#pragma unroll
            for (int n = 0; n < NU; n += 2) {
                bf16x8 pr;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float x = fast_exp2(sc[n + e / 4][e % 4] - m);
                    sum += x;
                    pr[e] = (bf16_t)x;
                }
#pragma unroll
                for (int i = 0; i < DT; ++i) {
                    const int row = n * kUnit + 4 * g + (hd >> 2), col = 16 * i + 4 * (hd & 3);
                    const char* const at = mine + (col & 7) * 2;
                    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + VTile<D>::off(row, col >> 3)));
                    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + VTile<D>::off(kUnit + row, col >> 3)));
                    typedef short s16x8 __attribute__((ext_vector_type(8)));
                    const s16x8 v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                    acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v), pr, acc[i], 0, 0, 0);
                }
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
    const int s = blockIdx.x / a.items;
    int idx = (blockIdx.x - s * a.items + s) % a.items;
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
    if (a.splits > 1 && (me.page < 0 || s * a.chunk > me.p / kUnit - me.lo / kUnit)) return;  // the merge knows
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
// over the chunks that hold part of the window (the others write nothing).  NG groups of D threads take every NG-th record each.
template <typename T, int D, int NG>
__global__ __launch_bounds__(D * NG) void decode_paged_combine_kernel(const PagedArgs a) {
    __shared__ float sm_o[NG][D], sm_m[NG], sm_l[NG];
    const size_t bh = blockIdx.x;
    const int col = threadIdx.x % D, grp = threadIdx.x / D;
    const Query me(a, (int)(bh / a.H));
    const int pieces = me.page < 0 ? 0 : (me.p / kUnit - me.lo / kUnit) / (sizeof(T) == 2 ? kTileUnits : 1) + 1;
    const int there = (pieces + a.chunk - 1) / a.chunk;
    const float* rec = a.part + bh * a.splits * record(D);
    float mm = kNone, ll = 0.f, oo = 0.f;
    constexpr int U = 8;  // records whose loads are in flight together
    for (int s0 = grp; s0 < there; s0 += U * NG) {
        float m[U], l[U], x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float* r = rec + (size_t)min(s0 + u * NG, there - 1) * record(D);
            m[u] = r[D];
            l[u] = s0 + u * NG < there ? r[D + 1] : 0.f;
            x[u] = r[col];
        }
        float mn = mm;
#pragma unroll
        for (int u = 0; u < U; ++u) mn = fmaxf(mn, m[u]);
        const float f0 = fast_exp2(mm - mn);
        ll *= f0;
        oo *= f0;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float f = s0 + u * NG < there ? fast_exp2(m[u] - mn) : 0.f;
            ll = fmaf(l[u], f, ll);
            oo = fmaf(x[u], f, oo);
        }
        mm = mn;
    }
    if (NG > 1) {
        sm_o[grp][col] = oo;
        if (col == 0) {
            sm_m[grp] = mm;
            sm_l[grp] = ll;
        }
        __syncthreads();
        if (grp > 0) return;
        float mn = mm;
#pragma unroll
        for (int k = 1; k < NG; ++k) mn = fmaxf(mn, sm_m[k]);
        ll = oo = 0.f;
#pragma unroll
        for (int k = 0; k < NG; ++k) {
            const float f = fast_exp2(sm_m[k] - mn);
            ll = fmaf(sm_l[k], f, ll);
            oo = fmaf(sm_o[k][col], f, oo);
        }
        mm = mn;
    }
    ((T*)a.o)[bh * D + col] = (T)(ll == 0.f ? 0.f : oo / ll);
    if (a.L != nullptr && col == 0) a.L[bh] = ll == 0.f ? -INFINITY : (mm + log2f(ll)) * kLn2;
}

// Units a window may touch, and the most chunks it is cut into.
int most_units(int page, int max_pages, int w) {
    const long long keys = (long long)max_pages * page;
    const long long span = w < keys ? w : keys;
    return (int)((span + kUnit - 2) / kUnit + 1);  // a window may begin inside a unit
}

// How a step is cut up; follows from the sizes alone, as the workspace does.
struct Plan {
    int GT, waves;          // query heads (fp32) and waves of a workgroup
    int chunk, splits;      // units (bf16: tiles) of a chunk, chunks
    long long items;        // workgroups of one chunk
    Plan(bool bf16, int B, int H, int Hkv, int d, int page, int max_pages, int w) {
        const int G = H / Hkv, units = most_units(page, max_pages, w);
        waves = 4;
        if (bf16) {
            const int tiles = (units + kTileUnits - 1) / kTileUnits;
            items = (long long)B * Hkv * ((G + 15) / 16);
            // Measured (us, four and eight waves, graphs of 21 steps; H 32, Hkv 8, d 128 unless named):
            //   * a window shorter than the table is about as long for every sequence.  Where one chunk each gives every compute unit two
            //     workgroups of four waves that is best (64 sequences, w 1024: one chunk 49, two 54); with half of that, one of eight
            //     waves (32 sequences: 26; two chunks of four waves 29); with fewer, chunks for two workgroups (8: 11.8, for one 13.0).
            //   * whole sequences are of any length: chunks of two tiles a wave, or as many as make 4096 workgroups, level that (16 of up
            //     to 8192: 70; 512 workgroups 79; H 32, Hkv 4, d 64, up to 16384: 41 and 53).
            //   * a window of three tiles a wave is not worth the merge (300 keys of one sequence: 4.4, in three chunks 6.3).
            const bool even = w < (long long)max_pages * page;
            long long S = 1;
            if (even && items >= 512) waves = 4;
            else if (tiles <= 24 || (even && items >= 256)) waves = 8;
            else {
                const long long want = even ? 512 : 4096, least = even ? waves : 2 * waves;
                S = (want + items - 1) / items;
                if (S > (tiles + least - 1) / least) S = (tiles + least - 1) / least;
            }
            chunk = (int)(((tiles + S - 1) / S + waves - 1) / waves * waves);
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
    const int f32 = Plan(false, B, H, Hkv, d, page, max_pages, w).splits, bf16 = Plan(true, B, H, Hkv, d, page, max_pages, w).splits;
    return (size_t)B * H * (f32 > bf16 ? f32 : bf16) * record(d) * sizeof(float);
}

template <typename T, int D>
static hipError_t launch(const PagedArgs& given, int B, hipStream_t s) {
    PagedArgs a = given;
    constexpr bool kShort = sizeof(T) == 2;
    const Plan plan(kShort, B, a.H, a.Hkv, D, a.page, a.max_pages, a.w);
    a.chunk = plan.chunk;
    a.splits = plan.splits;
    a.items = (int)plan.items;
    {
        ProfScope prof(kKernDecodePaged, s);
        auto go = [&](auto kernel, int threads) { hipLaunchKernelGGL(kernel, dim3((unsigned)(plan.items * a.splits)), dim3(threads), 0, s, a); };
        if constexpr (kShort) {
            const long long keys = (long long)a.max_pages * a.page, span = a.w < keys ? a.w : keys;
            const bool once = plan.items == (long long)B * a.Hkv && plan.items * span * D * 2 * (long long)sizeof(T) > kOnceBytes;
            if (plan.waves == 8) once ? go(decode_paged_mfma_kernel<D, 8, true>, 512) : go(decode_paged_mfma_kernel<D, 8, false>, 512);
            else once ? go(decode_paged_mfma_kernel<D, 4, true>, 256) : go(decode_paged_mfma_kernel<D, 4, false>, 256);
        }
        else plan.GT == 4 ? go(decode_paged_kernel<T, D, 4>, 256) : plan.GT == 2 ? go(decode_paged_kernel<T, D, 2>, 256) : go(decode_paged_kernel<T, D, 1>, 256);
    }
    if (a.splits > 1) {
        ProfScope prof(kKernDecodePagedCombine, s);
        if (a.splits > 16) hipLaunchKernelGGL((decode_paged_combine_kernel<T, D, 4>), dim3(B * a.H), dim3(4 * D), 0, s, a);
        else hipLaunchKernelGGL((decode_paged_combine_kernel<T, D, 1>), dim3(B * a.H), dim3(D), 0, s, a);
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
