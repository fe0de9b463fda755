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
constexpr float kNone = -3.0e38f;  // reference of no key yet: finite, so that differences of references are numbers, and below every score that counts

constexpr int kFewChunks = 16;  // chunks whose records all are written and merged by one group of threads (two rounds of loads)
constexpr long long kOnceWindows = 24 << 20;  // windows of more than this in all are not met in the L2s (32 MiB) again

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
    int splits, waves;  // chunks a window may be cut into, and waves of a workgroup
    int least, chunk;   // tiles of a chunk: at least, and at most
    int items;          // workgroups of one chunk
    int units_shift;    // log2 of the units of a page, -1: no power of two
};

// Tiles of a chunk of a window of `tiles`: what the longest window is cut into; but a sequence of less than an eighth of that (a table has columns
// for the longest one there may be) is cut into all the chunks there are, none smaller than the least.  (Eight sequences of 1000 tokens, H 32, Hkv 8,
// d 128, without a window in a table for 131072: 24.4 us in one chunk each, 13.5 in five.  Every sequence like that: 16 of up to 8192 in fp32 127 us
// against 125.)
__device__ __forceinline__ int chunk_of(const PagedArgs& a, int tiles) {
    if (tiles >= a.chunk * (long long)a.splits / 8) return a.chunk;
    const int c = ((tiles + a.splits - 1) / a.splits + a.waves - 1) / a.waves * a.waves;
    return min(max(c, a.least), a.chunk);
}

// A sequence's query position, the first position of its window, and once looked up the page and row that hold the query position.
struct Query {
    int p, lo, page = -1, row = 0;  // p < 0, or page -1: no token
    __device__ __forceinline__ Query(const PagedArgs& a, int b) {
        p = min(a.pos[b], a.max_pages * a.page - 1);
        lo = p < 0 ? 0 : max(0, p - a.w + 1);
    }
    // tiles of U units that the window touches
    template <int U>
    __device__ __forceinline__ int tiles() const {
        return p < 0 ? 0 : (p / kUnit - lo / kUnit) / U + 1;
    }
    __device__ __forceinline__ void look_up(const PagedArgs& a, int b) {
        if (p < 0) return;
        const int i = p / a.page, id = a.table[(size_t)b * a.max_pages + i];
        row = p - i * a.page;
        if (id >= 0 && id < a.pages) page = id;
    }
};

// Both products are on the matrix cores, 16x16 blocks, for up to 16 query heads of one key/value head:
//   S  [16 keys x 16 heads] = K [16 x D] Q^T           K as the A operand straight from memory (row: lane % 16)
//   O^T[D x 16 heads]      += V^T [D x keys] P^T       P as it leaves S: lane (head, g) has the keys 4 g + 0..3 of a unit
// A contraction may take its terms in any order, as long as both operands do: K and Q are taken 16 bytes a lane, and the keys in the order in which
// P's lanes have them, so neither is moved between lanes.  Heads past the group's are computed along on zeros.

// What differs between the storage types: a tile of UNITS units in registers, and its two products.
template <typename T, int D>
struct Tile;

// bf16 (16x16x32): two units make the 32 keys of the second product.  V^T goes through LDS, which hands out transposed pieces in P's order, 16-byte chunks
// permuted so that neither the row-wise writes nor the transposed reads meet in a bank.  A weight enters the product as two bf16 numbers, cut off and the
// rest, off by 2^-16 of it at most: one alone would be off by 2^-8, as much as the output's own rounding (against fp64, norm of the difference 1.9e-3 to
// 2.6e-3 instead of 1.7e-3; 64 sequences, w 1024, 45.2 us with one, 45.4 with two, one 7.6 and 7.75).  Neither part is negative, and the rest of a weight that is not zero is not
// zero either (2^-133 at least): an infinity among the values stays one, where the rest of a rounded weight would make 0 inf or inf - inf of it.  The matrix cores
// take 384 of the about 1700 cycles that a compute unit's share of the memory's rate gives the tile's 16 KiB (D = 128).
template <int D>
struct Tile<bf16_t, D> {
    static constexpr int kUnits = 2, kLds = 32 * D * 2;
    static constexpr int KS = D / 32, DT = D / 16, CPR = D / 8, RPI = 64 / CPR, VU = kUnit / RPI;  // CPR: chunks of a row, RPI: rows of a load
    bf16x8 k[kUnits][KS], v[kUnits][VU];
    struct Queries {
        bf16x8 x[KS];
        __device__ __forceinline__ void load(const bf16_t* q, int g, bool there) {
#pragma unroll
            for (int i = 0; i < KS; ++i) {
                x[i] = *reinterpret_cast<const bf16x8*>(q + 32 * i + 8 * g);
                if (!there) x[i] = bf16x8{};
            }
        }
    };
    template <bool ONCE>
    __device__ __forceinline__ void load(int n, const bf16_t* K, const bf16_t* V, int lane) {
#pragma unroll
        for (int i = 0; i < KS; ++i) k[n][i] = *reinterpret_cast<const bf16x8*>(K + (lane & 15) * D + 32 * i + 8 * (lane >> 4));
#pragma unroll
        for (int i = 0; i < VU; ++i) {
            const bf16x8* const from = reinterpret_cast<const bf16x8*>(V + (i * RPI + lane / CPR) * D + 8 * (lane % CPR));
            if constexpr (ONCE) v[n][i] = __builtin_nontemporal_load(from);
            else v[n][i] = *from;
        }
    }
    // values of masked keys do not enter the product, whatever they are.  there(k): key k of the unit counts
    template <typename F>
    __device__ __forceinline__ void mask(int n, int lane, F&& there) {
#pragma unroll
        for (int i = 0; i < VU; ++i)
            if (!there(i * RPI + lane / CPR)) v[n][i] = bf16x8{};
    }
    static __device__ __forceinline__ int off(int row, int chunk) {
        const int f = D == 128 ? ((row & 3) << 2 | ((row >> 2) & 1) << 1 | ((row >> 3) & 1))
                               : (((row >> 1) & 1) << 2 | ((row >> 2) & 1) << 1 | ((row >> 3) & 1));  // two rows share the banks' width
        return row * (D * 2) + ((chunk ^ f) << 4);
    }
    __device__ __forceinline__ void scores(f32x4 (&s)[kUnits], const Queries& q, char* lds, int lane) const {
#pragma unroll
        for (int n = 0; n < kUnits; ++n)
#pragma unroll
            for (int i = 0; i < VU; ++i) *reinterpret_cast<bf16x8*>(lds + off(n * kUnit + i * RPI + lane / CPR, lane % CPR)) = v[n][i];
#pragma unroll
        for (int n = 0; n < kUnits; ++n) {
            s[n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < KS; ++i) s[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[n][i], q.x[i], s[n], 0, 0, 0);
        }
    }
    struct Values {};  // in LDS
    __device__ __forceinline__ Values values() const { return {}; }
    static __device__ __forceinline__ void add(f32x4 (&acc)[DT], const f32x4 (&p)[kUnits], const Values&, const char* lds, int lane) {
        const int g = lane >> 4, hd = lane & 15;
        typedef unsigned short u16x8 __attribute__((ext_vector_type(8)));
        u16x8 cut;
        bf16x8 left;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float x = p[e / 4][e % 4];
            cut[e] = (unsigned short)(__float_as_uint(x) >> 16);
            left[e] = (bf16_t)(x - __uint_as_float(__float_as_uint(x) & 0xffff0000u));
        }
        const bf16x8 w = __builtin_bit_cast(bf16x8, cut);
        const bf16x8 rest = __builtin_bit_cast(bf16x8, __builtin_elementwise_max(__builtin_bit_cast(u16x8, left), __builtin_elementwise_min(cut, (u16x8)1)));
        asm volatile("" ::: "memory");
#pragma unroll
        for (int i = 0; i < DT; ++i) {
            const int row = 4 * g + (hd >> 2), col = 16 * i + 4 * (hd & 3);
            const char* const at = lds + (col & 7) * 2;
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + off(row, col >> 3)));
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + off(kUnit + row, col >> 3)));
            typedef short s16x8 __attribute__((ext_vector_type(8)));
            const s16x8 x = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
            acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), w, acc[i], 0, 0, 0);
            acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), rest, acc[i], 0, 0, 0);
        }
        asm volatile("" ::: "memory");
    }
    // O^T of the lane: head lane % 16, columns 16 i + 4 g + 0..3
    static __device__ __forceinline__ void put(float* out, const f32x4 (&acc)[DT], int lane) {
#pragma unroll
        for (int i = 0; i < DT; ++i) *reinterpret_cast<f32x4*>(out + 16 * i + 4 * (lane >> 4)) = acc[i];
    }
};

// fp32 (16x16x4, full fp32 products): step e of the second product takes the keys 4 g + e, so that a lane's V^T is element (key 4 g + e, column): four
// neighbouring columns of it, 64 h + 4 (lane % 16) + c, are one load and the rows of four of the product's tiles.  No LDS.  The matrix cores take
// 2048 cycles of each of the four SIMDs for 16 KiB (D = 128), a third of what the memory's rate gives them.
template <int D>
struct Tile<float, D> {
    static constexpr int kUnits = 1, kLds = 0;
    static constexpr int KS = D / 16, DT = D / 16, HS = D / 64;
    f32x4 k[1][KS], v[1][4][HS];
    struct Queries {
        f32x4 x[KS];
        __device__ __forceinline__ void load(const float* q, int g, bool there) {
#pragma unroll
            for (int i = 0; i < KS; ++i) {
                x[i] = *reinterpret_cast<const f32x4*>(q + 16 * i + 4 * g);
                if (!there) x[i] = f32x4{0.f, 0.f, 0.f, 0.f};
            }
        }
    };
    template <bool ONCE>
    __device__ __forceinline__ void load(int, const float* K, const float* V, int lane) {
#pragma unroll
        for (int i = 0; i < KS; ++i) k[0][i] = *reinterpret_cast<const f32x4*>(K + (lane & 15) * D + 16 * i + 4 * (lane >> 4));
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int h = 0; h < HS; ++h) {
                const f32x4* const from = reinterpret_cast<const f32x4*>(V + (4 * (lane >> 4) + e) * D + 64 * h + 4 * (lane & 15));
                if constexpr (ONCE) v[0][e][h] = __builtin_nontemporal_load(from);
                else v[0][e][h] = *from;
            }
    }
    template <typename F>
    __device__ __forceinline__ void mask(int, int lane, F&& there) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int h = 0; h < HS; ++h)
                if (!there(4 * (lane >> 4) + e)) v[0][e][h] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    __device__ __forceinline__ void scores(f32x4 (&s)[1], const Queries& q, char*, int) const {
        f32x4 part[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};  // two chains: each product waits for the one before it
#pragma unroll
        for (int i = 0; i < KS; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) part[e & 1] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[0][i][e], q.x[i][e], part[e & 1], 0, 0, 0);
        s[0] = part[0] + part[1];
    }
    struct Values {
        f32x4 x[4][HS];
    };
    __device__ __forceinline__ Values values() const {
        Values r;
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int h = 0; h < HS; ++h) r.x[e][h] = v[0][e][h];
        return r;
    }
    static __device__ __forceinline__ void add(f32x4 (&acc)[DT], const f32x4 (&p)[1], const Values& val, const char*, int) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int i = 0; i < DT; ++i) acc[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(val.x[e][i / 4][i % 4], p[0][e], acc[i], 0, 0, 0);
    }
    // tile 4 h + c, row 4 g + r of O^T: column 64 h + 16 g + 4 r + c
    static __device__ __forceinline__ void put(float* out, const f32x4 (&acc)[DT], int lane) {
#pragma unroll
        for (int h = 0; h < HS; ++h)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                *reinterpret_cast<f32x4*>(out + 64 * h + 16 * (lane >> 4) + 4 * r) = f32x4{acc[4 * h][r], acc[4 * h + 1][r], acc[4 * h + 2][r], acc[4 * h + 3][r]};
    }
};

typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));

// A workgroup takes one chunk of the window for up to 16 query heads of one key/value head, each wave every NW-th tile of it, newest first; loads of
// the next tile are on their way while a tile is worked on.  A head's weights are taken against a reference that is raised, and sums rescaled,
// only when a score exceeds it by 2^16.
// (The page numbers of the tile after that could be asked for ahead too: eight more registers, which bf16 at d = 128 does not have beside three waves a
// SIMD; when it was tried, whole sequences, H 32, Hkv 8, 4 of up to 8192 took 22.3 us with and 19.5 without, 16 of them 68.3 and 65.4, 128 windows of 512 keys
// 49.3 and 51.7.  Two tiles ahead: 22.1, 68.1 and 47.6, in fp32 past the registers.)
// ONCE: V is loaded past the caches.  No other workgroup reads it, and windows that no cache holds are read faster (us, bf16, H 32, Hkv 8, d 128,
// w 1024: 64 sequences 48.3 -> 45.4, 32 26.1 -> 22.4; fp32, 64 sequences 90 -> 83; H 32, Hkv 4, d 64, whole sequences of up to 16384 40.6 -> 34.3), those that
// the memory-side cache holds from call to call more slowly (12 sequences in three sets, 143 MB, 14.5 -> 15.0).  K's lines are asked for by two loads each:
// past the caches the 64 sequences take 48.3.
template <typename T, int D, int NW, bool ONCE>
__global__ __launch_bounds__(64 * NW, 2) void decode_paged_kernel(const PagedArgs a) {
    typedef Tile<T, D> Tl;
    constexpr int NU = Tl::kUnits, kHeads = 16, kPitch = D + 4;  // floats between the heads' sums when the waves merge
    constexpr int kWave = kHeads * kPitch * 4 > Tl::kLds ? kHeads * kPitch * 4 : Tl::kLds;
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
    Query me(a, b);
    const int tiles = me.tiles<NU>(), chunk = chunk_of(a, tiles);
    if (a.splits > 1 && s * chunk >= tiles) {  // nothing of the window here
        if (a.splits <= kFewChunks && (int)threadIdx.x < GT) {
            float* rec = a.part + (((size_t)b * a.H + h0 + threadIdx.x) * a.splits + s) * record(D);
            rec[D] = kNone;
            rec[D + 1] = 0.f;
        }
        return;
    }
    me.look_up(a, b);

    f32x4 acc[Tl::DT];
#pragma unroll
    for (int t = 0; t < Tl::DT; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = kNone, sum = 0.f;  // reference of the lane's head; its weights' sum over the lane's keys
    char* const mine = lds + wv * kWave;

    // the tiles of this chunk, counted from the newest unit back
    const int u_hi = me.p / kUnit, u_lo = me.lo / kUnit;
    const int t1 = me.page < 0 ? 0 : min((s + 1) * chunk, tiles);
    int t = s * chunk + wv;
    if (t < t1) {
        const T* const K = (const T*)a.Kp + (size_t)kvh * a.page * D;
        const T* const V = (const T*)a.Vp + (size_t)kvh * a.page * D;
        const float* const C = a.cp + (size_t)head * a.page;
        const int* const table = a.table + (size_t)b * a.max_pages;
        const float c0 = C[(size_t)me.page * a.H * a.page + me.row], to_log2 = a.scale * kLog2e;
        typename Tl::Queries q;
        q.load((const T*)a.q + ((size_t)b * a.H + head) * D, g, hd < GT);
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
        Tl tile;
        f32x4_any cf[NU];
        bool there[NU];
        auto issue = [&](int t) __attribute__((always_inline)) {
            Unit x[NU];
#pragma unroll
            for (int n = 0; n < NU; ++n) x[n] = unit(u_hi - NU * t - n);
#pragma unroll
            for (int n = 0; n < NU; ++n) {
                there[n] = x[n].there;
                const size_t at = ((size_t)x[n].page * a.Hkv * a.page + x[n].row) * D;
                tile.template load<ONCE>(n, K + at, V + at, lane);
                cf[n] = *reinterpret_cast<const f32x4_any*>(C + (size_t)x[n].page * a.H * a.page + x[n].row + 4 * g);
            }
        };
        issue(t);
        for (; t < t1; t += NW) {
            const int key0 = (u_hi - NU * t) * kUnit;  // first key of the newest unit
            bool whole = key0 - (NU - 1) * kUnit >= me.lo && key0 + kUnit - 1 <= me.p, was[NU];
#pragma unroll
            for (int n = 0; n < NU; ++n) {
                was[n] = there[n];
                whole = whole && there[n];
            }
            auto counts = [&](int n, int k) __attribute__((always_inline)) {
                const int key = key0 - n * kUnit + k;
                return was[n] && key >= me.lo && key <= me.p;
            };
            if (!whole) {
#pragma unroll
                for (int n = 0; n < NU; ++n) tile.mask(n, lane, [&](int k) { return counts(n, k); });
            }
            f32x4 sc[NU];
            float bias[NU][4];
            tile.scores(sc, q, mine, lane);
            const typename Tl::Values val = tile.values();
#pragma unroll
            for (int n = 0; n < NU; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) bias[n][e] = (cf[n][e] - c0) * kLog2e;
            if (t + NW < t1) issue(t + NW);
            __builtin_amdgcn_sched_barrier(0);
            float top = -INFINITY;
#pragma unroll
            for (int n = 0; n < NU; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float x = fmaf(sc[n][e], to_log2, bias[n][e]);
                    if (!whole) x = counts(n, 4 * g + e) ? x : -INFINITY;
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
                for (int i = 0; i < Tl::DT; ++i) acc[i] *= f;
                sum *= f;
            }
#pragma unroll
            for (int n = 0; n < NU; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    sc[n][e] = fast_exp2(sc[n][e] - m);
                    sum += sc[n][e];
                }
            Tl::add(acc, sc, val, mine, lane);
        }
    }
    // over the waves, through the space of their tiles
    Tl::put(reinterpret_cast<float*>(mine) + hd * kPitch, acc, lane);
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
// over the chunks.  NG groups of D threads take every NG-th record each.  Up to kFewChunks every chunk leaves a record, without sums where it holds
// nothing of the window; of more than that only those that do, and the merge asks for the position (H 32, Hkv 8, w 1024: without the look one
// conversation, nine chunks, 7.75 us instead of 7.84, eight 12.0 instead of 12.6; 16 whole sequences of H 32, Hkv 4, d 64 35.6 instead of 34.3).
template <typename T, int D, int NG>
__global__ __launch_bounds__(D * NG) void decode_paged_combine_kernel(const PagedArgs a) {
    __shared__ float sm_o[NG][D], sm_m[NG], sm_l[NG];
    const size_t bh = blockIdx.x;
    const int col = threadIdx.x % D, grp = threadIdx.x / D;
    int there = a.splits;
    if (NG > 1) {
        const Query me(a, (int)(bh / a.H));
        const int tiles = me.template tiles<Tile<T, D>::kUnits>(), chunk = chunk_of(a, tiles);
        there = (tiles + chunk - 1) / chunk;
    }
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
            oo = l[u] == 0.f ? oo : fmaf(x[u], f, oo);  // (no weight, no sums: an infinity there stays out)
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
    int waves;          // of a workgroup
    int chunk, splits;  // tiles of a chunk of the longest window, chunks
    int least;          // tiles of a chunk of shorter ones
    long long items;    // workgroups of one chunk
    Plan(bool bf16, int B, int H, int Hkv, int page, int max_pages, int w) {
        const int G = H / Hkv, units = most_units(page, max_pages, w), of = bf16 ? Tile<bf16_t, 128>::kUnits : Tile<float, 128>::kUnits;
        const int tiles = (units + of - 1) / of;
        items = (long long)B * Hkv * ((G + 15) / 16);
        waves = 4;
        // Measured (us, four and eight waves, graphs of 21 steps; H 32, Hkv 8, d 128 unless named):
        //   * a window shorter than the table is about as long for every sequence.  Where one chunk each gives every compute unit two
        //     workgroups of four waves that is best (64 sequences, w 1024: one chunk 45, two 53); with half of that, one of eight
        //     waves (32 sequences: 22.4; two chunks of four waves 25.2); with fewer, chunks for two workgroups (8: 12.0, for one 13.2).
        //   * whole sequences are of any length: chunks of two tiles a wave, or as many as make 4096 workgroups, level that (16 of up
        //     to 8192: 64; 512 workgroups 80; H 32, Hkv 4, d 64, up to 16384: 34 and 47).
        //   * a window of up to three tiles a wave goes in one chunk, without a merge: w 200, 300, 700 (one chunk / chunks of four waves) of 31 sequences
        //     8.4 / 11.3, 10.4 / 13.2, 17.2 / 20.0, of 16 7.3 / 9.2, 8.6 / 10.3, 14.7 either way, of 8 6.2 / 7.8, 8.5 either way, 13.3 / 10.6, of one 6.1 / 7.1,
        //     7.7 / 7.1, 11.9 / 7.3: up to about eight sequences windows of two and three tiles a wave would be better off in chunks.
        const bool even = w < (long long)max_pages * page;
        long long S = 1;
        least = waves;
        if (even && items >= 512) waves = 4;
        else if (tiles <= 24 || (even && items >= 256)) waves = 8;
        else {
            const long long want = even ? 512 : 4096;
            least = even ? waves : 2 * waves;
            S = (want + items - 1) / items;
            if (S > (tiles + least - 1) / least) S = (tiles + least - 1) / least;
        }
        chunk = (int)(((tiles + S - 1) / S + waves - 1) / waves * waves);
        splits = (tiles + chunk - 1) / chunk;
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
    const Plan plan(sizeof(T) == 2, B, a.H, a.Hkv, a.page, a.max_pages, a.w);
    a.chunk = plan.chunk;
    a.splits = plan.splits;
    a.least = plan.least;
    a.waves = plan.waves;
    a.items = (int)plan.items;
    {
        ProfScope prof(kKernDecodePaged, s);
        auto go = [&](auto kernel, int threads) { hipLaunchKernelGGL(kernel, dim3((unsigned)(plan.items * a.splits)), dim3(threads), 0, s, a); };
        const long long keys = (long long)a.max_pages * a.page, span = a.w < keys ? a.w : keys;
        const bool once = plan.items == (long long)B * a.Hkv && plan.items * span * D * 2 * (long long)sizeof(T) > kOnceWindows;
        if (plan.waves == 8) once ? go(decode_paged_kernel<T, D, 8, true>, 512) : go(decode_paged_kernel<T, D, 8, false>, 512);
        else once ? go(decode_paged_kernel<T, D, 4, true>, 256) : go(decode_paged_kernel<T, D, 4, false>, 256);
    }
    if (a.splits > 1) {
        ProfScope prof(kKernDecodePagedCombine, s);
        if (a.splits > kFewChunks) hipLaunchKernelGGL((decode_paged_combine_kernel<T, D, 4>), dim3(B * a.H), dim3(4 * D), 0, s, a);
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
