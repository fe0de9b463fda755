// New tokens of a batch of sequences into the paged key/value cache on gfx950: norm and rotation of their queries and keys, keys and
// values to their pages, and the gate's prefix carried on, in one launch.
//   * rows of queries, keys and values are held and worked on as in qk_norm_rope.hip; a row's sequence is looked up from the batch's
//     offsets and its page from the table, once for all its heads;
//   * the prefix is a scan along each sequence and goes to workgroups of its own, which the launch begins with (us, H 32, Hkv 8, d 128, one prompt of
//     8192 tokens: without gates 40.9, with the prefix in segments 48.4, by a wave for eight heads 190; 16 prompts of up to 2048 tokens 95.7 and 98.4).
#include "gfwa_internal.h"
#include "head_rows.h"

namespace gfwa {

namespace {

constexpr int kAppendWaves = 4;

struct AppendArgs {
    HeadsView q, k, v;
    const float *wq, *wk;
    float eps;
    const double* freq;
    int rot;
    bool norm, paired;
    const float* alpha;
    long long alpha_token, alpha_head;
    const int *start, *cached, *table;
    void *Q, *Kp, *Vp;
    float* cp;
    int rows, B, H, Hkv, pages, page, max_pages;
    int scan_blocks;   // workgroups of the prefix, in front
    int segments;      // pieces that a long sequence's prefix is cut into; 0: a wave for a whole sequence
    Shares shares;     // of tiles of 1024 / D rows
};

// The page that holds position p of sequence b, or -1: outside the table, or not there.
__device__ __forceinline__ int page_of(const AppendArgs& a, int b, long long p, int& row) {
    if (p < 0 || p >= (long long)a.max_pages * a.page) return -1;
    const int i = (int)p / a.page;
    row = (int)p - i * a.page;
    const int id = a.table[(size_t)b * a.max_pages + i];
    return id >= 0 && id < a.pages ? id : -1;
}

// The sequence b with start[b] <= row < start[b + 1], or -1, its first row and its tokens in the cache.  In a decoding step row b is sequence b's: that
// guess takes one round of loads where the search takes one for each halving of the batch.
__device__ __forceinline__ int sequence_of(const AppendArgs& a, int row, int& first, int& before) {
    const int guess = min(row, a.B - 1), next = a.start[guess + 1];
    first = a.start[guess];
    before = a.cached[guess];
    if ((first <= row) & (row < next)) return guess;
    int lo = 0, hi = a.B;
    while (hi - lo > 1) {
        const int mid = lo + (hi - lo) / 2;
        if (a.start[mid] <= row) lo = mid;
        else hi = mid;
    }
    first = a.start[lo];
    before = a.cached[lo];
    return first <= row && row < a.start[lo + 1] ? lo : -1;
}

// ---- the prefix: fp64 sums, each c rounded once

template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ double dpp_or_zero(double x) {  // lanes without a source, or in a row that ROWS leaves out, get 0
    typedef int i32x2 __attribute__((ext_vector_type(2)));
    const i32x2 v = __builtin_bit_cast(i32x2, x);
    return __builtin_bit_cast(double, i32x2{__builtin_amdgcn_update_dpp(0, v[0], CTRL, ROWS, 0xf, false),
                                            __builtin_amdgcn_update_dpp(0, v[1], CTRL, ROWS, 0xf, false)});
}
__device__ __forceinline__ double wave_scan(double x) {  // inclusive, over the 64 lanes
    x += dpp_or_zero<0x111>(x);
    x += dpp_or_zero<0x112>(x);
    x += dpp_or_zero<0x114>(x);
    x += dpp_or_zero<0x118>(x);
    x += dpp_or_zero<0x142, 0xa>(x);
    x += dpp_or_zero<0x143, 0xc>(x);
    return x;
}
__device__ __forceinline__ double lane_value(double x, int lane) {
    typedef int i32x2 __attribute__((ext_vector_type(2)));
    const i32x2 v = __builtin_bit_cast(i32x2, x);
    return __builtin_bit_cast(double, i32x2{__builtin_amdgcn_readlane(v[0], lane), __builtin_amdgcn_readlane(v[1], lane)});
}

constexpr int kScanHeads = 8;    // heads that are taken together
constexpr int kScanGroups = 8;   // groups of 64 tokens whose gates are on their way together
constexpr int kScanTokens = 64 * kScanGroups;

// A sequence's new rows n0 .. n1, how many tokens its cache holds, and the position of row 0, were it the sequence's.
struct NewTokens {
    int n0, n1;
    long long before, origin;
    __device__ __forceinline__ NewTokens(const AppendArgs& a, int b) {
        const int from = a.start[b], to = a.start[b + 1];
        n0 = min(max(from, 0), a.rows);
        n1 = min(max(to, n0), a.rows);
        before = a.cached[b];
        origin = before - from;
    }
};

// The prefix that sequence b's cache ends with.
__device__ __forceinline__ double cached_prefix(const AppendArgs& a, int b, long long before, int h) {
    int row = 0;
    const int id = page_of(a, b, before - 1, row);
    return id >= 0 ? (double)a.cp[((size_t)id * a.H + h) * a.page + row] : 0.0;
}

// c of the new tokens `from` .. `to` of sequence b for the heads h .. h + HEADS - 1, by one wave, 64 GROUPS tokens at a time; c: their prefixes in front
// of `from`.
template <int HEADS, int GROUPS>
__device__ __forceinline__ void prefix_heads(const AppendArgs& a, int b, const NewTokens& s, int h, int from, int to, double (&c)[HEADS]) {
    const int lane = threadIdx.x & 63;
    const long long last = (long long)a.max_pages * a.page - 1;
    for (int n = from; n < to; n += 64 * GROUPS) {
        float x[HEADS][GROUPS];
        int id[GROUPS], row[GROUPS];
#pragma unroll
        for (int u = 0; u < GROUPS; ++u) {  // (no condition at a load: all are on their way before the first one is waited for)
            const int t = min(n + 64 * u + lane, to - 1);
            const long long p = s.origin + t;
            const int at = (int)max(0LL, min(p, last)), i = at / a.page;
            row[u] = at - i * a.page;
            id[u] = a.table[(size_t)b * a.max_pages + i];
#pragma unroll
            for (int k = 0; k < HEADS; ++k) x[k][u] = a.alpha[t * a.alpha_token + min(h + k, a.H - 1) * a.alpha_head];
            if (p != at) row[u] = -1;  // outside the table
        }
#pragma unroll
        for (int u = 0; u < GROUPS; ++u) {
            const bool mine = n + 64 * u + lane < to, there = mine && row[u] >= 0 && id[u] >= 0 && id[u] < a.pages;
#pragma unroll
            for (int k = 0; k < HEADS; ++k) {
                const double sum = wave_scan(mine ? (double)x[k][u] : 0.0);
                if (there && h + k < a.H) a.cp[((size_t)id[u] * a.H + h + k) * a.page + row[u]] = (float)(c[k] + sum);
                c[k] += lane_value(sum, 63);
            }
        }
    }
}

// c of at most eight new tokens of sequence b for eight heads from h0 on, by one wave: a lane for each head and token.
constexpr int kFewTokens = 64 / kScanHeads;
__device__ void prefix_few(const AppendArgs& a, int b, const NewTokens& s, int h0) {
    const int lane = threadIdx.x & 63, t = lane / kScanHeads, h = h0 + lane % kScanHeads;
    const bool mine = s.n0 + t < s.n1 && h < a.H;
    int at = 0;
    const int id = mine ? page_of(a, b, s.origin + s.n0 + t, at) : -1;
    double c = mine ? a.alpha[(s.n0 + t) * a.alpha_token + h * a.alpha_head] : 0.f;
    if (s.n1 - s.n0 > 1) {
#pragma unroll
        for (int off = kScanHeads; off < 64; off *= 2) {
            const double x = __shfl_up(c, off, 64);
            if (lane >= off) c += x;
        }
    }
    if (!mine) return;
    c += cached_prefix(a, b, s.before, h);
    if (id >= 0) a.cp[((size_t)id * a.H + h) * a.page + at] = (float)c;
}

// c of all new tokens of sequence b for eight heads from h0 on, by one wave.
__device__ void prefix_short(const AppendArgs& a, int b, int h0) {
    const NewTokens s(a, b);
    if (s.n1 - s.n0 <= kFewTokens) return prefix_few(a, b, s, h0);
    double c[kScanHeads];
#pragma unroll
    for (int k = 0; k < kScanHeads; ++k) c[k] = cached_prefix(a, b, s.before, min(h0 + k, a.H - 1));
    prefix_heads<kScanHeads, 2>(a, b, s, h0, s.n0, s.n1, c);
}

// c of a segment of the new tokens of sequence b for eight heads from h0 on, by a workgroup: the gates in front of it are added up by all its threads (a
// line of them serves all eight heads), then every wave takes two heads.  Nothing waits for another workgroup; what that costs is that the gates
// are read as often as there are segments behind them.
__device__ void prefix_segment(const AppendArgs& a, int b, int h0, int segment) {
    const NewTokens s(a, b);
    const int n = s.n1 - s.n0, len = kScanTokens * ((n + kScanTokens * a.segments - 1) / (kScanTokens * a.segments));
    if (segment * len >= n) return;  // the same for the whole workgroup
    if (n <= kFewTokens) {
        if (threadIdx.x < 64) prefix_few(a, b, s, h0);
        return;
    }
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, from = s.n0 + segment * len;
    __shared__ double sums[kAppendWaves][kScanHeads];
    double sum = 0.0;
    const float* alpha = a.alpha + min(h0 + lane % kScanHeads, a.H - 1) * a.alpha_head;
    constexpr int kStep = 64 * kAppendWaves / kScanHeads, kLoads = 32;
    for (int t0 = s.n0 + (int)threadIdx.x / kScanHeads; t0 < from; t0 += kStep * kLoads) {
        float x[kLoads];
#pragma unroll
        for (int u = 0; u < kLoads; ++u) x[u] = alpha[min(t0 + kStep * u, from - 1) * a.alpha_token];
#pragma unroll
        for (int u = 0; u < kLoads; ++u) sum += t0 + kStep * u < from ? x[u] : 0.f;
    }
#pragma unroll
    for (int off = kScanHeads; off < 64; off *= 2) sum += __shfl_xor(sum, off, 64);
    if (lane < kScanHeads) sums[wv][lane] = sum;
    __syncthreads();
    static_assert(kScanHeads == 2 * kAppendWaves, "two heads to a wave");
    const int h = h0 + 2 * wv;
    if (h >= a.H) return;
    double c[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        c[k] = cached_prefix(a, b, s.before, min(h + k, a.H - 1));
#pragma unroll
        for (int i = 0; i < kAppendWaves; ++i) c[k] += sums[i][2 * wv + k];
    }
    prefix_heads<2, kScanGroups>(a, b, s, h, from, min(from + len, s.n1), c);
}

template <typename T, int D, bool ONCE>
__global__ __launch_bounds__(64 * kAppendWaves) void append_paged_kernel(const AppendArgs a) {
    constexpr int LPR = D / 16, HG = kSide<D>, RPW = 64 / LPR / HG;
    if ((int)blockIdx.x < a.scan_blocks) {
        const int block = xcd_remap(blockIdx.x, a.scan_blocks), units = (a.H + kScanHeads - 1) / kScanHeads;  // a sequence on one XCD: its heads share lines of alpha
        if (a.segments > 0) {
            const int i = block / units;
            prefix_segment(a, i / a.segments, (block - i * units) * kScanHeads, i % a.segments);
        } else {
            const int i = block * kAppendWaves + (threadIdx.x >> 6);
            if (i < a.B * units) prefix_short(a, i / units, i % units * kScanHeads);
        }
        return;
    }
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const LaneOfRow<D> l(lane % LPR, a.rot, a.paired);
    const int all = (a.Q != nullptr ? a.H : 0) + 2 * a.Hkv, keys = all - 2 * a.Hkv, values = all - a.Hkv;  // numbers of the first key, the first value
    for (int item = (blockIdx.x - a.scan_blocks) * kAppendWaves + wv; item < a.shares.items; item += (gridDim.x - a.scan_blocks) * kAppendWaves) {
        int tile;
        const HeadRange range = a.shares.range(item, tile);
        const int side = lane / LPR % HG;  // this lane's head of the HG next to each other
        const long long n = (long long)tile * RPW + lane / (LPR * HG), at = min(n, (long long)a.rows - 1);
        // the row's sequence, position and place in the cache, looked up while its first head is on its way
        int b = -2, row = 0, id = -1;
        long long p = 0;
        Angles angles;
        auto look_up = [&]() __attribute__((always_inline)) {
            if (b != -2) return;
            Frequencies freq;  // here, not in front of the loop: that takes three waves a SIMD where four have room (7168 tokens 47.3 us, 41.8)
            const bool turned = range.x0 < values && a.rot > 0;
            if (turned) freq.load(l, a.freq);
            int first, before;
            b = n < a.rows ? sequence_of(a, (int)n, first, before) : -1;
            if (b >= 0) {
                p = before + (n - first);
                if (range.x1 > keys) id = page_of(a, b, p, row);
            }
            if (turned) angles.at(l, (double)p, freq);
        };
        auto heads_of = [&](const HeadsView& in, const float* weight, void* out, int first, int count, auto kind) __attribute__((always_inline)) {
            constexpr HeadKind K = decltype(kind)::value;
            int h0, h1;
            if (!range.part(first, count, h0, h1)) return;
            const T* const from = (const T*)in.data + at * in.token;
            auto load = [&](LaneRow<T, D, ONCE>& r, int i) __attribute__((always_inline)) {
                r.load([&](int x) __attribute__((always_inline)) { return from + min(h0 + i * HG + x, h1 - 1) * in.head; }, side, l);
            };
            HeadWalk<LaneRow<T, D, ONCE>, decltype(load)> walk(0, (h1 - h0 + HG - 1) / HG, load);
            LaneVector<D> w;
            if (K != kValues && a.norm) w.load(weight, l);
            look_up();
            const bool there = K == kQueries ? b >= 0 : id >= 0;
            T* const to = (T*)out + (K == kQueries ? n * a.H * D : ((long long)max(id, 0) * a.Hkv * a.page + row) * D);
            const long long step = K == kQueries ? D : (long long)a.page * D;
            walk.run([&](LaneRow<T, D, ONCE>& r, int i) __attribute__((always_inline)) {
                if (K != kValues) {
                    r.arrive();
                    r.norm_and_turn(l, a.norm, a.eps, w, a.rot > 0, a.paired, angles);
                }
                const int h = h0 + i * HG + side;  // (with h0 + i * HG + x in its place: 16 prompts 97.2 us, 95.7)
                r.template store<ONCE>([&](int x) __attribute__((always_inline)) { return to + (h + (x - side)) * step; },
                                       [&](int x) __attribute__((always_inline)) { return there && h + (x - side) < h1; }, side, l, K != kValues);
            });
        };
        if (a.Q != nullptr) heads_of(a.q, a.wq, a.Q, 0, a.H, std::integral_constant<HeadKind, kQueries>{});
        heads_of(a.k, a.wk, a.Kp, keys, a.Hkv, std::integral_constant<HeadKind, kKeys>{});
        heads_of(a.v, nullptr, a.Vp, values, a.Hkv, std::integral_constant<HeadKind, kValues>{});
    }
}

}  // namespace

hipError_t append_paged(bool bf16, const HeadsView& q, const HeadsView& k, const HeadsView& v, const HeadRotation& how, const float* alpha,
                        long long alpha_token, long long alpha_head, const int* start, const int* cached, void* Q, const PagedCache& cache, int rows,
                        int B, int H, int Hkv, int d, hipStream_t s) {
    AppendArgs a{};
    a.q = q;
    a.k = k;
    a.v = v;
    a.wq = how.wq;
    a.wk = how.wk;
    a.eps = how.eps;
    a.freq = how.freq;
    a.rot = how.rot;
    a.norm = how.norm;
    a.paired = how.paired;
    a.alpha = alpha;
    a.alpha_token = alpha_token;
    a.alpha_head = alpha_head;
    a.start = start;
    a.cached = cached;
    a.table = cache.table;
    a.Q = Q;
    a.Kp = cache.Kp;
    a.Vp = cache.Vp;
    a.cp = cache.cp;
    a.rows = rows;
    a.B = B;
    a.H = H;
    a.Hkv = Hkv;
    a.pages = cache.pages;
    a.page = cache.page;
    a.max_pages = cache.max_pages;
    constexpr int kThreads = 64 * kAppendWaves;
    // The prefix.  Where sequences bring two tokens or fewer on average a wave takes eight heads of a sequence, however many tokens that has; otherwise a
    // workgroup does, for a segment of it: of 512 tokens, or as many as keep the segments to 64 and all sequences' to about 1024 workgroups.  (us, H 32,
    // Hkv 8, d 128, waves / workgroups: 512 sequences of two tokens 10.2 / 13.3, 256 of four 9.9 / 11.5, 299 of one and one of 512 18.0 / 11.3; 16 prompts in
    // up to 4096 workgroups 97.4, in up to 1024 95.7.)  Among many sequences a long one then is a single workgroup's for eight heads: one of 8192 tokens beside 31
    // of one 55.8, beside 255 80.0 (without gates 49.4 and 52.3; the 256 in up to 4096 workgroups 59.0).
    const int units = (H + kScanHeads - 1) / kScanHeads, sequences = B * units;
    if (alpha != nullptr && rows > 2LL * B) {
        const int most = sequences < 1024 ? 1024 / sequences : 1, want = (rows + kScanTokens - 1) / kScanTokens;
        a.segments = want < most ? want : most;
        if (a.segments > 64) a.segments = 64;
    }
    a.scan_blocks = alpha == nullptr ? 0 : a.segments > 0 ? sequences * a.segments : (sequences + kAppendWaves - 1) / kAppendWaves;
    const int side = d == 128 ? kSide<128> : kSide<64>;
    a.shares = Shares((int)(((long long)rows * side + 1024 / d - 1) / (1024 / d)), (Q != nullptr ? H : 0) + 2 * Hkv, side);
    long long blocks = ((long long)a.shares.items + kAppendWaves - 1) / kAppendWaves;
    if (blocks > 1 << 20) blocks = 1 << 20;
    ProfScope prof(kKernAppendPaged, s);
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)(a.scan_blocks + blocks)), dim3(kThreads), 0, s, a); };
    if (bf16) {
        const bool once = rows * ((Q != nullptr ? H : 0) + 2LL * Hkv) * d * 2 > kOnceBytes;  // of what is read
        if (d == 128) once ? launch(append_paged_kernel<bf16_t, 128, true>) : launch(append_paged_kernel<bf16_t, 128, false>);
        else once ? launch(append_paged_kernel<bf16_t, 64, true>) : launch(append_paged_kernel<bf16_t, 64, false>);
    } else {
        d == 128 ? launch(append_paged_kernel<float, 128, false>) : launch(append_paged_kernel<float, 64, false>);
    }
    return hipGetLastError();
}

}  // namespace gfwa
