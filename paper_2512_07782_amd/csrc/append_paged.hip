// New tokens of a batch of sequences into the paged key/value cache on gfx950: norm and rotation of their queries and keys, keys and
// values to their pages, and the gate's prefix carried on, in one launch.
//   * rows of queries, keys and values are held and worked on as in qk_norm_rope.hip; a row's sequence is looked up from the batch's
//     offsets and its page from the table, once for all its heads;
//   * the prefix is a scan along each sequence and goes to workgroups of its own, which the launch begins with.
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
    int scan_heads;    // heads that a wave of them takes: 8, or 1
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

constexpr int kShort = 8;       // new tokens, and heads, that a wave takes in one go
constexpr int kScanGroups = 8;  // groups of 64 tokens of a pass over a long sequence

// New tokens n0 .. n1 of sequence b, whose cache holds `before` tokens: c of one head, by one wave.  The gates and page ids of the next 512
// tokens are on their way while these are added up.
__device__ void prefix_long(const AppendArgs& a, int b, int h, int n0, int n1, long long before, double c) {
    const int lane = threadIdx.x & 63;
    const float* alpha = a.alpha + h * a.alpha_head;
    float x[2][kScanGroups];
    int id[2][kScanGroups];
    auto issue = [&](int n, auto buf) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < kScanGroups; ++u) {
            const int t = n + 64 * u + lane;
            x[decltype(buf)::value][u] = t < n1 ? alpha[t * a.alpha_token] : 0.f;
            int row;
            id[decltype(buf)::value][u] = t < n1 ? page_of(a, b, before + (t - n0), row) : -1;
        }
    };
    auto add = [&](int n, auto buf) __attribute__((always_inline)) {
        constexpr int k = decltype(buf)::value;
#pragma unroll
        for (int u = 0; u < kScanGroups; ++u) {
            const double s = wave_scan((double)x[k][u]);
            if (id[k][u] >= 0) {  // a position in the table: 32 bits
                const int p = (int)(before + (n - n0)) + 64 * u + lane;
                a.cp[((size_t)id[k][u] * a.H + h) * a.page + p % a.page] = (float)(c + s);
            }
            c += lane_value(s, 63);
        }
    };
    constexpr int kPass = 64 * kScanGroups;
    const std::integral_constant<int, 0> first;
    const std::integral_constant<int, 1> second;
    issue(n0, first);
    for (int n = n0; n < n1; n += 2 * kPass) {
        if (n1 - n > kPass) issue(n + kPass, second);
        add(n, first);
        if (n1 - n > kPass) {
            if (n1 - n > 2 * kPass) issue(n + 2 * kPass, first);
            add(n + kPass, second);
        }
    }
}

// c of the new tokens of sequence b for `heads` (1 or 8) heads from h0 on, by one wave.  A few tokens and eight heads: a lane for each of both.
__device__ void prefix_of(const AppendArgs& a, int b, int h0, int heads) {
    const int lane = threadIdx.x & 63;
    const int from = a.start[b], to = a.start[b + 1];
    const long long before = a.cached[b];
    const int n0 = min(max(from, 0), a.rows), n1 = min(max(to, n0), a.rows);
    if (n0 == n1) return;
    int row = 0;
    const int prev = page_of(a, b, before - 1, row);
    auto cached_c = [&](int h) { return prev >= 0 ? (double)a.cp[((size_t)prev * a.H + h) * a.page + row] : 0.0; };
    const int last = min(h0 + heads, a.H);
    if (heads == kShort && n1 - n0 <= kShort) {
        const int t = lane / kShort, h = h0 + lane % kShort;
        const bool mine = n0 + t < n1 && h < last;
        int at = 0;
        const int id = mine ? page_of(a, b, before + t, at) : -1;
        double c = mine ? a.alpha[(n0 + t) * a.alpha_token + h * a.alpha_head] : 0.f;
        if (n1 - n0 > 1) {
#pragma unroll
            for (int off = kShort; off < 64; off *= 2) {
                const double x = __shfl_up(c, off, 64);
                if (lane >= off) c += x;
            }
        }
        if (!mine) return;
        c += cached_c(h);
        if (id >= 0) a.cp[((size_t)id * a.H + h) * a.page + at] = (float)c;
        return;
    }
    for (int h = h0; h < last; ++h) prefix_long(a, b, h, n0, n1, before, cached_c(h));
}

template <typename T, int D, bool ONCE>
__global__ __launch_bounds__(64 * kAppendWaves) void append_paged_kernel(const AppendArgs a) {
    constexpr int LPR = D / 16, HG = kSide<D>, RPW = 64 / LPR / HG;
    if ((int)blockIdx.x < a.scan_blocks) {
        // the heads of a sequence on one XCD: they read the same lines of alpha
        const long long i = (long long)xcd_remap(blockIdx.x, a.scan_blocks) * kAppendWaves + (threadIdx.x >> 6);
        const int units = (a.H + a.scan_heads - 1) / a.scan_heads;
        if (i < (long long)a.B * units) prefix_of(a, (int)(i / units), (int)(i % units) * a.scan_heads, a.scan_heads);
        return;
    }
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const LaneOfRow<D> l(lane % LPR, a.rot, a.paired);
    const int all = (a.Q != nullptr ? a.H : 0) + 2 * a.Hkv, keys = all - 2 * a.Hkv, values = all - a.Hkv;  // numbers of the first key, the first value
    Frequencies freq;
    if (a.rot > 0) freq.load(l, a.freq);
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
            int first, before;
            b = n < a.rows ? sequence_of(a, (int)n, first, before) : -1;
            if (b >= 0) {
                p = (long long)before + ((int)n - first);
                if (before >= 0 && range.x1 > keys) id = page_of(a, b, p, row);
            }
            if (range.x0 < values && a.rot > 0) angles.at(l, (int)p, freq);
        };
        auto heads_of = [&](const HeadsView& in, const float* weight, void* out, int first, int count, auto kind) __attribute__((always_inline)) {
            constexpr HeadKind K = decltype(kind)::value;
            int h0, h1;
            if (!range.part(first, count, h0, h1)) return;
            const T* const from = (const T*)in.data + at * in.token;
            auto load = [&](LaneRow<T, D, ONCE>& r, int i) __attribute__((always_inline)) { r.load(from + min(h0 + i * HG + side, h1 - 1) * in.head, l); };
            HeadWalk<LaneRow<T, D, ONCE>, decltype(load)> walk(0, (h1 - h0 + HG - 1) / HG, load);
            LaneVector<D> w;
            if (K != kValues && a.norm) w.load(weight, l);
            look_up();
            const bool there = K == kQueries ? b >= 0 : id >= 0;
            T* const to = (T*)out + (K == kQueries ? n * a.H * D : ((long long)max(id, 0) * a.Hkv * a.page + row) * D);
            const size_t step = K == kQueries ? (size_t)D : (size_t)a.page * D;
            walk.run([&](LaneRow<T, D, ONCE>& r, int i) __attribute__((always_inline)) {
                const int h = h0 + i * HG + side;
                if (K != kValues) r.norm_and_turn(l, a.norm, a.eps, w, a.rot > 0, a.paired, angles);
                if (there && h < h1) r.template store<ONCE>(to + h * step, l);
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
    // a wave of the prefix takes one head where sequences bring many tokens (more than 16 on average: those with few leave
    // its lanes idle, those with many are bound by it), eight where they bring few
    a.scan_heads = rows > 16LL * B ? 1 : kShort;
    const long long scans = (long long)B * ((H + a.scan_heads - 1) / a.scan_heads);
    a.scan_blocks = alpha != nullptr ? (int)((scans + kAppendWaves - 1) / kAppendWaves) : 0;
    const int side = d == 128 ? kSide<128> : kSide<64>;
    a.shares = Shares((int)(((long long)rows * side + 1024 / d - 1) / (1024 / d)), (Q != nullptr ? H : 0) + 2 * Hkv, side);
    long long blocks = ((long long)a.shares.items + kAppendWaves - 1) / kAppendWaves;
    if (blocks > 1 << 20) blocks = 1 << 20;
    ProfScope prof(kKernAppendPaged, s);
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)(a.scan_blocks + blocks)), dim3(kThreads), 0, s, a); };
    if (bf16) {
        const bool once = rows * (H + 2LL * Hkv) * d * 2 > kOnceBytes;
        if (d == 128) once ? launch(append_paged_kernel<bf16_t, 128, true>) : launch(append_paged_kernel<bf16_t, 128, false>);
        else launch(append_paged_kernel<bf16_t, 64, false>);
    } else {
        d == 128 ? launch(append_paged_kernel<float, 128, false>) : launch(append_paged_kernel<float, 64, false>);
    }
    return hipGetLastError();
}

}  // namespace gfwa
