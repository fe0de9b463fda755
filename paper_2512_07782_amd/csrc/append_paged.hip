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
    long long items;   // row tiles x head ranges
    int ranges, heads;
};

// The page that holds position p of sequence b, or -1: outside the table, or not there.
__device__ __forceinline__ int page_of(const AppendArgs& a, int b, long long p, int& row) {
    if (p < 0 || p >= (long long)a.max_pages * a.page) return -1;
    const int i = (int)p / a.page;
    row = (int)p - i * a.page;
    const int id = a.table[(size_t)b * a.max_pages + i];
    return id >= 0 && id < a.pages ? id : -1;
}

// The sequence b with start[b] <= row < start[b + 1], or -1.
__device__ __forceinline__ int sequence_of(const int* start, int B, int row) {
    int lo = 0, hi = B;
    while (hi - lo > 1) {
        const int mid = lo + (hi - lo) / 2;
        if (start[mid] <= row) lo = mid;
        else hi = mid;
    }
    return start[lo] <= row && row < start[lo + 1] ? lo : -1;
}

// c_p of every new token of sequence b and head h, by one thread.
__device__ void prefix_of(const AppendArgs& a, int b, int h) {
    const int n0 = min(max(a.start[b], 0), a.rows), n1 = min(max(a.start[b + 1], n0), a.rows);
    const long long before = a.cached[b];
    double c = 0;
    int row = 0;
    const int prev = n1 > n0 ? page_of(a, b, before - 1, row) : -1;
    if (prev >= 0) c = a.cp[((size_t)prev * a.H + h) * a.page + row];
    for (int n = n0; n < n1; ++n) {
        c += a.alpha[n * a.alpha_token + h * a.alpha_head];
        const int id = page_of(a, b, before + (n - n0), row);
        if (id >= 0) a.cp[((size_t)id * a.H + h) * a.page + row] = (float)c;
    }
}

template <typename T, int D>
__global__ __launch_bounds__(64 * kAppendWaves) void append_paged_kernel(const AppendArgs a) {
    constexpr int LPR = D / 16, RPW = 64 / LPR;
    if ((int)blockIdx.x < a.scan_blocks) {
        const long long i = (long long)blockIdx.x * (64 * kAppendWaves) + threadIdx.x;
        if (i < (long long)a.B * a.H) prefix_of(a, (int)(i / a.H), (int)(i % a.H));
        return;
    }
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    const LaneOfRow<D> l(lane % LPR, a.rot, a.paired);
    const long long first = (long long)(blockIdx.x - a.scan_blocks) * kAppendWaves + wv;
    for (long long item = first; item < a.items; item += (long long)(gridDim.x - a.scan_blocks) * kAppendWaves) {
        const long long tile = item / a.ranges;
        const int x0 = (int)(item - tile * a.ranges) * a.heads, x1 = min(x0 + a.heads, a.H + 2 * a.Hkv);
        const long long n = tile * RPW + lane / LPR;
        const int b = n < a.rows ? sequence_of(a.start, a.B, (int)n) : -1;
        if (b < 0) continue;
        const int before = a.cached[b];
        const long long p = (long long)before + ((int)n - a.start[b]);
        int row = 0;
        const int id = before >= 0 ? page_of(a, b, p, row) : -1;
        Angles angles;
        if (x0 < a.H + a.Hkv && a.rot > 0) angles.at(l, (int)p, a.freq);
        // rows of `in` to `to`, `step` elements from head to head
        auto heads_of = [&](const HeadsView& in, const float* weight, T* to, size_t step, int first, int count, bool plain) __attribute__((always_inline)) {
            const int h0 = max(x0 - first, 0), h1 = min(x1 - first, count);
            if (h0 >= h1) return;
            const T* from = (const T*)in.data + n * in.token;
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
                ua.store(to + h * step + l.a);
                ub.store(to + h * step + l.b);
            }
        };
        if (a.Q != nullptr) heads_of(a.q, a.wq, (T*)a.Q + n * a.H * D, D, 0, a.H, false);
        if (id < 0) continue;
        const size_t at = ((size_t)id * a.Hkv * a.page + row) * D, step = (size_t)a.page * D;
        heads_of(a.k, a.wk, (T*)a.Kp + at, step, a.H, a.Hkv, false);
        heads_of(a.v, nullptr, (T*)a.Vp + at, step, a.H + a.Hkv, a.Hkv, true);
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
    a.scan_blocks = alpha != nullptr ? (int)(((long long)B * H + kThreads - 1) / kThreads) : 0;
    const int heads = H + 2 * Hkv;
    const long long tiles = (rows + 1024 / d - 1) / (1024 / d), waves = 16LL * device_cu_count();
    long long ranges = (waves + tiles - 1) / tiles;
    if (ranges > heads) ranges = heads;
    a.heads = (int)((heads + ranges - 1) / ranges);
    a.ranges = (heads + a.heads - 1) / a.heads;
    a.items = tiles * a.ranges;
    long long blocks = (a.items + kAppendWaves - 1) / kAppendWaves;
    if (blocks > 1 << 20) blocks = 1 << 20;
    ProfScope prof(kKernAppendPaged, s);
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)(a.scan_blocks + blocks)), dim3(kThreads), 0, s, a); };
    if (bf16) d == 128 ? launch(append_paged_kernel<bf16_t, 128>) : launch(append_paged_kernel<bf16_t, 64>);
    else d == 128 ? launch(append_paged_kernel<float, 128>) : launch(append_paged_kernel<float, 64>);
    return hipGetLastError();
}

}  // namespace gfwa
