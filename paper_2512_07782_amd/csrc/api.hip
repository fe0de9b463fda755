// C ABI of libgfwa (see include/gfwa.h): argument validation and dispatch.  No device memory is
// allocated here; everything is enqueued on the caller's stream.
#include <stdint.h>
#include <stdlib.h>
#include <string.h>
#include <algorithm>
#include <atomic>
#include <initializer_list>
#include <mutex>
#include <utility>

#include "../../include/gfwa.h"
#include "../../include/gfwa_layer.h"
#include "gfwa_internal.h"

namespace gfwa {

static thread_local char g_hip_msg[256] = "no HIP error recorded";

static int hip_status(hipError_t e) {
    if (e == hipSuccess) return GFWA_OK;
    snprintf(g_hip_msg, sizeof(g_hip_msg), "HIP error %d: %s", (int)e, hipGetErrorString(e));
    return GFWA_ERR_HIP;
}

static bool aligned(const void* p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

// Sizes every entry point shares.  Tile indices and per-head offsets are 32-bit in the kernels.
static int check_dims(int B, int H, int N, int d, int w, bool need_d) {
    if (B <= 0 || H <= 0 || N <= 0) return GFWA_ERR_DIM;
    if (need_d && (d <= 0 || w < 1)) return GFWA_ERR_DIM;
    const long long bh = (long long)B * H;
    if (bh > (1LL << 24) || (long long)N > (1LL << 24)) return GFWA_ERR_DIM;
    if (bh * ((N + 31) / 32) > 0x7fffffffLL) return GFWA_ERR_DIM;
    if (need_d && d != 64 && d != 128) return GFWA_ERR_UNSUPPORTED;
    return GFWA_OK;
}

// ---- what the operators around the attention check
static constexpr long long kMostOffset = 1LL << 40;  // elements: far beyond the memory there is, and safe to multiply

static int check_layer_dims(int B, int H, int Hkv, int N, int d) {
    if (int r = check_dims(B, H, N, d, 1, true)) return r;
    if (Hkv <= 0 || H % Hkv != 0 || (long long)B * N > 0x7fffffffLL) return GFWA_ERR_DIM;
    return GFWA_OK;
}

static int check_rotation(int dt, float eps, int rot, int flags, int d) {
    if (dt != GFWA_BF16 && dt != GFWA_F32) return GFWA_ERR_UNSUPPORTED;
    if (flags & ~(GFWA_HEAD_NORM | GFWA_ROPE_PAIRED)) return GFWA_ERR_UNSUPPORTED;
    if (rot < 0 || rot > d || rot % 16 != 0 || ((flags & GFWA_HEAD_NORM) && !(eps >= 0.0f))) return GFWA_ERR_DIM;
    return GFWA_OK;
}

// positions are 32-bit, offsets into the cache 64-bit; a launch holds less than 2^32 threads
static int check_cache(int B, int H, int pages, int page, int max_pages) {
    if (B <= 0 || pages <= 0 || page <= 0 || page % 16 != 0 || max_pages <= 0) return GFWA_ERR_DIM;
    if ((long long)B * H > (1LL << 22) || (long long)max_pages * page > 0x7fffffffLL) return GFWA_ERR_DIM;
    return GFWA_OK;
}

struct Bytes {
    const void* at;
    size_t count;
    bool meets(const Bytes& o) const { return at && o.at && overlap(at, count, o.at, o.count); }
};
// whether one of what a call writes meets another one or something that it reads
static bool any_meet(std::initializer_list<Bytes> writes, std::initializer_list<Bytes> reads) {
    for (const Bytes* w = writes.begin(); w != writes.end(); ++w) {
        for (const Bytes* o = writes.begin(); o != w; ++o)
            if (w->meets(*o)) return true;
        for (const Bytes& r : reads)
            if (w->meets(r)) return true;
    }
    return false;
}

// The strided tensor of `heads` heads that a caller describes; nullptr: none.
struct HeadsSpan {
    const gfwa_heads_t* t;
    int heads;
    int check(int B, int N, int d, size_t size) const {
        if (!t) return GFWA_OK;
        if (!aligned(t->data, 16)) return GFWA_ERR_ALIGN;
        const long long unit = 16 / (long long)size, strides[] = {t->batch, t->token, t->head}, counts[] = {B, N, heads};
        double last = 0;
        for (int i = 0; i < 3; ++i) {
            if (counts[i] == 1) continue;
            if (strides[i] < 0 || strides[i] > kMostOffset) return GFWA_ERR_DIM;
            if (strides[i] % unit != 0) return GFWA_ERR_ALIGN;
            last += (double)strides[i] * (double)(counts[i] - 1);
        }
        return last > (double)kMostOffset ? GFWA_ERR_DIM : GFWA_OK;
    }
    long long last_row(int B, int N) const {
        return (B > 1 ? t->batch * (B - 1) : 0) + (N > 1 ? t->token * (N - 1) : 0) + (heads > 1 ? t->head * (heads - 1) : 0);
    }
    Bytes bytes(int B, int N, int d, size_t size) const {
        return t ? Bytes{t->data, (size_t)(last_row(B, N) + d) * size} : Bytes{nullptr, 0};
    }
    // its dimensions by stride, the widest last, and what each reaches over
    struct Nest {
        long long dims[3][2];
        Nest(const gfwa_heads_t& t, int B, int N, int heads) : dims{{t.batch, B}, {t.token, N}, {t.head, heads}} {
            for (int i = 0; i < 2; ++i)
                for (int j = 0; j < 2 - i; ++j)
                    if (dims[j][0] > dims[j + 1][0]) std::swap(dims[j], dims[j + 1]);
        }
        // whether no two rows share an element: taken by stride, each dimension steps over all of the one below it
        bool disjoint(int d) const {
            long long reach = d;
            for (auto& x : dims) {
                if (x[1] == 1) continue;
                if (x[0] < reach) return false;
                reach += x[0] * (x[1] - 1);
            }
            return true;
        }
        // whether element `at`, counted from the first one, is in a row (of disjoint ones: the last one not behind it has it, or none)
        bool holds(long long at, int d) const {
            if (at < 0) return false;
            for (int i = 2; i >= 0; --i)
                if (dims[i][1] > 1 && at >= dims[i][0]) at -= dims[i][0] * std::min(at / dims[i][0], dims[i][1] - 1);
            return at < d;
        }
    };
    Nest nest(int B, int N) const { return Nest(*t, B, N, heads); }
    // whether its first or last row meets a row of o, a tensor of disjoint rows
    bool ends_meet(const HeadsSpan& o, const Nest& rows, int B, int N, int d, size_t size) const {
        const long long first = ((intptr_t)t->data - (intptr_t)o.t->data) / (long long)size, last = first + last_row(B, N);
        return rows.holds(first, d) || rows.holds(first + d - 1, d) || rows.holds(last, d) || rows.holds(last + d - 1, d);
    }
};

// whether outputs of one call are strided so that none of their rows meet
static bool rows_apart(const HeadsSpan* outs, int count, int B, int N, int d, size_t size) {
    for (int i = 0; i < count; ++i) {
        if (!outs[i].t) continue;
        const HeadsSpan::Nest rows = outs[i].nest(B, N);
        if (!rows.disjoint(d)) return false;
        for (int j = 0; j < count; ++j)
            if (j != i && outs[j].t && outs[j].ends_meet(outs[i], rows, B, N, d, size)) return false;
    }
    return true;
}

static HeadsView view(const gfwa_heads_t* t) { return t ? HeadsView{t->data, t->batch, t->token, t->head} : HeadsView{nullptr, 0, 0, 0}; }

// ---- optional per-kernel timing with HIP events on the caller's stream ----
namespace {
constexpr int kMaxRecords = 8192;
struct ProfRecord { int kernel; hipEvent_t start, stop; };
struct ProfState {
    std::atomic<bool> on{false};   // the only field read without the lock (every launch asks it)
    std::mutex lock;               // slot allocation, reset and read-out may come from different host threads
    int used = 0;
    int created = 0;
    ProfRecord rec[kMaxRecords];
};
ProfState g_prof;
}  // namespace

hipError_t allow_dynamic_lds(const void* kernel, size_t bytes, DeviceOnce& done) {
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    const unsigned long long bit = 1ull << (dev & 63);
    if (dev < 64 && (__atomic_load_n(&done.bits, __ATOMIC_ACQUIRE) & bit)) return hipSuccess;
    e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e == hipSuccess && dev < 64) __atomic_fetch_or(&done.bits, bit, __ATOMIC_RELEASE);
    return e;
}

int device_cu_count() {
    static int cached[64];  // 0: not asked yet
    int dev = 0, n = 0;
    if (hipGetDevice(&dev) != hipSuccess) return 256;
    if (dev >= 0 && dev < 64 && (n = __atomic_load_n(&cached[dev], __ATOMIC_RELAXED)) > 0) return n;
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0) return 256;
    if (dev >= 0 && dev < 64) __atomic_store_n(&cached[dev], n, __ATOMIC_RELAXED);
    return n;
}

ProfScope::ProfScope(int kernel, hipStream_t s) : slot_(-1), s_(s) {
    if (!g_prof.on.load(std::memory_order_relaxed)) return;
    std::lock_guard<std::mutex> hold(g_prof.lock);
    if (g_prof.used >= kMaxRecords) return;
    const int i = g_prof.used;
    if (i >= g_prof.created) {
        if (hipEventCreate(&g_prof.rec[i].start) != hipSuccess) return;
        if (hipEventCreate(&g_prof.rec[i].stop) != hipSuccess) return;
        g_prof.created = i + 1;
    }
    g_prof.rec[i].kernel = kernel;
    g_prof.used = i + 1;
    slot_ = i;
    (void)hipEventRecord(g_prof.rec[i].start, s_);
}
ProfScope::~ProfScope() {
    if (slot_ >= 0) (void)hipEventRecord(g_prof.rec[slot_].stop, s_);
}

}  // namespace gfwa

using namespace gfwa;

extern "C" {

int gfwa_gate_prefix(const float* alpha, float* c, int B, int H, int N, gfwa_stream_t stream) {
    if (!alpha || !c) return GFWA_ERR_NULL;
    if (int r = check_dims(B, H, N, 0, 1, false)) return r;
    if (!aligned(alpha, 4) || !aligned(c, 4)) return GFWA_ERR_ALIGN;
    return hip_status(gate_prefix(alpha, c, B * H, N, stream));
}

int gfwa_gate_activation_prefix(const float* hpre, const float* beta, float eps, float* c, int B, int H, int N,
                                gfwa_stream_t stream) {
    if (!hpre || !beta || !c) return GFWA_ERR_NULL;
    if (int r = check_dims(B, H, N, 0, 1, false)) return r;
    if (!(eps >= 0.0f)) return GFWA_ERR_DIM;
    if (!aligned(hpre, 4) || !aligned(beta, 4) || !aligned(c, 4)) return GFWA_ERR_ALIGN;
    return hip_status(gate_activation_prefix(hpre, beta, eps, c, B * H, N, stream));
}

size_t gfwa_gate_scan_workspace_bytes(int B, int H, int N) {
    if (check_dims(B, H, N, 0, 1, false) != GFWA_OK) return 0;
    return (gate_scan_workspace_bytes(B * H, N) + 255) & ~(size_t)255;
}

int gfwa_gate_prefix_stp(const float* in, const float* beta, float eps, float* c, void* workspace,
                         size_t workspace_bytes, int B, int H, int N, gfwa_stream_t stream) {
    if (!in || !c) return GFWA_ERR_NULL;
    if (int r = check_dims(B, H, N, 0, 1, false)) return r;
    if (beta && !(eps >= 0.0f)) return GFWA_ERR_DIM;
    if (!aligned(in, 4) || !aligned(c, 4) || (beta && !aligned(beta, 4))) return GFWA_ERR_ALIGN;
    if (!workspace || workspace_bytes < gfwa_gate_scan_workspace_bytes(B, H, N)) return GFWA_ERR_WORKSPACE;
    if (!aligned(workspace, 8)) return GFWA_ERR_ALIGN;
    return hip_status(gate_prefix_stp(in, beta, eps, c, (double*)workspace, B * H, N, stream));
}

int gfwa_gate_activation_backward(const float* hpre, const float* beta, float eps, const float* dalpha, float* dh,
                                  float* dbeta, int B, int H, int N, gfwa_stream_t stream) {
    if (!hpre || !beta || !dalpha || !dh || !dbeta) return GFWA_ERR_NULL;
    if (int r = check_dims(B, H, N, 0, 1, false)) return r;
    if (!(eps >= 0.0f)) return GFWA_ERR_DIM;
    if (!aligned(hpre, 4) || !aligned(beta, 4) || !aligned(dalpha, 4) || !aligned(dh, 4) || !aligned(dbeta, 4))
        return GFWA_ERR_ALIGN;
    return hip_status(gate_activation_backward(hpre, beta, eps, dalpha, dh, dbeta, (size_t)B * H * N, stream));
}

int gfwa_forward(gfwa_dtype_t dt, const void* Q, const void* K, const void* V, const float* c, void* O,
                 float* L, int B, int H, int N, int d, int w, float scale, gfwa_stream_t stream) {
    return gfwa_forward_gqa(dt, Q, K, V, c, O, L, B, H, H, N, d, w, scale, stream);
}

int gfwa_forward_gqa(gfwa_dtype_t dt, const void* Q, const void* K, const void* V, const float* c, void* O,
                     float* L, int B, int H, int Hkv, int N, int d, int w, float scale, gfwa_stream_t stream) {
    if (!Q || !K || !V || !c || !O || !L) return GFWA_ERR_NULL;
    if (int r = check_dims(B, H, N, d, w, true)) return r;
    if (Hkv <= 0 || H % Hkv != 0) return GFWA_ERR_DIM;
    if (dt != GFWA_BF16 && dt != GFWA_F32) return GFWA_ERR_UNSUPPORTED;
    if (!aligned(Q, 16) || !aligned(K, 16) || !aligned(V, 16) || !aligned(O, 16) || !aligned(c, 4) ||
        !aligned(L, 4))
        return GFWA_ERR_ALIGN;
    if (dt == GFWA_F32)
        return hip_status(forward_f32((const float*)Q, (const float*)K, (const float*)V, c, (float*)O, L,
                                      B, H, Hkv, N, d, w, scale, stream));
    return hip_status(forward_bf16(Q, K, V, c, O, L, B, H, Hkv, N, d, w, scale, stream));
}

size_t gfwa_backward_workspace_bytes(gfwa_dtype_t dt, int B, int H, int N, int d, int w) {
    if (check_dims(B, H, N, d, w, true) != GFWA_OK) return 0;
    if (dt != GFWA_BF16 && dt != GFWA_F32) return 0;
    // D, dc_col, dc_row: three fp32 vectors of B*H*N, each padded to 256 bytes; then the segment sums of the
    // gate-gradient scan (one fp64 per 4096 elements)
    const size_t one = (((size_t)B * H * N * sizeof(float)) + 255) & ~(size_t)255;
    return 3 * one + ((gate_scan_workspace_bytes(B * H, N) + 255) & ~(size_t)255);
}

size_t gfwa_backward_fast_workspace_bytes(gfwa_dtype_t dt, int B, int H, int N, int d, int w) {
    const size_t base = gfwa_backward_workspace_bytes(dt, B, H, N, d, w);
    if (base == 0 || dt != GFWA_BF16) return base;
    return base + backward_bf16_spill_bytes(B, H, N, d, w);
}

int gfwa_backward(gfwa_dtype_t dt, const void* Q, const void* K, const void* V, const void* O,
                  const void* dO, const float* c, const float* L, void* dQ, void* dK, void* dV,
                  float* dalpha, void* workspace, size_t workspace_bytes, int B, int H, int N, int d, int w,
                  float scale, gfwa_stream_t stream) {
    return gfwa_backward_gqa(dt, Q, K, V, O, dO, c, L, dQ, dK, dV, dalpha, workspace, workspace_bytes, B, H, H, N,
                             d, w, scale, stream);
}

int gfwa_backward_gqa(gfwa_dtype_t dt, const void* Q, const void* K, const void* V, const void* O,
                      const void* dO, const float* c, const float* L, void* dQ, void* dK, void* dV,
                      float* dalpha, void* workspace, size_t workspace_bytes, int B, int H, int Hkv, int N,
                      int d, int w, float scale, gfwa_stream_t stream) {
    if (!Q || !K || !V || !O || !dO || !c || !L || !dQ || !dK || !dV || !dalpha) return GFWA_ERR_NULL;
    if (int r = check_dims(B, H, N, d, w, true)) return r;
    if (Hkv <= 0 || H % Hkv != 0) return GFWA_ERR_DIM;
    if (dt != GFWA_BF16 && dt != GFWA_F32) return GFWA_ERR_UNSUPPORTED;
    const void* mats[] = {Q, K, V, O, dO, dQ, dK, dV};
    for (const void* p : mats)
        if (!aligned(p, 16)) return GFWA_ERR_ALIGN;
    if (!aligned(c, 4) || !aligned(L, 4) || !aligned(dalpha, 4)) return GFWA_ERR_ALIGN;
    const size_t need = gfwa_backward_workspace_bytes(dt, B, H, N, d, w);
    if (!workspace || workspace_bytes < need) return GFWA_ERR_WORKSPACE;
    if (!aligned(workspace, 16)) return GFWA_ERR_ALIGN;
    float* ws = (float*)workspace;
    if (dt == GFWA_F32)
        return hip_status(backward_f32((const float*)Q, (const float*)K, (const float*)V, (const float*)O,
                                       (const float*)dO, c, L, (float*)dQ, (float*)dK, (float*)dV, dalpha,
                                       ws, B, H, Hkv, N, d, w, scale, stream));
    const size_t fast = gfwa_backward_fast_workspace_bytes(dt, B, H, N, d, w);
    const bool spill = fast > need && workspace_bytes >= fast;
    return hip_status(
        backward_bf16(Q, K, V, O, dO, c, L, dQ, dK, dV, dalpha, ws, spill, B, H, Hkv, N, d, w, scale, stream));
}

size_t gfwa_decode_workspace_bytes(int B, int H, int T, int d, int w) {
    if (check_dims(B, H, T, d, w, true) != GFWA_OK) return 0;
    return (decode_workspace_bytes(B, H, T, d, w) + 255) & ~(size_t)255;
}

int gfwa_decode(gfwa_dtype_t dt, const void* q, const void* Kc, const void* Vc, float* c, const float* alpha_t,
                const int* pos, void* o, float* L, void* workspace, size_t workspace_bytes, int B, int H, int Hkv,
                int T, int d, int w, float scale, gfwa_stream_t stream) {
    if (!q || !Kc || !Vc || !c || !pos || !o) return GFWA_ERR_NULL;
    if (int r = check_dims(B, H, T, d, w, true)) return r;
    if (Hkv <= 0 || H % Hkv != 0) return GFWA_ERR_DIM;
    if (dt != GFWA_BF16 && dt != GFWA_F32) return GFWA_ERR_UNSUPPORTED;
    if (!aligned(q, 16) || !aligned(Kc, 16) || !aligned(Vc, 16) || !aligned(o, 16) || !aligned(c, 4) ||
        !aligned(pos, 4) || (alpha_t && !aligned(alpha_t, 4)) || (L && !aligned(L, 4)))
        return GFWA_ERR_ALIGN;
    if (!workspace || workspace_bytes < gfwa_decode_workspace_bytes(B, H, T, d, w)) return GFWA_ERR_WORKSPACE;
    if (!aligned(workspace, 16)) return GFWA_ERR_ALIGN;
    return hip_status(decode(dt == GFWA_BF16, q, Kc, Vc, c, alpha_t, pos, o, L, (float*)workspace, B, H, Hkv, T, d,
                             w, scale, stream));
}

int gfwa_decode_static(gfwa_dtype_t dt, const void* q, const void* Kc, const void* Vc, float* c,
                       const float* alpha_t, const int* pos, void* o, float* L, int B, int H, int Hkv, int T, int d,
                       int w, float scale, gfwa_stream_t stream) {
    if (!q || !Kc || !Vc || !c || !pos || !o) return GFWA_ERR_NULL;
    if (int r = check_dims(B, H, T, d, w, true)) return r;
    if (Hkv <= 0 || H % Hkv != 0) return GFWA_ERR_DIM;
    if (dt != GFWA_BF16 && dt != GFWA_F32) return GFWA_ERR_UNSUPPORTED;
    if (!aligned(q, 16) || !aligned(Kc, 16) || !aligned(Vc, 16) || !aligned(o, 16) || !aligned(c, 4) ||
        !aligned(pos, 4) || (alpha_t && !aligned(alpha_t, 4)) || (L && !aligned(L, 4)))
        return GFWA_ERR_ALIGN;
    if (gfwa_decode_workspace_bytes(B, H, T, d, w) > kDecodeStaticBytes) return GFWA_ERR_WORKSPACE;
    float* part = nullptr;
    if (hipError_t e = decode_static_scratch(&part)) return hip_status(e);
    return hip_status(decode(dt == GFWA_BF16, q, Kc, Vc, c, alpha_t, pos, o, L, part, B, H, Hkv, T, d, w, scale,
                             stream));
}

// ---- around the attention (gfwa_layer.h)

size_t gfwa_qk_norm_rope_backward_workspace_bytes(int B, int H, int Hkv, int N, int d) {
    if (check_layer_dims(B, H, Hkv, N, d) != GFWA_OK) return 0;
    return qk_norm_rope_backward_workspace_bytes(d);
}

int gfwa_qk_norm_rope(gfwa_dtype_t dt, const gfwa_heads_t* q, const gfwa_heads_t* k, const gfwa_heads_t* v, const float* wq,
                      const float* wk, float eps, const double* freq, int rot, const int* pos, int flags, void* Q, void* K,
                      void* V, int B, int H, int Hkv, int N, int d, gfwa_stream_t stream) {
    if (!q || !q->data || !k || !k->data || (v && (!v->data || !V)) || !Q || !K || (rot > 0 && !freq)) return GFWA_ERR_NULL;
    if (int r = check_layer_dims(B, H, Hkv, N, d)) return r;
    if (int r = check_rotation(dt, eps, rot, flags, d)) return r;
    const size_t size = dt == GFWA_BF16 ? 2 : 4, bytes = (size_t)B * N * d * size;
    const HeadsSpan spans[] = {{q, H}, {k, Hkv}, {v, Hkv}};
    for (const HeadsSpan& x : spans)
        if (int r = x.check(B, N, d, size)) return r;
    if (!v) V = nullptr;
    const Bytes outs[] = {{Q, bytes * H}, {K, bytes * Hkv}, {V, bytes * Hkv}};
    for (const Bytes& o : outs)
        if (!aligned(o.at, 16)) return GFWA_ERR_ALIGN;
    if (!aligned(wq, 4) || !aligned(wk, 4) || !aligned(pos, 4) || (rot > 0 && !aligned(freq, 8))) return GFWA_ERR_ALIGN;
    if (any_meet({outs[0], outs[1], outs[2]}, {spans[0].bytes(B, N, d, size), spans[1].bytes(B, N, d, size), spans[2].bytes(B, N, d, size), {wq, (size_t)d * 4},
                                               {wk, (size_t)d * 4}, {rot > 0 ? freq : nullptr, (size_t)rot * 4}, {pos, (size_t)B * N * 4}}))
        return GFWA_ERR_OVERLAP;
    const HeadRotation how{wq, wk, eps, freq, rot, pos, (flags & GFWA_HEAD_NORM) != 0, (flags & GFWA_ROPE_PAIRED) != 0};
    return hip_status(qk_norm_rope(dt == GFWA_BF16, view(q), view(k), view(v), how, Q, K, V, B, H, Hkv, N, d, stream));
}

int gfwa_qk_norm_rope_backward(gfwa_dtype_t dt, const gfwa_heads_t* q, const gfwa_heads_t* k, const float* wq, const float* wk,
                               float eps, const double* freq, int rot, const int* pos, int flags, const void* dQ, const void* dK,
                               const void* dV, const gfwa_heads_t* dq, const gfwa_heads_t* dk, const gfwa_heads_t* dv, float* dwq,
                               float* dwk, void* workspace, size_t workspace_bytes, int B, int H, int Hkv, int N, int d,
                               gfwa_stream_t stream) {
    const bool norm = (flags & GFWA_HEAD_NORM) != 0;
    if (!dQ || !dK || !dq || !dq->data || !dk || !dk->data || (norm && (!q || !q->data || !k || !k->data)) || (rot > 0 && !freq)) return GFWA_ERR_NULL;
    if ((dV != nullptr) != (dv != nullptr && dv->data != nullptr)) return GFWA_ERR_NULL;
    if (int r = check_layer_dims(B, H, Hkv, N, d)) return r;
    if (int r = check_rotation(dt, eps, rot, flags, d)) return r;
    if (!norm && (dwq || dwk)) return GFWA_ERR_UNSUPPORTED;
    if (!norm) q = k = nullptr;
    if (!dV) dv = nullptr;
    const size_t size = dt == GFWA_BF16 ? 2 : 4, bytes = (size_t)B * N * d * size;
    const HeadsSpan ins[] = {{q, H}, {k, Hkv}}, outs[] = {{dq, H}, {dk, Hkv}, {dv, Hkv}};
    for (const HeadsSpan& x : ins)
        if (int r = x.check(B, N, d, size)) return r;
    for (const HeadsSpan& x : outs)
        if (int r = x.check(B, N, d, size)) return r;
    if (!rows_apart(outs, 3, B, N, d, size)) return GFWA_ERR_OVERLAP;
    const Bytes grads[] = {{dQ, bytes * H}, {dK, bytes * Hkv}, {dV, bytes * Hkv}};
    for (const Bytes& g : grads)
        if (!aligned(g.at, 16)) return GFWA_ERR_ALIGN;
    if (!aligned(wq, 4) || !aligned(wk, 4) || !aligned(pos, 4) || !aligned(dwq, 4) || !aligned(dwk, 4) || (rot > 0 && !aligned(freq, 8)))
        return GFWA_ERR_ALIGN;
    for (const HeadsSpan& o : outs) {
        for (const HeadsSpan& x : ins)
            if (o.bytes(B, N, d, size).meets(x.bytes(B, N, d, size))) return GFWA_ERR_OVERLAP;
        for (const Bytes& g : grads)
            if (o.bytes(B, N, d, size).meets(g)) return GFWA_ERR_OVERLAP;
    }
    const Bytes wqs{wq, (size_t)d * 4}, wks{wk, (size_t)d * 4}, angles{rot > 0 ? freq : nullptr, (size_t)rot * 4}, positions{pos, (size_t)B * N * 4};
    for (const HeadsSpan& o : outs)
        if (any_meet({o.bytes(B, N, d, size)}, {wqs, wks, angles, positions})) return GFWA_ERR_OVERLAP;
    if (dwq || dwk) {
        const size_t scratch = gfwa_qk_norm_rope_backward_workspace_bytes(B, H, Hkv, N, d);
        if (!workspace || workspace_bytes < scratch) return GFWA_ERR_WORKSPACE;
        if (!aligned(workspace, 16)) return GFWA_ERR_ALIGN;
        if (any_meet({{dwq, (size_t)d * 4}, {dwk, (size_t)d * 4}, {workspace, scratch}},
                     {ins[0].bytes(B, N, d, size), ins[1].bytes(B, N, d, size), grads[0], grads[1], grads[2], outs[0].bytes(B, N, d, size),
                      outs[1].bytes(B, N, d, size), outs[2].bytes(B, N, d, size), wqs, wks, angles, positions}))
            return GFWA_ERR_OVERLAP;
    }
    const HeadRotation how{wq, wk, eps, freq, rot, pos, norm, (flags & GFWA_ROPE_PAIRED) != 0};
    return hip_status(qk_norm_rope_backward(dt == GFWA_BF16, view(q), view(k), how, dQ, dK, dV, view(dq), view(dk), view(dv), dwq, dwk,
                                            (float*)workspace, B, H, Hkv, N, d, stream));
}

int gfwa_append_paged(gfwa_dtype_t dt, const gfwa_heads_t* q, const gfwa_heads_t* k, const gfwa_heads_t* v, const float* wq,
                      const float* wk, float eps, const double* freq, int rot, int flags, const float* alpha, long long alpha_token,
                      long long alpha_head, const int* start, const int* cached, const int* table, void* Q, void* Kp, void* Vp,
                      float* cp, int rows, int B, int H, int Hkv, int d, int pages, int page, int max_pages,
                      gfwa_stream_t stream) {
    if ((q && (!q->data || !Q)) || !k || !k->data || !v || !v->data || (alpha && !cp) || !start || !cached || !table || !Kp || !Vp ||
        (rot > 0 && !freq))
        return GFWA_ERR_NULL;
    if (int r = check_layer_dims(1, H, Hkv, rows, d)) return r;
    if (int r = check_cache(B, H, pages, page, max_pages)) return r;
    if (int r = check_rotation(dt, eps, rot, flags, d)) return r;
    const size_t size = dt == GFWA_BF16 ? 2 : 4;
    if (!q) Q = nullptr;
    if (!alpha) cp = nullptr;
    const HeadsSpan ins[] = {{q, H}, {k, Hkv}, {v, Hkv}};
    for (const HeadsSpan& x : ins)
        if (int r = x.check(1, rows, d, size)) return r;
    if (alpha) {
        if (alpha_token < 0 || alpha_head < 0 || alpha_token > kMostOffset || alpha_head > kMostOffset ||
            (double)(rows - 1) * alpha_token + (double)(H - 1) * alpha_head > (double)kMostOffset)
            return GFWA_ERR_DIM;
    }
    if (!aligned(Q, 16) || !aligned(Kp, 16) || !aligned(Vp, 16) || !aligned(cp, 4) || !aligned(alpha, 4) || !aligned(start, 4) ||
        !aligned(cached, 4) || !aligned(table, 4) || !aligned(wq, 4) || !aligned(wk, 4) || (rot > 0 && !aligned(freq, 8)))
        return GFWA_ERR_ALIGN;
    const size_t per_head = (size_t)pages * page;
    const Bytes outs[] = {{Q, (size_t)rows * H * d * size}, {Kp, per_head * Hkv * d * size}, {Vp, per_head * Hkv * d * size}, {cp, per_head * H * 4}};
    const Bytes gate{alpha, alpha ? 4 * (size_t)((rows - 1) * alpha_token + (H - 1) * alpha_head + 1) : 0};
    if (any_meet({outs[0], outs[1], outs[2], outs[3]},
                 {ins[0].bytes(1, rows, d, size), ins[1].bytes(1, rows, d, size), ins[2].bytes(1, rows, d, size), gate, {wq, (size_t)d * 4}, {wk, (size_t)d * 4},
                  {rot > 0 ? freq : nullptr, (size_t)rot * 4}, {start, ((size_t)B + 1) * 4}, {cached, (size_t)B * 4}, {table, (size_t)B * max_pages * 4}}))
        return GFWA_ERR_OVERLAP;
    const HeadRotation how{wq, wk, eps, freq, rot, nullptr, (flags & GFWA_HEAD_NORM) != 0, (flags & GFWA_ROPE_PAIRED) != 0};
    const PagedCache cache{Kp, Vp, cp, table, pages, page, max_pages};
    return hip_status(append_paged(dt == GFWA_BF16, view(q), view(k), view(v), how, alpha, alpha_token, alpha_head, start, cached, Q, cache, rows,
                                   B, H, Hkv, d, stream));
}

size_t gfwa_decode_paged_workspace_bytes(int B, int H, int Hkv, int d, int page, int max_pages, int w) {
    if (check_layer_dims(B, H, Hkv, 1, d) != GFWA_OK || check_cache(B, H, 1, page, max_pages) != GFWA_OK || w < 1) return 0;
    return (decode_paged_workspace_bytes(B, H, Hkv, d, page, max_pages, w) + 255) & ~(size_t)255;
}

int gfwa_decode_paged(gfwa_dtype_t dt, const void* q, const void* Kp, const void* Vp, const float* cp, const int* table,
                      const int* pos, void* o, float* L, void* workspace, size_t workspace_bytes, int B, int H, int Hkv, int d,
                      int pages, int page, int max_pages, int w, float scale, gfwa_stream_t stream) {
    if (!q || !Kp || !Vp || !cp || !table || !pos || !o) return GFWA_ERR_NULL;
    if (int r = check_layer_dims(B, H, Hkv, 1, d)) return r;
    if (int r = check_cache(B, H, pages, page, max_pages)) return r;
    if (w < 1) return GFWA_ERR_DIM;
    if (dt != GFWA_BF16 && dt != GFWA_F32) return GFWA_ERR_UNSUPPORTED;
    if (!aligned(q, 16) || !aligned(Kp, 16) || !aligned(Vp, 16) || !aligned(o, 16) || !aligned(cp, 4) || !aligned(table, 4) ||
        !aligned(pos, 4) || !aligned(L, 4))
        return GFWA_ERR_ALIGN;
    const size_t scratch = gfwa_decode_paged_workspace_bytes(B, H, Hkv, d, page, max_pages, w);
    if (!workspace || workspace_bytes < scratch) return GFWA_ERR_WORKSPACE;
    if (!aligned(workspace, 16)) return GFWA_ERR_ALIGN;
    const size_t size = dt == GFWA_BF16 ? 2 : 4, row = (size_t)d * size, per_head = (size_t)pages * page, heads = (size_t)B * H;
    if (any_meet({{o, heads * row}, {L, heads * 4}, {workspace, scratch}},
                 {{q, heads * row}, {Kp, per_head * Hkv * row}, {Vp, per_head * Hkv * row}, {cp, per_head * H * 4}, {table, (size_t)B * max_pages * 4}, {pos, (size_t)B * 4}}))
        return GFWA_ERR_OVERLAP;
    const PagedCache cache{const_cast<void*>(Kp), const_cast<void*>(Vp), const_cast<float*>(cp), table, pages, page, max_pages};
    return hip_status(decode_paged(dt == GFWA_BF16, q, cache, pos, o, L, (float*)workspace, B, H, Hkv, d, w, scale, stream));
}

const char* gfwa_strerror(int code) {
    switch (code) {
        case GFWA_OK: return "ok";
        case GFWA_ERR_NULL: return "a required pointer is NULL";
        case GFWA_ERR_DIM: return "invalid size: B, H, N, d must be > 0, w >= 1, Hkv > 0 dividing H, within index range";
        case GFWA_ERR_UNSUPPORTED: return "unsupported head dimension (64 or 128) or dtype";
        case GFWA_ERR_ALIGN: return "pointer not sufficiently aligned (16 bytes matrices, 4 bytes vectors)";
        case GFWA_ERR_WORKSPACE:
            return "workspace missing or smaller than the matching gfwa_*_workspace_bytes() call asks for; for "
                   "gfwa_decode_static: the sizes need more than the library's 32 MiB of scratch";
        case GFWA_ERR_HIP: return g_hip_msg;
        case GFWA_ERR_OVERLAP: return "an output overlaps an input, another output or the workspace, or its own rows overlap";
        default: return "unknown status code";
    }
}

int gfwa_version(void) { return 100; }

int gfwa_probe_mfma(float* sink, int iterations, int workgroups, int random_operands, double* flops,
                    gfwa_stream_t stream) {
    if (!sink) return GFWA_ERR_NULL;
    if (iterations < 1 || workgroups < 1 || workgroups > (1 << 20) || iterations > (1 << 24)) return GFWA_ERR_DIM;
    if (!aligned(sink, 4)) return GFWA_ERR_ALIGN;
    if (random_operands < 0 || random_operands > 2) return GFWA_ERR_DIM;
    return hip_status(probe_mfma(sink, iterations, workgroups, random_operands, flops, stream));
}

int gfwa_probe_copy(const void* src, void* dst, size_t bytes, gfwa_stream_t stream) {
    if (!src || !dst) return GFWA_ERR_NULL;
    if (bytes < 16 || bytes % 16 != 0) return GFWA_ERR_DIM;
    if (!aligned(src, 16) || !aligned(dst, 16)) return GFWA_ERR_ALIGN;
    return hip_status(probe_copy(src, dst, bytes, stream));
}

int gfwa_profile_enable(int on) {
    std::lock_guard<std::mutex> hold(g_prof.lock);
    g_prof.on.store(on != 0, std::memory_order_relaxed);
    if (on) g_prof.used = 0;  // records stay readable after profiling is switched off
    return GFWA_OK;
}

int gfwa_profile_read(float* total_ms, int* launches, int n) {
    if (!total_ms || !launches) return GFWA_ERR_NULL;
    if (n < kKernFirstCount) return GFWA_ERR_DIM;
    for (int k = 0; k < n; ++k) {
        total_ms[k] = 0.f;
        launches[k] = 0;
    }
    std::lock_guard<std::mutex> hold(g_prof.lock);
    for (int i = 0; i < g_prof.used; ++i) {
        if (g_prof.rec[i].kernel >= n) continue;
        hipError_t e = hipEventSynchronize(g_prof.rec[i].stop);
        float ms = 0.f;
        if (e == hipSuccess) e = hipEventElapsedTime(&ms, g_prof.rec[i].start, g_prof.rec[i].stop);
        if (e != hipSuccess) return hip_status(e);
        total_ms[g_prof.rec[i].kernel] += ms;
        launches[g_prof.rec[i].kernel] += 1;
    }
    return GFWA_OK;
}

const char* gfwa_profile_kernel_name(int k) {
    static const char* names[kKernCount] = {"gate_prefix_scan", "forward", "bwd_rowdot", "bwd_dkv", "bwd_dq",
                                            "gate_grad_scan", "gate_activation_prefix_scan",
                                            "gate_activation_bwd", "decode_partial", "decode_combine", "scan_segment_sum", "scan_propagate",
                                            "gate_grad_segment_sum", "qk_norm_rope", "qk_norm_rope_bwd", "norm_weight_grad_sum", "append_paged",
                                            "decode_paged_partial", "decode_paged_combine"};
    return (k >= 0 && k < kKernCount) ? names[k] : "";
}

}  // extern "C"
