// Native half of the Python binding: checks torch tensors, allocates the outputs that were not given and calls
// the C ABI of libgfwa with raw pointers and the current HIP stream.  Small problems are bound by the host: through
// ctypes and Python-level checks a prefix + forward pair took 22 us of host time and a training step of ten tensors
// 75 us, more than its kernels; here a call costs its kernel launches plus about a microsecond.
//
// The module has no link-time dependency on libgfwa: binding.py hands over the addresses of its functions once
// (bind), so that the library named by GFWA_LIB is the one that is called.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/hip/EmptyTensor.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/DynamicTypes.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <initializer_list>
#include <optional>
#include <string>

#include "../../include/gfwa.h"
#include "../../include/gfwa_layer.h"

namespace {

// ---- the library's functions, by name, in the order bind() takes their addresses
struct Library {
    decltype(&gfwa_gate_prefix) gate_prefix;
    decltype(&gfwa_gate_activation_prefix) gate_activation_prefix;
    decltype(&gfwa_gate_activation_backward) gate_activation_backward;
    decltype(&gfwa_gate_scan_workspace_bytes) gate_scan_workspace_bytes;
    decltype(&gfwa_gate_prefix_stp) gate_prefix_stp;
    decltype(&gfwa_forward_gqa) forward_gqa;
    decltype(&gfwa_backward_workspace_bytes) backward_workspace_bytes;
    decltype(&gfwa_backward_gqa) backward_gqa;
    decltype(&gfwa_decode_workspace_bytes) decode_workspace_bytes;
    decltype(&gfwa_decode) decode;
    decltype(&gfwa_decode_static) decode_static;
    decltype(&gfwa_qk_norm_rope) qk_norm_rope;
    decltype(&gfwa_qk_norm_rope_backward_workspace_bytes) qk_norm_rope_backward_workspace_bytes;
    decltype(&gfwa_qk_norm_rope_backward) qk_norm_rope_backward;
    decltype(&gfwa_append_paged) append_paged;
    decltype(&gfwa_decode_paged_workspace_bytes) decode_paged_workspace_bytes;
    decltype(&gfwa_decode_paged) decode_paged;
};
constexpr Py_ssize_t kFunctions = sizeof(Library) / sizeof(void*);
Library lib;
PyObject* raise_status = nullptr;  // binding._check: turns a negative status into GfwaError

struct PyError {};  // a Python exception is set

// A scope without the interpreter lock, taken again however the scope is left (looking up the stream may throw).
struct Unlocked {
    PyThreadState* state = PyEval_SaveThread();
    Unlocked() = default;
    Unlocked(const Unlocked&) = delete;
    ~Unlocked() { PyEval_RestoreThread(state); }
};

[[noreturn]] void fail(PyObject* type, const std::string& text) {
    PyErr_SetString(type, text.c_str());
    throw PyError{};
}

std::string shape_text(at::IntArrayRef s) {  // as Python prints a tuple
    std::string r = "(";
    for (size_t i = 0; i < s.size(); ++i) r += (i ? ", " : "") + std::to_string(s[i]);
    return r + (s.size() == 1 ? ",)" : ")");
}
std::string dtype_text(at::ScalarType t) { return std::string("torch.") + torch::getTHPDtype(t)->name; }

const at::Tensor& tensor_of(PyObject* o, const char* name) {
    if (!THPVariable_Check(o)) fail(PyExc_TypeError, std::string(name) + " must be a tensor");
    return THPVariable_Unpack(o);
}

void need(const at::Tensor& t, at::IntArrayRef shape, at::ScalarType dtype, const char* name) {
    if (!t.is_cuda()) fail(PyExc_ValueError, std::string(name) + " must live on the GPU");
    if (t.sizes() != shape)
        fail(PyExc_ValueError, std::string(name) + " has shape " + shape_text(t.sizes()) + ", expected " + shape_text(shape));
    if (t.scalar_type() != dtype)
        fail(PyExc_TypeError, std::string(name) + " has dtype " + dtype_text(t.scalar_type()) + ", expected " + dtype_text(dtype));
    if (!t.is_contiguous()) fail(PyExc_ValueError, std::string(name) + " must be contiguous");
}

const void* input(PyObject* o, at::IntArrayRef shape, at::ScalarType dtype, const char* name) {
    const at::Tensor& t = tensor_of(o, name);
    need(t, shape, dtype, name);
    return t.const_data_ptr();
}

// without the interpreter lock, as torch.empty does it: an allocation may wait for the driver
at::Tensor fresh(at::IntArrayRef shape, at::ScalarType dtype, at::Device device) {
    Unlocked other_threads_may_run;
    return at::Tensor(at::detail::empty_cuda(shape, dtype, device, std::nullopt));
}

// An output: the caller's tensor, checked, or a fresh one.
struct Output {
    PyObject* given = nullptr;
    at::Tensor made;
    void* ptr = nullptr;
    Output(PyObject* o, at::IntArrayRef shape, at::ScalarType dtype, at::Device device, const char* name) {
        if (o == Py_None) {
            made = fresh(shape, dtype, device);
            ptr = made.data_ptr();
        } else {
            const at::Tensor& t = tensor_of(o, name);
            need(t, shape, dtype, name);
            given = o;
            ptr = t.data_ptr();
        }
    }
    PyObject* object() {
        if (given == nullptr) return THPVariable_Wrap(std::move(made));
        Py_INCREF(given);
        return given;
    }
};

// Scratch: the caller's tensor, or a fresh one of `bytes`.
struct Workspace {
    at::Tensor t;
    void* ptr;
    size_t bytes;
    Workspace(PyObject* o, size_t want, at::Device device) {
        if (o == Py_None) {
            t = fresh({(int64_t)want}, at::kByte, device);
        } else {
            t = tensor_of(o, "workspace");
            if (!t.is_cuda() || !t.is_contiguous()) fail(PyExc_ValueError, "workspace must be a contiguous GPU tensor");
        }
        ptr = t.data_ptr();
        bytes = t.nbytes();
    }
};

PyObject* tuple_of(std::initializer_list<Output*> outs) {
    PyObject* r = PyTuple_New((Py_ssize_t)outs.size());
    if (r == nullptr) throw PyError{};
    Py_ssize_t i = 0;
    for (Output* o : outs) {
        PyObject* x = o->object();
        if (x == nullptr) {
            Py_DECREF(r);
            throw PyError{};
        }
        PyTuple_SET_ITEM(r, i++, x);
    }
    return r;
}

// int(x) and float(x) of a Python number; integers are passed on modulo 2^32, as ctypes does for a C int
int as_int(PyObject* o) {
    PyObject* n = PyNumber_Long(o);
    if (n == nullptr) throw PyError{};
    const unsigned long long v = PyLong_AsUnsignedLongLongMask(n);
    Py_DECREF(n);
    if (PyErr_Occurred()) throw PyError{};
    return (int)(unsigned)v;
}
// A window of a cache whose positions are C ints: longer ones hold every sequence, as the longest int does.
int as_window(PyObject* o) {
    PyObject* n = PyNumber_Long(o);
    if (n == nullptr) throw PyError{};
    int past = 0;
    const long long v = PyLong_AsLongLongAndOverflow(n, &past);
    Py_DECREF(n);
    if (v == -1 && !past && PyErr_Occurred()) throw PyError{};
    return past > 0 || v > 0x7fffffffLL ? 0x7fffffff : past < 0 || v < 1 ? 0 : (int)v;  // 0: refused
}
float as_float(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw PyError{};
    return (float)v;
}

int storage_type(const at::Tensor& t) {
    if (t.scalar_type() == at::kBFloat16) return GFWA_BF16;
    if (t.scalar_type() == at::kFloat) return GFWA_F32;
    fail(PyExc_TypeError, "unsupported dtype " + dtype_text(t.scalar_type()) + ": bfloat16 or float32");
}

int kv_heads(int64_t H, int64_t Hkv) {
    if (Hkv <= 0 || H % Hkv != 0)
        fail(PyExc_ValueError, "the number of key/value heads (" + std::to_string(Hkv) +
                                   ") must divide the number of query heads (" + std::to_string(H) + ")");
    return (int)Hkv;
}

gfwa_stream_t stream() { return c10::hip::getCurrentHIPStream().stream(); }

// The library call itself, without the interpreter lock (other host threads may launch on other streams).
template <typename F>
void call(F&& f) {
    int status;
    {
        Unlocked other_threads_may_run;
        status = f();
    }
    if (status != 0) {
        PyObject* r = PyObject_CallFunction(raise_status, "i", status);
        Py_XDECREF(r);
        if (PyErr_Occurred()) throw PyError{};
    }
}

template <PyObject* (*F)(PyObject* const*), Py_ssize_t N>
PyObject* entry(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != N) {
        PyErr_Format(PyExc_TypeError, "%zd arguments expected", N);
        return nullptr;
    }
    try {
        return F(a);
    } catch (const PyError&) {
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

// [B,H,N] of a gate tensor
struct Rows {
    int B, H, N;
    Rows(const at::Tensor& t, const char* name) {
        if (t.dim() != 3) fail(PyExc_ValueError, std::string(name) + " must be [B,H,N]");
        B = (int)t.size(0);
        H = (int)t.size(1);
        N = (int)t.size(2);
    }
};

PyObject* gate_prefix(PyObject* const* a) {  // alpha, c
    const at::Tensor& alpha = tensor_of(a[0], "alpha");
    const Rows r(alpha, "alpha");
    const at::IntArrayRef shape = alpha.sizes();
    need(alpha, shape, at::kFloat, "alpha");
    Output c(a[1], shape, at::kFloat, alpha.device(), "c");
    call([&] { return lib.gate_prefix((const float*)alpha.const_data_ptr(), (float*)c.ptr, r.B, r.H, r.N, stream()); });
    return c.object();
}

PyObject* gate_activation_prefix(PyObject* const* a) {  // hpre, beta, eps, c
    const at::Tensor& hpre = tensor_of(a[0], "hpre");
    const Rows r(hpre, "hpre");
    const at::IntArrayRef shape = hpre.sizes();
    need(hpre, shape, at::kFloat, "hpre");
    const void* beta = input(a[1], shape, at::kFloat, "beta");
    const float eps = as_float(a[2]);
    Output c(a[3], shape, at::kFloat, hpre.device(), "c");
    call([&] {
        return lib.gate_activation_prefix((const float*)hpre.const_data_ptr(), (const float*)beta, eps, (float*)c.ptr, r.B, r.H,
                                          r.N, stream());
    });
    return c.object();
}

PyObject* gate_activation_backward(PyObject* const* a) {  // hpre, beta, eps, dalpha, dh, dbeta
    const at::Tensor& hpre = tensor_of(a[0], "hpre");
    const Rows r(hpre, "hpre");
    const at::IntArrayRef shape = hpre.sizes();
    need(hpre, shape, at::kFloat, "hpre");
    const void* beta = input(a[1], shape, at::kFloat, "beta");
    const float eps = as_float(a[2]);
    const void* dalpha = input(a[3], shape, at::kFloat, "dalpha");
    Output dh(a[4], shape, at::kFloat, hpre.device(), "dh");
    Output dbeta(a[5], shape, at::kFloat, hpre.device(), "dbeta");
    call([&] {
        return lib.gate_activation_backward((const float*)hpre.const_data_ptr(), (const float*)beta, eps, (const float*)dalpha,
                                            (float*)dh.ptr, (float*)dbeta.ptr, r.B, r.H, r.N, stream());
    });
    return tuple_of({&dh, &dbeta});
}

PyObject* gate_prefix_stp(PyObject* const* a) {  // x, beta, eps, c, workspace
    const at::Tensor& x = tensor_of(a[0], "x");
    const Rows r(x, "x");
    const at::IntArrayRef shape = x.sizes();
    need(x, shape, at::kFloat, "x");
    const void* beta = a[1] == Py_None ? nullptr : input(a[1], shape, at::kFloat, "beta");
    const float eps = as_float(a[2]);
    Output c(a[3], shape, at::kFloat, x.device(), "c");
    Workspace ws(a[4], a[4] == Py_None ? lib.gate_scan_workspace_bytes(r.B, r.H, r.N) : 0, x.device());
    call([&] {
        return lib.gate_prefix_stp((const float*)x.const_data_ptr(), (const float*)beta, eps, (float*)c.ptr, ws.ptr, ws.bytes,
                                   r.B, r.H, r.N, stream());
    });
    return c.object();
}

// sizes of the attention calls: Q [B,H,N,d], K [B,Hkv,N,d]; `grouped` lets Hkv differ from H
struct Sizes {
    int64_t B, H, N, d, Hkv;
    int64_t q[4], kv[4], rows[3];
    Sizes(const at::Tensor& Q, const at::Tensor& K, bool grouped) {
        if (Q.dim() != 4 || (grouped && K.dim() != 4))
            fail(PyExc_ValueError, grouped ? "Q must be [B,H,N,d] and K [B,Hkv,N,d]" : "Q must be [B,H,N,d]");
        B = Q.size(0);
        H = Q.size(1);
        N = Q.size(2);
        d = Q.size(3);
        Hkv = grouped ? kv_heads(H, K.size(1)) : H;
        q[0] = kv[0] = rows[0] = B;
        q[1] = rows[1] = H;
        kv[1] = Hkv;
        q[2] = kv[2] = rows[2] = N;
        q[3] = kv[3] = d;
    }
};

PyObject* forward(PyObject* const* a) {  // grouped, Q, K, V, c, w, scale, O, L
    const at::Tensor& Q = tensor_of(a[1], "Q");
    const at::Tensor& K = tensor_of(a[2], "K");
    const Sizes s(Q, K, a[0] == Py_True);
    const int dt = storage_type(Q);
    const at::ScalarType st = Q.scalar_type();
    need(Q, s.q, st, "Q");
    need(K, s.kv, st, "K");
    const void* V = input(a[3], s.kv, st, "V");
    const void* c = input(a[4], s.rows, at::kFloat, "c");
    const int w = as_int(a[5]);
    const float scale = as_float(a[6]);
    Output O(a[7], s.q, st, Q.device(), "O");
    Output L(a[8], s.rows, at::kFloat, Q.device(), "L");
    call([&] {
        return lib.forward_gqa(dt, Q.const_data_ptr(), K.const_data_ptr(), V, (const float*)c, O.ptr, (float*)L.ptr, (int)s.B,
                               (int)s.H, (int)s.Hkv, (int)s.N, (int)s.d, w, scale, stream());
    });
    return tuple_of({&O, &L});
}

PyObject* backward(PyObject* const* a) {  // grouped, Q, K, V, O, dO, c, L, w, scale, workspace, dQ, dK, dV, dalpha
    const at::Tensor& Q = tensor_of(a[1], "Q");
    const at::Tensor& K = tensor_of(a[2], "K");
    const Sizes s(Q, K, a[0] == Py_True);
    const int dt = storage_type(Q);
    const at::ScalarType st = Q.scalar_type();
    need(Q, s.q, st, "Q");
    need(K, s.kv, st, "K");
    const void* V = input(a[3], s.kv, st, "V");
    const void* O = input(a[4], s.q, st, "O");
    const void* dO = input(a[5], s.q, st, "dO");
    const void* c = input(a[6], s.rows, at::kFloat, "c");
    const void* L = input(a[7], s.rows, at::kFloat, "L");
    const int w = as_int(a[8]);
    const float scale = as_float(a[9]);
    Output dQ(a[11], s.q, st, Q.device(), "dQ");
    Output dK(a[12], s.kv, st, Q.device(), "dK");
    Output dV(a[13], s.kv, st, Q.device(), "dV");
    Output dalpha(a[14], s.rows, at::kFloat, Q.device(), "dalpha");
    Workspace ws(a[10], a[10] == Py_None ? lib.backward_workspace_bytes(dt, (int)s.B, (int)s.H, (int)s.N, (int)s.d, w) : 0,
                 Q.device());
    call([&] {
        return lib.backward_gqa(dt, Q.const_data_ptr(), K.const_data_ptr(), V, O, dO, (const float*)c, (const float*)L, dQ.ptr,
                                dK.ptr, dV.ptr, (float*)dalpha.ptr, ws.ptr, ws.bytes, (int)s.B, (int)s.H, (int)s.Hkv, (int)s.N,
                                (int)s.d, w, scale, stream());
    });
    return tuple_of({&dQ, &dK, &dV, &dalpha});
}

// the tensors both decoding calls take: q, Kc, Vc, c, pos, w, scale, alpha_t in a[0..7]
struct Step {
    const at::Tensor& q;
    int64_t B, H, Hkv, T, d, qs[3], heads[2];
    int dt, w;
    float scale;
    const void *Kc, *Vc, *alpha;
    float* c;
    const int* pos;
    explicit Step(PyObject* const* a) : q(tensor_of(a[0], "q")) {
        const at::Tensor& K = tensor_of(a[1], "Kc");
        if (q.dim() != 3 || K.dim() != 4) fail(PyExc_ValueError, "q must be [B,H,d] and Kc [B,Hkv,T,d]");
        B = q.size(0);
        H = q.size(1);
        d = q.size(2);
        T = K.size(2);
        Hkv = kv_heads(H, K.size(1));
        dt = storage_type(q);
        qs[0] = heads[0] = B;
        qs[1] = heads[1] = H;
        qs[2] = d;
        const int64_t cache[4] = {B, Hkv, T, d}, rows[3] = {B, H, T}, batch[1] = {B};
        need(q, qs, q.scalar_type(), "q");
        need(K, cache, q.scalar_type(), "Kc");
        Kc = K.const_data_ptr();
        Vc = input(a[2], cache, q.scalar_type(), "Vc");
        const at::Tensor& ct = tensor_of(a[3], "c");
        need(ct, rows, at::kFloat, "c");
        c = (float*)ct.data_ptr();
        pos = (const int*)input(a[4], batch, at::kInt, "pos");
        w = as_int(a[5]);
        scale = as_float(a[6]);
        alpha = a[7] == Py_None ? nullptr : input(a[7], heads, at::kFloat, "alpha_t");
    }
};

PyObject* decode(PyObject* const* a) {  // q, Kc, Vc, c, pos, w, scale, alpha_t, o, L, workspace
    const Step s(a);
    Output o(a[8], s.qs, s.q.scalar_type(), s.q.device(), "o");
    Output L(a[9], s.heads, at::kFloat, s.q.device(), "L");
    Workspace ws(a[10], a[10] == Py_None ? lib.decode_workspace_bytes((int)s.B, (int)s.H, (int)s.T, (int)s.d, s.w) : 0,
                 s.q.device());
    call([&] {
        return lib.decode(s.dt, s.q.const_data_ptr(), s.Kc, s.Vc, s.c, (const float*)s.alpha, s.pos, o.ptr, (float*)L.ptr, ws.ptr,
                          ws.bytes, (int)s.B, (int)s.H, (int)s.Hkv, (int)s.T, (int)s.d, s.w, s.scale, stream());
    });
    return tuple_of({&o, &L});
}

PyObject* decode_static(PyObject* const* a) {  // q, Kc, Vc, c, pos, w, scale, alpha_t, o, L
    const Step s(a);
    const at::Tensor& o = tensor_of(a[8], "o");
    const at::Tensor& L = tensor_of(a[9], "L");
    need(o, s.qs, s.q.scalar_type(), "o");
    need(L, s.heads, at::kFloat, "L");
    call([&] {
        return lib.decode_static(s.dt, s.q.const_data_ptr(), s.Kc, s.Vc, s.c, (const float*)s.alpha, s.pos, o.data_ptr(),
                                 (float*)L.data_ptr(), (int)s.B, (int)s.H, (int)s.Hkv, (int)s.T, (int)s.d, s.w, s.scale, stream());
    });
    return PyTuple_Pack(2, a[8], a[9]);
}

// ---- around the attention (gfwa_layer.h)

// Every tensor of a call on one GPU, and that the current one: its current stream is where the call goes.
struct OneDevice {
    at::Device device;
    explicit OneDevice(const at::Tensor& t) : device(t.device()) {}
    void also(const at::Tensor& t, const char* name) const {
        if (t.device() != device)
            fail(PyExc_ValueError, std::string(name) + " is on " + t.device().str() + ", the first tensor on " + device.str());
    }
    void is_current() const {
        const int now = c10::hip::current_device();
        if (device.index() != now)
            fail(PyExc_ValueError, "the tensors are on " + device.str() + ", the current device is " + std::to_string(now));
    }
};

const at::Tensor& dense(PyObject* o, at::IntArrayRef shape, at::ScalarType dtype, const OneDevice& dev, const char* name) {
    const at::Tensor& t = tensor_of(o, name);
    need(t, shape, dtype, name);
    dev.also(t, name);
    return t;
}
const void* optional_input(PyObject* o, at::IntArrayRef shape, at::ScalarType dtype, const OneDevice& dev, const char* name) {
    return o == Py_None ? nullptr : dense(o, shape, dtype, dev, name).const_data_ptr();
}
// sizes that are passed on as C ints
void fits_int(at::IntArrayRef sizes) {
    for (int64_t n : sizes)
        if (n > 0x7fffffffLL) fail(PyExc_ValueError, "a size of " + std::to_string(n) + " is too large");
}

// A strided tensor of heads, [B,N,heads,d] (or [rows,heads,d]): anything whose last dimension is contiguous.
struct Heads {
    gfwa_heads_t t{};
    bool given = false;
    Heads() = default;
    Heads(const at::Tensor& x, at::IntArrayRef shape, at::ScalarType dtype, const OneDevice& dev, const char* name, bool write) {
        if (!x.is_cuda()) fail(PyExc_ValueError, std::string(name) + " must live on the GPU");
        if (x.sizes() != shape)
            fail(PyExc_ValueError, std::string(name) + " has shape " + shape_text(x.sizes()) + ", expected " + shape_text(shape));
        if (x.scalar_type() != dtype)
            fail(PyExc_TypeError, std::string(name) + " has dtype " + dtype_text(x.scalar_type()) + ", expected " + dtype_text(dtype));
        const int64_t n = x.dim();
        if (x.stride(n - 1) != 1) fail(PyExc_ValueError, std::string(name) + " must be contiguous in its last dimension");
        dev.also(x, name);
        t.data = write ? x.data_ptr() : const_cast<void*>(x.const_data_ptr());
        t.head = x.stride(n - 2);
        t.token = x.stride(n - 3);
        t.batch = n == 4 ? x.stride(0) : 0;
        given = true;
    }
    const gfwa_heads_t* get() const { return given ? &t : nullptr; }
};

// Norm and rotation: wq, wk, eps, freq, norm, paired
struct Rotation {
    const float *wq, *wk;
    float eps;
    const double* freq = nullptr;
    int rot = 0, flags = 0;
    Rotation(PyObject* const* a, int64_t d, const OneDevice& dev) {
        const int64_t weights[1] = {d};
        wq = (const float*)optional_input(a[0], weights, at::kFloat, dev, "wq");
        wk = (const float*)optional_input(a[1], weights, at::kFloat, dev, "wk");
        eps = as_float(a[2]);
        if (a[3] != Py_None) {
            const at::Tensor& f = tensor_of(a[3], "freq");
            if (f.dim() != 1) fail(PyExc_ValueError, "freq must be [rot / 2]");
            const int64_t half[1] = {f.size(0)};
            freq = (const double*)dense(a[3], half, at::kDouble, dev, "freq").const_data_ptr();
            fits_int({2 * half[0]});
            rot = (int)(2 * half[0]);
        }
        const int norm = PyObject_IsTrue(a[4]), paired = PyObject_IsTrue(a[5]);
        if (norm < 0 || paired < 0) throw PyError{};
        flags = (norm ? GFWA_HEAD_NORM : 0) | (paired ? GFWA_ROPE_PAIRED : 0);
        if (!norm && (a[0] != Py_None || a[1] != Py_None)) fail(PyExc_ValueError, "wq and wk are weights of the norm, which norm=False leaves out");
    }
};

PyObject* none_or(Output* o) {
    if (o == nullptr) Py_RETURN_NONE;
    return o->object();
}
template <size_t N>
PyObject* tuple_or_none(Output* const (&outs)[N]) {
    PyObject* r = PyTuple_New((Py_ssize_t)N);
    if (r == nullptr) throw PyError{};
    for (size_t i = 0; i < N; ++i) {
        PyObject* x = none_or(outs[i]);
        if (x == nullptr) {
            Py_DECREF(r);
            throw PyError{};
        }
        PyTuple_SET_ITEM(r, (Py_ssize_t)i, x);
    }
    return r;
}

PyObject* qk_norm_rope(PyObject* const* a) {  // q, k, v, wq, wk, eps, freq, norm, paired, pos, Q, K, V
    const at::Tensor &q = tensor_of(a[0], "q"), &k = tensor_of(a[1], "k");
    if (q.dim() != 4 || k.dim() != 4) fail(PyExc_ValueError, "q must be [B,N,H,d] and k [B,N,Hkv,d]");
    const int64_t B = q.size(0), N = q.size(1), H = q.size(2), d = q.size(3), Hkv = kv_heads(H, k.size(2));
    fits_int({B, N, H, d});
    const int dt = storage_type(q);
    const at::ScalarType st = q.scalar_type();
    const OneDevice dev(q);
    const int64_t qs[4] = {B, N, H, d}, ks[4] = {B, N, Hkv, d}, Qs[4] = {B, H, N, d}, Ks[4] = {B, Hkv, N, d}, ps[2] = {B, N};
    const Heads hq(q, qs, st, dev, "q", false), hk(k, ks, st, dev, "k", false);
    const Heads hv = a[2] == Py_None ? Heads() : Heads(tensor_of(a[2], "v"), ks, st, dev, "v", false);
    const Rotation how(a + 3, d, dev);
    const void* pos = optional_input(a[9], ps, at::kInt, dev, "pos");
    for (int i = 10; i < 13; ++i)
        if (a[i] != Py_None) dev.also(tensor_of(a[i], "an output"), "an output");
    dev.is_current();
    Output Q(a[10], Qs, st, q.device(), "Q"), K(a[11], Ks, st, q.device(), "K");
    std::optional<Output> V;
    if (hv.given) V.emplace(a[12], Ks, st, q.device(), "V");
    call([&] {
        return lib.qk_norm_rope(dt, hq.get(), hk.get(), hv.get(), how.wq, how.wk, how.eps, how.freq, how.rot, (const int*)pos, how.flags,
                                Q.ptr, K.ptr, V ? V->ptr : nullptr, (int)B, (int)H, (int)Hkv, (int)N, (int)d, stream());
    });
    return tuple_or_none({&Q, &K, V ? &*V : nullptr});
}

// A gradient of heads: the caller's strided tensor, checked, or a fresh dense one.
struct HeadsOutput {
    std::optional<Output> made;
    PyObject* given = nullptr;
    Heads h;
    HeadsOutput(PyObject* o, at::IntArrayRef shape, at::ScalarType dtype, const OneDevice& dev, const char* name) {
        if (o == Py_None) {
            made.emplace(o, shape, dtype, dev.device, name);
            h = Heads(made->made, shape, dtype, dev, name, true);
        } else {
            h = Heads(tensor_of(o, name), shape, dtype, dev, name, true);
            given = o;
        }
    }
    PyObject* object() {
        if (made) return made->object();
        Py_INCREF(given);
        return given;
    }
};

// q, k, dQ, dK, dV, wq, wk, eps, freq, norm, paired, pos, dq, dk, dv, dwq, dwk, workspace
PyObject* qk_norm_rope_backward(PyObject* const* a) {
    const int norm = PyObject_IsTrue(a[9]);
    if (norm < 0) throw PyError{};
    const bool with_q = norm || a[0] != Py_None, with_k = norm || a[1] != Py_None;  // without the norm neither is read, and the gradients have their sizes
    const at::Tensor &q = with_q ? tensor_of(a[0], "q") : tensor_of(a[2], "dQ"), &k = with_k ? tensor_of(a[1], "k") : tensor_of(a[3], "dK");
    if (q.dim() != 4 || k.dim() != 4) fail(PyExc_ValueError, "q must be [B,N,H,d] and k [B,N,Hkv,d], dQ [B,H,N,d] and dK [B,Hkv,N,d]");
    const int64_t B = q.size(0), N = q.size(with_q ? 1 : 2), H = q.size(with_q ? 2 : 1), d = q.size(3), Hkv = kv_heads(H, k.size(with_k ? 2 : 1));
    fits_int({B, N, H, d});
    const int dt = storage_type(q);
    const at::ScalarType st = q.scalar_type();
    const OneDevice dev(q);
    const int64_t qs[4] = {B, N, H, d}, ks[4] = {B, N, Hkv, d}, Qs[4] = {B, H, N, d}, Ks[4] = {B, Hkv, N, d}, ps[2] = {B, N}, ws[1] = {d};
    const Heads hq = with_q ? Heads(q, qs, st, dev, "q", false) : Heads(), hk = with_k ? Heads(k, ks, st, dev, "k", false) : Heads();
    const void *dQ = dense(a[2], Qs, st, dev, "dQ").const_data_ptr(), *dK = dense(a[3], Ks, st, dev, "dK").const_data_ptr();
    const void* dV = optional_input(a[4], Ks, st, dev, "dV");
    const Rotation how(a + 5, d, dev);
    const void* pos = optional_input(a[11], ps, at::kInt, dev, "pos");
    for (int i = 15; i < 18; ++i)
        if (a[i] != Py_None) dev.also(tensor_of(a[i], "an output"), "an output");
    const bool wants[2] = {a[5] != Py_None || a[15] != Py_None, a[6] != Py_None || a[16] != Py_None};
    if (!(how.flags & GFWA_HEAD_NORM) && (wants[0] || wants[1])) fail(PyExc_ValueError, "dwq and dwk belong to the norm, which norm=False leaves out");
    if (a[4] == Py_None && a[14] != Py_None) fail(PyExc_ValueError, "dv without dV");
    dev.is_current();
    HeadsOutput dq(a[12], qs, st, dev, "dq"), dk(a[13], ks, st, dev, "dk");
    std::optional<HeadsOutput> dv;
    if (a[4] != Py_None) dv.emplace(a[14], ks, st, dev, "dv");
    std::optional<Output> dw[2];
    for (int i = 0; i < 2; ++i)
        if (wants[i]) dw[i].emplace(a[15 + i], ws, at::kFloat, dev.device, i ? "dwk" : "dwq");
    std::optional<Workspace> scratch;
    if (wants[0] || wants[1])
        scratch.emplace(a[17], a[17] == Py_None ? lib.qk_norm_rope_backward_workspace_bytes((int)B, (int)H, (int)Hkv, (int)N, (int)d) : 0, dev.device);
    call([&] {
        return lib.qk_norm_rope_backward(dt, hq.get(), hk.get(), how.wq, how.wk, how.eps, how.freq, how.rot, (const int*)pos, how.flags, dQ, dK, dV,
                                         dq.h.get(), dk.h.get(), dv ? dv->h.get() : nullptr, dw[0] ? (float*)dw[0]->ptr : nullptr,
                                         dw[1] ? (float*)dw[1]->ptr : nullptr, scratch ? scratch->ptr : nullptr, scratch ? scratch->bytes : 0,
                                         (int)B, (int)H, (int)Hkv, (int)N, (int)d, stream());
    });
    PyObject* out[5] = {dq.object(), dk.object(), dv ? dv->object() : none_or(nullptr), none_or(dw[0] ? &*dw[0] : nullptr),
                        none_or(dw[1] ? &*dw[1] : nullptr)};
    PyObject* r = PyTuple_New(5);
    for (int i = 0; i < 5; ++i) {
        if (r == nullptr || out[i] == nullptr) {
            for (int k2 = i; k2 < 5; ++k2) Py_XDECREF(out[k2]);
            Py_XDECREF(r);
            throw PyError{};
        }
        PyTuple_SET_ITEM(r, i, out[i]);
    }
    return r;
}

// the paged cache both calls take: Kp, Vp [pages,Hkv,page,d], cp [pages,H,page] or None, table [B,max_pages]
struct Pages {
    int64_t pages, page, max_pages;
    void *Kp, *Vp;
    float* cp = nullptr;
    const int* table;
    Pages(PyObject* K, PyObject* V, PyObject* c, PyObject* t, int64_t B, int64_t H, int64_t Hkv, int64_t d, at::ScalarType st, const OneDevice& dev,
          bool write) {
        const at::Tensor& k = tensor_of(K, "Kp");
        const at::Tensor& tab = tensor_of(t, "table");
        if (k.dim() != 4 || tab.dim() != 2) fail(PyExc_ValueError, "Kp must be [pages,Hkv,page,d] and table [B,max_pages]");
        pages = k.size(0);
        page = k.size(2);
        max_pages = tab.size(1);
        const int64_t ks[4] = {pages, Hkv, page, d}, cs[3] = {pages, H, page}, ts[2] = {B, max_pages};
        const at::Tensor& kt = dense(K, ks, st, dev, "Kp");
        const at::Tensor& vt = dense(V, ks, st, dev, "Vp");
        Kp = write ? kt.data_ptr() : const_cast<void*>(kt.const_data_ptr());
        Vp = write ? vt.data_ptr() : const_cast<void*>(vt.const_data_ptr());
        if (c != Py_None) {
            const at::Tensor& ct = dense(c, cs, at::kFloat, dev, "cp");
            cp = (float*)(write ? ct.data_ptr() : const_cast<void*>(ct.const_data_ptr()));
        }
        table = (const int*)dense(t, ts, at::kInt, dev, "table").const_data_ptr();
        fits_int({pages, page, max_pages, B, H, Hkv, d});
    }
};

// k, v, Kp, Vp, start, cached, table, q, wq, wk, eps, freq, norm, paired, alpha, cp, Q
PyObject* append_paged(PyObject* const* a) {
    const at::Tensor& k = tensor_of(a[0], "k");
    if (k.dim() != 3) fail(PyExc_ValueError, "k must be [rows,Hkv,d]");
    const int64_t rows = k.size(0), Hkv = k.size(1), d = k.size(2);
    int64_t H = Hkv;
    const bool gated = a[14] != Py_None;
    if (a[7] != Py_None) {
        const at::Tensor& q = tensor_of(a[7], "q");
        if (q.dim() != 3) fail(PyExc_ValueError, "q must be [rows,H,d]");
        H = q.size(1);
    } else if (gated) {
        const at::Tensor& al = tensor_of(a[14], "alpha");
        if (al.dim() != 2) fail(PyExc_ValueError, "alpha must be [rows,H]");
        H = al.size(1);
    }
    kv_heads(H, Hkv);
    fits_int({rows});
    const int dt = storage_type(k);
    const at::ScalarType st = k.scalar_type();
    const OneDevice dev(k);
    const at::Tensor& cached = tensor_of(a[5], "cached");
    if (cached.dim() != 1) fail(PyExc_ValueError, "cached must be [B]");
    const int64_t B = cached.size(0), qs[3] = {rows, H, d}, ks[3] = {rows, Hkv, d}, bs[1] = {B}, ss[1] = {B + 1}, as[2] = {rows, H};
    const Heads hk(k, ks, st, dev, "k", false), hv(tensor_of(a[1], "v"), ks, st, dev, "v", false);
    const Heads hq = a[7] == Py_None ? Heads() : Heads(tensor_of(a[7], "q"), qs, st, dev, "q", false);
    const void *start = dense(a[4], ss, at::kInt, dev, "start").const_data_ptr(), *before = dense(a[5], bs, at::kInt, dev, "cached").const_data_ptr();
    const Rotation how(a + 8, d, dev);
    const float* alpha = nullptr;
    int64_t alpha_token = 0, alpha_head = 0;
    if (gated) {
        const at::Tensor& al = tensor_of(a[14], "alpha");
        if (!al.is_cuda()) fail(PyExc_ValueError, "alpha must live on the GPU");
        if (al.sizes() != at::IntArrayRef(as))
            fail(PyExc_ValueError, "alpha has shape " + shape_text(al.sizes()) + ", expected " + shape_text(as));
        if (al.scalar_type() != at::kFloat) fail(PyExc_TypeError, "alpha has dtype " + dtype_text(al.scalar_type()) + ", expected torch.float32");
        dev.also(al, "alpha");
        alpha = (const float*)al.const_data_ptr();
        alpha_token = rows > 1 ? al.stride(0) : 0;
        alpha_head = H > 1 ? al.stride(1) : 0;
        if (a[15] == Py_None) fail(PyExc_ValueError, "alpha without cp");
    }
    const Pages cache(a[2], a[3], gated ? a[15] : Py_None, a[6], B, H, Hkv, d, st, dev, true);
    if (a[16] != Py_None) dev.also(tensor_of(a[16], "Q"), "Q");
    dev.is_current();
    std::optional<Output> Q;
    if (hq.given) Q.emplace(a[16], qs, st, dev.device, "Q");
    call([&] {
        return lib.append_paged(dt, hq.get(), hk.get(), hv.get(), how.wq, how.wk, how.eps, how.freq, how.rot, how.flags, alpha, alpha_token,
                                alpha_head, (const int*)start, (const int*)before, cache.table, Q ? Q->ptr : nullptr, cache.Kp, cache.Vp, cache.cp,
                                (int)rows, (int)B, (int)H, (int)Hkv, (int)d, (int)cache.pages, (int)cache.page, (int)cache.max_pages,
                                stream());
    });
    return none_or(Q ? &*Q : nullptr);
}

PyObject* decode_paged(PyObject* const* a) {  // q, Kp, Vp, cp, table, pos, w, scale, o, L, workspace
    const at::Tensor& q = tensor_of(a[0], "q");
    const at::Tensor& k = tensor_of(a[1], "Kp");
    if (q.dim() != 3 || k.dim() != 4) fail(PyExc_ValueError, "q must be [B,H,d] and Kp [pages,Hkv,page,d]");
    const int64_t B = q.size(0), H = q.size(1), d = q.size(2), Hkv = kv_heads(H, k.size(1)), qs[3] = {B, H, d}, heads[2] = {B, H}, bs[1] = {B};
    const int dt = storage_type(q);
    const OneDevice dev(q);
    need(q, qs, q.scalar_type(), "q");
    if (a[3] == Py_None) fail(PyExc_TypeError, "cp must be a tensor");
    const Pages cache(a[1], a[2], a[3], a[4], B, H, Hkv, d, q.scalar_type(), dev, false);
    const void* pos = dense(a[5], bs, at::kInt, dev, "pos").const_data_ptr();
    const int w = as_window(a[6]);
    const float scale = as_float(a[7]);
    for (int i = 8; i < 11; ++i)
        if (a[i] != Py_None) dev.also(tensor_of(a[i], "an output"), "an output");
    dev.is_current();
    Output o(a[8], qs, q.scalar_type(), dev.device, "o"), L(a[9], heads, at::kFloat, dev.device, "L");
    Workspace ws(a[10], a[10] == Py_None ? lib.decode_paged_workspace_bytes((int)B, (int)H, (int)Hkv, (int)d, (int)cache.page, (int)cache.max_pages, w) : 0,
                 dev.device);
    call([&] {
        return lib.decode_paged(dt, q.const_data_ptr(), cache.Kp, cache.Vp, cache.cp, cache.table, (const int*)pos, o.ptr, (float*)L.ptr, ws.ptr,
                                ws.bytes, (int)B, (int)H, (int)Hkv, (int)d, (int)cache.pages, (int)cache.page, (int)cache.max_pages, w, scale,
                                stream());
    });
    return tuple_of({&o, &L});
}

// bind(check, (address, ...)): binding._check and the functions of `Library`, in its order
PyObject* bind(PyObject* const* a) {
    if (!PyTuple_Check(a[1]) || PyTuple_GET_SIZE(a[1]) != kFunctions)
        fail(PyExc_TypeError, "a tuple of " + std::to_string(kFunctions) + " addresses expected");
    void* addr[kFunctions];
    for (Py_ssize_t i = 0; i < kFunctions; ++i) {
        addr[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(a[1], i));
        if (PyErr_Occurred()) throw PyError{};
    }
    memcpy(&lib, addr, sizeof(lib));
    Py_INCREF(a[0]);
    Py_XDECREF(raise_status);
    raise_status = a[0];
    Py_RETURN_NONE;
}

#define GFWA_ENTRY(f, n) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&entry<f, n>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {GFWA_ENTRY(bind, 2),
                         GFWA_ENTRY(gate_prefix, 2),
                         GFWA_ENTRY(gate_activation_prefix, 4),
                         GFWA_ENTRY(gate_activation_backward, 6),
                         GFWA_ENTRY(gate_prefix_stp, 5),
                         GFWA_ENTRY(forward, 9),
                         GFWA_ENTRY(backward, 15),
                         GFWA_ENTRY(decode, 11),
                         GFWA_ENTRY(decode_static, 10),
                         GFWA_ENTRY(qk_norm_rope, 13),
                         GFWA_ENTRY(qk_norm_rope_backward, 18),
                         GFWA_ENTRY(append_paged, 17),
                         GFWA_ENTRY(decode_paged, 11),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_gfwa_call", "Checked calls of libgfwa on torch tensors.", -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__gfwa_call(void) { return PyModule_Create(&module); }
