// The Python binding's short way into libpsgd: the calls of a training loop with plain device tensors, checked and passed on
// without building Python objects for every shape and pointer (psgd.py's own way takes 2.5 to 3 us of a 5.5 to 10 us call).
// A call that is not plainly in order is not answered here: NOT_MINE sends it psgd.py's way, which checks it argument by argument
// and raises what there is to raise, as it does for the library's refusals of an argument; other failures psgd.py raises at once.  Nothing is kept between calls but the addresses of the library's functions.
#include <Python.h>

#include <torch/csrc/autograd/python_variable.h>

#include <c10/core/Allocator.h>
#include <c10/hip/HIPStream.h>

#include <cmath>
#include <cstdint>
#include <initializer_list>

#include "psgd.h"
#include "psgd_attention.h"
#include "psgd_layers.h"

namespace {

constexpr long NOT_MINE = 1;   // the library's own statuses are zero and negative

struct Library {
    decltype(&psgd_mix_step_deg) mix_step_deg = nullptr;
    decltype(&psgd_mix_step_d1d) mix_step_d1d = nullptr;
    decltype(&psgd_mix_full) mix_full = nullptr;
    decltype(&psgd_build_mixing_device) build_mixing_device = nullptr;
    decltype(&psgd_consensus_dist_ex) consensus_dist_ex = nullptr;
    decltype(&psgd_synth_grad_ex) synth_grad_ex = nullptr;
    decltype(&psgd_consensus_dist) consensus_dist = nullptr;
} lib;

// A plain strided tensor on device `dev` whose pointer means what it says: no subclass, no tensor of a transform or a trace.
const at::Tensor* plain(PyObject* o, int dev) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.defined() || !t.is_cuda() || t.layout() != at::kStrided || t.get_device() != dev || !t.has_storage()) return nullptr;
    const at::TensorImpl* impl = t.unsafeGetTensorImpl();
    if (impl->is_python_dispatch()) return nullptr;
    const c10::DispatchKeySet ks = t.key_set();
    using K = c10::DispatchKey;
    for (K k : {K::FuncTorchBatched, K::FuncTorchGradWrapper, K::Functionalize, K::Conjugate, K::Negative, K::ZeroTensor, K::Python})
        if (ks.has(k)) return nullptr;
    return &t;
}

struct Rows {
    void* p;
    int64_t ld;
};
// [n, d] with unit stride along d; the first tensor says what n and d are (n < 0 on entry).
bool rows(PyObject* o, int dev, c10::ScalarType type, int64_t& n, int64_t& d, Rows& r) {
    const at::Tensor* t = plain(o, dev);
    if (!t || t->scalar_type() != type || t->dim() != 2) return false;
    const int64_t tn = t->size(0), td = t->size(1);
    if (n < 0) {
        n = tn;
        d = td;
    }
    if (tn != n || td != d || n < 1 || n > PSGD_MAX_N || (d > 1 && t->stride(1) != 1)) return false;
    r.p = t->data_ptr();
    r.ld = n > 1 ? t->stride(0) : d;
    return true;
}
// A contiguous table of `type` with a whole number of slots per row.
bool table(PyObject* o, int dev, c10::ScalarType type, int64_t n, int64_t& deg, void*& p) {
    const at::Tensor* t = plain(o, dev);
    if (!t || t->scalar_type() != type || !t->is_contiguous() || t->numel() < n || t->numel() % n || t->numel() / n > PSGD_MAX_DEG)
        return false;
    if (deg < 0) deg = t->numel() / n;
    p = t->data_ptr();
    return deg == t->numel() / n;
}
bool scalar_out(PyObject* o, int dev, double*& p) {
    p = nullptr;
    if (o == Py_None) return true;
    const at::Tensor* t = plain(o, dev);
    if (!t || t->scalar_type() != at::kDouble || t->numel() < 1) return false;
    p = static_cast<double*>(t->data_ptr());
    return true;
}
// The stream's handle: the current one for None, else the object's own.
bool stream_of(PyObject* o, int dev, void*& s) {
    if (o == Py_None) {
        s = c10::hip::getCurrentHIPStream(static_cast<c10::DeviceIndex>(dev)).stream();
        return true;
    }
    PyObject* h = PyObject_GetAttrString(o, "cuda_stream");
    if (!h) {
        PyErr_Clear();
        return false;
    }
    s = PyLong_AsVoidPtr(h);
    Py_DECREF(h);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        return false;
    }
    return true;
}
bool number(PyObject* o, float& v) {
    if (!PyFloat_CheckExact(o)) return false;
    v = static_cast<float>(PyFloat_AS_DOUBLE(o));
    return true;
}
bool integer(PyObject* o, int64_t& v) {
    if (!PyLong_CheckExact(o)) return false;
    int over = 0;
    v = PyLong_AsLongLongAndOverflow(o, &over);
    return !over;
}
int device() { return lib.mix_full ? static_cast<int>(c10::hip::current_device()) : -1; }
PyObject* answer(long rc) { return PyLong_FromLong(rc); }

// Errors of torch's own accessors (C++ exceptions) are not for Python's C API to meet: such a call goes the long way.
template <typename F> PyObject* guarded(const F& f) {
    try {
        return answer(f());
    } catch (...) {
        return answer(NOT_MINE);
    }
}

// The library's calls run without the interpreter's lock, as through ctypes.
struct Unlocked {
    PyThreadState* state = PyEval_SaveThread();
    ~Unlocked() { PyEval_RestoreThread(state); }
};

bool gradient_type(PyObject* o, c10::ScalarType& type, int& bf16) {
    if (!THPVariable_CheckExact(o)) return false;
    type = THPVariable_Unpack(o).scalar_type();
    bf16 = type != at::kFloat;
    return type == at::kFloat || type == at::kBFloat16;
}

// mix_step(X, X_out, G, nbr, w, lr, delay_mode, stream, cdist_out)
PyObject* mix_step(PyObject*, PyObject* const* a, Py_ssize_t count) {
    return guarded([&]() -> long {
        const int dev = device();
        int64_t n = -1, d = 0, deg = -1, mode = 0;
        Rows x, o, g;
        void *nbr, *w, *s;
        double* cd;
        float lr;
        c10::ScalarType type;
        int bf16 = 0;
        if (count != 9 || dev < 0 || !gradient_type(a[2], type, bf16) || !rows(a[0], dev, at::kFloat, n, d, x) ||
            !rows(a[1], dev, at::kFloat, n, d, o) || !rows(a[2], dev, type, n, d, g) || !table(a[3], dev, at::kInt, n, deg, nbr) ||
            !table(a[4], dev, at::kFloat, n, deg, w) || !number(a[5], lr) || !integer(a[6], mode) || mode < 0 || mode > 1 ||
            !stream_of(a[7], dev, s) || !scalar_out(a[8], dev, cd))
            return NOT_MINE;
        Unlocked run;
        return lib.mix_step_deg(static_cast<float*>(x.p), x.ld, static_cast<float*>(o.p), o.ld, g.p, g.ld, bf16,
                                static_cast<int32_t*>(nbr), static_cast<float*>(w), static_cast<int>(deg), static_cast<int>(n), d, lr,
                                static_cast<int>(mode), cd, s);
    });
}

// mix_full(X, X_out, G, lr, delay_mode, stream, cdist_out)
PyObject* mix_full(PyObject*, PyObject* const* a, Py_ssize_t count) {
    return guarded([&]() -> long {
        const int dev = device();
        int64_t n = -1, d = 0, mode = 0;
        Rows x, o, g;
        void* s;
        double* cd;
        float lr;
        c10::ScalarType type;
        int bf16 = 0;
        if (count != 7 || dev < 0 || !gradient_type(a[2], type, bf16) || !rows(a[0], dev, at::kFloat, n, d, x) ||
            !rows(a[1], dev, at::kFloat, n, d, o) || !rows(a[2], dev, type, n, d, g) || !number(a[3], lr) || !integer(a[4], mode) ||
            mode < 0 || mode > 1 || !stream_of(a[5], dev, s) || !scalar_out(a[6], dev, cd))
            return NOT_MINE;
        Unlocked run;
        return lib.mix_full(static_cast<float*>(x.p), x.ld, static_cast<float*>(o.p), o.ld, g.p, g.ld, bf16, static_cast<int>(n), d, lr,
                            static_cast<int>(mode), cd, s);
    });
}

// mix_step_d1d(X, X_out, G, nbr, w, lr, noise, G_next, c, stream, cdist_out)
PyObject* mix_step_d1d(PyObject*, PyObject* const* a, Py_ssize_t count) {
    return guarded([&]() -> long {
        const int dev = device();
        int64_t n = -1, d = 0, deg = -1;
        Rows x, o, g, z, h;
        void *nbr, *w, *s;
        double* cd;
        float lr, c;
        if (count != 11 || dev < 0 || !rows(a[0], dev, at::kFloat, n, d, x) || !rows(a[1], dev, at::kFloat, n, d, o) ||
            !rows(a[2], dev, at::kFloat, n, d, g) || !table(a[3], dev, at::kInt, n, deg, nbr) || !table(a[4], dev, at::kFloat, n, deg, w) ||
            !number(a[5], lr) || !rows(a[6], dev, at::kFloat, n, d, z) || !rows(a[7], dev, at::kFloat, n, d, h) || !number(a[8], c) ||
            !stream_of(a[9], dev, s) || !scalar_out(a[10], dev, cd))
            return NOT_MINE;
        Unlocked run;
        return lib.mix_step_d1d(static_cast<float*>(x.p), x.ld, static_cast<float*>(o.p), o.ld, static_cast<float*>(g.p), g.ld,
                                static_cast<int32_t*>(nbr), static_cast<float*>(w), static_cast<int>(deg), static_cast<int>(n), d, lr,
                                static_cast<float*>(z.p), z.ld, static_cast<float*>(h.p), h.ld, c, cd, s);
    });
}

// build_mixing_device(topology, n, seed, nbr, w, step_dev, step_offset, advance, stream)
PyObject* build_mixing_device(PyObject*, PyObject* const* a, Py_ssize_t count) {
    return guarded([&]() -> long {
        const int dev = device();
        int64_t topology, n, seed, offset, advance, deg = PSGD_DEG;
        void *nbr, *w, *s;
        uint64_t* step = nullptr;
        if (count != 9 || dev < 0 || !integer(a[0], topology) || !integer(a[1], n) || !integer(a[2], seed) || topology < 0 ||
            topology > 2 || n < 1 || n > PSGD_MAX_N || !table(a[3], dev, at::kInt, n, deg, nbr) || !table(a[4], dev, at::kFloat, n, deg, w) ||
            !integer(a[6], offset) || !integer(a[7], advance) || advance < 0 || advance > INT32_MAX || !stream_of(a[8], dev, s))
            return NOT_MINE;
        if (a[5] != Py_None) {
            const at::Tensor* t = plain(a[5], dev);
            if (!t || (t->scalar_type() != at::kLong && t->scalar_type() != at::kUInt64) || t->numel() < 1) return NOT_MINE;
            step = static_cast<uint64_t*>(t->data_ptr());
        }
        Unlocked run;
        return lib.build_mixing_device(static_cast<int>(topology), static_cast<int>(n), static_cast<uint64_t>(seed), step,
                                       static_cast<uint64_t>(offset), static_cast<int>(advance), static_cast<int32_t*>(nbr),
                                       static_cast<float*>(w), s);
    });
}

// consensus_dist_async(X, out, stream)
PyObject* consensus_dist_async(PyObject*, PyObject* const* a, Py_ssize_t count) {
    return guarded([&]() -> long {
        const int dev = device();
        int64_t n = -1, d = 0;
        Rows x;
        double* out;
        void* s;
        if (count != 3 || dev < 0 || a[1] == Py_None || !rows(a[0], dev, at::kFloat, n, d, x) || !scalar_out(a[1], dev, out) ||
            !stream_of(a[2], dev, s))
            return NOT_MINE;
        Unlocked run;
        return lib.consensus_dist_ex(static_cast<float*>(x.p), x.ld, static_cast<int>(n), d, out, s);
    });
}

// consensus_dist(X): the value, or None where the call is not answered here
PyObject* consensus_dist(PyObject*, PyObject* const* a, Py_ssize_t count) {
    double v = 0.0;
    bool mine = false;
    try {
        const int dev = device();
        int64_t n = -1, d = 0;
        Rows x;
        if (count == 1 && dev >= 0 && rows(a[0], dev, at::kFloat, n, d, x) && THPVariable_Unpack(a[0]).is_contiguous()) {
            Unlocked run;
            v = lib.consensus_dist(static_cast<float*>(x.p), static_cast<int>(n), d);
            mine = true;
        }
    } catch (...) {
    }
    if (!mine) Py_RETURN_NONE;
    return PyFloat_FromDouble(v);
}

// synth_grad(X_prev, noise, G, c, stream)
PyObject* synth_grad(PyObject*, PyObject* const* a, Py_ssize_t count) {
    return guarded([&]() -> long {
        const int dev = device();
        int64_t n = -1, d = 0;
        Rows x, z, g;
        float c;
        void* s;
        if (count != 5 || dev < 0 || !rows(a[0], dev, at::kFloat, n, d, x) || !rows(a[1], dev, at::kFloat, n, d, z) ||
            !rows(a[2], dev, at::kFloat, n, d, g) || !number(a[3], c) || !stream_of(a[4], dev, s))
            return NOT_MINE;
        Unlocked run;
        return lib.synth_grad_ex(static_cast<float*>(x.p), x.ld, static_cast<float*>(z.p), z.ld, static_cast<float*>(g.p), g.ld,
                                 static_cast<int>(n), d, c, s);
    });
}

// ------------------------------------------------------------------------------------------------ layers and losses (psgd_layers.h)
struct Layers {
    decltype(&psgd_layer_norm) layer_norm = nullptr;
    decltype(&psgd_layer_norm_grad) layer_norm_grad = nullptr;
    decltype(&psgd_layer_norm_grad_workspace) layer_norm_grad_workspace = nullptr;
    decltype(&psgd_linear) linear = nullptr;
    decltype(&psgd_linear_workspace) linear_workspace = nullptr;
    decltype(&psgd_linear_grad) linear_grad = nullptr;
    decltype(&psgd_linear_grad_workspace) linear_grad_workspace = nullptr;
    decltype(&psgd_token_logprobs) token_logprobs = nullptr;
    decltype(&psgd_distill) distill = nullptr;
} layers;
int layers_device() { return layers.distill ? static_cast<int>(c10::hip::current_device()) : -1; }

// An operand as the library takes it; None is no operand.
struct Operand {
    psgd_view v{};
    bool there = false;
    const psgd_view* get() const { return there ? &v : nullptr; }
};
// The sizes in `shape` that are negative are taken from the tensor, the others have to be its.
bool operand(PyObject* o, int dev, std::initializer_list<int64_t*> shape, Operand& x, bool optional = false) {
    if (o == Py_None) return optional;
    const at::Tensor* t = plain(o, dev);
    if (!t || t->dim() != static_cast<int64_t>(shape.size())) return false;
    int64_t dims = 0;
    for (int64_t* size : shape) {
        const int64_t have = t->size(dims++);
        if (*size < 0) *size = have;
        if (*size != have) return false;
    }
    const c10::ScalarType type = t->scalar_type();
    if (type != at::kFloat && type != at::kBFloat16 && type != at::kInt) return false;
    if (t->size(dims - 1) > 1 && t->stride(dims - 1) != 1) return false;
    x.v.data = t->data_ptr();
    x.v.learner = t->size(0) > 1 ? t->stride(0) : 0;
    x.v.row = dims == 3 && t->size(1) > 1 ? t->stride(1) : 0;
    x.v.type = type == at::kFloat ? PSGD_F32 : type == at::kBFloat16 ? PSGD_BF16 : PSGD_I32;
    x.there = true;
    return true;
}
template <typename T> bool vector(PyObject* o, int dev, int64_t numel, c10::ScalarType type, T*& p) {
    p = nullptr;
    if (o == Py_None) return true;
    const at::Tensor* t = plain(o, dev);
    if (!t || t->scalar_type() != type || t->numel() != numel || !t->is_contiguous()) return false;
    p = static_cast<T*>(t->data_ptr());
    return true;
}
// `bytes` of torch's allocator for work on stream `s`: kept until the call has returned, after which the stream's order keeps it.  Only for the current
// stream, on which the allocator hands them out.
bool workspace(int dev, size_t bytes, void* s, c10::DataPtr& room) {
    if (!bytes) return true;
    if (s != c10::hip::getCurrentHIPStream(static_cast<c10::DeviceIndex>(dev)).stream()) return false;
    room = c10::GetAllocator(c10::kCUDA)->allocate(bytes);
    return room.get() != nullptr;
}

// layer_norm(x, gain, bias, y, eps, mean, rstd, stream)
PyObject* layer_norm(PyObject*, PyObject* const* a, Py_ssize_t count) {
    return guarded([&]() -> long {
        const int dev = layers_device();
        int64_t n = -1, t = -1, c = -1;
        Operand x, g, b, y;
        float eps, *mean, *rstd;
        void* s;
        if (count != 8 || dev < 0 || !operand(a[0], dev, {&n, &t, &c}, x) || !operand(a[1], dev, {&n, &c}, g) ||
            !operand(a[2], dev, {&n, &c}, b, true) || !operand(a[3], dev, {&n, &t, &c}, y) || !number(a[4], eps) || n > PSGD_MAX_N ||
            !vector(a[5], dev, n * t, at::kFloat, mean) || !vector(a[6], dev, n * t, at::kFloat, rstd) || !stream_of(a[7], dev, s))
            return NOT_MINE;
        Unlocked run;
        return layers.layer_norm(x.get(), g.get(), b.get(), y.get(), mean, rstd, static_cast<int>(n), t, c, eps, s);
    });
}

// layer_norm_grad(dy, x, gain, mean, rstd, dx, dgain, dbias, add, stream)
PyObject* layer_norm_grad(PyObject*, PyObject* const* a, Py_ssize_t count) {
    return guarded([&]() -> long {
        const int dev = layers_device();
        int64_t n = -1, t = -1, c = -1;
        Operand dy, x, g, dx, dg, db, add;
        float *mean, *rstd;
        void* s;
        c10::DataPtr room;
        if (count != 10 || dev < 0 || !operand(a[0], dev, {&n, &t, &c}, dy) || !operand(a[1], dev, {&n, &t, &c}, x) ||
            !operand(a[2], dev, {&n, &c}, g) || n > PSGD_MAX_N || !vector(a[3], dev, n * t, at::kFloat, mean) ||
            !vector(a[4], dev, n * t, at::kFloat, rstd) || !operand(a[5], dev, {&n, &t, &c}, dx) || !operand(a[6], dev, {&n, &c}, dg, true) ||
            !operand(a[7], dev, {&n, &c}, db, true) || !operand(a[8], dev, {&n, &t, &c}, add, true) || !stream_of(a[9], dev, s))
            return NOT_MINE;
        const size_t need = dg.there || db.there ? layers.layer_norm_grad_workspace(static_cast<int>(n), t, c) : 0;
        if (!workspace(dev, need, s, room)) return NOT_MINE;
        Unlocked run;
        return layers.layer_norm_grad(dy.get(), x.get(), g.get(), mean, rstd, add.get(), dx.get(), dg.get(), db.get(), static_cast<int>(n), t, c,
                                      room.get(), need, s);
    });
}

// linear(x, w, y, bias, act, residual, z, stream)
PyObject* linear(PyObject*, PyObject* const* a, Py_ssize_t count) {
    return guarded([&]() -> long {
        const int dev = layers_device();
        int64_t n = -1, t = -1, i = -1, o = -1, act;
        Operand x, w, y, b, r, z;
        void* s;
        c10::DataPtr room;
        if (count != 8 || dev < 0 || !operand(a[0], dev, {&n, &t, &i}, x) || !operand(a[1], dev, {&n, &o, &i}, w) || n > PSGD_MAX_N ||
            !operand(a[2], dev, {&n, &t, &o}, y) || !operand(a[3], dev, {&n, &o}, b, true) || !integer(a[4], act) ||
            !operand(a[5], dev, {&n, &t, &o}, r, true) || !operand(a[6], dev, {&n, &t, &o}, z, true) || !stream_of(a[7], dev, s))
            return NOT_MINE;
        const size_t need = layers.linear_workspace(x.get(), w.get(), static_cast<int>(n), t, i, o);
        if (!workspace(dev, need, s, room)) return NOT_MINE;
        Unlocked run;
        return layers.linear(x.get(), w.get(), b.get(), r.get(), y.get(), z.get(), static_cast<int>(act), static_cast<int>(n), t, i, o,
                             room.get(), need, s);
    });
}

// linear_grad(dy, x, w, dx, dw, db, act, z, stream)
PyObject* linear_grad(PyObject*, PyObject* const* a, Py_ssize_t count) {
    return guarded([&]() -> long {
        const int dev = layers_device();
        int64_t n = -1, t = -1, i = -1, o = -1, act;
        Operand dy, x, w, dx, dw, db, z;
        void* s;
        c10::DataPtr room;
        if (count != 9 || dev < 0 || !operand(a[0], dev, {&n, &t, &o}, dy) || !operand(a[1], dev, {&n, &t, &i}, x) ||
            !operand(a[2], dev, {&n, &o, &i}, w) || n > PSGD_MAX_N || !operand(a[3], dev, {&n, &t, &i}, dx, true) ||
            !operand(a[4], dev, {&n, &o, &i}, dw, true) || !operand(a[5], dev, {&n, &o}, db, true) || !integer(a[6], act) ||
            !operand(a[7], dev, {&n, &t, &o}, z, true) || !stream_of(a[8], dev, s))
            return NOT_MINE;
        const size_t need = layers.linear_grad_workspace(dy.get(), x.get(), w.get(), dx.get(), dw.get(), db.get(), static_cast<int>(act),
                                                         static_cast<int>(n), t, i, o);
        if (!workspace(dev, need, s, room)) return NOT_MINE;
        Unlocked run;
        return layers.linear_grad(dy.get(), z.get(), x.get(), w.get(), dx.get(), dw.get(), db.get(), static_cast<int>(act), static_cast<int>(n),
                                  t, i, o, room.get(), need, s);
    });
}

// token_logprobs(logits, tokens, logp, entropy, top_logp, top_idx, stream)
PyObject* token_logprobs(PyObject*, PyObject* const* a, Py_ssize_t count) {
    return guarded([&]() -> long {
        const int dev = layers_device();
        int64_t n = -1, t = -1, v = -1, k = 0;
        Operand x, tok;
        float *logp, *entropy, *top;
        int32_t* idx;
        void* s;
        if (count != 7 || dev < 0 || !operand(a[0], dev, {&n, &t, &v}, x) || n > PSGD_MAX_N) return NOT_MINE;
        const at::Tensor* given = plain(a[1], dev);
        if (!given || given->scalar_type() != at::kInt || given->dim() != 2 || given->size(0) != n || given->size(1) != t) return NOT_MINE;
        tok.v = psgd_view{given->data_ptr(), n > 1 ? given->stride(0) : 0, t > 1 ? given->stride(1) : 0, PSGD_I32};
        if (a[5] != Py_None) {
            const at::Tensor* at = plain(a[5], dev);
            if (!at || at->dim() != 3) return NOT_MINE;
            k = at->size(2);
        }
        if ((a[4] == Py_None) != (a[5] == Py_None) || k > PSGD_MAX_TOP || !vector(a[2], dev, n * t, at::kFloat, logp) ||
            !vector(a[3], dev, n * t, at::kFloat, entropy) || !vector(a[4], dev, n * t * k, at::kFloat, top) ||
            !vector(a[5], dev, n * t * k, at::kInt, idx) || !stream_of(a[6], dev, s))
            return NOT_MINE;
        Unlocked run;
        return layers.token_logprobs(x.get(), &tok.v, logp, entropy, top, idx, static_cast<int>(k), static_cast<int>(n), t, v, s);
    });
}

// distill(logits, top_idx, top_logit, loss, tau, weight, dlogits, stream)
PyObject* distill(PyObject*, PyObject* const* a, Py_ssize_t count) {
    return guarded([&]() -> long {
        const int dev = layers_device();
        int64_t n = -1, t = -1, v = -1, k = -1;
        Operand x, idx, top, g;
        float tau, *loss, *weight;
        void* s;
        if (count != 8 || dev < 0 || !operand(a[0], dev, {&n, &t, &v}, x) || n > PSGD_MAX_N || !operand(a[1], dev, {&n, &t, &k}, idx) ||
            !operand(a[2], dev, {&n, &t, &k}, top) || k > PSGD_MAX_SLOTS || !vector(a[3], dev, n * t, at::kFloat, loss) || !number(a[4], tau) ||
            !vector(a[5], dev, n * t, at::kFloat, weight) || !operand(a[6], dev, {&n, &t, &v}, g, true) || !stream_of(a[7], dev, s))
            return NOT_MINE;
        Unlocked run;
        return layers.distill(x.get(), idx.get(), top.get(), weight, loss, g.get(), tau, static_cast<int>(k), static_cast<int>(n), t, v, s);
    });
}

// bind_layers(addresses of the functions, in the order of struct Layers)
PyObject* bind_layers(PyObject*, PyObject* const* a, Py_ssize_t count) {
    void* p[9];
    if (count != 9) return answer(NOT_MINE);
    for (int i = 0; i < 9; ++i) {
        p[i] = PyLong_AsVoidPtr(a[i]);
        if (PyErr_Occurred()) return nullptr;
    }
    layers.layer_norm = reinterpret_cast<decltype(layers.layer_norm)>(p[0]);
    layers.layer_norm_grad = reinterpret_cast<decltype(layers.layer_norm_grad)>(p[1]);
    layers.layer_norm_grad_workspace = reinterpret_cast<decltype(layers.layer_norm_grad_workspace)>(p[2]);
    layers.linear = reinterpret_cast<decltype(layers.linear)>(p[3]);
    layers.linear_workspace = reinterpret_cast<decltype(layers.linear_workspace)>(p[4]);
    layers.linear_grad = reinterpret_cast<decltype(layers.linear_grad)>(p[5]);
    layers.linear_grad_workspace = reinterpret_cast<decltype(layers.linear_grad_workspace)>(p[6]);
    layers.token_logprobs = reinterpret_cast<decltype(layers.token_logprobs)>(p[7]);
    layers.distill = reinterpret_cast<decltype(layers.distill)>(p[8]);
    return answer(0);
}

// bind(addresses of the functions, in the order of struct Library)
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t count) {
    void* p[7];
    if (count != 7) return answer(NOT_MINE);
    for (int i = 0; i < 7; ++i) {
        p[i] = PyLong_AsVoidPtr(a[i]);
        if (PyErr_Occurred()) return nullptr;
    }
    lib.mix_step_deg = reinterpret_cast<decltype(lib.mix_step_deg)>(p[0]);
    lib.mix_step_d1d = reinterpret_cast<decltype(lib.mix_step_d1d)>(p[1]);
    lib.mix_full = reinterpret_cast<decltype(lib.mix_full)>(p[2]);
    lib.build_mixing_device = reinterpret_cast<decltype(lib.build_mixing_device)>(p[3]);
    lib.consensus_dist_ex = reinterpret_cast<decltype(lib.consensus_dist_ex)>(p[4]);
    lib.synth_grad_ex = reinterpret_cast<decltype(lib.synth_grad_ex)>(p[5]);
    lib.consensus_dist = reinterpret_cast<decltype(lib.consensus_dist)>(p[6]);
    return answer(0);
}

// ------------------------------------------------------------------------------------------------ attention blocks (psgd_attention.h)
struct Attention {
    decltype(&psgd_qk_norm_rope) qk_norm_rope = nullptr;
    decltype(&psgd_qk_norm_rope_grad) qk_norm_rope_grad = nullptr;
    decltype(&psgd_qk_norm_rope_grad_workspace) qk_norm_rope_grad_workspace = nullptr;
    decltype(&psgd_attention) attention = nullptr;
    decltype(&psgd_attention_grad) attention_grad = nullptr;
    decltype(&psgd_attention_grad_workspace) attention_grad_workspace = nullptr;
    decltype(&psgd_attention_step) attention_step = nullptr;
    decltype(&psgd_attention_step_workspace) attention_step_workspace = nullptr;
    decltype(&psgd_dropout) dropout = nullptr;
} blocks;
int blocks_device() { return blocks.dropout ? static_cast<int>(c10::hip::current_device()) : -1; }

// What the calls have in common: n learners of t tokens, heads of the queries and of the keys.
struct Heads {
    int64_t n = -1, t = -1, cq = -1, ck = -1, heads, kv, head;
    // After the queries have said what n, t and cq are.
    bool of(PyObject* h, PyObject* k) {
        if (!integer(h, heads) || !integer(k, kv) || heads < 1 || kv < 1 || cq % heads || n > PSGD_MAX_N) return false;
        head = cq / heads;
        ck = kv * head;
        return heads <= INT32_MAX && kv <= INT32_MAX && head <= PSGD_MAX_HEAD;
    }
};
// [rows, cols] int32 of any strides.
bool numbers(PyObject* o, int dev, int64_t rows, int64_t cols, Operand& x, bool optional = false) {
    if (o == Py_None) return optional;
    const at::Tensor* t = plain(o, dev);
    if (!t || t->scalar_type() != at::kInt || t->dim() != 2 || t->size(0) != rows || t->size(1) != cols) return false;
    x.v = psgd_view{t->data_ptr(), rows > 1 ? t->stride(0) : 0, cols > 1 ? t->stride(1) : 0, PSGD_I32};
    x.there = true;
    return true;
}
bool starts_of(PyObject* o, int dev, int64_t n, Operand& x, int64_t& sequences) {
    sequences = 0;
    if (o == Py_None) return true;
    const at::Tensor* t = plain(o, dev);
    if (!t || t->scalar_type() != at::kInt || t->dim() != 2 || t->size(0) != n || t->size(1) < 2 || t->stride(1) != 1) return false;
    x.v = psgd_view{t->data_ptr(), n > 1 ? t->stride(0) : 0, 0, PSGD_I32};
    x.there = true;
    sequences = t->size(1) - 1;
    return sequences <= INT32_MAX;
}
bool small(PyObject* o, int& v) {
    int64_t x;
    if (!integer(o, x) || x < INT32_MIN || x > INT32_MAX) return false;
    v = static_cast<int>(x);
    return true;
}
bool real(PyObject* o, double& v) {
    if (!PyFloat_CheckExact(o)) return false;
    v = PyFloat_AS_DOUBLE(o);
    return true;
}
// None: head ** -0.5, in 64 bits as Python has it
bool scale_of(PyObject* o, int64_t head, float& v) {
    if (o != Py_None) return number(o, v);
    v = static_cast<float>(std::pow(static_cast<double>(head), -0.5));
    return true;
}
bool word_of(PyObject* o, uint64_t& v) {
    if (!PyLong_CheckExact(o)) return false;
    v = PyLong_AsUnsignedLongLongMask(o);
    return true;
}

// qk_norm_rope(q, k, q_out, k_out, heads, kv, positions, q_gain, k_gain, eps, rotary, base, pairs, stream)
PyObject* qk_norm_rope(PyObject*, PyObject* const* a, Py_ssize_t count) {
    return guarded([&]() -> long {
        const int dev = blocks_device();
        Heads s;
        Operand q, k, qo, ko, pos, gq, gk;
        float eps;
        double base;
        int rotary, pairs;
        void* st;
        if (count != 14 || dev < 0 || !operand(a[0], dev, {&s.n, &s.t, &s.cq}, q) || !s.of(a[4], a[5]) || !operand(a[1], dev, {&s.n, &s.t, &s.ck}, k) ||
            !operand(a[2], dev, {&s.n, &s.t, &s.cq}, qo) || !operand(a[3], dev, {&s.n, &s.t, &s.ck}, ko) || !numbers(a[6], dev, s.n, s.t, pos, true) ||
            !operand(a[7], dev, {&s.n, &s.head}, gq, true) || !operand(a[8], dev, {&s.n, &s.head}, gk, true) || !number(a[9], eps) || !small(a[10], rotary) ||
            !real(a[11], base) || !small(a[12], pairs) || !stream_of(a[13], dev, st))
            return NOT_MINE;
        Unlocked run;
        return blocks.qk_norm_rope(q.get(), k.get(), pos.get(), gq.get(), gk.get(), qo.get(), ko.get(), static_cast<int>(s.heads), static_cast<int>(s.kv),
                                   static_cast<int>(s.head), rotary, pairs, base, eps, static_cast<int>(s.n), s.t, st);
    });
}

// qk_norm_rope_grad(dq_out, dk_out, q, k, dq, dk, heads, kv, positions, q_gain, k_gain, dq_gain, dk_gain, eps, rotary, base, pairs, stream)
PyObject* qk_norm_rope_grad(PyObject*, PyObject* const* a, Py_ssize_t count) {
    return guarded([&]() -> long {
        const int dev = blocks_device();
        Heads s;
        Operand qo, ko, q, k, dq, dk, pos, gq, gk, dgq, dgk;
        float eps;
        double base;
        int rotary, pairs;
        void* st;
        c10::DataPtr room;
        if (count != 18 || dev < 0 || !operand(a[0], dev, {&s.n, &s.t, &s.cq}, qo) || !s.of(a[6], a[7]) || !operand(a[1], dev, {&s.n, &s.t, &s.ck}, ko) ||
            !operand(a[2], dev, {&s.n, &s.t, &s.cq}, q, true) || !operand(a[3], dev, {&s.n, &s.t, &s.ck}, k, true) || !operand(a[4], dev, {&s.n, &s.t, &s.cq}, dq) ||
            !operand(a[5], dev, {&s.n, &s.t, &s.ck}, dk) || !numbers(a[8], dev, s.n, s.t, pos, true) || !operand(a[9], dev, {&s.n, &s.head}, gq, true) ||
            !operand(a[10], dev, {&s.n, &s.head}, gk, true) || !operand(a[11], dev, {&s.n, &s.head}, dgq, true) || !operand(a[12], dev, {&s.n, &s.head}, dgk, true) ||
            (!gq.there && (dgq.there || dgk.there)) || !number(a[13], eps) || !small(a[14], rotary) || !real(a[15], base) || !small(a[16], pairs) ||
            !stream_of(a[17], dev, st))
            return NOT_MINE;
        const size_t need = dgq.there || dgk.there ? blocks.qk_norm_rope_grad_workspace(static_cast<int>(s.n), s.t, static_cast<int>(s.head)) : 0;
        if (!workspace(dev, need, st, room)) return NOT_MINE;
        Unlocked run;
        return blocks.qk_norm_rope_grad(qo.get(), ko.get(), q.get(), k.get(), pos.get(), gq.get(), gk.get(), dq.get(), dk.get(), dgq.get(), dgk.get(),
                                        static_cast<int>(s.heads), static_cast<int>(s.kv), static_cast<int>(s.head), rotary, pairs, base, eps,
                                        static_cast<int>(s.n), s.t, room.get(), need, st);
    });
}

// attention(q, k, v, out, heads, kv, lse, starts, window, sinks, scale, stream)
PyObject* attention(PyObject*, PyObject* const* a, Py_ssize_t count) {
    return guarded([&]() -> long {
        const int dev = blocks_device();
        Heads s;
        Operand q, k, v, o, st;
        float *lse, scale;
        int window, sinks;
        int64_t sequences;
        void* stream;
        if (count != 12 || dev < 0 || !operand(a[0], dev, {&s.n, &s.t, &s.cq}, q) || !s.of(a[4], a[5]) || !operand(a[1], dev, {&s.n, &s.t, &s.ck}, k) ||
            !operand(a[2], dev, {&s.n, &s.t, &s.ck}, v) || !operand(a[3], dev, {&s.n, &s.t, &s.cq}, o) || !vector(a[6], dev, s.n * s.heads * s.t, at::kFloat, lse) ||
            !starts_of(a[7], dev, s.n, st, sequences) || !small(a[8], window) || !small(a[9], sinks) || !scale_of(a[10], s.head, scale) || !stream_of(a[11], dev, stream))
            return NOT_MINE;
        Unlocked run;
        return blocks.attention(q.get(), k.get(), v.get(), st.get(), o.get(), lse, static_cast<int>(s.heads), static_cast<int>(s.kv), static_cast<int>(s.head), window,
                                sinks, scale, static_cast<int>(sequences), static_cast<int>(s.n), s.t, stream);
    });
}

// attention_grad(dout, q, k, v, out, lse, dq, dk, dv, heads, kv, starts, window, sinks, scale, stream)
PyObject* attention_grad(PyObject*, PyObject* const* a, Py_ssize_t count) {
    return guarded([&]() -> long {
        const int dev = blocks_device();
        Heads s;
        Operand d, q, k, v, o, st, dq, dk, dv;
        float *lse, scale;
        int window, sinks;
        int64_t sequences;
        void* stream;
        c10::DataPtr room;
        if (count != 16 || dev < 0 || !operand(a[1], dev, {&s.n, &s.t, &s.cq}, q) || !s.of(a[9], a[10]) || !operand(a[0], dev, {&s.n, &s.t, &s.cq}, d) ||
            !operand(a[2], dev, {&s.n, &s.t, &s.ck}, k) || !operand(a[3], dev, {&s.n, &s.t, &s.ck}, v) || !operand(a[4], dev, {&s.n, &s.t, &s.cq}, o) ||
            !vector(a[5], dev, s.n * s.heads * s.t, at::kFloat, lse) || !operand(a[6], dev, {&s.n, &s.t, &s.cq}, dq) || !operand(a[7], dev, {&s.n, &s.t, &s.ck}, dk) ||
            !operand(a[8], dev, {&s.n, &s.t, &s.ck}, dv) || !starts_of(a[11], dev, s.n, st, sequences) || !small(a[12], window) || !small(a[13], sinks) ||
            !scale_of(a[14], s.head, scale) || !stream_of(a[15], dev, stream))
            return NOT_MINE;
        const size_t need = blocks.attention_grad_workspace(static_cast<int>(s.heads), static_cast<int>(s.kv), static_cast<int>(s.head), window, sinks,
                                                            static_cast<int>(sequences), static_cast<int>(s.n), s.t);
        if (!workspace(dev, need, stream, room)) return NOT_MINE;
        Unlocked run;
        return blocks.attention_grad(d.get(), q.get(), k.get(), v.get(), o.get(), lse, st.get(), dq.get(), dk.get(), dv.get(), static_cast<int>(s.heads),
                                     static_cast<int>(s.kv), static_cast<int>(s.head), window, sinks, scale, static_cast<int>(sequences), static_cast<int>(s.n), s.t,
                                     room.get(), need, stream);
    });
}

bool cache_of(PyObject* o, int dev, const Heads& s, int64_t& slots, psgd_cache& c) {
    const at::Tensor* t = plain(o, dev);
    if (!t || t->dim() != 4 || t->size(0) != s.n || t->size(1) != s.t || t->size(2) < 1 || t->size(3) != s.ck || (s.ck > 1 && t->stride(3) != 1)) return false;
    if (t->scalar_type() != at::kFloat && t->scalar_type() != at::kBFloat16) return false;
    if (slots < 0) slots = t->size(2);
    c = psgd_cache{t->data_ptr(), s.n > 1 ? t->stride(0) : 0, s.t > 1 ? t->stride(1) : 0, slots > 1 ? t->stride(2) : 0,
                   t->scalar_type() == at::kFloat ? PSGD_F32 : PSGD_BF16};
    return t->size(2) == slots;
}

// attention_step(q, k, v, cache_k, cache_v, lengths, out, heads, kv, window, sinks, scale, stream)
PyObject* attention_step(PyObject*, PyObject* const* a, Py_ssize_t count) {
    return guarded([&]() -> long {
        const int dev = blocks_device();
        Heads s;
        Operand q, k, v, o, len;
        psgd_cache ck, cv;
        float scale;
        int window, sinks;
        int64_t slots = -1;
        void* stream;
        c10::DataPtr room;
        if (count != 13 || dev < 0 || !operand(a[0], dev, {&s.n, &s.t, &s.cq}, q) || !s.of(a[7], a[8]) || !operand(a[1], dev, {&s.n, &s.t, &s.ck}, k) ||
            !operand(a[2], dev, {&s.n, &s.t, &s.ck}, v) || !cache_of(a[3], dev, s, slots, ck) || !cache_of(a[4], dev, s, slots, cv) ||
            !numbers(a[5], dev, s.n, s.t, len) || !operand(a[6], dev, {&s.n, &s.t, &s.cq}, o) || !small(a[9], window) || !small(a[10], sinks) ||
            !scale_of(a[11], s.head, scale) || !stream_of(a[12], dev, stream))
            return NOT_MINE;
        const size_t need = blocks.attention_step_workspace(static_cast<int>(s.heads), static_cast<int>(s.kv), static_cast<int>(s.head), window, sinks,
                                                            static_cast<int>(s.n), s.t, slots);
        if (!workspace(dev, need, stream, room)) return NOT_MINE;
        Unlocked run;
        return blocks.attention_step(q.get(), k.get(), v.get(), &ck, &cv, len.get(), o.get(), static_cast<int>(s.heads), static_cast<int>(s.kv),
                                     static_cast<int>(s.head), window, sinks, scale, static_cast<int>(s.n), s.t, slots, room.get(), need, stream);
    });
}

// dropout(x, y, p, seed, step, residual, step_dev, stream)
PyObject* dropout(PyObject*, PyObject* const* a, Py_ssize_t count) {
    return guarded([&]() -> long {
        const int dev = blocks_device();
        int64_t n = -1, t = -1, c = -1;
        Operand x, y, r;
        float p;
        uint64_t seed, step;
        uint64_t* counter = nullptr;
        void* stream;
        if (count != 8 || dev < 0 || !operand(a[0], dev, {&n, &t, &c}, x) || n > PSGD_MAX_N || !operand(a[1], dev, {&n, &t, &c}, y) || !number(a[2], p) ||
            !word_of(a[3], seed) || !word_of(a[4], step) || !operand(a[5], dev, {&n, &t, &c}, r, true) || !stream_of(a[7], dev, stream))
            return NOT_MINE;
        if (a[6] != Py_None) {
            const at::Tensor* d = plain(a[6], dev);
            if (!d || (d->scalar_type() != at::kLong && d->scalar_type() != at::kUInt64) || d->numel() < 1) return NOT_MINE;
            counter = static_cast<uint64_t*>(d->data_ptr());
        }
        Unlocked run;
        return blocks.dropout(x.get(), r.get(), y.get(), p, seed, step, counter, static_cast<int>(n), t, c, stream);
    });
}

// bind_attention(addresses of the functions, in the order of struct Attention)
PyObject* bind_attention(PyObject*, PyObject* const* a, Py_ssize_t count) {
    void* p[9];
    if (count != 9) return answer(NOT_MINE);
    for (int i = 0; i < 9; ++i) {
        p[i] = PyLong_AsVoidPtr(a[i]);
        if (PyErr_Occurred()) return nullptr;
    }
    blocks.qk_norm_rope = reinterpret_cast<decltype(blocks.qk_norm_rope)>(p[0]);
    blocks.qk_norm_rope_grad = reinterpret_cast<decltype(blocks.qk_norm_rope_grad)>(p[1]);
    blocks.qk_norm_rope_grad_workspace = reinterpret_cast<decltype(blocks.qk_norm_rope_grad_workspace)>(p[2]);
    blocks.attention = reinterpret_cast<decltype(blocks.attention)>(p[3]);
    blocks.attention_grad = reinterpret_cast<decltype(blocks.attention_grad)>(p[4]);
    blocks.attention_grad_workspace = reinterpret_cast<decltype(blocks.attention_grad_workspace)>(p[5]);
    blocks.attention_step = reinterpret_cast<decltype(blocks.attention_step)>(p[6]);
    blocks.attention_step_workspace = reinterpret_cast<decltype(blocks.attention_step_workspace)>(p[7]);
    blocks.dropout = reinterpret_cast<decltype(blocks.dropout)>(p[8]);
    return answer(0);
}

#define PSGD_METHOD(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {PSGD_METHOD(mix_step),  PSGD_METHOD(mix_full), PSGD_METHOD(mix_step_d1d), PSGD_METHOD(build_mixing_device),
                         PSGD_METHOD(consensus_dist_async), PSGD_METHOD(consensus_dist), PSGD_METHOD(synth_grad), PSGD_METHOD(bind),
                         PSGD_METHOD(layer_norm), PSGD_METHOD(layer_norm_grad), PSGD_METHOD(linear), PSGD_METHOD(linear_grad),
                         PSGD_METHOD(token_logprobs), PSGD_METHOD(distill), PSGD_METHOD(bind_layers),
                         PSGD_METHOD(qk_norm_rope), PSGD_METHOD(qk_norm_rope_grad), PSGD_METHOD(attention), PSGD_METHOD(attention_grad), PSGD_METHOD(attention_step),
                         PSGD_METHOD(dropout), PSGD_METHOD(bind_attention), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__call(void) { return PyModule_Create(&module); }
