// The plain calls of binding.py in native code: checks, outputs and the launch of one call on ordinary tensors, current
// stream, outputs allocated here.  Any other call, and any that the checks or the library refuse, gives None, and the
// Python function behind it does what it always did (and raises what it always raised).
//
// A small call is bound by this work: two calls of a training step on two 256-token sequences take 12.7 us on the GPU.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <cstdint>

namespace {

typedef int (*FwdFn)(const void *, const void *, const void *, void *, const int32_t *, const float *, float, int, int, int, int, void *);
typedef int (*BwdFn)(const void *, const void *, const void *, const void *, void *, void *, void *, const int32_t *, const float *, float,
                     int, int, int, int, void *, size_t, void *);
typedef size_t (*BytesFn)(int, int, int, int);

FwdFn fwd_fn;
BwdFn bwd_fn;
BytesFn bytes_fn;

// An ordinary GPU tensor: exactly torch.Tensor, and nothing that a transform or a mode of torch has wrapped.
bool plain(PyObject *o, at::Tensor &t) {
    if (!THPVariable_CheckExact(o)) return false;
    t = THPVariable_Unpack(o);
    const auto keys = t.unsafeGetTensorImpl()->key_set();
    return t.defined() && t.is_cuda() && t.layout() == at::kStrided &&
           !keys.has_any(c10::DispatchKeySet({c10::DispatchKey::Python, c10::DispatchKey::FuncTorchBatched, c10::DispatchKey::FuncTorchGradWrapper,
                                              c10::DispatchKey::Functionalize, c10::DispatchKey::Batched, c10::DispatchKey::Negative,
                                              c10::DispatchKey::Conjugate, c10::DispatchKey::ZeroTensor}));
}

bool rows(PyObject *o, at::Tensor &t, const at::Tensor *like) {
    return plain(o, t) && t.scalar_type() == at::kBFloat16 && t.is_contiguous() && t.dim() == 4 && (!like || t.sizes() == like->sizes());
}

bool vec(PyObject *o, at::Tensor &t, int64_t n, at::ScalarType type) {
    return plain(o, t) && t.scalar_type() == type && t.is_contiguous() && t.dim() == 1 && t.size(0) == n;
}

bool ordinary_state() {            // no mode that would want to see the calls of the Python function
    return !c10::impl::TorchDispatchModeTLS::any_modes_set() && !at::impl::torch_function_mode_enabled() &&
           !c10::impl::tls_local_dispatch_key_set().included_.has_any(c10::DispatchKeySet({c10::DispatchKey::FuncTorchDynamicLayerFrontMode, c10::DispatchKey::Functionalize, c10::DispatchKey::Python}));
}

struct Call {
    at::Tensor q, k, v, g, seqlens, bias;
    float scale;
    int B, N, H, d;
};

// q, k, v, [d_o,] seqlens, bias, scale
bool read(PyObject *const *args, Py_ssize_t n, bool backward, Call &c) {
    if (n != (backward ? 7 : 6) || !ordinary_state()) return false;
    const int m = backward ? 4 : 3;
    if (!rows(args[0], c.q, nullptr) || !rows(args[1], c.k, &c.q) || !rows(args[2], c.v, &c.q)) return false;
    if (backward && !rows(args[3], c.g, &c.q)) return false;
    for (int i = 0; i < 4; ++i)
        if (c.q.size(i) > INT32_MAX) return false;
    c.B = (int)c.q.size(0); c.N = (int)c.q.size(1); c.H = (int)c.q.size(2); c.d = (int)c.q.size(3);
    if (!vec(args[m], c.seqlens, c.B, at::kInt) || !vec(args[m + 1], c.bias, c.B, at::kFloat)) return false;
    if (!PyFloat_CheckExact(args[m + 2])) return false;
    c.scale = (float)PyFloat_AS_DOUBLE(args[m + 2]);
    return true;
}

void *current_stream() { return static_cast<void *>(c10::hip::getCurrentHIPStream().stream()); }

template <class T>
T *data(const at::Tensor &t) { return static_cast<T *>(t.data_ptr()); }

PyObject *none() {                 // with no Python error behind it, which what threw may have left
    PyErr_Clear();
    Py_RETURN_NONE;
}

struct WithoutGil {                // other threads of the interpreter run while memory is found and the launch is made
    PyThreadState *state = PyEval_SaveThread();
    ~WithoutGil() { PyEval_RestoreThread(state); }
};

PyObject *fwd(PyObject *, PyObject *const *args, Py_ssize_t n) {
    try {
        Call c;
        if (!fwd_fn || !read(args, n, false, c)) return none();
        at::Tensor o;
        int rc;
        {
            WithoutGil released;
            o = at::empty_like(c.q);
            rc = fwd_fn(data<void>(c.q), data<void>(c.k), data<void>(c.v), data<void>(o), data<int32_t>(c.seqlens), data<float>(c.bias),
                        c.scale, c.B, c.N, c.H, c.d, current_stream());
        }
        return rc ? none() : THPVariable_Wrap(std::move(o));
    } catch (...) {                // out of memory and the like: the Python function meets it again and reports it
        return none();
    }
}

PyObject *bwd(PyObject *, PyObject *const *args, Py_ssize_t n) {
    try {
        Call c;
        if (!bwd_fn || !bytes_fn || !read(args, n, true, c)) return none();
        const size_t need = bytes_fn(c.B, c.N, c.H, c.d);
        if (need && c.q.get_device() != c10::hip::current_device()) return none();   // scratch belongs to a stream of its own device
        at::Tensor dq, dk, dv, ws;
        int rc;
        {
            WithoutGil released;
            dq = at::empty_like(c.q);
            dk = at::empty_like(c.q);
            dv = at::empty_like(c.q);
            if (need) ws = at::empty({(int64_t)need}, c.q.options().dtype(at::kByte).requires_grad(false));
            rc = bwd_fn(data<void>(c.q), data<void>(c.k), data<void>(c.v), data<void>(c.g), data<void>(dq), data<void>(dk), data<void>(dv),
                        data<int32_t>(c.seqlens), data<float>(c.bias), c.scale, c.B, c.N, c.H, c.d, need ? data<void>(ws) : nullptr,
                        need, current_stream());
        }
        if (rc) return none();
        PyObject *out = PyTuple_New(3);
        at::Tensor *const grads[3] = {&dq, &dk, &dv};
        for (int i = 0; out && i < 3; ++i) {
            PyObject *const t = THPVariable_Wrap(std::move(*grads[i]));
            if (t) PyTuple_SET_ITEM(out, i, t);
            else Py_CLEAR(out);
        }
        return out;                // nullptr with the error that PyTuple_New or THPVariable_Wrap has set
    } catch (...) {
        return none();
    }
}

// The library's functions, as addresses: sigmoid_attn_fwd, sigmoid_attn_bwd, sigmoid_attn_bwd_onepass_workspace_bytes.
PyObject *use(PyObject *, PyObject *args) {
    unsigned long long f, b, s;
    if (!PyArg_ParseTuple(args, "KKK", &f, &b, &s)) return nullptr;
    fwd_fn = reinterpret_cast<FwdFn>(f);
    bwd_fn = reinterpret_cast<BwdFn>(b);
    bytes_fn = reinterpret_cast<BytesFn>(s);
    Py_RETURN_NONE;
}

// ---- the calls with a relative position bias (bit 0 of `kind`) and with dropout (bit 1)
//   (kind, q, k, v, [d_o,] seqlens_q, seqlens_k, bias, scale, [table, buckets, q_start or None,] [p, rng])
typedef int (*RelFwd)(const void *, const void *, const void *, void *, const int32_t *, const int32_t *, const float *, float,
                      const void *, const int32_t *, int, int, const int32_t *, int, int, int, int, int, void *, size_t, void *);
typedef int (*DropFwd)(const void *, const void *, const void *, void *, const int32_t *, const int32_t *, const float *, float,
                       float, const uint64_t *, int, int, int, int, int, void *);
typedef int (*BothFwd)(const void *, const void *, const void *, void *, const int32_t *, const int32_t *, const float *, float,
                       const void *, const int32_t *, int, int, const int32_t *, float, const uint64_t *, int, int, int, int, int, void *);
typedef int (*RelBwd)(const void *, const void *, const void *, const void *, void *, void *, void *, void *, const int32_t *, const int32_t *,
                      const float *, float, const void *, const int32_t *, int, int, const int32_t *, int, int, int, int, int, void *, size_t, void *);
typedef int (*DropBwd)(const void *, const void *, const void *, const void *, void *, void *, void *, const int32_t *, const int32_t *,
                       const float *, float, float, const uint64_t *, int, int, int, int, int, void *);
typedef int (*BothBwd)(const void *, const void *, const void *, const void *, void *, void *, void *, void *, const int32_t *, const int32_t *,
                       const float *, float, const void *, const int32_t *, int, int, const int32_t *, float, const uint64_t *, int, int, int, int, int,
                       void *, size_t, void *);
typedef size_t (*FwdBytes)(int, int, int, int, int);
typedef size_t (*BwdBytes)(int, int, int, int, int, int);
struct {
    RelFwd rel_fwd;
    DropFwd drop_fwd;
    BothFwd both_fwd;
    RelBwd rel_bwd;
    DropBwd drop_bwd;
    BothBwd both_bwd;
    FwdBytes fwd_bytes;
    BwdBytes bwd_bytes;
} mods;

struct ModCall {
    at::Tensor q, k, v, g, nq, nk, bias, table, buckets, start, rng;
    bool rel, drop;
    float scale, p;
    int B, Lq, Lk, H, d, num, reach;
    const void *at_table() const { return table.const_data_ptr(); }
    const int32_t *at_buckets() const { return static_cast<const int32_t *>(buckets.const_data_ptr()); }
    const int32_t *at_start() const { return start.defined() ? static_cast<const int32_t *>(start.const_data_ptr()) : nullptr; }
    const uint64_t *at_rng() const { return static_cast<const uint64_t *>(rng.const_data_ptr()); }
};

bool read_mod(PyObject *const *args, Py_ssize_t n, bool backward, ModCall &c) {
    if (n < 1 || !PyLong_CheckExact(args[0]) || !ordinary_state()) return false;
    const long kind = PyLong_AsLong(args[0]);
    c.rel = kind & 1;
    c.drop = kind & 2;
    if (n != 8 + backward + 3 * c.rel + 2 * c.drop) return false;
    PyObject *const *a = args + 1;
    if (!rows(*a++, c.q, nullptr) || !rows(*a++, c.k, nullptr) || !rows(*a++, c.v, &c.k)) return false;
    if (c.q.size(0) != c.k.size(0) || c.q.size(2) != c.k.size(2) || c.q.size(3) != c.k.size(3)) return false;
    if (backward && !rows(*a++, c.g, &c.q)) return false;
    for (int i = 0; i < 4; ++i)
        if (c.q.size(i) > INT32_MAX || c.k.size(i) > INT32_MAX) return false;
    c.B = (int)c.q.size(0); c.Lq = (int)c.q.size(1); c.Lk = (int)c.k.size(1); c.H = (int)c.q.size(2); c.d = (int)c.q.size(3);
    if (!vec(*a++, c.nq, c.B, at::kInt) || !vec(*a++, c.nk, c.B, at::kInt) || !vec(*a++, c.bias, c.B, at::kFloat)) return false;
    if (!PyFloat_CheckExact(*a)) return false;
    c.scale = (float)PyFloat_AS_DOUBLE(*a++);
    if (c.rel) {
        if (!plain(*a++, c.table) || c.table.scalar_type() != at::kBFloat16 || !c.table.is_contiguous() || c.table.dim() != 2 || c.table.size(1) != c.H) return false;
        if (!plain(*a++, c.buckets) || c.buckets.scalar_type() != at::kInt || !c.buckets.is_contiguous() || c.buckets.dim() != 1 || c.buckets.size(0) % 2 != 1) return false;
        if (c.table.size(0) > INT32_MAX || c.buckets.size(0) > INT32_MAX) return false;
        c.num = (int)c.table.size(0);
        c.reach = (int)(c.buckets.size(0) / 2);
        if (*a != Py_None && !vec(*a, c.start, c.B, at::kInt)) return false;
        ++a;
    }
    if (c.drop) {
        if (!PyFloat_CheckExact(*a)) return false;
        c.p = (float)PyFloat_AS_DOUBLE(*a++);
        if (!vec(*a++, c.rng, 2, at::kLong)) return false;
    }
    const auto here = c10::hip::current_device();
    for (const at::Tensor *t : {&c.q, &c.k, &c.v, &c.g, &c.nq, &c.nk, &c.bias, &c.table, &c.buckets, &c.start, &c.rng})
        if (t->defined() && t->get_device() != here) return false;
    return true;
}

at::Tensor scratch(const at::Tensor &like, size_t bytes) { return at::empty({(int64_t)bytes}, like.options().dtype(at::kByte).requires_grad(false)); }

PyObject *mod_fwd(PyObject *, PyObject *const *args, Py_ssize_t n) {
    try {
        ModCall c;
        if (!mods.rel_fwd || !read_mod(args, n, false, c)) return none();
        at::Tensor o, ws;
        int rc;
        {
            WithoutGil released;
            o = at::empty_like(c.q);
            void *const q = data<void>(c.q), *const k = data<void>(c.k), *const v = data<void>(c.v), *const out = data<void>(o), *const s = current_stream();
            const int32_t *const nq = data<int32_t>(c.nq), *const nk = data<int32_t>(c.nk);
            const float *const b = data<float>(c.bias);
            if (c.rel && c.drop) {
                rc = mods.both_fwd(q, k, v, out, nq, nk, b, c.scale, c.at_table(), c.at_buckets(), c.num, c.reach, c.at_start(), c.p, c.at_rng(), c.B, c.Lq, c.Lk, c.H, c.d, s);
            } else if (c.rel) {
                const size_t need = mods.fwd_bytes(c.B, c.Lq, c.Lk, c.H, c.d);
                if (need) ws = scratch(c.q, need);
                rc = mods.rel_fwd(q, k, v, out, nq, nk, b, c.scale, c.at_table(), c.at_buckets(), c.num, c.reach, c.at_start(), c.B, c.Lq, c.Lk, c.H, c.d,
                                  need ? data<void>(ws) : nullptr, need, s);
            } else {
                rc = mods.drop_fwd(q, k, v, out, nq, nk, b, c.scale, c.p, c.at_rng(), c.B, c.Lq, c.Lk, c.H, c.d, s);
            }
        }
        return rc ? none() : THPVariable_Wrap(std::move(o));
    } catch (...) {
        return none();
    }
}

PyObject *mod_bwd(PyObject *, PyObject *const *args, Py_ssize_t n) {
    try {
        ModCall c;
        if (!mods.rel_fwd || !read_mod(args, n, true, c)) return none();
        at::Tensor dq, dk, dv, dtable, ws;
        int rc;
        {
            WithoutGil released;
            dq = at::empty_like(c.q);
            dk = at::empty_like(c.k);
            dv = at::empty_like(c.v);
            size_t need = 0;
            if (c.rel) {
                dtable = at::empty_like(c.table);
                need = mods.bwd_bytes(c.B, c.Lq, c.Lk, c.H, c.d, c.reach);
                if (need) ws = scratch(c.q, need);
            }
            void *const q = data<void>(c.q), *const k = data<void>(c.k), *const v = data<void>(c.v), *const g = data<void>(c.g), *const s = current_stream();
            void *const oq = data<void>(dq), *const ok = data<void>(dk), *const ov = data<void>(dv), *const w = need ? data<void>(ws) : nullptr;
            const int32_t *const nq = data<int32_t>(c.nq), *const nk = data<int32_t>(c.nk);
            const float *const b = data<float>(c.bias);
            if (c.rel && c.drop)
                rc = mods.both_bwd(q, k, v, g, oq, ok, ov, data<void>(dtable), nq, nk, b, c.scale, c.at_table(), c.at_buckets(), c.num, c.reach, c.at_start(),
                                   c.p, c.at_rng(), c.B, c.Lq, c.Lk, c.H, c.d, w, need, s);
            else if (c.rel)
                rc = mods.rel_bwd(q, k, v, g, oq, ok, ov, data<void>(dtable), nq, nk, b, c.scale, c.at_table(), c.at_buckets(), c.num, c.reach, c.at_start(),
                                  c.B, c.Lq, c.Lk, c.H, c.d, w, need, s);
            else
                rc = mods.drop_bwd(q, k, v, g, oq, ok, ov, nq, nk, b, c.scale, c.p, c.at_rng(), c.B, c.Lq, c.Lk, c.H, c.d, s);
        }
        if (rc) return none();
        const int count = c.rel ? 4 : 3;
        PyObject *out = PyTuple_New(count);
        at::Tensor *const grads[4] = {&dq, &dk, &dv, &dtable};
        for (int i = 0; out && i < count; ++i) {
            PyObject *const t = THPVariable_Wrap(std::move(*grads[i]));
            if (t) PyTuple_SET_ITEM(out, i, t);
            else Py_CLEAR(out);
        }
        return out;
    } catch (...) {
        return none();
    }
}

// The addresses of sigmoid_attn_rel_fwd, _dropout_fwd, _rel_dropout_fwd, the three _bwd, _rel_fwd_workspace_bytes and _rel_bwd_workspace_bytes.
PyObject *use_mod(PyObject *, PyObject *args) {
    unsigned long long a[8];
    if (!PyArg_ParseTuple(args, "KKKKKKKK", a, a + 1, a + 2, a + 3, a + 4, a + 5, a + 6, a + 7)) return nullptr;
    mods = {reinterpret_cast<RelFwd>(a[0]), reinterpret_cast<DropFwd>(a[1]), reinterpret_cast<BothFwd>(a[2]), reinterpret_cast<RelBwd>(a[3]),
            reinterpret_cast<DropBwd>(a[4]), reinterpret_cast<BothBwd>(a[5]), reinterpret_cast<FwdBytes>(a[6]), reinterpret_cast<BwdBytes>(a[7])};
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"fwd", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(fwd)), METH_FASTCALL, nullptr},
    {"bwd", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(bwd)), METH_FASTCALL, nullptr},
    {"use", use, METH_VARARGS, nullptr},
    {"mod_fwd", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(mod_fwd)), METH_FASTCALL, nullptr},
    {"mod_bwd", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(mod_bwd)), METH_FASTCALL, nullptr},
    {"use_mod", use_mod, METH_VARARGS, nullptr},
    {nullptr, nullptr, 0, nullptr},
};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fastcall", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fastcall(void) { return PyModule_Create(&module); }
