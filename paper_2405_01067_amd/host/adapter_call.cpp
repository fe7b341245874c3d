// The calls of a layer with adapters and of the norm in front of it from Python, in native code, as layer_call.cpp has those of a factored layer: what
// binding.lr_adapters_fwd, lr_adapters_fwd_q8, lr_adapters_bwd, lr_rms_norm_fwd and lr_rms_norm_bwd do for plain tensors that fit each other, with the
// outputs and the workspace allocated here.  Anything else is answered with None, and the Python code goes on as if it had not asked.
//
// A step of single tokens is bound by this: through Python alone a call of one token's layer takes 16 us of host time and 9 us of the GPU's.
#include "call_util.h"

#include "abtrain.h"

namespace {

using namespace native_call;

decltype(&lr_adapters_fwd) fwd_fn;
decltype(&lr_adapters_fwd_q8) fwd_q8_fn;
decltype(&lr_adapters_fwd_workspace_bytes) fwd_bytes_fn;
decltype(&lr_adapters_bwd) bwd_fn;
decltype(&lr_adapters_bwd_workspace_bytes) bwd_bytes_fn;
decltype(&lr_rms_norm_fwd) norm_fwd_fn;
decltype(&lr_rms_norm_bwd) norm_bwd_fn;
decltype(&lr_rms_norm_bwd_workspace_bytes) norm_bwd_bytes_fn;

bool is(const at::Tensor* t, at::ScalarType dtype, std::initializer_list<int64_t> shape) {
    return t && t->scalar_type() == dtype && t->sizes() == at::IntArrayRef(shape.begin(), shape.size());
}

// A, B, row_adapter, ranks, scales in args[0 .. 4]; false: not for this code
bool adapters_of(PyObject* const* args, int64_t M, int64_t m, int64_t n, abt_adapters& ad, const int32_t*& ids) {
    const at::Tensor *A = plain(args[0], 3), *B = plain(args[1], 3), *rows = plain(args[2], 1);
    const at::Tensor *ranks = args[3] == Py_None ? nullptr : plain(args[3], 1), *scales = args[4] == Py_None ? nullptr : plain(args[4], 1);
    if (!A || !B || !rows || (!ranks && args[3] != Py_None) || (!scales && args[4] != Py_None)) return false;
    const int64_t count = A->size(0), r = A->size(2);
    if (!is(A, at::kBFloat16, {count, m, r}) || !is(B, at::kBFloat16, {count, r, n}) || !is(rows, at::kInt, {M}) || (ranks && !is(ranks, at::kInt, {count})) ||
        (scales && !is(scales, at::kFloat, {count})) || count > INT32_MAX || r > INT32_MAX)
        return false;
    ad = abt_adapters{A->data_ptr(), B->data_ptr(), ranks ? (const int32_t*)ranks->data_ptr() : nullptr, scales ? (const float*)scales->data_ptr() : nullptr,
                      (int32_t)count, (int32_t)r};
    ids = (const int32_t*)rows->data_ptr();
    return true;
}

at::Tensor space(size_t bytes, const at::TensorOptions& opt) { return at::empty({(int64_t)(bytes < 256 ? 256 : bytes)}, opt.dtype(at::kByte)); }

// (X, W, A, B, row_adapter, ranks, scales, save_T) -> (Y, T or None), or None
PyObject* fwd(PyObject*, PyObject* const* args, Py_ssize_t k) {
    if (k != 8) { PyErr_SetString(PyExc_TypeError, "fwd takes 8 arguments"); return nullptr; }
    void *stream, *x, *w, *y, *t = nullptr;
    int64_t M, m, n;
    abt_adapters ad;
    const int32_t* ids;
    at::Tensor Y, T, ws;
    PyObject* results;
    try {
        const at::Tensor *X = plain(args[0]), *W = plain(args[1]);
        const int save = PyObject_IsTrue(args[7]);
        if (save < 0) return nullptr;
        if (!X || !W || watched()) Py_RETURN_NONE;
        M = X->size(0); n = X->size(1); m = W->size(0);
        if (!is(X, at::kBFloat16, {M, n}) || !is(W, at::kBFloat16, {m, n}) || !adapters_of(args + 2, M, m, n, ad, ids)) Py_RETURN_NONE;
        if (!current_stream(&stream)) return nullptr;
        const auto opt = X->options().requires_grad(false);
        Y = at::empty({M, m}, opt);
        if (save) { T = at::empty({M, ad.r}, opt.dtype(at::kFloat)); t = T.data_ptr(); }
        ws = space(fwd_bytes_fn(M, m, n, ad.r, ad.count), opt);
        x = X->data_ptr(); w = W->data_ptr(); y = Y.data_ptr();
        results = Py_BuildValue("(NN)", THPVariable_Wrap(Y), wrap_or_none(T));
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;                                  // out of memory and the like: the Python code meets it again and says so
    }
    if (!results) return nullptr;
    int code;
    Py_BEGIN_ALLOW_THREADS
    code = fwd_fn(x, w, &ad, ids, y, (float*)t, M, m, n, ABT_BF16, ws.data_ptr(), (size_t)ws.numel(), stream);
    Py_END_ALLOW_THREADS
    return finished(results, code, "lr_adapters_fwd");
}

// (X, Xq, x_scale, Wq, w_scale, A, B, row_adapter, ranks, scales) -> Y, or None
PyObject* fwd_q8(PyObject*, PyObject* const* args, Py_ssize_t k) {
    if (k != 10) { PyErr_SetString(PyExc_TypeError, "fwd_q8 takes 10 arguments"); return nullptr; }
    void *stream, *in[5], *y;
    int64_t M, m, n;
    abt_adapters ad;
    const int32_t* ids;
    at::Tensor Y, ws;
    PyObject* results;
    try {
        const at::Tensor *X = plain(args[0]), *Xq = plain(args[1]), *xs = plain(args[2], 1), *Wq = plain(args[3]), *wsc = plain(args[4], 1);
        if (!X || !Wq || watched()) Py_RETURN_NONE;
        M = X->size(0); n = X->size(1); m = Wq->size(0);
        if (!is(X, at::kBFloat16, {M, n}) || !is(Xq, at::kFloat8_e4m3fn, {M, n}) || !is(xs, at::kFloat, {M}) || !is(Wq, at::kFloat8_e4m3fn, {m, n}) ||
            !is(wsc, at::kFloat, {m}) || !adapters_of(args + 5, M, m, n, ad, ids))
            Py_RETURN_NONE;
        if (!current_stream(&stream)) return nullptr;
        const auto opt = X->options().requires_grad(false);
        Y = at::empty({M, m}, opt);
        ws = space(fwd_bytes_fn(M, m, n, ad.r, ad.count), opt);
        const at::Tensor* operands[5] = {X, Xq, xs, Wq, wsc};
        for (int i = 0; i < 5; ++i) in[i] = operands[i]->data_ptr();
        y = Y.data_ptr();
        results = THPVariable_Wrap(Y);
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    if (!results) return nullptr;
    int code;
    Py_BEGIN_ALLOW_THREADS
    code = fwd_q8_fn(in[0], in[1], (const float*)in[2], in[3], (const float*)in[4], &ad, ids, y, M, m, n, ws.data_ptr(), (size_t)ws.numel(), stream);
    Py_END_ALLOW_THREADS
    return finished(results, code, "lr_adapters_fwd_q8");
}

// (dY, X, T, W, A, B, row_adapter, ranks, scales, need_dX, need_dA, need_dB) -> (dX, dA, dB), or None
PyObject* bwd(PyObject*, PyObject* const* args, Py_ssize_t k) {
    if (k != 12) { PyErr_SetString(PyExc_TypeError, "bwd takes 12 arguments"); return nullptr; }
    void *stream, *dy, *x, *w, *t = nullptr, *to[3];
    int64_t M, m, n;
    int need[3];
    abt_adapters ad;
    const int32_t* ids;
    at::Tensor out[3], ws;
    PyObject* results;
    try {
        const at::Tensor *dY = plain(args[0]), *X = plain(args[1]), *W = plain(args[3]);
        const at::Tensor* T = args[2] == Py_None ? nullptr : plain(args[2]);
        if (!dY || !X || !W || (!T && args[2] != Py_None) || watched()) Py_RETURN_NONE;
        for (int i = 0; i < 3; ++i)
            if ((need[i] = PyObject_IsTrue(args[9 + i])) < 0) return nullptr;
        M = X->size(0); n = X->size(1); m = W->size(0);
        if (!is(X, at::kBFloat16, {M, n}) || !is(W, at::kBFloat16, {m, n}) || !is(dY, at::kBFloat16, {M, m}) || !adapters_of(args + 4, M, m, n, ad, ids) ||
            (T && !is(T, at::kFloat, {M, ad.r})))
            Py_RETURN_NONE;
        if (!current_stream(&stream)) return nullptr;
        const auto opt = X->options().requires_grad(false);
        if (need[0]) out[0] = at::empty({M, n}, opt);
        if (need[1]) out[1] = at::empty({ad.count, m, ad.r}, opt.dtype(at::kFloat));
        if (need[2]) out[2] = at::empty({ad.count, ad.r, n}, opt.dtype(at::kFloat));
        ws = space(bwd_bytes_fn(M, m, n, ad.r, ad.count), opt);
        dy = dY->data_ptr(); x = X->data_ptr(); w = W->data_ptr();
        if (T) t = T->data_ptr();
        for (int i = 0; i < 3; ++i) to[i] = out[i].defined() ? out[i].data_ptr() : nullptr;
        results = Py_BuildValue("(NNN)", wrap_or_none(out[0]), wrap_or_none(out[1]), wrap_or_none(out[2]));
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    if (!results) return nullptr;
    int code;
    Py_BEGIN_ALLOW_THREADS
    code = bwd_fn(dy, x, (const float*)t, w, &ad, ids, to[0], (float*)to[1], (float*)to[2], M, m, n, ABT_BF16, 0, ws.data_ptr(), (size_t)ws.numel(), stream);
    Py_END_ALLOW_THREADS
    return finished(results, code, "lr_adapters_bwd");
}

// bf16 or fp32
bool type_of(const at::Tensor& t, int& dt) {
    dt = t.scalar_type() == at::kBFloat16 ? ABT_BF16 : ABT_F32;
    return dt == ABT_BF16 || t.scalar_type() == at::kFloat;
}

// (X, gain, eps, residual, quantize) -> (Y, H, Yq, y_scale), or None
PyObject* norm_fwd(PyObject*, PyObject* const* args, Py_ssize_t k) {
    if (k != 5) { PyErr_SetString(PyExc_TypeError, "norm_fwd takes 5 arguments"); return nullptr; }
    void *stream, *x, *g, *r = nullptr, *h = nullptr, *y, *yq = nullptr, *s = nullptr;
    int64_t M, n;
    int dt;
    double eps;
    at::Tensor Y, H, Yq, S;
    PyObject* results;
    try {
        const at::Tensor *X = plain(args[0]), *gain = plain(args[1], 1), *R = args[3] == Py_None ? nullptr : plain(args[3]);
        eps = PyFloat_AsDouble(args[2]);
        if (eps == -1.0 && PyErr_Occurred()) return nullptr;
        const int quantize = PyObject_IsTrue(args[4]);
        if (quantize < 0) return nullptr;
        if (!X || !gain || (!R && args[3] != Py_None) || watched() || !type_of(*X, dt)) Py_RETURN_NONE;
        M = X->size(0); n = X->size(1);
        if (!is(gain, at::kFloat, {n}) || (R && !is(R, X->scalar_type(), {M, n}))) Py_RETURN_NONE;
        if (!current_stream(&stream)) return nullptr;
        const auto opt = X->options().requires_grad(false);
        Y = at::empty({M, n}, opt);
        if (R) { H = at::empty({M, n}, opt); h = H.data_ptr(); r = R->data_ptr(); }
        if (quantize) {
            Yq = at::empty({M, n}, opt.dtype(at::kFloat8_e4m3fn));
            S = at::empty({M}, opt.dtype(at::kFloat));
            yq = Yq.data_ptr(); s = S.data_ptr();
        }
        x = X->data_ptr(); g = gain->data_ptr(); y = Y.data_ptr();
        PyObject* kept = R ? THPVariable_Wrap(H) : args[0];
        if (!R) Py_INCREF(kept);
        results = Py_BuildValue("(NNNN)", THPVariable_Wrap(Y), kept, wrap_or_none(Yq), wrap_or_none(S));
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    if (!results) return nullptr;
    const int code = norm_fwd_fn(x, r, (const float*)g, eps, h, y, yq, (float*)s, M, n, dt, stream);
    return finished(results, code, "lr_rms_norm_fwd");
}

// (dY, H, gain, eps, dH) -> (dX, dgain), or None
PyObject* norm_bwd(PyObject*, PyObject* const* args, Py_ssize_t k) {
    if (k != 5) { PyErr_SetString(PyExc_TypeError, "norm_bwd takes 5 arguments"); return nullptr; }
    void *stream, *dy, *h, *g, *dh = nullptr, *dx, *dg;
    int64_t M, n;
    int dt;
    double eps;
    at::Tensor dX, dG, ws;
    PyObject* results;
    try {
        const at::Tensor *dY = plain(args[0]), *H = plain(args[1]), *gain = plain(args[2], 1), *dH = args[4] == Py_None ? nullptr : plain(args[4]);
        eps = PyFloat_AsDouble(args[3]);
        if (eps == -1.0 && PyErr_Occurred()) return nullptr;
        if (!dY || !H || !gain || (!dH && args[4] != Py_None) || watched() || !type_of(*H, dt)) Py_RETURN_NONE;
        M = H->size(0); n = H->size(1);
        if (!is(dY, H->scalar_type(), {M, n}) || !is(gain, at::kFloat, {n}) || (dH && !is(dH, H->scalar_type(), {M, n}))) Py_RETURN_NONE;
        if (!current_stream(&stream)) return nullptr;
        const auto opt = H->options().requires_grad(false);
        dX = at::empty({M, n}, opt);
        dG = at::empty({n}, opt.dtype(at::kFloat));
        ws = space(norm_bwd_bytes_fn(M, n, dt), opt);
        dy = dY->data_ptr(); h = H->data_ptr(); g = gain->data_ptr(); dx = dX.data_ptr(); dg = dG.data_ptr();
        if (dH) dh = dH->data_ptr();
        results = Py_BuildValue("(NN)", THPVariable_Wrap(dX), THPVariable_Wrap(dG));
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    if (!results) return nullptr;
    const int code = norm_bwd_fn(dy, h, (const float*)g, eps, dh, dx, (float*)dg, M, n, dt, 0, ws.data_ptr(), (size_t)ws.numel(), stream);
    return finished(results, code, "lr_rms_norm_bwd");
}

// (addresses in the order of the functions above, the three callables)
PyObject* setup(PyObject*, PyObject* args) {
    unsigned long long a[8];
    if (!PyArg_ParseTuple(args, "KKKKKKKKOOO", a, a + 1, a + 2, a + 3, a + 4, a + 5, a + 6, a + 7, &get_device, &get_stream, &check)) return nullptr;
    Py_INCREF(get_device); Py_INCREF(get_stream); Py_INCREF(check);
    fwd_fn = reinterpret_cast<decltype(fwd_fn)>(a[0]); fwd_q8_fn = reinterpret_cast<decltype(fwd_q8_fn)>(a[1]); fwd_bytes_fn = reinterpret_cast<decltype(fwd_bytes_fn)>(a[2]);
    bwd_fn = reinterpret_cast<decltype(bwd_fn)>(a[3]); bwd_bytes_fn = reinterpret_cast<decltype(bwd_bytes_fn)>(a[4]);
    norm_fwd_fn = reinterpret_cast<decltype(norm_fwd_fn)>(a[5]); norm_bwd_fn = reinterpret_cast<decltype(norm_bwd_fn)>(a[6]);
    norm_bwd_bytes_fn = reinterpret_cast<decltype(norm_bwd_bytes_fn)>(a[7]);
    Py_RETURN_NONE;
}

template <class F>
PyCFunction fast(F f) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)); }

PyMethodDef methods[] = {{"fwd", fast(fwd), METH_FASTCALL, nullptr}, {"fwd_q8", fast(fwd_q8), METH_FASTCALL, nullptr}, {"bwd", fast(bwd), METH_FASTCALL, nullptr},
                         {"norm_fwd", fast(norm_fwd), METH_FASTCALL, nullptr}, {"norm_bwd", fast(norm_bwd), METH_FASTCALL, nullptr},
                         {"setup", setup, METH_VARARGS, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "adapter_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_adapter_call() { return PyModule_Create(&module); }
