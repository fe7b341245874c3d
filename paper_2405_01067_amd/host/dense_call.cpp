// The calls of the dense layer, of dropout and of the group norm from Python, in native code, as adapter_call.cpp has those of a layer with adapters: what
// binding.lr_dense_fwd, lr_dense_bwd, lr_dropout, lr_group_norm_fwd and lr_group_norm_bwd do for plain tensors that fit each other, with the outputs and the
// workspace allocated here.  Anything else is answered with None, and the Python code goes on as if it had not asked.
#include "call_util.h"

#include "abtrain.h"

namespace {

using namespace native_call;

decltype(&lr_dense_fwd) dense_fwd_fn;
decltype(&lr_dense_fwd_workspace_bytes) dense_fwd_bytes_fn;
decltype(&lr_dense_bwd) dense_bwd_fn;
decltype(&lr_dense_bwd_workspace_bytes) dense_bwd_bytes_fn;
decltype(&lr_dropout) dropout_fn;
decltype(&lr_group_norm_fwd) group_fwd_fn;
decltype(&lr_group_norm_bwd) group_bwd_fn;
decltype(&lr_group_norm_workspace_bytes) group_bytes_fn;
PyTypeObject* dropout_type;

bool is(const at::Tensor* t, at::ScalarType dtype, std::initializer_list<int64_t> shape) {
    return t && t->scalar_type() == dtype && t->sizes() == at::IntArrayRef(shape.begin(), shape.size());
}
// None: NULL and true; false: not for this code
bool optional(PyObject* o, const at::Tensor** t, int64_t dim = 2) {
    *t = o == Py_None ? nullptr : plain(o, dim);
    return *t || o == Py_None;
}
bool activation(PyObject* o, int& act) {
    static const char* const names[] = {"none", "relu", "gelu", "gelu_tanh", "silu"};         // in the order of abt_activation
    if (!PyUnicode_CheckExact(o)) return false;
    for (act = 0; act < 5; ++act)
        if (PyUnicode_CompareWithASCIIString(o, names[act]) == 0) return true;
    return false;
}
// A binding.Dropout whose state is on this device, or None
bool dropout_of(PyObject* o, const at::Tensor& beside, const abt_dropout** d) {
    *d = nullptr;
    if (o == Py_None) return true;
    if (Py_TYPE(o) != dropout_type) return false;
    PyObject* const state = PyObject_GetAttrString(o, "state");
    PyObject* const address = state ? PyObject_GetAttrString(o, "address") : nullptr;
    const at::Tensor* const t = state ? plain(state, 1) : nullptr;
    const bool fine = address && t && t->device() == beside.device() && PyLong_Check(address);
    if (fine) *d = reinterpret_cast<const abt_dropout*>(PyLong_AsSize_t(address));
    const bool ours = fine && *d && (*d)->state == t->data_ptr();
    Py_XDECREF(state);
    Py_XDECREF(address);
    if (PyErr_Occurred()) PyErr_Clear();
    return ours;
}
// Are they all where X is, and is that the current device?  And its current stream.
bool stream_of(const at::Tensor& X, std::initializer_list<const at::Tensor*> others, void** s) {
    for (const at::Tensor* t : others)
        if (t && t->device() != X.device()) return false;
    PyObject* dev = PyObject_CallNoArgs(get_device);
    const bool here = dev && PyLong_AsLong(dev) == X.device().index();
    Py_XDECREF(dev);
    if (here && current_stream(s)) return true;
    PyErr_Clear();
    return false;
}
// undefined where none is needed
at::Tensor space(size_t bytes, const at::TensorOptions& opt) { return bytes ? at::empty({(int64_t)bytes}, opt.dtype(at::kByte)) : at::Tensor(); }
size_t bytes_of(const at::Tensor& t) { return t.defined() ? (size_t)t.numel() : 0; }
bool type_of(const at::Tensor& t, int& dt) {
    dt = t.scalar_type() == at::kBFloat16 ? ABT_BF16 : ABT_F32;
    return dt == ABT_BF16 || t.scalar_type() == at::kFloat;
}
void* address(const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }
void* address(const at::Tensor* t) { return t ? t->data_ptr() : nullptr; }
bool wants(PyObject* const* args, int count, int* need) {
    for (int i = 0; i < count; ++i)
        if ((need[i] = PyObject_IsTrue(args[i])) < 0) return false;
    return true;
}

// (X, W, bias, act, dropout, residual, save_Z) -> (Y, Z or None), or None
PyObject* dense_fwd(PyObject*, PyObject* const* args, Py_ssize_t k) {
    if (k != 7) { PyErr_SetString(PyExc_TypeError, "dense_fwd takes 7 arguments"); return nullptr; }
    void *stream, *x, *w, *b, *r, *y, *z;
    int64_t M, m, n;
    int act, save;
    const abt_dropout* drop;
    at::Tensor Y, Z, ws;
    PyObject* results;
    try {
        const at::Tensor *X = plain(args[0]), *W = plain(args[1]), *bias, *R;
        if (!wants(args + 6, 1, &save)) return nullptr;
        if (!X || !W || !optional(args[2], &bias, 1) || !optional(args[5], &R) || !activation(args[3], act) || watched()) Py_RETURN_NONE;
        M = X->size(0); n = X->size(1); m = W->size(0);
        if (!is(X, at::kBFloat16, {M, n}) || !is(W, at::kBFloat16, {m, n}) || (bias && !is(bias, at::kFloat, {m})) || (R && !is(R, at::kBFloat16, {M, m})) ||
            !dropout_of(args[4], *X, &drop) || !stream_of(*X, {W, bias, R}, &stream))
            Py_RETURN_NONE;
        const auto opt = X->options().requires_grad(false);
        Y = at::empty({M, m}, opt);
        if (save) Z = at::empty({M, m}, opt);
        ws = space(dense_fwd_bytes_fn(M, m, n), opt);
        x = address(X); w = address(W); b = address(bias); r = address(R); y = address(Y); z = address(Z);
        results = Py_BuildValue("(NN)", THPVariable_Wrap(Y), wrap_or_none(Z));
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;                                  // out of memory and the like: the Python code meets it again and says so
    }
    if (!results) return nullptr;
    return finished(results, dense_fwd_fn(x, w, (const float*)b, r, y, z, M, m, n, act, drop, ABT_BF16, address(ws), bytes_of(ws), stream),
                    "lr_dense_fwd");
}

// (dY, X, W, Z, act, dropout, need_dX, need_dW, need_dbias) -> (dX, dW, dbias), or None
PyObject* dense_bwd(PyObject*, PyObject* const* args, Py_ssize_t k) {
    if (k != 9) { PyErr_SetString(PyExc_TypeError, "dense_bwd takes 9 arguments"); return nullptr; }
    void *stream, *dy, *x, *w, *z, *to[3];
    int64_t M, m, n;
    int act, need[3];
    const abt_dropout* drop;
    at::Tensor out[3], ws;
    PyObject* results;
    try {
        const at::Tensor *dY = plain(args[0]), *X = plain(args[1]), *W = plain(args[2]), *Z;
        if (!wants(args + 6, 3, need)) return nullptr;
        if (!dY || !X || !W || !optional(args[3], &Z) || !activation(args[4], act) || watched()) Py_RETURN_NONE;
        M = X->size(0); n = X->size(1); m = W->size(0);
        if (!is(X, at::kBFloat16, {M, n}) || !is(W, at::kBFloat16, {m, n}) || !is(dY, at::kBFloat16, {M, m}) || (Z && !is(Z, at::kBFloat16, {M, m})) || (act && !Z) ||
            !dropout_of(args[5], *X, &drop) || !stream_of(*X, {dY, W, Z}, &stream))
            Py_RETURN_NONE;
        const auto opt = X->options().requires_grad(false);
        if (need[0]) out[0] = at::empty({M, n}, opt);
        if (need[1]) out[1] = at::empty({m, n}, opt.dtype(at::kFloat));
        if (need[2]) out[2] = at::empty({m}, opt.dtype(at::kFloat));
        ws = space(dense_bwd_bytes_fn(M, m, n), opt);
        dy = address(dY); x = address(X); w = address(W); z = address(Z);
        for (int i = 0; i < 3; ++i) to[i] = address(out[i]);
        results = Py_BuildValue("(NNN)", wrap_or_none(out[0]), wrap_or_none(out[1]), wrap_or_none(out[2]));
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    if (!results) return nullptr;
    return finished(results, dense_bwd_fn(dy, x, w, z, to[0], (float*)to[1], (float*)to[2], M, m, n, act, drop, ABT_BF16, 0, address(ws), bytes_of(ws), stream), "lr_dense_bwd");
}

// (X, dropout, residual) -> Y, or None
PyObject* dropout(PyObject*, PyObject* const* args, Py_ssize_t k) {
    if (k != 3) { PyErr_SetString(PyExc_TypeError, "dropout takes 3 arguments"); return nullptr; }
    void *stream, *x, *r, *y;
    int64_t count;
    int dt;
    const abt_dropout* drop;
    at::Tensor Y;
    PyObject* results;
    try {
        const int64_t dim = THPVariable_CheckExact(args[0]) ? THPVariable_Unpack(args[0]).dim() : -1;
        const at::Tensor *X = plain(args[0], dim), *R;
        if (!X || !optional(args[2], &R, dim) || watched() || !type_of(*X, dt) || (R && (R->scalar_type() != X->scalar_type() || R->sizes() != X->sizes())) || X->numel() == 0 ||
            args[1] == Py_None || !dropout_of(args[1], *X, &drop) || !stream_of(*X, {R}, &stream))
            Py_RETURN_NONE;
        count = X->numel();
        Y = at::empty(X->sizes(), X->options().requires_grad(false));
        x = address(X); r = address(R); y = address(Y);
        results = THPVariable_Wrap(Y);
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    if (!results) return nullptr;
    return finished(results, dropout_fn(x, r, y, count, drop, dt, stream), "lr_dropout");
}

// [N, ..., C]
const at::Tensor* images(PyObject* o, int64_t& N, int64_t& pixels, int64_t& C) {
    const int64_t dim = THPVariable_CheckExact(o) ? THPVariable_Unpack(o).dim() : 0;
    const at::Tensor* const X = dim >= 2 ? plain(o, dim) : nullptr;
    if (!X || X->numel() == 0) return nullptr;
    N = X->size(0); C = X->size(dim - 1);
    pixels = X->numel() / (N * C);
    return X;
}

// (X, gain, shift, groups, eps, act) -> (Y, mean, rstd), or None
PyObject* group_fwd(PyObject*, PyObject* const* args, Py_ssize_t k) {
    if (k != 6) { PyErr_SetString(PyExc_TypeError, "group_fwd takes 6 arguments"); return nullptr; }
    void *stream, *in[3], *to[3];
    int64_t N, pixels, C, groups;
    int dt, act;
    double eps;
    at::Tensor out[3], ws;
    PyObject* results;
    try {
        const at::Tensor *X = images(args[0], N, pixels, C), *gain = plain(args[1], 1), *shift = plain(args[2], 1);
        if (!X || !PyLong_CheckExact(args[3]) || !PyFloat_CheckExact(args[4]) || !activation(args[5], act) || watched() || !type_of(*X, dt) || !is(gain, at::kFloat, {C}) ||
            !is(shift, at::kFloat, {C}))
            Py_RETURN_NONE;
        groups = PyLong_AsSsize_t(args[3]);
        eps = PyFloat_AS_DOUBLE(args[4]);
        if (PyErr_Occurred()) { PyErr_Clear(); Py_RETURN_NONE; }
        if (groups < 1 || C % 8 || C % groups) Py_RETURN_NONE;
        const size_t need = group_bytes_fn(N, pixels, C, groups, dt, 0);
        if (!stream_of(*X, {gain, shift}, &stream)) Py_RETURN_NONE;
        const auto opt = X->options().requires_grad(false);
        out[0] = at::empty(X->sizes(), opt);
        out[1] = at::empty({N, groups}, opt.dtype(at::kFloat));
        out[2] = at::empty({N, groups}, opt.dtype(at::kFloat));
        ws = space(need, opt);
        in[0] = address(X); in[1] = address(gain); in[2] = address(shift);
        for (int i = 0; i < 3; ++i) to[i] = address(out[i]);
        results = Py_BuildValue("(NNN)", THPVariable_Wrap(out[0]), THPVariable_Wrap(out[1]), THPVariable_Wrap(out[2]));
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    if (!results) return nullptr;
    return finished(results, group_fwd_fn(in[0], (const float*)in[1], (const float*)in[2], eps, to[0], (float*)to[1], (float*)to[2], N, pixels, C, groups, act, dt, address(ws),
                                          bytes_of(ws), stream), "lr_group_norm_fwd");
}

// (dY, X, gain, shift, mean, rstd, act, need_dX, need_dgain, need_dshift) -> (dX, dgain, dshift), or None
PyObject* group_bwd(PyObject*, PyObject* const* args, Py_ssize_t k) {
    if (k != 10) { PyErr_SetString(PyExc_TypeError, "group_bwd takes 10 arguments"); return nullptr; }
    void *stream, *in[6], *to[3];
    int64_t N, pixels, C, groups;
    int dt, act, need[3];
    at::Tensor out[3], ws;
    PyObject* results;
    try {
        if (!wants(args + 7, 3, need)) return nullptr;
        const at::Tensor* const X = images(args[1], N, pixels, C);
        if (!X) Py_RETURN_NONE;
        const at::Tensor* const t[6] = {plain(args[0], X->dim()), X, plain(args[2], 1), plain(args[3], 1), plain(args[4]), plain(args[5])};
        if (!t[0] || !t[4] || !activation(args[6], act) || watched() || !type_of(*X, dt)) Py_RETURN_NONE;
        groups = t[4]->size(1);
        if (t[0]->scalar_type() != X->scalar_type() || t[0]->sizes() != X->sizes() || !is(t[2], at::kFloat, {C}) || !is(t[3], at::kFloat, {C}) || !is(t[4], at::kFloat, {N, groups}) ||
            !is(t[5], at::kFloat, {N, groups}))
            Py_RETURN_NONE;
        if (groups < 1 || C % 8 || C % groups) Py_RETURN_NONE;
        const size_t bytes = group_bytes_fn(N, pixels, C, groups, dt, 1);
        if (!stream_of(*X, {t[0], t[2], t[3], t[4], t[5]}, &stream)) Py_RETURN_NONE;
        const auto opt = X->options().requires_grad(false);
        if (need[0]) out[0] = at::empty(X->sizes(), opt);
        for (int i = 1; i < 3; ++i)
            if (need[i]) out[i] = at::empty({C}, opt.dtype(at::kFloat));
        ws = space(bytes, opt);
        for (int i = 0; i < 6; ++i) in[i] = address(t[i]);
        for (int i = 0; i < 3; ++i) to[i] = address(out[i]);
        results = Py_BuildValue("(NNN)", wrap_or_none(out[0]), wrap_or_none(out[1]), wrap_or_none(out[2]));
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    if (!results) return nullptr;
    return finished(results, group_bwd_fn(in[0], in[1], (const float*)in[2], (const float*)in[3], (const float*)in[4], (const float*)in[5], to[0], (float*)to[1], (float*)to[2], N, pixels, C,
                                          groups, act, dt, 0, address(ws), bytes_of(ws), stream), "lr_group_norm_bwd");
}

// (addresses in the order of the functions above, the three callables); the type of binding.Dropout by itself
PyObject* setup(PyObject*, PyObject* args) {
    unsigned long long a[8];
    if (!PyArg_ParseTuple(args, "KKKKKKKKOOO", a, a + 1, a + 2, a + 3, a + 4, a + 5, a + 6, a + 7, &get_device, &get_stream, &check)) return nullptr;
    Py_INCREF(get_device); Py_INCREF(get_stream); Py_INCREF(check);
    dense_fwd_fn = reinterpret_cast<decltype(dense_fwd_fn)>(a[0]); dense_fwd_bytes_fn = reinterpret_cast<decltype(dense_fwd_bytes_fn)>(a[1]);
    dense_bwd_fn = reinterpret_cast<decltype(dense_bwd_fn)>(a[2]); dense_bwd_bytes_fn = reinterpret_cast<decltype(dense_bwd_bytes_fn)>(a[3]);
    dropout_fn = reinterpret_cast<decltype(dropout_fn)>(a[4]); group_fwd_fn = reinterpret_cast<decltype(group_fwd_fn)>(a[5]);
    group_bwd_fn = reinterpret_cast<decltype(group_bwd_fn)>(a[6]); group_bytes_fn = reinterpret_cast<decltype(group_bytes_fn)>(a[7]);
    Py_RETURN_NONE;
}
PyObject* dropout_class(PyObject*, PyObject* type) {
    if (!PyType_Check(type)) { PyErr_SetString(PyExc_TypeError, "a type"); return nullptr; }
    Py_INCREF(type);
    dropout_type = reinterpret_cast<PyTypeObject*>(type);
    Py_RETURN_NONE;
}

template <class F>
PyCFunction fast(F f) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)); }

PyMethodDef methods[] = {{"dense_fwd", fast(dense_fwd), METH_FASTCALL, nullptr}, {"dense_bwd", fast(dense_bwd), METH_FASTCALL, nullptr},
                         {"dropout", fast(dropout), METH_FASTCALL, nullptr}, {"group_fwd", fast(group_fwd), METH_FASTCALL, nullptr},
                         {"group_bwd", fast(group_bwd), METH_FASTCALL, nullptr}, {"dropout_class", dropout_class, METH_O, nullptr},
                         {"setup", setup, METH_VARARGS, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "dense_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_dense_call() { return PyModule_Create(&module); }
