// Descriptors of LayerBuffers objects (binding.py), written straight into an array of squant_layer: in
// Python this takes about 2 us a layer, longer than the GPU needs for the layers of a small model.
// fill(list, start, address) writes descriptors from element `start` on and returns the index of the first
// element it leaves to the Python code: one that is not made of plain tensors, or that the Python code
// would reject.  It neither keeps nor caches anything.
// linear(), linear_backward(), checkpoint() and restore() make whole calls of the linear operators (linear.py) for plain
// tensors of the current device: about 20 us in Python, longer than the GPU needs for few tokens.  They return None for
// whatever they leave to the Python code, which checks the arguments anew and has the errors' texts.
#include <Python.h>

#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/core/grad_mode.h>
#include <ATen/ops/empty.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstddef>
#include <limits>

#include "squant.h"

namespace {

PyObject *s_names[8];   // w, codes, scales, kernel_err, channel_err, dequant, dequant_bf16, scales_in

// A reference that goes with its scope, also when data_ptr() throws.
struct Held {
    PyObject *p = nullptr;
    Held() = default;
    Held(const Held &) = delete;
    Held &operator=(const Held &) = delete;
    ~Held() { Py_XDECREF(p); }
};

// The tensor behind attribute i of o: 1 found, 0 None, -1 not a plain tensor (or no such attribute).
int tensor_of(PyObject *o, int i, const at::Tensor *&t, Held &held)
{
    held.p = PyObject_GetAttr(o, s_names[i]);
    if (!held.p) {
        PyErr_Clear();
        return -1;
    }
    if (held.p == Py_None) return 0;
    if (!THPVariable_CheckExact(held.p)) return -1;   // subclasses may have their own idea of data_ptr()
    t = &THPVariable_Unpack(held.p);
    return 1;
}

// One descriptor.  False: left to the Python code.
bool descriptor(PyObject *o, squant_layer &l)
{
    void *ptr[8] = {};
    bool ok = true;
    const at::Tensor *w = nullptr;
    Held held[8];
    for (int i = 0; i < 8 && ok; ++i) {
        const at::Tensor *t = nullptr;
        const int kind = tensor_of(o, i, t, held[i]);
        if (kind < 0 || (i == 0 && kind == 0)) { ok = false; break; }
        if (kind == 0) continue;
        ptr[i] = t->data_ptr();
        if (i == 0) {
            w = t;
            const auto s = w->sizes();
            if (s.size() < 2 || s.size() > 4) { ok = false; break; }
            int32_t d[4] = {1, 1, 1, 1};
            for (size_t k = 0; k < s.size(); ++k) {
                if (s[k] > std::numeric_limits<int32_t>::max()) ok = false;
                d[k] = static_cast<int32_t>(s[k]);
            }
            l.cout = d[0]; l.cin = d[1]; l.kh = d[2]; l.kw = d[3];
        } else if (i == 7) {
            ok = t->scalar_type() == at::kFloat && t->numel() == l.cout && t->is_contiguous() && t->device() == w->device();
        }
    }
    if (ok) {
        l.w = static_cast<const float *>(ptr[0]);
        l.codes = static_cast<int8_t *>(ptr[1]);
        l.scales = static_cast<float *>(ptr[2]);
        l.kernel_err = static_cast<float *>(ptr[3]);
        l.channel_err = static_cast<float *>(ptr[4]);
        l.dequant = static_cast<float *>(ptr[5]);
        l.dequant_bf16 = static_cast<uint16_t *>(ptr[6]);
        l.scales_in = static_cast<const float *>(ptr[7]);
    }
    return ok;
}

PyObject *fill(PyObject *, PyObject *args)
{
    PyObject *list = nullptr;
    Py_ssize_t start = 0;
    unsigned long long address = 0;
    if (!PyArg_ParseTuple(args, "O!nK", &PyList_Type, &list, &start, &address)) return nullptr;
    squant_layer *out = reinterpret_cast<squant_layer *>(static_cast<uintptr_t>(address));
    Py_ssize_t i = start;
    if (!at::impl::torch_function_mode_enabled()) {
        for (; i < PyList_GET_SIZE(list); ++i) {
            bool ok = false;
            try {
                ok = descriptor(PyList_GET_ITEM(list, i), out[i]);
            } catch (const std::exception &) {   // a tensor without storage: the Python code raises its error
                ok = false;
            }
            if (!ok) break;
        }
    }
    return PyLong_FromSsize_t(i);
}

// ---- linear operators

using LinearFn = int (*)(const squant_linear_args *, void *);
using LinearNeedFn = int64_t (*)(const squant_linear_args *);
using GradFn = int (*)(const squant_linear_grad_args *, void *);
using GradNeedFn = int64_t (*)(const squant_linear_grad_args *);
using CheckpointFn = int (*)(const void *, int64_t, int32_t, int64_t, const squant_checkpoint_data *, void *);
using RestoreFn = int (*)(const squant_checkpoint_data *, int64_t, int32_t, void *, int64_t, void *);

constexpr int64_t kMostRows = std::numeric_limits<int32_t>::max();

// The library's functions, as use() was told them.
struct Library {
    LinearFn linear;
    LinearNeedFn linear_need;
    GradFn grad;
    GradNeedFn grad_need;
    CheckpointFn checkpoint;
    RestoreFn restore;
} s_lib;

PyObject *use(PyObject *, PyObject *args)
{
    unsigned long long a[6];
    if (!PyArg_ParseTuple(args, "KKKKKK", &a[0], &a[1], &a[2], &a[3], &a[4], &a[5])) return nullptr;
    const auto at = [&](int i) { return static_cast<uintptr_t>(a[i]); };
    s_lib = {reinterpret_cast<LinearFn>(at(0)), reinterpret_cast<LinearNeedFn>(at(1)), reinterpret_cast<GradFn>(at(2)),
             reinterpret_cast<GradNeedFn>(at(3)), reinterpret_cast<CheckpointFn>(at(4)), reinterpret_cast<RestoreFn>(at(5))};
    Py_RETURN_NONE;
}

void *stream_of(unsigned long long handle) { return reinterpret_cast<void *>(static_cast<uintptr_t>(handle)); }

// Whether a result would have to be part of an autograd graph, which these calls make none of: the Python code refuses it.
bool wants_graph(std::initializer_list<const at::Tensor *> inputs)
{
    if (!at::GradMode::is_enabled()) return false;
    for (const at::Tensor *t : inputs)
        if (t && t->requires_grad()) return true;
    return false;
}

// The tensor itself; null for None; false where it is anything but a plain tensor.
bool plain(PyObject *o, const at::Tensor *&t)
{
    t = nullptr;
    if (o == Py_None) return true;
    if (!THPVariable_CheckExact(o)) return false;
    t = &THPVariable_Unpack(o);
    return true;
}

// [..., features] as rows: two dimensions with neighbouring features, or a contiguous tensor.
bool rows_of(const at::Tensor &t, int64_t &rows, int64_t &features, int64_t &stride)
{
    const auto s = t.sizes();
    if (s.size() < 2) return false;
    features = s.back();
    if (features < 1 || features > kMostRows) return false;
    if (s.size() == 2) {
        if (features > 1 && t.stride(1) != 1) return false;
        rows = s[0];
        stride = t.stride(0);
        return true;
    }
    if (!t.is_contiguous()) return false;
    rows = 1;
    for (size_t i = 0; i + 1 < s.size(); ++i) rows *= s[i];
    stride = features;
    return true;
}

bool vector_ok(const at::Tensor *t, int64_t n, const at::Device &d)
{
    return !t || (t->scalar_type() == at::kFloat && t->dim() == 1 && t->numel() == n && t->is_contiguous() && t->device() == d);
}

bool codes_ok(const at::Tensor &codes, int64_t cout, int64_t cin, bool packed, const at::Device &d)
{
    return codes.scalar_type() == at::kChar && codes.dim() >= 2 && codes.size(0) == cout && codes.numel() == cout * (packed ? (cin + 1) / 2 : cin) &&
           codes.is_contiguous() && codes.device() == d;
}

bool checkpoint_ok(const at::Tensor *codes, const at::Tensor *exps, int64_t rows, int64_t features, const at::Device &d)
{
    const int64_t groups = (features + 31) / 32;
    return codes && exps && codes->scalar_type() == at::kChar && exps->scalar_type() == at::kByte && codes->dim() == 2 && exps->dim() == 2 &&
           codes->size(0) == rows && codes->size(1) == 32 * groups && exps->size(0) == rows && exps->size(1) == groups &&
           codes->is_contiguous() && exps->is_contiguous() && codes->device() == d && exps->device() == d;
}

PyObject *none() { Py_RETURN_NONE; }
PyObject *tensor_or_none(const at::Tensor &t) { return t.defined() ? THPVariable_Wrap(t) : none(); }

// Runs a call; whatever throws inside (an allocation, a tensor without storage) leaves it to the Python code.
template <typename Body>
PyObject *guarded(const Body &body)
{
    if (at::impl::torch_function_mode_enabled()) Py_RETURN_NONE;
    try {
        return body();
    } catch (const std::exception &) {
        if (PyErr_Occurred()) PyErr_Clear();
        Py_RETURN_NONE;
    }
}

at::Tensor new_tensor(at::IntArrayRef shape, at::ScalarType type, const at::Device &d)
{
    return at::empty(shape, at::TensorOptions().dtype(type).device(d));
}

PyObject *linear(PyObject *, PyObject *args)
{
    unsigned long long stream;
    PyObject *po[6];   // x, codes, scales, bias, residual, out
    int device, act, packed, save;
    if (!PyArg_ParseTuple(args, "KiOOOOOOipp", &stream, &device, &po[0], &po[1], &po[2], &po[3], &po[4], &po[5], &act, &packed, &save))
        return nullptr;
    return guarded([&]() -> PyObject * {
        const at::Tensor *t[6];
        for (int i = 0; i < 6; ++i)
            if (!plain(po[i], t[i])) return none();
        if (!t[0] || !t[1] || !t[2] || act < 0 || wants_graph({t[0], t[2], t[3], t[4], t[5]})) return none();
        const at::Tensor &x = *t[0];
        const at::Device d = x.device();
        const auto type = x.scalar_type();
        if (!d.is_cuda() || d.index() != device || (type != at::kBFloat16 && type != at::kHalf) || t[1]->dim() < 2) return none();
        squant_linear_args a{};
        int64_t cin = 0;
        const int64_t cout = t[1]->size(0);
        if (!rows_of(x, a.tokens, cin, a.x_stride) || cout > kMostRows) return none();
        if (!codes_ok(*t[1], cout, cin, packed, d) || !vector_ok(t[2], cout, d) || !vector_ok(t[3], cout, d)) return none();
        auto shape = x.sizes().vec();
        shape.back() = cout;
        int64_t rows = 0, features = 0;
        for (int i = 4; i < 6; ++i)
            if (t[i] && (t[i]->scalar_type() != type || t[i]->sizes() != at::IntArrayRef(shape) || t[i]->device() != d)) return none();
        if (t[4] && !rows_of(*t[4], rows, features, a.residual_stride)) return none();
        at::Tensor y = t[5] ? *t[5] : new_tensor(shape, type, d);
        if (!rows_of(y, rows, features, a.y_stride)) return none();
        a.cin = static_cast<int32_t>(cin);
        a.cout = static_cast<int32_t>(cout);
        a.dtype = type == at::kHalf ? SQUANT_FP16 : SQUANT_BF16;
        a.act = static_cast<uint32_t>(act);
        a.flags = packed ? SQUANT_FLAG_PACK_INT4 : 0;
        a.x = x.data_ptr();
        a.codes = static_cast<const int8_t *>(t[1]->data_ptr());
        a.scales = static_cast<const float *>(t[2]->data_ptr());
        a.bias = t[3] ? static_cast<const float *>(t[3]->data_ptr()) : nullptr;
        a.residual = t[4] ? t[4]->data_ptr() : nullptr;
        a.y = y.data_ptr();
        at::Tensor codes, exps, workspace;
        if (save) {
            const int64_t groups = (cout + 31) / 32;
            codes = new_tensor({a.tokens, 32 * groups}, at::kChar, d);
            exps = new_tensor({a.tokens, groups}, at::kByte, d);
            a.z = {static_cast<int8_t *>(codes.data_ptr()), static_cast<uint8_t *>(exps.data_ptr())};
        }
        const int64_t bytes = s_lib.linear_need(&a);
        if (bytes < 0) return none();
        if (bytes > 0) {
            workspace = new_tensor({bytes}, at::kByte, d);
            a.workspace = workspace.data_ptr();
            a.workspace_bytes = bytes;
        }
        const int rc = s_lib.linear(&a, stream_of(stream));
        if (rc != SQUANT_OK) return PyLong_FromLong(rc);
        if (t[5] && !y.is_inference()) y.unsafeGetTensorImpl()->bump_version();   // written in place, as autograd has to know
        if (!save) {
            if (!t[5]) return THPVariable_Wrap(y);
            Py_INCREF(po[5]);
            return po[5];
        }
        PyObject *first = po[5];
        if (t[5]) Py_INCREF(first);
        else first = THPVariable_Wrap(y);
        return Py_BuildValue("(NNN)", first, THPVariable_Wrap(codes), THPVariable_Wrap(exps));
    });
}

PyObject *linear_backward(PyObject *, PyObject *args)
{
    unsigned long long stream;
    PyObject *po[8];   // dy, codes, scales, bias, z codes, z exps, x codes, x exps
    int device, act, packed, want_dx, want_dw, want_db, want_ds;
    long long cin;
    if (!PyArg_ParseTuple(args, "KiOOOOOOOOLippppp", &stream, &device, &po[0], &po[1], &po[2], &po[3], &po[4], &po[5], &po[6], &po[7],
                          &cin, &act, &packed, &want_dx, &want_dw, &want_db, &want_ds))
        return nullptr;
    return guarded([&]() -> PyObject * {
        const at::Tensor *t[8];
        for (int i = 0; i < 8; ++i)
            if (!plain(po[i], t[i])) return none();
        if (!t[0] || !t[1] || !t[2] || act < 0 || wants_graph({t[0]})) return none();
        const at::Tensor &dy = *t[0];
        const at::Device d = dy.device();
        if (!d.is_cuda() || d.index() != device || dy.scalar_type() != at::kBFloat16 || cin < 1 || cin > kMostRows) return none();
        squant_linear_grad_args a{};
        int64_t cout = 0;
        if (!rows_of(dy, a.tokens, cout, a.dy_stride)) return none();
        if (!codes_ok(*t[1], cout, cin, packed, d) || !vector_ok(t[2], cout, d) || !vector_ok(t[3], cout, d)) return none();
        if ((t[4] || t[5]) && !checkpoint_ok(t[4], t[5], a.tokens, cout, d)) return none();
        if ((t[6] || t[7]) && !checkpoint_ok(t[6], t[7], a.tokens, cin, d)) return none();
        if ((!t[4] && (act || want_ds)) || (!t[6] && want_dw)) return none();
        auto shape = dy.sizes().vec();
        shape.back() = cin;
        at::Tensor dx, dw, db, ds, workspace;
        if (want_dx) dx = new_tensor(shape, at::kBFloat16, d);
        if (want_dw) dw = new_tensor({cout, cin}, at::kBFloat16, d);
        if (want_db) db = new_tensor({cout}, at::kFloat, d);
        if (want_ds) ds = new_tensor({cout}, at::kFloat, d);
        a.cin = static_cast<int32_t>(cin);
        a.cout = static_cast<int32_t>(cout);
        a.act = static_cast<uint32_t>(act);
        a.flags = packed ? SQUANT_FLAG_PACK_INT4 : 0;
        a.dy = dy.data_ptr();
        a.codes = static_cast<const int8_t *>(t[1]->data_ptr());
        a.scales = static_cast<const float *>(t[2]->data_ptr());
        a.bias = t[3] ? static_cast<const float *>(t[3]->data_ptr()) : nullptr;
        if (t[4]) a.z = {static_cast<int8_t *>(t[4]->data_ptr()), static_cast<uint8_t *>(t[5]->data_ptr())};
        if (t[6]) a.x = {static_cast<int8_t *>(t[6]->data_ptr()), static_cast<uint8_t *>(t[7]->data_ptr())};
        a.dx = want_dx ? dx.data_ptr() : nullptr;
        a.dweight = want_dw ? dw.data_ptr() : nullptr;
        a.dx_stride = a.dweight_stride = cin;
        a.dbias = want_db ? static_cast<float *>(db.data_ptr()) : nullptr;
        a.dscales = want_ds ? static_cast<float *>(ds.data_ptr()) : nullptr;
        const int64_t bytes = s_lib.grad_need(&a);
        if (bytes < 0) return none();
        if (bytes > 0) {
            workspace = new_tensor({bytes}, at::kByte, d);
            a.workspace = workspace.data_ptr();
            a.workspace_bytes = bytes;
        }
        const int rc = s_lib.grad(&a, stream_of(stream));
        if (rc != SQUANT_OK) return PyLong_FromLong(rc);
        return Py_BuildValue("(NNNN)", tensor_or_none(dx), tensor_or_none(dw), tensor_or_none(db), tensor_or_none(ds));
    });
}

PyObject *checkpoint(PyObject *, PyObject *args)
{
    unsigned long long stream;
    PyObject *px;
    int device;
    if (!PyArg_ParseTuple(args, "KiO", &stream, &device, &px)) return nullptr;
    return guarded([&]() -> PyObject * {
        const at::Tensor *x;
        int64_t rows, features, stride;
        if (!plain(px, x) || !x || !x->is_cuda() || x->device().index() != device || x->scalar_type() != at::kBFloat16 ||
            !rows_of(*x, rows, features, stride)) return none();
        const int64_t groups = (features + 31) / 32;
        at::Tensor codes = new_tensor({rows, 32 * groups}, at::kChar, x->device()), exps = new_tensor({rows, groups}, at::kByte, x->device());
        const squant_checkpoint_data to{static_cast<int8_t *>(codes.data_ptr()), static_cast<uint8_t *>(exps.data_ptr())};
        const int rc = s_lib.checkpoint(x->data_ptr(), rows, static_cast<int32_t>(features), stride, &to, stream_of(stream));
        if (rc != SQUANT_OK) return PyLong_FromLong(rc);
        return Py_BuildValue("(NNL)", THPVariable_Wrap(codes), THPVariable_Wrap(exps), static_cast<long long>(features));
    });
}

PyObject *restore(PyObject *, PyObject *args)
{
    unsigned long long stream;
    PyObject *pc, *pe;
    int device;
    long long features;
    if (!PyArg_ParseTuple(args, "KiOOL", &stream, &device, &pc, &pe, &features)) return nullptr;
    return guarded([&]() -> PyObject * {
        const at::Tensor *codes, *exps;
        if (!plain(pc, codes) || !plain(pe, exps) || !codes || !exps || !codes->is_cuda() || codes->device().index() != device || codes->dim() != 2 ||
            features < 1 || features > kMostRows || !checkpoint_ok(codes, exps, codes->size(0), features, codes->device())) return none();
        const int64_t rows = codes->size(0);
        at::Tensor out = new_tensor({rows, features}, at::kBFloat16, codes->device());
        const squant_checkpoint_data from{static_cast<int8_t *>(codes->data_ptr()), static_cast<uint8_t *>(exps->data_ptr())};
        const int rc = s_lib.restore(&from, rows, static_cast<int32_t>(features), out.data_ptr(), features, stream_of(stream));
        return rc != SQUANT_OK ? PyLong_FromLong(rc) : THPVariable_Wrap(out);
    });
}

PyMethodDef methods[] = {{"use", use, METH_VARARGS, "addresses of the library's functions"},
                         {"linear", linear, METH_VARARGS, "one call of squant_linear: the output (with its checkpoint's codes and exponents), an error code, or None"},
                         {"linear_backward", linear_backward, METH_VARARGS, "one call of squant_linear_backward: four gradients, an error code, or None"},
                         {"checkpoint", checkpoint, METH_VARARGS, "one call of squant_checkpoint: codes, exponents and features, an error code, or None"},
                         {"restore", restore, METH_VARARGS, "one call of squant_checkpoint_restore: the values, an error code, or None"},
                         {"fill", fill, METH_VARARGS, "fill(list, start, address) -> index of the first element left out"},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void)
{
    const char *names[8] = {"w", "codes", "scales", "kernel_err", "channel_err", "dequant", "dequant_bf16", "scales_in"};
    for (int i = 0; i < 8; ++i) {
        s_names[i] = PyUnicode_InternFromString(names[i]);
        if (!s_names[i]) return nullptr;
    }
    PyObject *m = PyModule_Create(&module);
    if (!m) return nullptr;
    // Size of a descriptor and the places of its fields as this extension was built with them, in the order of
    // squant.h: the Python code compares them with its own before it hands over an array.
    using L = squant_layer;
    PyObject *layout = Py_BuildValue("(nnnnnnnnnnnnn)", sizeof(L), offsetof(L, w), offsetof(L, cout), offsetof(L, cin), offsetof(L, kh), offsetof(L, kw),
                                     offsetof(L, codes), offsetof(L, scales), offsetof(L, kernel_err), offsetof(L, channel_err),
                                     offsetof(L, dequant), offsetof(L, dequant_bf16), offsetof(L, scales_in));
    if (PyModule_AddIntConstant(m, "linear_bytes", sizeof(squant_linear_args)) != 0 ||
        PyModule_AddIntConstant(m, "linear_grad_bytes", sizeof(squant_linear_grad_args)) != 0) {
        Py_XDECREF(layout);
        Py_DECREF(m);
        return nullptr;
    }
    if (!layout || PyModule_AddObject(m, "layout", layout) != 0) {
        Py_XDECREF(layout);
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
