// Host path of the Python binding: what happens between a Python call and the C entry point.
//
// A product at the small sizes takes 2-4 us on the GPU, so a call's time is the host's.  Checking the
// arguments, allocating the result, finding the stream and marshalling through ctypes took 6-7 us of
// interpreted code a call; here the same checks read the tensors' fields and the C entry point is called
// through its address.  Python keeps the names, the defaults and the rare paths (lending scratch).
//
// The C library is the one the Python side has loaded: bind() takes its entry points' addresses, so this
// module does not link to it and a process always talks to one library.
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/hip/EmptyTensor.h>
#include <ATen/ops/empty.h>
#include <c10/hip/HIPStream.h>

#include <vector>

#include "bsr_spmm.h"

namespace {

bsr_status (*g_spmm)(const bsr_matrix*, int64_t, const void*, void*, bsr_dtype, bsr_path, void*) = nullptr;
bsr_status (*g_spmm_static)(const bsr_matrix*, int64_t, const void*, void*, bsr_dtype, void*) = nullptr;
bsr_status (*g_sddmm)(const bsr_matrix*, int64_t, const void*, const void*, void*, bsr_dtype, void*, size_t, void*) = nullptr;
bsr_status (*g_sddmm_workspace)(const bsr_matrix*, int64_t, size_t*) = nullptr;
bsr_status (*g_scratch_size)(const bsr_matrix*, int64_t, size_t*) = nullptr;
bsr_status (*g_spmm_epilogue)(const bsr_matrix*, int64_t, const void*, void*, bsr_dtype, const bsr_epilogue*, void*) = nullptr;
bsr_status (*g_backward)(int64_t, int64_t, bsr_act, bsr_dtype, const void*, const void*, bsr_dtype, void*, float*, void*, size_t, void*) = nullptr;
bsr_status (*g_backward_workspace)(int64_t, int64_t, size_t*) = nullptr;
bsr_status (*g_adamw_step)(const bsr_adamw*, const bsr_adamw_hyper*, void*) = nullptr;
bsr_status (*g_adamw_moments)(const bsr_adamw*, bsr_dtype, void* const*, void* const*, void*) = nullptr;
bsr_status (*g_spmm_gated)(const bsr_matrix*, int64_t, const void*, void*, bsr_dtype, const bsr_gated*, void*, size_t, void*) = nullptr;
bsr_status (*g_gated_workspace)(const bsr_matrix*, int64_t, bsr_dtype, size_t*) = nullptr;
bsr_status (*g_gated_backward)(int64_t, int64_t, int32_t, bsr_act, bsr_dtype, const void*, const void*, bsr_dtype, void*, float*, void*, size_t, void*) = nullptr;
bsr_status (*g_gated_backward_workspace)(int64_t, int64_t, int32_t, size_t*) = nullptr;
bsr_status (*g_norm)(int64_t, int64_t, bsr_dtype, const void*, bsr_dtype, const void*, void*, void*, const bsr_residual*, void*) = nullptr;
bsr_status (*g_norm_backward)(int64_t, int64_t, bsr_dtype, const void*, bsr_dtype, const void*, const void*, const void*, void*, void*, const bsr_residual*,
                              const bsr_residual_grads*, void*, size_t, void*) = nullptr;
bsr_status (*g_norm_backward_workspace)(int64_t, int64_t, size_t*) = nullptr;
bsr_status (*g_muon_step)(const bsr_muon*, const bsr_muon_hyper*, void*) = nullptr;
PyObject* g_error = nullptr;                          // BsrError(status, where)

// What the calls need to know of a matrix; owned by the Python object that owns the handle.
struct core_object {
    PyObject_HEAD
    bsr_matrix* handle;
    int64_t n, k, nnzb;
    int64_t bs_r, bs_c;
    int dtype;
    size_t scratch_bytes;                             // what has been lent so far
    uintptr_t known;                                  // the stream that was given work last, which the owner knows; to begin with its own
};

constexpr at::ScalarType kTypes[3] = {at::kFloat, at::kHalf, at::kBFloat16};

int core_init(PyObject* self, PyObject* args, PyObject*)
{
    core_object* c = reinterpret_cast<core_object*>(self);
    unsigned long long handle = 0, known = 0;
    long long n, k, nnzb, bs_r, bs_c;
    if (!PyArg_ParseTuple(args, "KLLLLLiK", &handle, &n, &k, &nnzb, &bs_r, &bs_c, &c->dtype, &known)) return -1;
    c->known = (uintptr_t)known;
    c->handle = reinterpret_cast<bsr_matrix*>(handle);
    c->n = n; c->k = k; c->nnzb = nnzb; c->bs_r = bs_r; c->bs_c = bs_c;
    c->scratch_bytes = 0;
    return 0;
}

PyObject* core_lent(PyObject* self, PyObject* bytes)
{
    const size_t v = PyLong_AsSize_t(bytes);
    if (PyErr_Occurred()) return nullptr;
    reinterpret_cast<core_object*>(self)->scratch_bytes = v;
    Py_RETURN_NONE;
}

PyObject* core_closed(PyObject* self, PyObject*)
{
    reinterpret_cast<core_object*>(self)->handle = nullptr;
    Py_RETURN_NONE;
}

PyMethodDef core_methods[] = {
    {"lent", core_lent, METH_O, "The handle has been lent this many bytes of scratch."},
    {"closed", core_closed, METH_NOARGS, "The handle has been destroyed."},
    {nullptr, nullptr, 0, nullptr}};

PyTypeObject core_type = {PyVarObject_HEAD_INIT(nullptr, 0)};

PyObject* value_error(const char* text)
{
    PyErr_SetString(PyExc_ValueError, text);
    return nullptr;
}

// Code of a tensor's type, -1 with KeyError(dtype) for a type the library has not.
int type_code(const at::Tensor& t, PyObject* obj)
{
    const at::ScalarType s = t.scalar_type();
    for (int i = 0; i < 3; ++i)
        if (s == kTypes[i]) return i;
    PyObject* d = PyObject_GetAttrString(obj, "dtype");
    if (d) { PyErr_SetObject(PyExc_KeyError, d); Py_DECREF(d); }
    return -1;
}

// Code of a type's name ("f32" | "f16" | "bf16"; None or "": `fallback`), -1 with KeyError(name).
int name_code(PyObject* name, int fallback)
{
    if (name == Py_None) return fallback;
    if (PyUnicode_Check(name)) {
        Py_ssize_t len = 0;
        const char* s = PyUnicode_AsUTF8AndSize(name, &len);
        if (!s) return -1;
        if (len == 0) return fallback;
        if (!strcmp(s, "f32")) return BSR_F32;
        if (!strcmp(s, "f16")) return BSR_F16;
        if (!strcmp(s, "bf16")) return BSR_BF16;
    }
    PyErr_SetObject(PyExc_KeyError, name);
    return -1;
}

bool tensor_of(PyObject* obj, const char* what, const at::Tensor** out)
{
    if (!THPVariable_Check(obj)) {
        PyErr_Format(PyExc_TypeError, "%s must be a torch.Tensor", what);
        return false;
    }
    *out = &THPVariable_Unpack(obj);
    return true;
}

core_object* core_of(PyObject* obj)
{
    if (Py_TYPE(obj) == &core_type) return reinterpret_cast<core_object*>(obj);
    PyErr_SetString(PyExc_TypeError, "W must be a BsrMatrix");
    return nullptr;
}

PyObject* failed(bsr_status st, const char* where)
{
    PyObject* e = PyObject_CallFunction(g_error, "is", (int)st, where);
    if (e) { PyErr_SetObject(reinterpret_cast<PyObject*>(Py_TYPE(e)), e); Py_DECREF(e); }
    return nullptr;
}

// Scratch the product with m rows wants and the handle has not been lent: W.ensure_scratch(m), in Python.
bool ensure_scratch(PyObject* W, const core_object* c, int64_t m)
{
    size_t need = 0;
    const bsr_status st = g_scratch_size(c->handle, m, &need);
    if (st != BSR_OK) { failed(st, "bsr_scratch_size"); return false; }
    if (need <= c->scratch_bytes) return true;
    PyObject* r = PyObject_CallMethod(W, "ensure_scratch", "L", (long long)m);
    Py_XDECREF(r);
    return r != nullptr;
}

void* stream() { return c10::hip::getCurrentHIPStream().stream(); }

// A call on another stream than the one before it (`known`; to begin with the one on which the owner's buffers -- plan, moments --
// were made): the owner has the allocator told, once a stream (its _on_stream), or that would give them away, as soon as the
// owner is dropped, to what their own stream is given next, while this call is still to read its tables.  False with an error set.
bool told_of_stream(PyObject* owner, uintptr_t known, uintptr_t* now_known = nullptr)
{
    const uintptr_t now = reinterpret_cast<uintptr_t>(stream());
    if (now == known) return true;
    PyObject* done = PyObject_CallMethod(owner, "_on_stream", "K", (unsigned long long)now);
    if (!done) return false;
    Py_DECREF(done);
    if (now_known) *now_known = now;
    return true;
}

// A result: through torch's dispatcher, so that its modes and its deterministic fill see it.
at::Tensor result(at::IntArrayRef shape, int code, const at::Tensor& like)
{
    return at::empty(shape, at::TensorOptions().dtype(kTypes[code]).device(like.device()));
}

bool dims2(const at::Tensor& t, int64_t rows, int64_t cols)
{
    return t.dim() == 2 && t.size(0) == rows && t.size(1) == cols;
}

// spmm(W, core, X, Y or None, y_dtype or None, path) -> Y
PyObject* spmm(PyObject*, PyObject* const* a, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    if (nargs != 6) return value_error("spmm takes 6 arguments");
    core_object* c = core_of(a[1]);
    const at::Tensor *X = nullptr, *Y = nullptr;
    if (!c || !tensor_of(a[2], "X", &X)) return nullptr;
    if (X->dim() != 2 || X->size(1) != c->k) return value_error("X must be (m, k)");
    const int x_code = type_code(*X, a[2]);
    if (x_code < 0) return nullptr;
    if (x_code != c->dtype || !X->is_contiguous()) return value_error("X must be contiguous and of W's dtype");
    const int64_t m = X->size(0);
    const int y_code = name_code(a[4], c->dtype);
    if (y_code < 0 || !ensure_scratch(a[0], c, m)) return nullptr;
    const long path = PyLong_AsLong(a[5]);
    if ((path == -1 && PyErr_Occurred()) || !told_of_stream(a[0], c->known, &c->known)) return nullptr;
    at::Tensor fresh;
    PyObject* out = a[3];
    if (out == Py_None) {
        fresh = result({m, c->n}, y_code, *X);
        Y = &fresh;
    } else {
        if (!tensor_of(out, "Y", &Y)) return nullptr;
        if (!dims2(*Y, m, c->n) || !Y->is_contiguous() || Y->scalar_type() != kTypes[y_code])
            return value_error("Y must be a contiguous (m, n) tensor of y_dtype");
    }
    const void* xp = X->data_ptr();
    void* yp = Y->data_ptr();
    bsr_status st;
    {
        pybind11::gil_scoped_release no_gil;
        st = g_spmm(c->handle, m, xp, yp, (bsr_dtype)y_code, (bsr_path)path, stream());
    }
    if (st != BSR_OK) return failed(st, "bsr_spmm");
    if (out == Py_None) return THPVariable_Wrap(std::move(fresh));
    Py_INCREF(out);
    return out;
    END_HANDLE_TH_ERRORS
}

// spmm_static(W, core, X, Y) -> Y
PyObject* spmm_static(PyObject*, PyObject* const* a, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    if (nargs != 4) return value_error("spmm_static takes 4 arguments");
    core_object* c = core_of(a[1]);
    const at::Tensor *X = nullptr, *Y = nullptr;
    if (!c || !tensor_of(a[2], "X", &X) || !tensor_of(a[3], "Y", &Y)) return nullptr;
    const int x_code = type_code(*X, a[2]);
    if (x_code < 0) return nullptr;
    if (X->dim() != 2 || X->size(1) != c->k || x_code != c->dtype || !X->is_contiguous())
        return value_error("X must be a contiguous (m, k) tensor of W's dtype");
    const int64_t m = X->size(0);
    if (!dims2(*Y, m, c->n) || Y->scalar_type() != at::kFloat || !Y->is_contiguous())
        return value_error("Y must be a contiguous (m, n) fp32 tensor");
    if (!told_of_stream(a[0], c->known, &c->known)) return nullptr;
    const void* xp = X->data_ptr();
    void* yp = Y->data_ptr();
    bsr_status st;
    {
        pybind11::gil_scoped_release no_gil;
        st = g_spmm_static(c->handle, m, xp, yp, BSR_F32, stream());
    }
    if (st != BSR_OK) return failed(st, "bsr_spmm_static");
    Py_INCREF(a[3]);
    return a[3];
    END_HANDLE_TH_ERRORS
}

// sddmm(W, core, G, X, D or None, d_dtype or None, lend_scratch) -> D
PyObject* sddmm(PyObject*, PyObject* const* a, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    if (nargs != 7) return value_error("sddmm takes 7 arguments");
    core_object* c = core_of(a[1]);
    const at::Tensor *G = nullptr, *X = nullptr, *D = nullptr;
    if (!c || !tensor_of(a[2], "G", &G) || !tensor_of(a[3], "X", &X)) return nullptr;
    if (G->dim() != 2 || X->dim() != 2 || G->size(0) != X->size(0) || G->size(1) != c->n || X->size(1) != c->k)
        return value_error("G must be (m, n) and X (m, k)");
    const int g_code = type_code(*G, a[2]);
    if (g_code < 0) return nullptr;
    const int x_code = type_code(*X, a[3]);
    if (x_code < 0) return nullptr;
    if (g_code != c->dtype || x_code != c->dtype || !G->is_contiguous() || !X->is_contiguous())
        return value_error("G and X must be contiguous and of W's dtype");
    const int64_t m = G->size(0);
    const int d_code = name_code(a[5], c->dtype);
    if (d_code < 0) return nullptr;
    const int lend = PyObject_IsTrue(a[6]);
    if (lend < 0 || (lend && !ensure_scratch(a[0], c, m)) || !told_of_stream(a[0], c->known, &c->known)) return nullptr;
    at::Tensor fresh;
    PyObject* out = a[4];
    if (out == Py_None) {
        fresh = result({c->nnzb, c->bs_r, c->bs_c}, d_code, *G);
        D = &fresh;
    } else {
        if (!tensor_of(out, "D", &D)) return nullptr;
        if (D->dim() != 3 || D->size(0) != c->nnzb || D->size(1) != c->bs_r || D->size(2) != c->bs_c ||
            D->scalar_type() != kTypes[d_code] || !D->is_contiguous())
            return value_error("D must be a contiguous (nnzb, bs_r, bs_c) tensor of d_dtype");
    }
    const void *gp = G->data_ptr(), *xp = X->data_ptr();
    void* dp = D->data_ptr();
    // This call's workspace: from torch's allocator, which hands it on in stream order once the call has returned.  The
    // product runs without it too: a caller that lends nothing gets nothing allocated, and memory that is not there is
    // no error.
    size_t ws_bytes = 0;
    at::Tensor ws;
    if (lend) {
        pybind11::gil_scoped_release no_gil;          // the first one of a pattern builds the product's plan: milliseconds
        if (g_sddmm_workspace(c->handle, m, &ws_bytes) != BSR_OK) ws_bytes = 0;
    }
    if (ws_bytes > 0) {
        try {
            ws = at::Tensor(at::detail::empty_cuda({(int64_t)ws_bytes}, at::kByte, G->device(), std::nullopt));
        } catch (const c10::OutOfMemoryError&) {
            ws_bytes = 0;
        }
    }
    bsr_status st;
    {
        pybind11::gil_scoped_release no_gil;
        st = g_sddmm(c->handle, m, gp, xp, dp, (bsr_dtype)d_code, ws_bytes ? ws.data_ptr() : nullptr, ws_bytes, stream());
    }
    if (st != BSR_OK) return failed(st, "bsr_sddmm");
    if (out == Py_None) return THPVariable_Wrap(std::move(fresh));
    Py_INCREF(out);
    return out;
    END_HANDLE_TH_ERRORS
}

// Code of an activation's name (None: none), -1 with KeyError(name).
int act_code(PyObject* name)
{
    static const char* const names[] = {"none", "relu", "gelu", "gelu_tanh", "silu"};
    if (name == Py_None) return BSR_ACT_NONE;
    if (PyUnicode_Check(name)) {
        const char* s = PyUnicode_AsUTF8(name);
        if (!s) return -1;
        for (int i = 0; i < 5; ++i)
            if (!strcmp(s, names[i])) return i;
    }
    PyErr_SetObject(PyExc_KeyError, name);
    return -1;
}

// Whether the kernels of this call may touch the tensor: they run on the current device's current stream, X's or G's, which
// is checked against the current device first (`device`: its number, else -1).
bool here(const at::Tensor& t, const char* what, int device = -1)
{
    if (t.is_cuda() && t.get_device() == (device < 0 ? (int)c10::hip::current_device() : device)) return true;
    PyErr_Format(PyExc_ValueError, "%s must be on the current GPU", what);
    return false;
}

// An optional contiguous (rows, cols) tensor of type `code` on `device`; false with an error set.
bool matrix_of(PyObject* obj, const char* what, int64_t rows, int64_t cols, int code, int device, const at::Tensor** out)
{
    *out = nullptr;
    if (obj == Py_None) return true;
    const at::Tensor* t = nullptr;
    if (!tensor_of(obj, what, &t)) return false;
    if (!dims2(*t, rows, cols) || !t->is_contiguous() || t->scalar_type() != kTypes[code]) {
        PyErr_Format(PyExc_ValueError, "%s must be a contiguous (%lld, %lld) tensor of the result's type", what, (long long)rows, (long long)cols);
        return false;
    }
    *out = t;
    return here(*t, what, device);
}

// spmm_epilogue(W, core, X, Y or None, y_dtype or None, bias or None, act or None, residual or None, through or None,
//               Z or None, keep_z) -> Y, or (Y, Z) where Z or keep_z is given
PyObject* spmm_epilogue(PyObject*, PyObject* const* a, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    if (nargs != 11) return value_error("spmm_epilogue takes 11 arguments");
    core_object* c = core_of(a[1]);
    const at::Tensor *X = nullptr, *Y = nullptr, *bias = nullptr, *residual = nullptr, *through = nullptr, *Z = nullptr;
    if (!c || !tensor_of(a[2], "X", &X)) return nullptr;
    if (X->dim() != 2 || X->size(1) != c->k) return value_error("X must be (m, k)");
    const int x_code = type_code(*X, a[2]);
    if (x_code < 0) return nullptr;
    if (x_code != c->dtype || !X->is_contiguous()) return value_error("X must be contiguous and of W's dtype");
    if (!here(*X, "X")) return nullptr;
    const int device = (int)X->get_device();
    const int64_t m = X->size(0);
    const int y_code = name_code(a[4], c->dtype);
    if (y_code < 0) return nullptr;
    bsr_epilogue ep{};
    const int act = act_code(a[6]);
    if (act < 0) return nullptr;
    ep.act = (bsr_act)act;
    if (a[5] != Py_None) {
        if (!tensor_of(a[5], "bias", &bias)) return nullptr;
        const int code = type_code(*bias, a[5]);
        if (code < 0) return nullptr;
        if (bias->dim() != 1 || bias->size(0) != c->n || !bias->is_contiguous() || (code != c->dtype && code != BSR_F32))
            return value_error("bias must be a contiguous (n,) tensor of W's dtype or fp32");
        if (!here(*bias, "bias", device)) return nullptr;
        ep.bias_dev = bias->data_ptr();
        ep.bias_dtype = (bsr_dtype)code;
    }
    if (a[7] != Py_None) {
        if (!tensor_of(a[7], "residual", &residual)) return nullptr;
        if (!dims2(*residual, m, c->n) || residual->scalar_type() != kTypes[y_code] ||
            (c->n > 1 && residual->stride(1) != 1) || (m > 1 && residual->stride(0) < c->n))
            return value_error("residual must be an (m, n) tensor of the result's type, its rows contiguous");
        if (!here(*residual, "residual", device)) return nullptr;
        ep.residual_dev = residual->data_ptr();
        ep.residual_ld = m > 1 ? residual->stride(0) : 0;
    }
    if (!matrix_of(a[8], "through", m, c->n, y_code, device, &through) || !matrix_of(a[9], "Z", m, c->n, y_code, device, &Z) ||
        !matrix_of(a[3], "Y", m, c->n, y_code, device, &Y)) return nullptr;
    if (through) ep.through_dev = through->data_ptr();
    const int keep_z = PyObject_IsTrue(a[10]);
    if (keep_z < 0 || !ensure_scratch(a[0], c, m) || !told_of_stream(a[0], c->known, &c->known)) return nullptr;
    at::Tensor fresh_y, fresh_z;
    if (!Y) {
        fresh_y = result({m, c->n}, y_code, *X);
        Y = &fresh_y;
    }
    if (!Z && keep_z) {
        fresh_z = result({m, c->n}, y_code, *X);
        Z = &fresh_z;
    }
    if (Z) ep.z_dev = Z->data_ptr();
    const void* xp = X->data_ptr();
    void* yp = Y->data_ptr();
    bsr_status st;
    {
        pybind11::gil_scoped_release no_gil;
        st = g_spmm_epilogue(c->handle, m, xp, yp, (bsr_dtype)y_code, &ep, stream());
    }
    if (st != BSR_OK) return failed(st, "bsr_spmm_epilogue");
    PyObject* y_obj = a[3];
    if (y_obj == Py_None) y_obj = THPVariable_Wrap(std::move(fresh_y));
    else Py_INCREF(y_obj);
    if (!Z || !y_obj) return y_obj;
    PyObject* z_obj = a[9];
    if (z_obj == Py_None) z_obj = THPVariable_Wrap(std::move(fresh_z));
    else Py_INCREF(z_obj);
    if (!z_obj) { Py_DECREF(y_obj); return nullptr; }
    PyObject* pair = PyTuple_Pack(2, y_obj, z_obj);
    Py_DECREF(y_obj);
    Py_DECREF(z_obj);
    return pair;
    END_HANDLE_TH_ERRORS
}

// epilogue_backward(G, Z or None, act or None, DZ or None, dz_dtype or None, DB or None, need_dz, need_db) -> (DZ or None, DB or None)
PyObject* epilogue_backward(PyObject*, PyObject* const* a, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    if (nargs != 8) return value_error("epilogue_backward takes 8 arguments");
    const at::Tensor *G = nullptr, *Z = nullptr, *DZ = nullptr, *DB = nullptr;
    if (!tensor_of(a[0], "G", &G)) return nullptr;
    const int g_code = type_code(*G, a[0]);
    if (g_code < 0) return nullptr;
    if (G->dim() != 2 || !G->is_contiguous()) return value_error("G must be a contiguous (m, n) tensor");
    if (!here(*G, "G")) return nullptr;
    const int device = (int)G->get_device();
    const int64_t m = G->size(0), n = G->size(1);
    const int act = act_code(a[2]);
    if (act < 0) return nullptr;
    if (!matrix_of(a[1], "Z", m, n, g_code, device, &Z)) return nullptr;
    if (!Z && act != BSR_ACT_NONE) return value_error("Z must be given unless act is none");
    const int dz_code = name_code(a[4], g_code);
    if (dz_code < 0) return nullptr;
    if (dz_code != g_code && g_code != BSR_F32) return value_error("dz_dtype must be G's type unless that is fp32");
    if (!matrix_of(a[3], "DZ", m, n, dz_code, device, &DZ)) return nullptr;
    if (a[5] != Py_None) {
        if (!tensor_of(a[5], "DB", &DB)) return nullptr;
        if (DB->dim() != 1 || DB->size(0) != n || !DB->is_contiguous() || DB->scalar_type() != at::kFloat)
            return value_error("DB must be a contiguous (n,) fp32 tensor");
        if (!here(*DB, "DB", device)) return nullptr;
    }
    const int need_dz = PyObject_IsTrue(a[6]), need_db = PyObject_IsTrue(a[7]);
    if (need_dz < 0 || need_db < 0) return nullptr;
    // without an activation dZ is G: nothing to compute unless its type changes or a buffer of its own is given
    const bool dz_is_g = !DZ && need_dz && act == BSR_ACT_NONE && dz_code == g_code;
    at::Tensor fresh_dz, fresh_db, ws;
    if (!DZ && need_dz && !dz_is_g) {
        fresh_dz = result({m, n}, dz_code, *G);
        DZ = &fresh_dz;
    }
    if (!DB && need_db) {
        fresh_db = result({n}, BSR_F32, *G);
        DB = &fresh_db;
    }
    if (DZ || DB) {
        size_t ws_bytes = 0;
        if (DB) {
            const bsr_status st = g_backward_workspace(m, n, &ws_bytes);
            if (st != BSR_OK) return failed(st, "bsr_epilogue_backward_workspace_size");
            if (ws_bytes) ws = at::Tensor(at::detail::empty_cuda({(int64_t)ws_bytes}, at::kByte, G->device(), std::nullopt));
        }
        bsr_status st;
        {
            pybind11::gil_scoped_release no_gil;
            st = g_backward(m, n, (bsr_act)act, (bsr_dtype)g_code, G->data_ptr(), Z ? Z->data_ptr() : nullptr, (bsr_dtype)dz_code,
                            DZ ? DZ->data_ptr() : nullptr, DB ? DB->data_ptr<float>() : nullptr, ws_bytes ? ws.data_ptr() : nullptr,
                            ws_bytes, stream());
        }
        if (st != BSR_OK) return failed(st, "bsr_epilogue_backward");
    }
    auto object = [](PyObject* given, at::Tensor& fresh) -> PyObject* {
        if (given == Py_None && fresh.defined()) return THPVariable_Wrap(std::move(fresh));
        Py_INCREF(given);
        return given;
    };
    PyObject* dz_obj = dz_is_g ? object(a[0], fresh_dz) : object(a[3], fresh_dz);
    if (!dz_obj) return nullptr;
    PyObject* db_obj = object(a[5], fresh_db);
    if (!db_obj) { Py_DECREF(dz_obj); return nullptr; }
    PyObject* pair = PyTuple_Pack(2, dz_obj, db_obj);
    Py_DECREF(dz_obj);
    Py_DECREF(db_obj);
    return pair;
    END_HANDLE_TH_ERRORS
}

// Memory for one call, from torch's allocator, which hands it on in stream order once the call has returned.
at::Tensor call_workspace(size_t bytes, const at::Tensor& like)
{
    return at::Tensor(at::detail::empty_cuda({(int64_t)bytes}, at::kByte, like.device(), std::nullopt));
}

// The object of a result: the one that was given, else the new tensor (None where there is neither).
PyObject* result_object(PyObject* given, at::Tensor& fresh)
{
    if (given == Py_None && fresh.defined()) return THPVariable_Wrap(std::move(fresh));
    Py_INCREF(given);
    return given;
}
PyObject* pair_of(PyObject* first, PyObject* second)  // takes both references
{
    PyObject* pair = first && second ? PyTuple_Pack(2, first, second) : nullptr;
    Py_XDECREF(first);
    Py_XDECREF(second);
    return pair;
}

// spmm_gated(W, core, X, H or None, h_dtype or None, bias or None, act or None, Z or None, keep_z) -> H, or (H, Z) where Z or
// keep_z is given
PyObject* spmm_gated(PyObject*, PyObject* const* a, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    if (nargs != 9) return value_error("spmm_gated takes 9 arguments");
    core_object* c = core_of(a[1]);
    const at::Tensor *X = nullptr, *H = nullptr, *bias = nullptr, *Z = nullptr;
    if (!c || !tensor_of(a[2], "X", &X)) return nullptr;
    if (X->dim() != 2 || X->size(1) != c->k) return value_error("X must be (m, k)");
    const int x_code = type_code(*X, a[2]);
    if (x_code < 0) return nullptr;
    if (x_code != c->dtype || !X->is_contiguous()) return value_error("X must be contiguous and of W's dtype");
    if (!here(*X, "X")) return nullptr;
    if (c->bs_r <= 0 || (c->n / c->bs_r) % 2 != 0) return value_error("W must hold a gate's and another matrix's block-rows in turn");
    const int device = (int)X->get_device();
    const int64_t m = X->size(0), n = c->n / 2;
    const int h_code = name_code(a[4], c->dtype);
    if (h_code < 0) return nullptr;
    bsr_gated how{};
    const int act = act_code(a[6]);
    if (act < 0) return nullptr;
    how.act = (bsr_act)act;
    if (a[5] != Py_None) {
        if (!tensor_of(a[5], "bias", &bias)) return nullptr;
        const int code = type_code(*bias, a[5]);
        if (code < 0) return nullptr;
        if (bias->dim() != 1 || bias->size(0) != c->n || !bias->is_contiguous() || (code != c->dtype && code != BSR_F32))
            return value_error("bias must be a contiguous (2n,) tensor of W's dtype or fp32");
        if (!here(*bias, "bias", device)) return nullptr;
        how.bias_dev = bias->data_ptr();
        how.bias_dtype = (bsr_dtype)code;
    }
    if (!matrix_of(a[7], "Z", m, c->n, h_code, device, &Z) || !matrix_of(a[3], "H", m, n, h_code, device, &H)) return nullptr;
    const int keep_z = PyObject_IsTrue(a[8]);
    if (keep_z < 0 || !ensure_scratch(a[0], c, m) || !told_of_stream(a[0], c->known, &c->known)) return nullptr;
    at::Tensor fresh_h, fresh_z, ws;
    if (!H) {
        fresh_h = result({m, n}, h_code, *X);
        H = &fresh_h;
    }
    if (!Z && keep_z) {
        fresh_z = result({m, c->n}, h_code, *X);
        Z = &fresh_z;
    }
    if (Z) how.z_dev = Z->data_ptr();
    size_t ws_bytes = 0;
    if (!Z || h_code != BSR_F32) {                    // (fp32 sums that are kept are their own workspace)
        const bsr_status st = g_gated_workspace(c->handle, m, (bsr_dtype)h_code, &ws_bytes);
        if (st != BSR_OK) return failed(st, "bsr_spmm_gated_workspace_size");
        if (ws_bytes) ws = call_workspace(ws_bytes, *X);
    }
    const void* xp = X->data_ptr();
    void* hp = H->data_ptr();
    bsr_status st;
    {
        pybind11::gil_scoped_release no_gil;
        st = g_spmm_gated(c->handle, m, xp, hp, (bsr_dtype)h_code, &how, ws_bytes ? ws.data_ptr() : nullptr, ws_bytes, stream());
    }
    if (st != BSR_OK) return failed(st, "bsr_spmm_gated");
    PyObject* h_obj = result_object(a[3], fresh_h);
    return Z ? pair_of(h_obj, result_object(a[7], fresh_z)) : h_obj;
    END_HANDLE_TH_ERRORS
}

// An optional contiguous (n,) tensor of fp32 for sums.
bool sums_of(PyObject* obj, const char* what, int64_t n, int device, const at::Tensor** out)
{
    *out = nullptr;
    if (obj == Py_None) return true;
    const at::Tensor* t = nullptr;
    if (!tensor_of(obj, what, &t)) return false;
    if (t->dim() != 1 || t->size(0) != n || !t->is_contiguous() || t->scalar_type() != at::kFloat) {
        PyErr_Format(PyExc_ValueError, "%s must be a contiguous (%lld,) fp32 tensor", what, (long long)n);
        return false;
    }
    *out = t;
    return here(*t, what, device);
}

// gated_backward(G, Z, unit, act or None, DZ or None, dz_dtype or None, DB or None, need_dz, need_db) -> (DZ or None, DB or None)
PyObject* gated_backward(PyObject*, PyObject* const* a, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    if (nargs != 9) return value_error("gated_backward takes 9 arguments");
    const at::Tensor *G = nullptr, *Z = nullptr, *DZ = nullptr, *DB = nullptr;
    if (!tensor_of(a[0], "G", &G) || !tensor_of(a[1], "Z", &Z)) return nullptr;
    const int g_code = type_code(*G, a[0]);
    if (g_code < 0) return nullptr;
    if (G->dim() != 2 || !G->is_contiguous()) return value_error("G must be a contiguous (m, n) tensor");
    if (!here(*G, "G")) return nullptr;
    const int device = (int)G->get_device();
    const int64_t m = G->size(0), n = G->size(1);
    const long long unit = PyLong_AsLongLong(a[2]);
    if (unit == -1 && PyErr_Occurred()) return nullptr;
    if (unit < 1 || unit > INT32_MAX || n % unit != 0) return value_error("bs_r must divide G's columns");
    const int act = act_code(a[3]);
    if (act < 0 || !matrix_of(a[1], "Z", m, 2 * n, g_code, device, &Z)) return nullptr;
    const int dz_code = name_code(a[5], g_code);
    if (dz_code < 0) return nullptr;
    if (dz_code != g_code && g_code != BSR_F32) return value_error("dz_dtype must be G's type unless that is fp32");
    if (!matrix_of(a[4], "DZ", m, 2 * n, dz_code, device, &DZ) || !sums_of(a[6], "DB", 2 * n, device, &DB)) return nullptr;
    const int need_dz = PyObject_IsTrue(a[7]), need_db = PyObject_IsTrue(a[8]);
    if (need_dz < 0 || need_db < 0) return nullptr;
    at::Tensor fresh_dz, fresh_db, ws;
    if (!DZ && need_dz) {
        fresh_dz = result({m, 2 * n}, dz_code, *G);
        DZ = &fresh_dz;
    }
    if (!DB && need_db) {
        fresh_db = result({2 * n}, BSR_F32, *G);
        DB = &fresh_db;
    }
    if (DZ || DB) {
        size_t ws_bytes = 0;
        if (DB) {
            const bsr_status st = g_gated_backward_workspace(m, n, (int32_t)unit, &ws_bytes);
            if (st != BSR_OK) return failed(st, "bsr_gated_backward_workspace_size");
            if (ws_bytes) ws = call_workspace(ws_bytes, *G);
        }
        bsr_status st;
        {
            pybind11::gil_scoped_release no_gil;
            st = g_gated_backward(m, n, (int32_t)unit, (bsr_act)act, (bsr_dtype)g_code, G->data_ptr(), Z->data_ptr(), (bsr_dtype)dz_code,
                                  DZ ? DZ->data_ptr() : nullptr, DB ? DB->data_ptr<float>() : nullptr, ws_bytes ? ws.data_ptr() : nullptr, ws_bytes,
                                  stream());
        }
        if (st != BSR_OK) return failed(st, "bsr_gated_backward");
    }
    return pair_of(result_object(a[4], fresh_dz), result_object(a[6], fresh_db));
    END_HANDLE_TH_ERRORS
}

// Code of a norm's name (None: none), -1 with KeyError(name).
int norm_code(PyObject* name)
{
    if (name == Py_None) return BSR_NORM_NONE;
    if (PyUnicode_Check(name)) {
        const char* s = PyUnicode_AsUTF8(name);
        if (!s) return -1;
        if (!strcmp(s, "none")) return BSR_NORM_NONE;
        if (!strcmp(s, "rms")) return BSR_NORM_RMS;
        if (!strcmp(s, "layer")) return BSR_NORM_LAYER;
    }
    PyErr_SetObject(PyExc_KeyError, name);
    return -1;
}

const char* const kVectors[5] = {"post_weight", "post_bias", "gate", "pre_weight", "pre_bias"};

// The settings a[0 .. 9] = post, pre, the five vectors or None, eps, stream_scale, branch_scale; n columns, B's type `code`.
bool norm_settings(PyObject* const* a, int64_t n, int code, int device, bsr_residual* how, const at::Tensor* (&vec)[5])
{
    const int post = norm_code(a[0]);
    const int pre = post < 0 ? -1 : norm_code(a[1]);
    if (pre < 0) return false;
    how->post = (bsr_norm)post;
    how->pre = (bsr_norm)pre;
    how->w_dtype = (bsr_dtype)code;
    const void* at[5] = {};
    int type = -1;
    for (int i = 0; i < 5; ++i) {
        vec[i] = nullptr;
        if (a[2 + i] == Py_None) continue;
        if (!tensor_of(a[2 + i], kVectors[i], &vec[i])) return false;
        const int c = type_code(*vec[i], a[2 + i]);
        if (c < 0) return false;
        if (vec[i]->dim() != 1 || vec[i]->size(0) != n || !vec[i]->is_contiguous() || (c != code && c != BSR_F32) || (type >= 0 && c != type)) {
            PyErr_Format(PyExc_ValueError, "%s must be a contiguous (%lld,) tensor of B's dtype or fp32, all vectors of one type", kVectors[i], (long long)n);
            return false;
        }
        if (!here(*vec[i], kVectors[i], device)) return false;
        type = c;
        at[i] = vec[i]->data_ptr();
    }
    if (type >= 0) how->w_dtype = (bsr_dtype)type;
    how->post_weight_dev = at[0];
    how->post_bias_dev = at[1];
    how->gate_dev = at[2];
    how->pre_weight_dev = at[3];
    how->pre_bias_dev = at[4];
    how->eps = PyFloat_AsDouble(a[7]);
    how->stream_scale = (float)PyFloat_AsDouble(a[8]);
    how->branch_scale = (float)PyFloat_AsDouble(a[9]);
    return !PyErr_Occurred();
}

// residual_norm(S, B or None, 10 settings, out or None, U or None, u_dtype or None, need_sum) -> (S' or None, U or None)
PyObject* residual_norm(PyObject*, PyObject* const* a, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    if (nargs != 16) return value_error("residual_norm takes 16 arguments");
    const at::Tensor *S = nullptr, *B = nullptr, *out = nullptr, *U = nullptr, *vec[5];
    if (!tensor_of(a[0], "S", &S)) return nullptr;
    const int s_code = type_code(*S, a[0]);
    if (s_code < 0) return nullptr;
    if (S->dim() != 2 || !S->is_contiguous()) return value_error("S must be a contiguous (m, n) tensor");
    if (!here(*S, "S")) return nullptr;
    const int device = (int)S->get_device();
    const int64_t m = S->size(0), n = S->size(1);
    int b_code = s_code;
    if (a[1] != Py_None) {
        if (!tensor_of(a[1], "B", &B) || (b_code = type_code(*B, a[1])) < 0) return nullptr;
        if (a[14] != Py_None && name_code(a[14], -1) != b_code) return PyErr_Occurred() ? nullptr : value_error("u_dtype must be B's type");
    } else if ((b_code = name_code(a[14], s_code)) < 0) {
        return nullptr;
    }
    if (s_code != b_code && s_code != BSR_F32) return value_error("S must be of B's type or fp32");
    bsr_residual how{};
    if (!matrix_of(a[1], "B", m, n, b_code, device, &B) || !norm_settings(a + 2, n, b_code, device, &how, vec) ||
        !matrix_of(a[12], "out", m, n, s_code, device, &out) || !matrix_of(a[13], "U", m, n, b_code, device, &U)) return nullptr;
    if (U && how.pre == BSR_NORM_NONE) return value_error("U is pre's result: pre must be rms or layer");
    const int need_sum = PyObject_IsTrue(a[15]);
    if (need_sum < 0) return nullptr;
    at::Tensor fresh_s, fresh_u;
    // without a branch and a scale S' is S: nothing to compute unless a buffer of its own is given
    const bool sum_is_s = !out && !B && need_sum && how.stream_scale == 1.f;
    if (!out && need_sum && !sum_is_s) {
        fresh_s = result({m, n}, s_code, *S);
        out = &fresh_s;
    }
    if (!U && how.pre != BSR_NORM_NONE) {
        fresh_u = result({m, n}, b_code, *S);
        U = &fresh_u;
    }
    if (out || U) {
        bsr_status st;
        {
            pybind11::gil_scoped_release no_gil;
            st = g_norm(m, n, (bsr_dtype)s_code, S->data_ptr(), (bsr_dtype)b_code, B ? B->data_ptr() : nullptr, out ? out->data_ptr() : nullptr,
                        U ? U->data_ptr() : nullptr, &how, stream());
        }
        if (st != BSR_OK) return failed(st, "bsr_residual_norm");
    }
    return pair_of(result_object(sum_is_s ? a[0] : a[12], fresh_s), result_object(a[13], fresh_u));
    END_HANDLE_TH_ERRORS
}

// residual_norm_backward(S or None, B or None, GS or None, GU or None, 10 settings, DS or None, DB or None, need_ds, need_db,
//                        list of five: a buffer, None or True (a new one)) -> (DS or None, DB or None, list of five)
PyObject* residual_norm_backward(PyObject*, PyObject* const* a, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    if (nargs != 19 || !PyList_Check(a[18]) || PyList_GET_SIZE(a[18]) != 5) return value_error("residual_norm_backward takes 18 arguments and a list of 5");
    const at::Tensor *given[4] = {}, *DS = nullptr, *DB = nullptr, *vec[5];   // S, B, GS, GU
    const char* const names[4] = {"S", "B", "GS", "GU"};
    int code[4] = {-1, -1, -1, -1};
    const at::Tensor* like = nullptr;
    for (int i = 0; i < 4; ++i) {
        if (a[i] == Py_None) continue;
        if (!tensor_of(a[i], names[i], &given[i]) || (code[i] = type_code(*given[i], a[i])) < 0) return nullptr;
        if (given[i]->dim() != 2) return value_error("S, B, GS and GU must be (m, n)");
        if (!like) like = given[i];
    }
    if (!like) return value_error("none of S, B, GS and GU is given");
    if (!here(*like, "S, B, GS or GU")) return nullptr;
    const int device = (int)like->get_device();
    const int64_t m = like->size(0), n = like->size(1);
    int s_code = code[0] >= 0 ? code[0] : code[2], b_code = code[1] >= 0 ? code[1] : code[3];
    if (s_code < 0) s_code = b_code;
    if (b_code < 0) b_code = s_code;
    if (s_code != b_code && s_code != BSR_F32) return value_error("S must be of B's type or fp32");
    bsr_residual how{};
    for (int i = 0; i < 4; ++i)
        if (!matrix_of(a[i], names[i], m, n, i == 0 || i == 2 ? s_code : b_code, device, &given[i])) return nullptr;
    if (!norm_settings(a + 4, n, b_code, device, &how, vec) || !matrix_of(a[14], "DS", m, n, s_code, device, &DS) ||
        !matrix_of(a[15], "DB", m, n, b_code, device, &DB)) return nullptr;
    const at::Tensor *S = given[0], *B = given[1], *GS = given[2], *GU = given[3];
    if (!S && how.pre != BSR_NORM_NONE) return value_error("S must be given unless pre is none");
    if (GU && how.pre == BSR_NORM_NONE) return value_error("GU is the gradient of pre's result: pre must be rms or layer");
    const int need_ds = PyObject_IsTrue(a[16]), need_db = PyObject_IsTrue(a[17]);
    if (need_ds < 0 || need_db < 0) return nullptr;
    at::Tensor fresh_ds, fresh_db, fresh[5], ws;
    float* to[5] = {};
    bool sums = false;
    for (int i = 0; i < 5; ++i) {
        PyObject* obj = PyList_GET_ITEM(a[18], i);
        if (obj == Py_None) continue;
        const at::Tensor* t = nullptr;
        if (obj == Py_True) {
            fresh[i] = result({n}, BSR_F32, *like);
            t = &fresh[i];
        } else if (!sums_of(obj, kVectors[i], n, device, &t)) {
            return nullptr;
        }
        to[i] = t->data_ptr<float>();
        sums = true;
    }
    if (!DS && need_ds) {
        fresh_ds = result({m, n}, s_code, *like);
        DS = &fresh_ds;
    }
    if (!DB && need_db && B) {
        fresh_db = result({m, n}, b_code, *like);
        DB = &fresh_db;
    }
    if (DS || DB || sums) {
        size_t ws_bytes = 0;
        const bsr_status size = g_norm_backward_workspace(m, n, &ws_bytes);
        if (size != BSR_OK) return failed(size, "bsr_residual_norm_backward_workspace_size");
        if (!sums && n <= 8192) ws_bytes = 0;
        if (ws_bytes) ws = call_workspace(ws_bytes, *like);
        const bsr_residual_grads grads{to[0], to[1], to[2], to[3], to[4]};
        auto at = [](const at::Tensor* t) { return t ? t->data_ptr() : nullptr; };
        bsr_status st;
        {
            pybind11::gil_scoped_release no_gil;
            st = g_norm_backward(m, n, (bsr_dtype)s_code, at(S), (bsr_dtype)b_code, at(B), at(GS), at(GU), at(DS), at(DB), &how, &grads,
                                 ws_bytes ? ws.data_ptr() : nullptr, ws_bytes, stream());
        }
        if (st != BSR_OK) return failed(st, "bsr_residual_norm_backward");
    }
    PyObject* list = PyList_New(5);
    if (!list) return nullptr;
    for (int i = 0; i < 5; ++i) {
        PyObject* obj = PyList_GET_ITEM(a[18], i);
        PyObject* mine = result_object(obj == Py_True ? Py_None : obj, fresh[i]);
        if (!mine) { Py_DECREF(list); return nullptr; }
        PyList_SET_ITEM(list, i, mine);
    }
    PyObject* ds_obj = result_object(a[14], fresh_ds);
    PyObject* db_obj = result_object(a[15], fresh_db);
    PyObject* all = ds_obj && db_obj ? PyTuple_Pack(3, ds_obj, db_obj, list) : nullptr;
    Py_XDECREF(ds_obj);
    Py_XDECREF(db_obj);
    Py_DECREF(list);
    return all;
    END_HANDLE_TH_ERRORS
}

// A setting of a step: a number, or one element of `type` on `device`, whose address is taken.  False with an error set.
template <typename N, typename P>
bool setting(PyObject* obj, const char* what, at::ScalarType type, int device, N (*number)(PyObject*), N* value, const P** at_device)
{
    if (!THPVariable_Check(obj)) {
        *value = number(obj);
        return !PyErr_Occurred();
    }
    const at::Tensor& t = THPVariable_Unpack(obj);
    if (t.scalar_type() != type || t.numel() != 1 || !t.is_cuda() || t.get_device() != device) {
        PyErr_Format(PyExc_ValueError, "%s on the GPU must be one %s of the handle's device", what, type == at::kLong ? "int64" : "fp32");
        return false;
    }
    *at_device = static_cast<const P*>(t.data_ptr());
    return true;
}
long long integer(PyObject* o)                        // whatever int() takes
{
    PyObject* i = PyNumber_Long(o);
    if (!i) return -1;
    const long long v = PyLong_AsLongLong(i);
    Py_DECREF(i);
    return v;
}
double real(PyObject* o) { return PyFloat_AsDouble(o); }

// Of an optimizer's owner, as above; a call that the entry point refuses (closed, or not on its device) is not told of.
// (Its owner keeps the stream that it knows.)
bool told_of_stream(PyObject* owner, const void* opt, int device, PyObject* known)
{
    const unsigned long long address = PyLong_AsUnsignedLongLong(known);
    if (PyErr_Occurred()) return false;
    return !opt || (int)c10::hip::current_device() != device || told_of_stream(owner, (uintptr_t)address);
}

const bsr_adamw* adamw_of(PyObject* address)          // 0: closed, which the entry points refuse
{
    return reinterpret_cast<const bsr_adamw*>(PyLong_AsUnsignedLongLong(address));
}

// adamw_step(owner, handle's address, device, stream the owner knows, step, lr, beta1, beta2, eps, grad_scale, seed)
PyObject* adamw_step(PyObject*, PyObject* const* a, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    if (nargs != 11) return value_error("adamw_step takes 11 arguments");
    PyObject *owner = a[0], *known = a[3];
    const bsr_adamw* opt = adamw_of(a[1]);
    const int device = (int)PyLong_AsLong(a[2]);
    if (PyErr_Occurred()) return nullptr;
    a += 2;                                           // the settings' places below
    bsr_adamw_hyper h{};
    long long step = 1;
    double grad_scale = 1.0;
    if (!setting(a[2], "step", at::kLong, device, integer, &step, &h.step_dev) || !setting(a[3], "lr", at::kFloat, device, real, &h.lr, &h.lr_dev) ||
        !setting(a[7], "grad_scale", at::kFloat, device, real, &grad_scale, &h.grad_scale_dev)) return nullptr;
    h.step = step;
    h.grad_scale = (float)grad_scale;
    h.beta1 = real(a[4]);
    h.beta2 = real(a[5]);
    h.eps = real(a[6]);
    h.seed = (uint32_t)PyLong_AsUnsignedLongLongMask(a[8]);
    if (PyErr_Occurred() || !told_of_stream(owner, opt, device, known)) return nullptr;
    bsr_status st;
    {
        pybind11::gil_scoped_release no_gil;
        st = g_adamw_step(opt, &h, stream());
    }
    if (st != BSR_OK) return failed(st, "bsr_adamw_step");
    Py_RETURN_NONE;
    END_HANDLE_TH_ERRORS
}

// adamw_moments(owner, handle's address, device, stream the owner knows, tuple of the tensors' elements, list of pairs of tensors)
PyObject* adamw_moments(PyObject*, PyObject* const* a, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    if (nargs != 6 || !PyTuple_Check(a[4]) || !PyList_Check(a[5]))
        return value_error("adamw_moments takes an owner, an address, a device, a stream, a tuple and a list");
    PyObject *owner = a[0], *known = a[3];
    const bsr_adamw* opt = adamw_of(a[1]);
    const int device = (int)PyLong_AsLong(a[2]);
    if (PyErr_Occurred()) return nullptr;
    a += 2;
    const Py_ssize_t n = PyTuple_GET_SIZE(a[2]);
    if (PyList_GET_SIZE(a[3]) != n) return value_error("out: a pair of tensors a parameter");
    std::vector<void*> out[2];
    int code = -1;
    for (Py_ssize_t i = 0; i < n; ++i) {
        PyObject* pair = PyList_GET_ITEM(a[3], i);
        if (!(PyTuple_Check(pair) || PyList_Check(pair)) || PySequence_Fast_GET_SIZE(pair) != 2) return value_error("out: a pair of tensors a parameter");
        const long long count = PyLong_AsLongLong(PyTuple_GET_ITEM(a[2], i));
        for (int k = 0; k < 2; ++k) {
            const at::Tensor* t = nullptr;
            PyObject* obj = PySequence_Fast_GET_ITEM(pair, k);
            if (!tensor_of(obj, "out", &t)) return nullptr;
            if (code < 0 && (code = type_code(*t, obj)) < 0) return nullptr;
            if (t->scalar_type() != kTypes[code] || t->numel() != count || !t->is_contiguous() || !t->is_cuda() || t->get_device() != device) {
                PyErr_Format(PyExc_ValueError, "out[%lld]: contiguous tensors of one type, %lld elements each, on the handle's device", (long long)i, count);
                return nullptr;
            }
            out[k].push_back(t->data_ptr());
        }
    }
    if (!told_of_stream(owner, opt, device, known)) return nullptr;
    out[0].push_back(nullptr);                        // an address for an empty list
    out[1].push_back(nullptr);
    bsr_status st;
    {
        pybind11::gil_scoped_release no_gil;
        st = g_adamw_moments(opt, code < 0 ? BSR_F32 : (bsr_dtype)code, out[0].data(), out[1].data(), stream());
    }
    if (st != BSR_OK) return failed(st, "bsr_adamw_moments");
    Py_RETURN_NONE;
    END_HANDLE_TH_ERRORS
}

// muon_step(owner, handle's address, device, stream the owner knows, step, lr, momentum, nesterov, ns_steps, a, b, c, eps, grad_scale, seed)
PyObject* muon_step(PyObject*, PyObject* const* a, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    if (nargs != 15) return value_error("muon_step takes 15 arguments");
    const bsr_muon* opt = reinterpret_cast<const bsr_muon*>(PyLong_AsUnsignedLongLong(a[1]));   // 0: closed, which the entry point refuses
    const int device = (int)PyLong_AsLong(a[2]);
    if (PyErr_Occurred()) return nullptr;
    bsr_muon_hyper h{};
    long long step = 1;
    double grad_scale = 1.0;
    if (!setting(a[4], "step", at::kLong, device, integer, &step, &h.step_dev) || !setting(a[5], "lr", at::kFloat, device, real, &h.lr, &h.lr_dev) ||
        !setting(a[13], "grad_scale", at::kFloat, device, real, &grad_scale, &h.grad_scale_dev)) return nullptr;
    h.step = step;
    h.grad_scale = (float)grad_scale;
    h.momentum = real(a[6]);
    h.nesterov = PyObject_IsTrue(a[7]);
    const long long steps = integer(a[8]);
    h.ns_steps = steps < 0 || steps > INT32_MAX ? -1 : (int32_t)steps;
    h.a = (float)real(a[9]);
    h.b = (float)real(a[10]);
    h.c = (float)real(a[11]);
    h.eps = real(a[12]);
    h.seed = (uint32_t)PyLong_AsUnsignedLongLongMask(a[14]);
    if (PyErr_Occurred() || !told_of_stream(a[0], opt, device, a[3])) return nullptr;
    bsr_status st;
    {
        pybind11::gil_scoped_release no_gil;
        st = g_muon_step(opt, &h, stream());
    }
    if (st != BSR_OK) return failed(st, "bsr_muon_step");
    Py_RETURN_NONE;
    END_HANDLE_TH_ERRORS
}

// bind(address of bsr_spmm_ex, bsr_spmm_static, bsr_sddmm_ws, bsr_scratch_size, bsr_sddmm_workspace_size,
//      bsr_spmm_epilogue, bsr_epilogue_backward, bsr_epilogue_backward_workspace_size, bsr_adamw_step, bsr_adamw_moments, bsr_spmm_gated,
//      bsr_spmm_gated_workspace_size, bsr_gated_backward, bsr_gated_backward_workspace_size, bsr_residual_norm,
//      bsr_residual_norm_backward, bsr_residual_norm_backward_workspace_size, bsr_muon_step, BsrError)
PyObject* bind(PyObject*, PyObject* args)
{
    unsigned long long f[18];
    PyObject* error = nullptr;
    if (!PyArg_ParseTuple(args, "KKKKKKKKKKKKKKKKKKO", &f[0], &f[1], &f[2], &f[3], &f[4], &f[5], &f[6], &f[7], &f[8], &f[9], &f[10], &f[11], &f[12], &f[13],
                          &f[14], &f[15], &f[16], &f[17], &error)) return nullptr;
    g_spmm = reinterpret_cast<decltype(g_spmm)>(f[0]);
    g_spmm_static = reinterpret_cast<decltype(g_spmm_static)>(f[1]);
    g_sddmm = reinterpret_cast<decltype(g_sddmm)>(f[2]);
    g_scratch_size = reinterpret_cast<decltype(g_scratch_size)>(f[3]);
    g_sddmm_workspace = reinterpret_cast<decltype(g_sddmm_workspace)>(f[4]);
    g_spmm_epilogue = reinterpret_cast<decltype(g_spmm_epilogue)>(f[5]);
    g_backward = reinterpret_cast<decltype(g_backward)>(f[6]);
    g_backward_workspace = reinterpret_cast<decltype(g_backward_workspace)>(f[7]);
    g_adamw_step = reinterpret_cast<decltype(g_adamw_step)>(f[8]);
    g_adamw_moments = reinterpret_cast<decltype(g_adamw_moments)>(f[9]);
    g_spmm_gated = reinterpret_cast<decltype(g_spmm_gated)>(f[10]);
    g_gated_workspace = reinterpret_cast<decltype(g_gated_workspace)>(f[11]);
    g_gated_backward = reinterpret_cast<decltype(g_gated_backward)>(f[12]);
    g_gated_backward_workspace = reinterpret_cast<decltype(g_gated_backward_workspace)>(f[13]);
    g_norm = reinterpret_cast<decltype(g_norm)>(f[14]);
    g_norm_backward = reinterpret_cast<decltype(g_norm_backward)>(f[15]);
    g_norm_backward_workspace = reinterpret_cast<decltype(g_norm_backward_workspace)>(f[16]);
    g_muon_step = reinterpret_cast<decltype(g_muon_step)>(f[17]);
    Py_INCREF(error);
    Py_XDECREF(g_error);
    g_error = error;
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"bind", bind, METH_VARARGS, "Take the C library's entry points and the error class."},
    {"spmm", reinterpret_cast<PyCFunction>(spmm), METH_FASTCALL, "spmm(W, core, X, Y, y_dtype, path) -> Y"},
    {"spmm_static", reinterpret_cast<PyCFunction>(spmm_static), METH_FASTCALL, "spmm_static(W, core, X, Y) -> Y"},
    {"sddmm", reinterpret_cast<PyCFunction>(sddmm), METH_FASTCALL, "sddmm(W, core, G, X, D, d_dtype, lend) -> D"},
    {"spmm_epilogue", reinterpret_cast<PyCFunction>(spmm_epilogue), METH_FASTCALL,
     "spmm_epilogue(W, core, X, Y, y_dtype, bias, act, residual, through, Z, keep_z) -> Y or (Y, Z)"},
    {"epilogue_backward", reinterpret_cast<PyCFunction>(epilogue_backward), METH_FASTCALL,
     "epilogue_backward(G, Z, act, DZ, dz_dtype, DB, need_dz, need_db) -> (DZ, DB)"},
    {"adamw_step", reinterpret_cast<PyCFunction>(adamw_step), METH_FASTCALL,
     "adamw_step(owner, handle, device, stream, step, lr, beta1, beta2, eps, grad_scale, seed)"},
    {"adamw_moments", reinterpret_cast<PyCFunction>(adamw_moments), METH_FASTCALL, "adamw_moments(owner, handle, device, stream, counts, out)"},
    {"spmm_gated", reinterpret_cast<PyCFunction>(spmm_gated), METH_FASTCALL,
     "spmm_gated(W, core, X, H, h_dtype, bias, act, Z, keep_z) -> H or (H, Z)"},
    {"gated_backward", reinterpret_cast<PyCFunction>(gated_backward), METH_FASTCALL,
     "gated_backward(G, Z, unit, act, DZ, dz_dtype, DB, need_dz, need_db) -> (DZ, DB)"},
    {"residual_norm", reinterpret_cast<PyCFunction>(residual_norm), METH_FASTCALL,
     "residual_norm(S, B, post, pre, post_weight, post_bias, gate, pre_weight, pre_bias, eps, stream_scale, branch_scale, out, U, u_dtype, need_sum)"
     " -> (S', U)"},
    {"residual_norm_backward", reinterpret_cast<PyCFunction>(residual_norm_backward), METH_FASTCALL,
     "residual_norm_backward(S, B, GS, GU, post, ..., branch_scale, DS, DB, need_ds, need_db, sums) -> (DS, DB, sums)"},
    {"muon_step", reinterpret_cast<PyCFunction>(muon_step), METH_FASTCALL,
     "muon_step(owner, handle, device, stream, step, lr, momentum, nesterov, ns_steps, a, b, c, eps, grad_scale, seed)"},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", "Native host path of the binding.", -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__binding()
{
    core_type.tp_name = "_binding.Core";
    core_type.tp_basicsize = sizeof(core_object);
    core_type.tp_flags = Py_TPFLAGS_DEFAULT;
    core_type.tp_new = PyType_GenericNew;
    core_type.tp_init = core_init;
    core_type.tp_methods = core_methods;
    if (PyType_Ready(&core_type) < 0) return nullptr;
    PyObject* m = PyModule_Create(&module);
    if (!m) return nullptr;
    Py_INCREF(&core_type);
    if (PyModule_AddObject(m, "Core", reinterpret_cast<PyObject*>(&core_type)) < 0) return nullptr;
    return m;
}
