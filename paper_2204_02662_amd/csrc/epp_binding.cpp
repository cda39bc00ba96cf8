// CPython entry points of the calls that a training loop makes on every layer of every pass: argument
// checks on the tensors' C++ objects, current stream, call of the C ABI (include/epp.h).
//
// On a small graph such a call is all host work: a kernel of 4 us, and 7.5 us to check five arguments,
// look up the stream and marshal the call from Python through ctypes.  Here the same steps take 1.5 us beside the
// launch itself.  Messages and exceptions are those of the module that imports this one (__init__.py).
//
// What PyTorch's C++ throws (a tensor of unknown shape, as tracing makes them, asked for its sizes) leaves
// every entry point as the Python exception it stands for: past a C function it would end the process.

#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <c10/core/impl/VirtualGuardImpl.h>
#include <c10/hip/HIPCachingAllocator.h>

#include <atomic>
#include <vector>

#include "epp.h"

namespace {

PyObject* g_error = nullptr;       // EppError(code, message)
PyObject* g_raw_stream = nullptr;  // torch._C._cuda_getCurrentRawStream(device index)
PyObject *s_handle, *s_cached_n, *s_n;

// Positional and keyword arguments of a call, in the order of `names`.
// (`required`: how many of them have to be given; the others are nullptr where they are not.  -1: all)
bool take_args(const char* fn, PyObject* const* args, Py_ssize_t n, PyObject* kw, const char* const* names, int count,
               PyObject** out, int required = -1) {
    for (int i = 0; i < count; ++i) out[i] = i < n ? args[i] : nullptr;
    if (n > count) {
        PyErr_Format(PyExc_TypeError, "%s() takes %d arguments (%zd given)", fn, count, n);
        return false;
    }
    const Py_ssize_t n_kw = kw ? PyTuple_GET_SIZE(kw) : 0;
    for (Py_ssize_t j = 0; j < n_kw; ++j) {
        PyObject* key = PyTuple_GET_ITEM(kw, j);
        int i = 0;
        while (i < count && PyUnicode_CompareWithASCIIString(key, names[i]) != 0) ++i;
        if (i == count || out[i]) {
            PyErr_Format(PyExc_TypeError, "%s() got an unexpected or repeated argument '%U'", fn, key);
            return false;
        }
        out[i] = args[n + j];
    }
    for (int i = 0; i < (required < 0 ? count : required); ++i) {
        if (!out[i]) {
            PyErr_Format(PyExc_TypeError, "%s() misses the argument '%s'", fn, names[i]);
            return false;
        }
    }
    return true;
}

// Library handle of a path or of all paths.
void* handle_of(PyObject* o) {
    PyObject* h = PyObject_GetAttr(o, s_handle);
    if (!h) return nullptr;
    void* p = h == Py_None ? nullptr : PyLong_AsVoidPtr(h);
    Py_DECREF(h);
    if (!p && !PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "the handle has been released");
    return p;
}

// Vertices of its graph (cached by the object), -1 on an error.
int64_t vertices_of(PyObject* o) {
    PyObject* n = PyObject_GetAttr(o, s_cached_n);
    if (n && n == Py_None) {
        Py_DECREF(n);
        n = PyObject_GetAttr(o, s_n);
    }
    if (!n) return -1;
    const int64_t v = PyLong_AsLongLong(n);
    Py_DECREF(n);
    return v;
}

const at::Tensor* bad_tensor(const at::Tensor& t, const char* dtype) {
    const std::string got = std::string(c10::toString(t.scalar_type())), on = t.device().str();
    PyErr_Format(PyExc_ValueError, "expected a contiguous CUDA tensor of %s, got %s on %s", dtype, got.c_str(), on.c_str());
    return nullptr;
}

const at::Tensor* float_tensor(PyObject* o) {
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "expected a tensor, got %s", Py_TYPE(o)->tp_name);
        return nullptr;
    }
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.scalar_type() != at::kFloat || !t.is_contiguous()) return bad_tensor(t, "torch.float32");
    return &t;
}

const at::Tensor* matrix(PyObject* o, const char* what) {
    const at::Tensor* t = float_tensor(o);
    if (t && t->dim() != 2) {
        PyErr_Format(PyExc_ValueError, "%s must be a matrix", what);
        return nullptr;
    }
    return t;
}

// The current stream of the current device; false on an error.
bool current_stream(void** stream) {
    static const c10::impl::DeviceGuardImplInterface* const guard = c10::impl::getDeviceGuardImpl(c10::DeviceType::CUDA);
    PyObject* dev = PyLong_FromLong(guard->getDevice().index());
    if (!dev) return false;
    PyObject* raw = PyObject_CallOneArg(g_raw_stream, dev);
    Py_DECREF(dev);
    if (!raw) return false;
    *stream = PyLong_AsVoidPtr(raw);
    Py_DECREF(raw);
    return !PyErr_Occurred();
}

PyObject* finish(int rc) {
    if (rc >= 0) Py_RETURN_NONE;
    PyObject* e = PyObject_CallFunction(g_error, "is", rc, epp_last_error());
    if (e) {
        PyErr_SetObject(g_error, e);
        Py_DECREF(e);
    }
    return nullptr;
}

int32_t width(const at::Tensor& t, int d) { return (int32_t)t.size(d); }

template <bool FULL>
PyObject* aggregate(PyObject*, PyObject* const* args, Py_ssize_t n, PyObject* kw) {
    static const char* const names[2][3] = {{"path", "grad_in", "grad_out"}, {"full", "grad_in", "grad_out"}};
    PyObject* a[3];
    if (!take_args(FULL ? "epp_full_aggregate" : "epp_backward_aggregate", args, n, kw, names[FULL], 3, a)) return nullptr;
    const at::Tensor *in = float_tensor(a[1]), *out = in ? float_tensor(a[2]) : nullptr;
    if (!out) return nullptr;
    if (in->dim() != 2 || in->sizes() != out->sizes()) {
        PyErr_SetString(PyExc_ValueError, "grad_in and grad_out must be n x F matrices of the same shape");
        return nullptr;
    }
    const int64_t vertices = vertices_of(a[0]);
    if (vertices < 0) return nullptr;
    if (in->size(0) != vertices) {  // the kernels index rows by vertex id: fewer rows would be read out of bounds
        PyErr_Format(PyExc_ValueError, "gradient matrices have %lld rows, the graph has %lld vertices",
                     (long long)in->size(0), (long long)vertices);
        return nullptr;
    }
    epp_path_t* path = static_cast<epp_path_t*>(handle_of(a[0]));
    void* s;
    if (!path || !current_stream(&s)) return nullptr;
    const float* src = in->const_data_ptr<float>();
    float* dst = out->mutable_data_ptr<float>();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = FULL ? epp_full_aggregate(path, src, dst, width(*in, 1), s) : epp_backward_aggregate(path, src, dst, width(*in, 1), s);
    Py_END_ALLOW_THREADS
    return finish(rc);
}

template <bool STATIC>
PyObject* weight_gradient(PyObject*, PyObject* const* args, Py_ssize_t n, PyObject* kw) {
    static const char* const names[] = {"paths", "k", "Y", "grad_X", "grad_W", "workspace"};
    PyObject* a[6];
    if (!take_args(STATIC ? "epp_weight_gradient_static" : "epp_weight_gradient", args, n, kw, names, STATIC ? 5 : 6, a))
        return nullptr;
    const at::Tensor* Y = matrix(a[2], "Y");
    const at::Tensor* G = Y ? matrix(a[3], "grad_X") : nullptr;
    const at::Tensor* W = G ? matrix(a[4], "grad_W") : nullptr;
    const int64_t vertices = W ? vertices_of(a[0]) : -1;
    if (vertices < 0) return nullptr;
    if (Y->size(0) != vertices || G->size(0) != vertices || W->size(0) != Y->size(1) || W->size(1) != G->size(1)) {
        PyErr_SetString(PyExc_ValueError, "shapes: Y n x F_in, grad_X n x F_out, grad_W F_in x F_out");
        return nullptr;
    }
    void* ws = nullptr;
    int64_t ws_bytes = 0;
    if (!STATIC) {
        if (!THPVariable_Check(a[5]) || !THPVariable_Unpack(a[5]).is_cuda() ||
            THPVariable_Unpack(a[5]).scalar_type() != at::kByte || !THPVariable_Unpack(a[5]).is_contiguous()) {
            PyErr_SetString(PyExc_ValueError, "workspace must be a contiguous CUDA uint8 tensor");
            return nullptr;
        }
        ws = THPVariable_Unpack(a[5]).mutable_data_ptr();
        ws_bytes = THPVariable_Unpack(a[5]).numel();
    }
    const int k = (int)PyLong_AsLong(a[1]);
    if (k == -1 && PyErr_Occurred()) return nullptr;
    epp_paths_t* paths = static_cast<epp_paths_t*>(handle_of(a[0]));
    void* s;
    if (!paths || !current_stream(&s)) return nullptr;
    const float *y = Y->const_data_ptr<float>(), *g = G->const_data_ptr<float>();
    float* w = W->mutable_data_ptr<float>();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = STATIC ? epp_weight_gradient_static(paths, k, y, width(*Y, 1), g, width(*G, 1), w, s)
                : epp_weight_gradient(paths, k, y, width(*Y, 1), g, width(*G, 1), w, ws, ws_bytes, s);
    Py_END_ALLOW_THREADS
    return finish(rc);
}

PyObject* input_gradient(PyObject*, PyObject* const* args, Py_ssize_t n, PyObject* kw) {
    static const char* const names[] = {"paths", "k", "grad_X", "W", "grad_Y"};
    PyObject* a[5];
    if (!take_args("epp_input_gradient", args, n, kw, names, 5, a)) return nullptr;
    const at::Tensor* G = matrix(a[2], "grad_X");
    const at::Tensor* W = G ? matrix(a[3], "W") : nullptr;
    const at::Tensor* Y = W ? matrix(a[4], "grad_Y") : nullptr;
    const int64_t vertices = Y ? vertices_of(a[0]) : -1;
    if (vertices < 0) return nullptr;
    if (G->size(0) != vertices || W->size(1) != G->size(1) || Y->size(0) != G->size(0) || Y->size(1) != W->size(0)) {
        PyErr_SetString(PyExc_ValueError, "shapes: grad_X n x F_out, W F_in x F_out, grad_Y n x F_in");
        return nullptr;
    }
    const int k = (int)PyLong_AsLong(a[1]);
    if (k == -1 && PyErr_Occurred()) return nullptr;
    epp_paths_t* paths = static_cast<epp_paths_t*>(handle_of(a[0]));
    void* s;
    if (!paths || !current_stream(&s)) return nullptr;
    const float *g = G->const_data_ptr<float>(), *w = W->const_data_ptr<float>();
    float* y = Y->mutable_data_ptr<float>();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = epp_input_gradient(paths, k, g, width(*G, 1), w, width(*W, 0), y, s);
    Py_END_ALLOW_THREADS
    return finish(rc);
}

// ---- rows that belong to groups, all gradients together: tensors of several types, rows with a stride, lists that may be missing

// The device that calls are made on.
c10::DeviceIndex current_device() {
    static const c10::impl::DeviceGuardImplInterface* const guard = c10::impl::getDeviceGuardImpl(c10::DeviceType::CUDA);
    return guard->getDevice().index();
}

// A tensor on the current device; its memory is what the kernels of the current stream use.  (any_sign: also one that stands for the
// negative of its memory)
const at::Tensor* device_tensor(PyObject* o, const char* what, bool any_sign = false) {
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "%s: expected a tensor, got %s", what, Py_TYPE(o)->tp_name);
        return nullptr;
    }
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.layout() != at::kStrided) {
        const std::string on = t.device().str();
        PyErr_Format(PyExc_ValueError, "%s: expected a dense CUDA tensor, got one on %s", what, on.c_str());
        return nullptr;
    }
    if (t.device().index() != current_device()) {
        const std::string on = t.device().str();
        PyErr_Format(PyExc_ValueError, "%s is on %s, the current device is cuda:%d", what, on.c_str(), (int)current_device());
        return nullptr;
    }
    if (t.is_neg() && !any_sign) {
        PyErr_Format(PyExc_ValueError, "%s is a view that stands for the negative of its memory (resolve_neg() gives a tensor that does not)", what);
        return nullptr;
    }
    return &t;
}

int element_type(const at::Tensor& t) {  // -1: none that the library has
    switch (t.scalar_type()) {
        case at::kFloat: return EPP_FLOAT32;
        case at::kBFloat16: return EPP_BFLOAT16;
        case at::kHalf: return EPP_FLOAT16;
        default: return -1;
    }
}

// float32, bfloat16 or float16, of `dims` dimensions (0: any).
const at::Tensor* numbers(PyObject* o, const char* what, int dims, int* type, bool any_sign = false) {
    const at::Tensor* t = device_tensor(o, what, any_sign);
    if (!t) return nullptr;
    *type = element_type(*t);
    if (*type < 0) {
        const std::string got = c10::toString(t->scalar_type());
        PyErr_Format(PyExc_ValueError, "%s: expected float32, bfloat16 or float16, got %s", what, got.c_str());
        return nullptr;
    }
    if (dims && t->dim() != dims) {
        PyErr_Format(PyExc_ValueError, "%s must have %d dimensions, has %d", what, dims, (int)t->dim());
        return nullptr;
    }
    return t;
}

// A contiguous vector of int32 (None or missing: no list); false on an error.
bool indexes(PyObject* o, const char* what, const int32_t** p, int64_t* n, bool may_miss) {
    *p = nullptr;
    *n = -1;
    if (may_miss && (!o || o == Py_None)) return true;
    const at::Tensor* t = device_tensor(o, what);
    if (!t) return false;
    if (t->scalar_type() != at::kInt || t->dim() != 1 || !t->is_contiguous()) {
        PyErr_Format(PyExc_ValueError, "%s must be a contiguous vector of int32", what);
        return false;
    }
    *n = t->numel();
    // (an empty tensor has no address, and is a list all the same)
    static const int32_t none = 0;
    *p = *n ? static_cast<const int32_t*>(t->const_data_ptr()) : &none;
    return true;
}

bool workspace_of(PyObject* o, void** p, int64_t* bytes) {
    const at::Tensor* t = device_tensor(o, "workspace");
    if (!t) return false;
    if (t->scalar_type() != at::kByte || !t->is_contiguous()) {
        PyErr_SetString(PyExc_ValueError, "workspace must be a contiguous CUDA uint8 tensor");
        return false;
    }
    *p = t->mutable_data_ptr();
    *bytes = t->numel();
    return true;
}

// A matrix, rows of consecutive elements with any distance from row to row.
const at::Tensor* rows_of(PyObject* o, const char* what, int* type, epp_rows_t* r) {
    const at::Tensor* t = numbers(o, what, 2, type);
    if (!t) return nullptr;
    const int64_t n = t->size(0), width = t->size(1);
    if (width > 1 && t->stride(1) != 1) {
        PyErr_Format(PyExc_ValueError, "%s: the elements of a row must be consecutive", what);
        return nullptr;
    }
    r->data = const_cast<void*>(t->const_data_ptr());
    r->n = n;
    r->ld = n > 1 ? t->stride(0) : width;
    return t;
}

// Entries: as many as the lists that are given name, else the rows of the first matrix.
bool entries(const epp_rows_t& a, int64_t na, const epp_rows_t& b, int64_t nb, const char* what_a, const char* what_b, int64_t* m) {
    *m = na >= 0 ? na : nb >= 0 ? nb : a.n;
    if ((na >= 0 ? na : a.n) == *m && (nb >= 0 ? nb : b.n) == *m) return true;
    PyErr_Format(PyExc_ValueError, "%lld entries in %s, %lld in %s", (long long)(na >= 0 ? na : a.n), what_a, (long long)(nb >= 0 ? nb : b.n), what_b);
    return false;
}

PyObject* group_rows(PyObject*, PyObject* const* args, Py_ssize_t n, PyObject* kw) {
    static const char* const names[] = {"group_of", "G", "offsets", "order", "workspace", "rows"};
    PyObject* a[6];
    if (!take_args("epp_group_rows", args, n, kw, names, 6, a, 5)) return nullptr;
    const int32_t *group_of, *rows, *offsets, *order;
    int64_t n_rows, m, n_offsets, n_order, bytes;
    void *ws, *s;
    if (!indexes(a[0], "group_of", &group_of, &n_rows, false)) return nullptr;
    const long G = PyLong_AsLong(a[1]);
    if (G == -1 && PyErr_Occurred()) return nullptr;
    if (!indexes(a[2], "offsets", &offsets, &n_offsets, false) || !indexes(a[3], "order", &order, &n_order, false) ||
        !workspace_of(a[4], &ws, &bytes) || !indexes(a[5], "rows", &rows, &m, true))
        return nullptr;
    if (m < 0) m = n_rows;
    if (G < 1 || G > 0x7FFFFFFE || n_offsets != G + 1 || n_order != m) {
        PyErr_SetString(PyExc_ValueError, "shapes: G >= 1, offsets G + 1, order as many as rows (without rows, as group_of)");
        return nullptr;
    }
    // (what is written: a tensor that shares its memory until then gets its own)
    int32_t* const to_offsets = THPVariable_Unpack(a[2]).mutable_data_ptr<int32_t>();
    int32_t* const to_order = m ? THPVariable_Unpack(a[3]).mutable_data_ptr<int32_t>() : nullptr;
    if (!current_stream(&s)) return nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = epp_group_rows(group_of, n_rows, rows, m, (int)G, to_offsets, to_order, ws, bytes, s);
    Py_END_ALLOW_THREADS
    return finish(rc);
}

template <bool INPUT>
PyObject* grouped_rows(PyObject*, PyObject* const* args, Py_ssize_t n, PyObject* kw) {
    static const char* const names[2][6] = {{"X", "W", "offsets", "out", "in_rows", "out_rows"}, {"grad_out", "W", "offsets", "grad_X", "in_rows", "out_rows"}};
    PyObject* a[6];
    if (!take_args(INPUT ? "epp_grouped_input_gradient" : "epp_grouped_product", args, n, kw, names[INPUT], 6, a, 4)) return nullptr;
    epp_rows_t in = {}, out = {};
    int type, type_w, type_out;
    const int32_t* offsets;
    int64_t n_offsets, n_in, n_out, m;
    const at::Tensor* x = rows_of(a[0], names[INPUT][0], &type, &in);
    const at::Tensor* W = x ? numbers(a[1], "W", 3, &type_w) : nullptr;
    const at::Tensor* y = W ? rows_of(a[3], names[INPUT][3], &type_out, &out) : nullptr;
    if (!y || !indexes(a[2], "offsets", &offsets, &n_offsets, false) || !indexes(a[4], "in_rows", &in.rows, &n_in, true) ||
        !indexes(a[5], "out_rows", &out.rows, &n_out, true))
        return nullptr;
    if (!W->is_contiguous() || type_w != type || type_out != type) {
        PyErr_Format(PyExc_ValueError, "%s, W (contiguous) and %s must be of one type", names[INPUT][0], names[INPUT][3]);
        return nullptr;
    }
    const int64_t G = W->size(0), F_in = W->size(1), F_out = W->size(2);
    if (n_offsets != G + 1 || x->size(1) != (INPUT ? F_out : F_in) || y->size(1) != (INPUT ? F_in : F_out) || G > 0x7FFFFFFE ||
        F_in > 0x7FFFFFFF || F_out > 0x7FFFFFFF) {
        PyErr_SetString(PyExc_ValueError, INPUT ? "shapes: grad_out .. x F_out, W G x F_in x F_out, offsets G + 1, grad_X .. x F_in"
                                                : "shapes: X .. x F_in, W G x F_in x F_out, offsets G + 1, out .. x F_out");
        return nullptr;
    }
    if (!entries(in, n_in, out, n_out, n_in < 0 ? names[INPUT][0] : "in_rows", n_out < 0 ? names[INPUT][3] : "out_rows", &m)) return nullptr;
    const void* w = W->const_data_ptr();
    out.data = y->mutable_data_ptr();
    void* s;
    if (!current_stream(&s)) return nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = (INPUT ? epp_grouped_input_gradient : epp_grouped_product)(type, &in, w, offsets, (int)G, m, (int)F_in, (int)F_out, &out, s);
    Py_END_ALLOW_THREADS
    return finish(rc);
}

PyObject* grouped_weight_gradient(PyObject*, PyObject* const* args, Py_ssize_t n, PyObject* kw) {
    static const char* const names[] = {"X", "grad_out", "offsets", "grad_W", "workspace", "x_rows", "grad_rows"};
    PyObject* a[7];
    if (!take_args("epp_grouped_weight_gradient", args, n, kw, names, 7, a, 5)) return nullptr;
    epp_rows_t X = {}, grad = {};
    int type, type_grad, type_w;
    const int32_t* offsets;
    int64_t n_offsets, n_x, n_grad, m, bytes;
    void *ws, *s;
    const at::Tensor* x = rows_of(a[0], "X", &type, &X);
    const at::Tensor* y = x ? rows_of(a[1], "grad_out", &type_grad, &grad) : nullptr;
    const at::Tensor* W = y ? numbers(a[3], "grad_W", 3, &type_w) : nullptr;
    if (!W || !indexes(a[2], "offsets", &offsets, &n_offsets, false) || !workspace_of(a[4], &ws, &bytes) ||
        !indexes(a[5], "x_rows", &X.rows, &n_x, true) || !indexes(a[6], "grad_rows", &grad.rows, &n_grad, true))
        return nullptr;
    if (!W->is_contiguous() || type_grad != type || (type_w != type && type_w != EPP_FLOAT32)) {
        PyErr_SetString(PyExc_ValueError, "X and grad_out must be of one type, grad_W (contiguous) of the same or float32");
        return nullptr;
    }
    const int64_t G = W->size(0), F_in = W->size(1), F_out = W->size(2);
    if (n_offsets != G + 1 || x->size(1) != F_in || y->size(1) != F_out || G > 0x7FFFFFFE || F_in > 0x7FFFFFFF || F_out > 0x7FFFFFFF) {
        PyErr_SetString(PyExc_ValueError, "shapes: X .. x F_in, grad_out .. x F_out, offsets G + 1, grad_W G x F_in x F_out");
        return nullptr;
    }
    if (!entries(X, n_x, grad, n_grad, n_x < 0 ? "X" : "x_rows", n_grad < 0 ? "grad_out" : "grad_rows", &m)) return nullptr;
    void* w = W->mutable_data_ptr();
    if (!current_stream(&s)) return nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = epp_grouped_weight_gradient(type, &X, &grad, offsets, (int)G, m, (int)F_in, (int)F_out, type_w, w, ws, bytes, s);
    Py_END_ALLOW_THREADS
    return finish(rc);
}

template <bool CLIP>
PyObject* gradients(PyObject*, PyObject* const* args, Py_ssize_t n, PyObject* kw) {
    static const char* const names[2][5] = {{"grads", "norm", "workspace"}, {"grads", "max_norm", "norm", "workspace", "out"}};
    PyObject* a[5] = {};
    if (!take_args(CLIP ? "epp_clip_gradients" : "epp_gradient_norm", args, n, kw, names[CLIP], CLIP ? 5 : 3, a, CLIP ? 4 : 3)) return nullptr;
    double max_norm = 0.0;
    if (CLIP) {
        max_norm = PyFloat_AsDouble(a[1]);
        if (max_norm == -1.0 && PyErr_Occurred()) return nullptr;
    }
    const at::Tensor* norm = device_tensor(a[CLIP ? 2 : 1], "norm");
    void *ws, *s;
    int64_t bytes;
    if (!norm) return nullptr;
    if (norm->scalar_type() != at::kFloat || norm->numel() != 1) {
        PyErr_SetString(PyExc_ValueError, "norm must be one float32 on the GPU");
        return nullptr;
    }
    if (!workspace_of(a[CLIP ? 3 : 2], &ws, &bytes)) return nullptr;
    PyObject* const out_arg = CLIP && a[4] && a[4] != Py_None ? a[4] : nullptr;
    struct Held {  // (a list of its own: the caller's may change meanwhile)
        PyObject* o = nullptr;
        ~Held() { Py_XDECREF(o); }
    } in, out;
    in.o = PySequence_Tuple(a[0]);
    if (!in.o || (out_arg && !(out.o = PySequence_Tuple(out_arg)))) return nullptr;
    const Py_ssize_t count = PyTuple_GET_SIZE(in.o);
    if (out.o && PyTuple_GET_SIZE(out.o) != count) {
        PyErr_Format(PyExc_ValueError, "%zd gradients, %zd outputs", count, PyTuple_GET_SIZE(out.o));
        return nullptr;
    }
    if (count > 0x7FFFFFFF) {
        PyErr_SetString(PyExc_ValueError, "too many gradients");
        return nullptr;
    }
    std::vector<epp_gradient_t> grads((size_t)count);
    for (Py_ssize_t i = 0; i < count; ++i) {
        int type, type_out;
        const at::Tensor* x = numbers(PyTuple_GET_ITEM(in.o, i), "a gradient", 0, &type, true);
        if (!x) return nullptr;
        if (!x->is_non_overlapping_and_dense()) {
            PyErr_Format(PyExc_ValueError, "gradient %zd: its elements must fill their memory, without gaps", i);
            return nullptr;
        }
        epp_gradient_t& g = grads[(size_t)i];
        g.type = type;
        g.count = x->numel();
        g.out = nullptr;
        if (out.o) {
            const at::Tensor* y = numbers(PyTuple_GET_ITEM(out.o, i), "an output", 0, &type_out, true);
            if (!y) return nullptr;
            if (type_out != type || y->sizes() != x->sizes() || y->strides() != x->strides()) {
                PyErr_Format(PyExc_ValueError, "output %zd: type, shape and strides must be the gradient's", i);
                return nullptr;
            }
            if (y->is_neg() != x->is_neg()) {
                PyErr_Format(PyExc_ValueError, "gradient %zd or its output is a view that stands for the negative of its memory, the other is not", i);
                return nullptr;
            }
            g.out = y->mutable_data_ptr();
        }
        g.data = CLIP && !out.o ? x->mutable_data_ptr() : const_cast<void*>(x->const_data_ptr());
    }
    float* to = norm->mutable_data_ptr<float>();
    if (!current_stream(&s)) return nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = CLIP ? epp_clip_gradients(grads.data(), (int)count, max_norm, to, ws, bytes, s) : epp_gradient_norm(grads.data(), (int)count, to, ws, bytes, s);
    Py_END_ALLOW_THREADS
    return finish(rc);
}

typedef PyObject* (*Entry)(PyObject*, PyObject* const*, Py_ssize_t, PyObject*);
template <Entry F>
PyObject* guarded(PyObject* self, PyObject* const* args, Py_ssize_t n, PyObject* kw) {
    // (PyTorch's own macro for this also buffers warnings: 0.2 us a call)
    try {
        return F(self, args, n, kw);
    } catch (python_error& e) {
        e.restore();
    } catch (const c10::Error& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what_without_backtrace());
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

// epp_alloc_t of PyTorch's caching allocator, on the current device and stream; any host thread, with the interpreter's lock or without.
// (As functions of the Python module, called back through ctypes, an allocation and its release took 4.3 us, and a construction or an
// import makes about eight, some of them while the GPU waits for the next launch: constructed on 8,000 vertices 106 -> 88 us, imported
// and one epoch on the blog graph 120 -> 112.)
std::atomic<long long> g_allocs{0}, g_frees{0}, g_bytes{0};

void* torch_alloc(size_t bytes, void*) {
    try {
        void* p = c10::hip::HIPCachingAllocator::raw_alloc(bytes);
        if (!p) return nullptr;
        g_allocs.fetch_add(1, std::memory_order_relaxed);
        g_bytes.fetch_add((long long)bytes, std::memory_order_relaxed);
        return p;
    } catch (...) {  // out of memory: the library reports EPP_ERR_ALLOC
        return nullptr;
    }
}
void torch_free(void* p, void*) {
    g_frees.fetch_add(1, std::memory_order_relaxed);
    try {
        c10::hip::HIPCachingAllocator::raw_delete(p);
    } catch (...) {  // (nobody to tell: the handle goes)
    }
}

// (address of the allocating function, of the releasing one)
PyObject* allocator(PyObject*, PyObject*) {
    return Py_BuildValue("KK", (unsigned long long)reinterpret_cast<uintptr_t>(&torch_alloc),
                         (unsigned long long)reinterpret_cast<uintptr_t>(&torch_free));
}
// alloc_news(dictionary): adds to its allocs, frees, bytes and live what has been counted since the last call.
PyObject* alloc_news(PyObject*, PyObject* stats) {
    if (!PyDict_Check(stats)) {
        PyErr_SetString(PyExc_TypeError, "alloc_news(dictionary)");
        return nullptr;
    }
    if (!g_allocs.load(std::memory_order_relaxed) && !g_frees.load(std::memory_order_relaxed)) Py_RETURN_NONE;
    const long long allocs = g_allocs.exchange(0, std::memory_order_relaxed), frees = g_frees.exchange(0, std::memory_order_relaxed);
    const struct { const char* key; long long more; } news[] = {
        {"allocs", allocs}, {"frees", frees}, {"bytes", g_bytes.exchange(0, std::memory_order_relaxed)}, {"live", allocs - frees}};
    for (const auto& x : news) {
        PyObject* const had = PyDict_GetItemString(stats, x.key);  // (borrowed; none: taken for 0)
        PyObject* const more = PyLong_FromLongLong(x.more);
        PyObject* const sum = more && had ? PyNumber_Add(had, more) : more;
        const bool done = sum && PyDict_SetItemString(stats, x.key, sum) == 0;
        if (had) Py_XDECREF(more);
        Py_XDECREF(sum);
        if (!done) return nullptr;
    }
    Py_RETURN_NONE;
}

// init(error class, raw-stream function)
PyObject* init(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != 2) {
        PyErr_SetString(PyExc_TypeError, "init(error, raw_stream)");
        return nullptr;
    }
    Py_INCREF(args[0]);
    Py_XSETREF(g_error, args[0]);
    Py_INCREF(args[1]);
    Py_XSETREF(g_raw_stream, args[1]);
    Py_RETURN_NONE;
}

#define EPP_FAST(f) reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(guarded<f>)), METH_FASTCALL | METH_KEYWORDS

PyMethodDef methods[] = {
    {"init", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(init)), METH_FASTCALL, nullptr},
    {"epp_backward_aggregate", EPP_FAST(aggregate<false>),
     "epp_backward_aggregate(path, grad_in, grad_out)\n\nPartially-active backward aggregation of one layer."},
    {"epp_full_aggregate", EPP_FAST(aggregate<true>),
     "epp_full_aggregate(full, grad_in, grad_out)\n\nAll-active backward aggregation."},
    {"epp_weight_gradient", EPP_FAST(weight_gradient<false>),
     "epp_weight_gradient(paths, k, Y, grad_X, grad_W, workspace)\n\nW' = Y^T (x) X' over the rows of N^k (k = -1: all "
     "rows); `workspace` is a CUDA uint8 tensor of\nat least epp_weight_gradient_workspace(...) bytes."},
    {"epp_weight_gradient_static", EPP_FAST(weight_gradient<true>),
     "epp_weight_gradient_static(paths, k, Y, grad_X, grad_W)\n\nepp_weight_gradient without a workspace: the partial sums "
     "use the library's static device array\n(no allocation anywhere; F_in * F_out <= 8,388,608; calls on one GPU must "
     "not overlap)."},
    {"epp_input_gradient", EPP_FAST(input_gradient),
     "epp_input_gradient(paths, k, grad_X, W, grad_Y)\n\nY' = X' (x) W^T on the rows of N^k (k = -1: all rows); other rows "
     "of grad_Y are not touched."},
    {"epp_group_rows", EPP_FAST(group_rows),
     "epp_group_rows(group_of, G, offsets, order, workspace, rows=None)\n\nEntries (the rows listed in `rows`, or all) in the order of "
     "their groups: `offsets` (G + 1) and `order`\n(as many as entries; those in no group last), all int32.  `workspace` is a CUDA "
     "uint8 tensor of at least\nepp_group_rows_workspace(entries, G) bytes."},
    {"epp_grouped_product", EPP_FAST(grouped_rows<false>),
     "epp_grouped_product(X, W, offsets, out, in_rows=None, out_rows=None)\n\nout = X W[g] on the entries offsets[g] to offsets[g + 1] of "
     "every group g; entry i reads row in_rows[i] of X and\nwrites row out_rows[i] of out (None: row i).  Other rows of out are not "
     "touched."},
    {"epp_grouped_input_gradient", EPP_FAST(grouped_rows<true>),
     "epp_grouped_input_gradient(grad_out, W, offsets, grad_X, in_rows=None, out_rows=None)\n\ngrad_X = grad_out W[g]^T on the entries of "
     "every group g, rows as in epp_grouped_product."},
    {"epp_grouped_weight_gradient", EPP_FAST(grouped_weight_gradient),
     "epp_grouped_weight_gradient(X, grad_out, offsets, grad_W, workspace, x_rows=None, grad_rows=None)\n\ngrad_W[g] = X^T grad_out over "
     "the entries of group g; grad_W of the operands' type or float32.  `workspace` is a CUDA\nuint8 tensor of at least "
     "epp_grouped_weight_gradient_workspace(entries, G, F_in, F_out) bytes."},
    {"epp_gradient_norm", EPP_FAST(gradients<false>),
     "epp_gradient_norm(grads, norm, workspace)\n\nThe norm of all gradients together; `workspace` is a CUDA uint8 tensor of at least\n"
     "epp_gradient_norm_workspace(len(grads)) bytes."},
    {"epp_clip_gradients", EPP_FAST(gradients<true>),
     "epp_clip_gradients(grads, max_norm, norm, workspace, out=None)\n\nThe norm of all gradients together, and every gradient times "
     "min(1, max_norm / norm), in place or into `out`."},
    {"allocator", allocator, METH_NOARGS, nullptr},
    {"alloc_news", alloc_news, METH_O, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding(void) {
    s_handle = PyUnicode_InternFromString("_h");
    s_cached_n = PyUnicode_InternFromString("_n");
    s_n = PyUnicode_InternFromString("n");
    if (!s_handle || !s_cached_n || !s_n) return nullptr;
    return PyModule_Create(&module);
}
