// The 8-bit operators from Python: checks of tensors, new results and the call into the C ABI.
//
// A call's kernel takes a few microseconds, as much as a handful of calls into torch from Python:
// 1 x 2048 bf16, us a call with all this in Python and ctypes / here: quantise 7.7 / 4.0, read back 6.4 / 4.0, norm
// with residual 11.0 / 4.8, of which a launch is 3.2.  No stream is looked up here: the handle has asked torch for it.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/core/grad_mode.h>
#include <ATen/hip/EmptyTensor.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/functions/basic_ops.h>
#include <torch/csrc/autograd/python_variable.h>

#include "shifter.h"

namespace {

PyObject* g_matrix = nullptr;                       // the class Q8Matrix, whose slots these name
PyObject *g_q, *g_scale, *g_rows, *g_cols, *g_ld;
PyObject* g_failed = nullptr;                       // raises for a code of the C ABI

// Where a call runs: what the handle passes first.
struct Handle {
    shifter_ctx* ctx;
    c10::DeviceIndex device;
};

bool is_none(PyObject* o) { return o == Py_None; }

struct PythonError {};                              // a Python exception is set

struct Owned {                                      // a reference given back at the end
    PyObject* p;
    explicit Owned(PyObject* o) : p(o) { if (!p) throw PythonError(); }
    Owned(const Owned&) = delete;
    ~Owned() { Py_XDECREF(p); }
    PyObject* release() { PyObject* o = p; p = nullptr; return o; }
};

const at::Tensor& tensor_of(PyObject* o, const char* what) {
    TORCH_CHECK_VALUE(THPVariable_Check(o), what, " must be a tensor");
    return THPVariable_Unpack(o);
}

void here(const Handle& h, const at::Tensor& x, const char* what) {
    const c10::Device d = x.device();
    TORCH_CHECK_VALUE(d.is_cuda() && d.index() == h.device, what, " is not on cuda:", (int)h.device);
}

// No operator passes gradients on.  An 8-bit matrix is a constant to autograd, as whole numbers are; where elements are made
// from elements that need a gradient, that would be lost without a word.
bool needs_gradient(const at::Tensor& x) { return x.defined() && x.requires_grad() && at::GradMode::is_enabled(); }

// A new result of such elements has an error for its backward pass.
at::Tensor tied(at::Tensor&& result, const at::Tensor& a, const at::Tensor& b, const char* fn) {
    if (!needs_gradient(a) && !needs_gradient(b)) return std::move(result);
    torch::autograd::variable_list all{std::move(result), a, b};
    const auto error = std::make_shared<torch::autograd::DelayedError>(std::string("q8.") + fn + " passes no gradients on", 3);
    return (*error)(std::move(all))[0];
}

// What a caller gives to be written has no such place: neither it nor what it is made from may need a gradient.
void constant(const at::Tensor& x, const char* what) {
    TORCH_CHECK_VALUE(!needs_gradient(x), what, " needs a gradient, which a call that writes a given tensor does not pass on: "
                      "detach it, or call under torch.no_grad()");
}
void written(const at::Tensor& x) {
    if (!x.is_inference()) x.unsafeGetTensorImpl()->bump_version();
}

int code_of(at::ScalarType t) {
    switch (t) {
        case at::kFloat: return SHIFTER_F32;
        case at::kBFloat16: return SHIFTER_BF16;
        case at::kHalf: return SHIFTER_F16;
        default: return -1;
    }
}

// A matrix of elements, or of the mask's bytes.
struct Rows {
    void* p = nullptr;
    int dtype = 0;
    uint64_t rows = 0, cols = 0, ld = 0;
};

void lay_out(Rows& r, const Handle& h, const at::Tensor& x, const char* what) {
    const int64_t rows = x.size(0), cols = x.size(1), ld = rows < 2 ? cols : x.stride(0);
    TORCH_CHECK_VALUE((cols <= 1 || x.stride(1) == 1) && ld >= cols, "the columns of ", what,
                      " must lie side by side, rows one after another");
    here(h, x, what);
    r.p = x.data_ptr();
    r.rows = (uint64_t)rows;
    r.cols = (uint64_t)cols;
    r.ld = (uint64_t)ld;
}

Rows rows_of(const Handle& h, const at::Tensor& x, const char* what) {
    Rows r;
    r.dtype = x.dim() == 2 ? code_of(x.scalar_type()) : -1;
    TORCH_CHECK_VALUE(r.dtype >= 0, what, " must be a two-dimensional fp32, bf16 or fp16 tensor");
    lay_out(r, h, x, what);
    return r;
}

void same(const at::Tensor& a, uint64_t rows, uint64_t cols, at::ScalarType t, const char* what) {
    TORCH_CHECK_VALUE(a.dim() == 2 && (uint64_t)a.size(0) == rows && (uint64_t)a.size(1) == cols && a.scalar_type() == t, what,
                      " must have shape (", rows, ", ", cols, ") and type ", t);
}

const float* vector_of(const Handle& h, PyObject* o, uint64_t n, const char* what) {
    const at::Tensor& v = tensor_of(o, what);
    TORCH_CHECK_VALUE(v.scalar_type() == at::kFloat && v.dim() == 1 && (uint64_t)v.size(0) == n && v.is_contiguous(), what,
                      " must be a contiguous float32 vector of ", n);
    here(h, v, what);
    return static_cast<const float*>(v.data_ptr());
}

// A new tensor straight from the device's allocator (at::empty finds its way there in 0.3 us more).
at::Tensor new_tensor(const Handle& h, at::IntArrayRef sizes, at::ScalarType t) {
    return at::Tensor(at::detail::empty_cuda(sizes, t, c10::Device(c10::DeviceType::CUDA, h.device), std::nullopt));
}

at::Tensor new_rows(const Handle& h, uint64_t rows, uint64_t cols, at::ScalarType t) {
    return new_tensor(h, {(int64_t)rows, (int64_t)cols}, t);
}

// An 8-bit matrix as the C ABI takes it.
struct Codes {
    int8_t* q = nullptr;
    float* scale = nullptr;
    uint64_t rows = 0, cols = 0, ld = 0;
};

uint64_t number_at(PyObject* o, PyObject* name) {
    const Owned v(PyObject_GetAttr(o, name));
    const unsigned long long n = PyLong_AsUnsignedLongLong(v.p);
    if (PyErr_Occurred()) throw PythonError();
    return n;
}

Codes codes_of(const Handle& h, PyObject* o, const char* what) {
    TORCH_CHECK_VALUE(PyObject_TypeCheck(o, reinterpret_cast<PyTypeObject*>(g_matrix)), what, " must be a Q8Matrix");
    Codes m;
    const Owned q(PyObject_GetAttr(o, g_q)), scale(PyObject_GetAttr(o, g_scale));
    const at::Tensor& codes = tensor_of(q.p, what);
    here(h, codes, what);
    m.q = static_cast<int8_t*>(codes.data_ptr());
    m.scale = static_cast<float*>(tensor_of(scale.p, what).data_ptr());
    m.rows = number_at(o, g_rows);
    m.cols = number_at(o, g_cols);
    m.ld = number_at(o, g_ld);
    return m;
}

void put(PyObject* o, PyObject* name, PyObject* value) {
    const Owned v(value);
    if (PyObject_SetAttr(o, name, v.p) < 0) throw PythonError();
}

// A new 8-bit matrix of Python's class, as its __init__ would leave it, its codes and its scales in one allocation.
PyObject* new_codes(const Handle& h, uint64_t rows, uint64_t cols, Codes& m) {
    m.rows = rows;
    m.cols = cols;
    m.ld = (cols + 15u) / 16u * 16u;
    const int64_t bytes = (int64_t)(rows * m.ld);
    at::Tensor q = new_tensor(h, {bytes + 4 * (int64_t)rows}, at::kChar);
    at::Tensor scale = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(q.storage()), q.key_set(), caffe2::TypeMeta::Make<float>());
    scale.unsafeGetTensorImpl()->set_storage_offset(bytes / 4);
    scale.unsafeGetTensorImpl()->set_sizes_contiguous({(int64_t)rows});
    q.unsafeGetTensorImpl()->set_sizes_contiguous({(int64_t)rows, (int64_t)m.ld});
    m.q = static_cast<int8_t*>(q.data_ptr());
    m.scale = static_cast<float*>(scale.data_ptr());
    PyTypeObject* type = reinterpret_cast<PyTypeObject*>(g_matrix);
    Owned o(type->tp_alloc(type, 0));
    put(o.p, g_q, THPVariable_Wrap(std::move(q)));
    put(o.p, g_scale, THPVariable_Wrap(std::move(scale)));
    put(o.p, g_rows, PyLong_FromUnsignedLongLong(rows));
    put(o.p, g_cols, PyLong_FromUnsignedLongLong(cols));
    put(o.p, g_ld, PyLong_FromUnsignedLongLong(m.ld));
    return o.release();
}

// `out` of a call, or a new matrix.
PyObject* room(const Handle& h, uint64_t rows, uint64_t cols, PyObject* out, Codes& m) {
    if (is_none(out)) return new_codes(h, rows, cols, m);
    m = codes_of(h, out, "out");
    TORCH_CHECK_VALUE(m.rows == rows && m.cols == cols, "out is an 8-bit matrix of another size");
    Py_INCREF(out);
    return out;
}

// A given 8-bit matrix has been written.
void written(PyObject* out) {
    if (is_none(out)) return;
    const Owned q(PyObject_GetAttr(out, g_q)), scale(PyObject_GetAttr(out, g_scale));
    written(tensor_of(q.p, "out"));
    written(tensor_of(scale.p, "out"));
}

// The same for elements: their type is out's, or dtype.
at::Tensor result(const Handle& h, uint64_t rows, uint64_t cols, PyObject* dtype, PyObject* out, Rows& r) {
    at::Tensor x;
    if (is_none(out)) {
        const int code = THPDtype_Check(dtype) ? code_of(reinterpret_cast<THPDtype*>(dtype)->scalar_type) : -1;
        TORCH_CHECK_VALUE(code >= 0, "dtype must be fp32, bf16 or fp16");
        x = new_rows(h, rows, cols, reinterpret_cast<THPDtype*>(dtype)->scalar_type);
    } else {
        x = tensor_of(out, "out");
        constant(x, "out");
        same(x, rows, cols, x.scalar_type(), "out");
    }
    r = rows_of(h, x, "out");
    return x;
}

// What a call returns once it has been enqueued.
PyObject* wrap(PyObject* out, at::Tensor&& x) {
    if (is_none(out)) return THPVariable_Wrap(std::move(x));
    written(x);
    Py_INCREF(out);
    return out;
}

Handle handle_of(PyObject* const* args) {
    Handle h;
    h.ctx = static_cast<shifter_ctx*>(PyLong_AsVoidPtr(args[0]));
    h.device = (c10::DeviceIndex)PyLong_AsLong(args[1]);
    if (PyErr_Occurred()) throw PythonError();
    return h;
}

bool truth(PyObject* o) {
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw PythonError();
    return v != 0;
}

void check(int rc, PyObject* ctx) {
    if (rc == SHIFTER_OK) return;
    const Owned none(PyObject_CallFunction(g_failed, "iO", rc, ctx));       // raises
    TORCH_CHECK(false, "call failed with code ", rc);
}

// The call itself, without the interpreter's lock (a full queue makes a launch wait).
template <typename F>
void enqueue(PyObject* ctx, F call) {
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = call();
    Py_END_ALLOW_THREADS
    check(rc, ctx);
}

// A function of N arguments whose exceptions become Python's.
template <Py_ssize_t N, PyObject* (*F)(PyObject* const*)>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != N) {
        PyErr_Format(PyExc_TypeError, "%zd arguments expected, got %zd", N, n);
        return nullptr;
    }
    try {
        return F(args);
    } catch (const PythonError&) {
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

// ctx, device, x, relu, out -> matrix
PyObject* quantize(PyObject* const* a) {
    const Handle h = handle_of(a);
    const Rows x = rows_of(h, tensor_of(a[2], "x"), "x");
    const uint32_t flags = truth(a[3]) ? SHIFTER_Q8_RELU : 0u;
    Codes m;
    Owned out(room(h, x.rows, x.cols, a[4], m));
    enqueue(a[0], [&] { return shifter_quantize_q8(h.ctx, x.p, x.dtype, x.ld, x.rows, x.cols, flags, m.q, m.ld, m.scale); });
    written(a[4]);
    return out.release();
}

// ctx, device, m, dtype, out -> elements
PyObject* dequantize(PyObject* const* a) {
    const Handle h = handle_of(a);
    const Codes m = codes_of(h, a[2], "m");
    Rows r;
    at::Tensor x = result(h, m.rows, m.cols, a[3], a[4], r);
    enqueue(a[0], [&] { return shifter_dequantize_q8(h.ctx, m.q, m.ld, m.scale, m.rows, m.cols, r.p, r.dtype, r.ld); });
    return wrap(a[4], std::move(x));
}

// ctx, device, x, weight, eps, residual, h, out -> (matrix, h)
PyObject* rms_norm(PyObject* const* a) {
    const Handle h = handle_of(a);
    const at::Tensor& tx = tensor_of(a[2], "x");
    if (!is_none(a[5]) && !is_none(a[6])) {    // without a residual the stream is x itself, with its graph
        constant(tx, "x");
        constant(tensor_of(a[5], "residual"), "residual");
        constant(tensor_of(a[6], "h"), "h");
    }
    const Rows x = rows_of(h, tx, "x");
    const float* weight = vector_of(h, a[3], x.cols, "weight");
    const double eps = PyFloat_AsDouble(a[4]);
    if (PyErr_Occurred()) throw PythonError();
    Rows residual, stream;
    at::Tensor sum;
    if (!is_none(a[5])) {
        const at::Tensor& t = tensor_of(a[5], "residual");
        same(t, x.rows, x.cols, tx.scalar_type(), "residual");
        residual = rows_of(h, t, "residual");
        if (is_none(a[6])) {
            sum = new_rows(h, x.rows, x.cols, tx.scalar_type());
        } else {
            sum = tensor_of(a[6], "h");
            same(sum, x.rows, x.cols, tx.scalar_type(), "h");
        }
        stream = rows_of(h, sum, "h");
    } else {
        TORCH_CHECK_VALUE(is_none(a[6]), "h without a residual: the stream is x itself");
    }
    Codes m;
    Owned out(room(h, x.rows, x.cols, a[7], m));
    enqueue(a[0], [&] {
        return shifter_rms_norm_q8(h.ctx, x.p, x.ld, residual.p, residual.ld, x.dtype, x.rows, x.cols, weight, (float)eps, stream.p,
                                   stream.ld, m.q, m.ld, m.scale);
    });
    written(a[7]);
    if (!is_none(a[5]) && is_none(a[6])) sum = tied(std::move(sum), tx, tensor_of(a[5], "residual"), "rms_norm");
    Owned held(is_none(a[5]) ? (Py_INCREF(a[2]), a[2]) : wrap(a[6], std::move(sum)));
    Owned both(PyTuple_New(2));
    PyTuple_SET_ITEM(both.p, 0, out.release());
    PyTuple_SET_ITEM(both.p, 1, held.release());
    return both.release();
}

// ctx, device, a, b, bias, relu, dtype, out -> elements
PyObject* matmul(PyObject* const* v) {
    const Handle h = handle_of(v);
    if (!is_none(v[4]) && !is_none(v[7])) constant(tensor_of(v[4], "bias"), "bias");
    const Codes a = codes_of(h, v[2], "a"), b = codes_of(h, v[3], "b");
    TORCH_CHECK_VALUE(a.cols == b.cols, "a and b have different numbers of columns");
    const float* bias = is_none(v[4]) ? nullptr : vector_of(h, v[4], b.rows, "bias");
    const uint32_t flags = truth(v[5]) ? SHIFTER_Q8_RELU : 0u;
    Rows r;
    at::Tensor c = result(h, a.rows, b.rows, v[6], v[7], r);
    enqueue(v[0], [&] {
        return shifter_matmul_q8(h.ctx, a.q, a.ld, a.scale, b.q, b.ld, b.scale, a.rows, b.rows, a.cols, bias, flags, r.p, r.dtype, r.ld);
    });
    if (!is_none(v[4]) && is_none(v[7])) c = tied(std::move(c), tensor_of(v[4], "bias"), at::Tensor(), "matmul");
    return wrap(v[7], std::move(c));
}

// ctx, device, g, x, mask, dtype, out, accumulate, room -> dw.  room(bytes) gives a workspace, where one is needed.
PyObject* weight_grad(PyObject* const* a) {
    const Handle h = handle_of(a);
    const at::Tensor& tg = tensor_of(a[2], "g");
    if (!is_none(a[6])) constant(tg, "g");
    const Rows g = rows_of(h, tg, "g");
    const Codes x = codes_of(h, a[3], "x");
    TORCH_CHECK_VALUE(x.rows == g.rows, "g and x have different numbers of rows");
    Rows mask, r;
    if (!is_none(a[4])) {
        const at::Tensor& t = tensor_of(a[4], "mask");
        same(t, g.cols, x.cols, at::kByte, "mask");
        lay_out(mask, h, t, "mask");
    }
    const uint32_t flags = truth(a[7]) ? SHIFTER_Q8_ACCUMULATE : 0u;
    TORCH_CHECK_VALUE(!flags || !is_none(a[6]), "accumulate without out");
    TORCH_CHECK_VALUE(is_none(a[6]) || tensor_of(a[6], "out").scalar_type() == at::kFloat, "out must be float32");
    at::Tensor dw = result(h, g.cols, x.cols, a[5], a[6], r);
    uint64_t need = 0;
    check(shifter_weight_grad_q8_layout(g.rows, g.cols, x.cols, &need), Py_None);
    void* work = nullptr;
    PyObject* held = nullptr;
    if (need) {
        held = PyObject_CallFunction(a[8], "K", (unsigned long long)need);
        if (!held) throw PythonError();
    }
    const Owned keep(held ? held : (Py_INCREF(Py_None), Py_None));
    if (held) work = tensor_of(held, "work").data_ptr();
    // with the interpreter's lock: the launches share the handle's workspace, and another thread's stay out from between them
    check(shifter_weight_grad_q8(h.ctx, g.p, g.dtype, g.ld, x.q, x.ld, x.scale, g.rows, g.cols, x.cols,
                                 static_cast<const uint8_t*>(mask.p), mask.ld, flags, static_cast<float*>(r.p), r.ld, work, need), a[0]);
    if (is_none(a[6])) dw = tied(std::move(dw), tg, at::Tensor(), "weight_grad");
    return wrap(a[6], std::move(dw));
}

// Q8Matrix, failed(code, ctx): what the functions below make and raise.
PyObject* bind(PyObject* const* a) {
    Py_INCREF(a[0]);
    Py_XSETREF(g_matrix, a[0]);
    Py_INCREF(a[1]);
    Py_XSETREF(g_failed, a[1]);
    Py_RETURN_NONE;
}

#define Q8_ENTRY(name, n) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&entry<n, name>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {Q8_ENTRY(bind, 2), Q8_ENTRY(quantize, 5), Q8_ENTRY(dequantize, 5), Q8_ENTRY(rms_norm, 8),
                         Q8_ENTRY(matmul, 8), Q8_ENTRY(weight_grad, 9), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_q8", "The 8-bit operators' calls; see q8.py.", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__q8() {
    struct { PyObject** at; const char* name; } const names[] = {{&g_q, "q"}, {&g_scale, "scale"}, {&g_rows, "rows"}, {&g_cols, "cols"}, {&g_ld, "ld"}};
    for (const auto& n : names)
        if (!(*n.at = PyUnicode_InternFromString(n.name))) return nullptr;
    return PyModule_Create(&module);
}
