// The 8-bit operators and those beside them from Python: checks of tensors, new results and the call into the C ABI.
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

// ---- what a network answers with, and what it is trained on ----

// A workspace of `need` bytes at least, from room(need); nothing where none is needed.
struct Work {
    PyObject* held = nullptr;
    void* p = nullptr;
    Work(PyObject* room, uint64_t need) {
        if (!need) return;
        held = PyObject_CallFunction(room, "K", (unsigned long long)need);
        if (!held) throw PythonError();
        p = tensor_of(held, "work").data_ptr();
    }
    Work(const Work&) = delete;
    ~Work() { Py_XDECREF(held); }
};

float number_of(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (PyErr_Occurred()) throw PythonError();
    return (float)v;
}

// A vector of whole numbers, one a row: targets, adapters.
const int64_t* numbers_of(const Handle& h, PyObject* o, uint64_t n, const char* what) {
    const at::Tensor& v = tensor_of(o, what);
    TORCH_CHECK_VALUE(v.scalar_type() == at::kLong && v.dim() == 1 && (uint64_t)v.size(0) == n && v.is_contiguous(), what,
                      " must be a contiguous int64 vector of ", n);
    here(h, v, what);
    return static_cast<const int64_t*>(v.data_ptr());
}

// ctx, device, x, target, scale, entropy, top, room -> (logp, lse, entropy, top, index, norm), None for what is not asked for
PyObject* log_probs(PyObject* const* a) {
    const Handle h = handle_of(a);
    const at::Tensor& tx = tensor_of(a[2], "x");
    const Rows x = rows_of(h, tx, "x");
    shifter_log_probs_args g{};
    g.d_x = x.p;
    g.ld_x = x.ld;
    g.rows = x.rows;
    g.cols = x.cols;
    g.dtype = x.dtype;
    g.scale = number_of(a[4]);
    const bool entropy = truth(a[5]);
    const long top = PyLong_AsLong(a[6]);
    if (PyErr_Occurred()) throw PythonError();
    TORCH_CHECK_VALUE(top >= 0 && top <= (long)SHIFTER_LOG_PROBS_MAX_TOP && (uint64_t)top <= x.cols, "top must be 0 to ",
                      SHIFTER_LOG_PROBS_MAX_TOP, " and not above the columns");
    g.top = (uint32_t)top;
    const bool given = !is_none(a[3]);
    if (given) g.d_target = numbers_of(h, a[3], x.rows, "target");
    const int64_t rows = (int64_t)x.rows;
    at::Tensor out[6];
    // the vectors in one allocation
    out[5] = new_tensor(h, {rows * (3 + given + entropy)}, at::kFloat);
    float* at = static_cast<float*>(out[5].data_ptr());
    int64_t used = 2 * rows;
    auto vector = [&](at::Tensor& v) {
        v = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(out[5].storage()), out[5].key_set(), out[5].dtype());
        v.unsafeGetTensorImpl()->set_storage_offset(used);
        v.unsafeGetTensorImpl()->set_sizes_contiguous({rows});
        float* p = at + used;
        used += rows;
        return p;
    };
    g.d_norm = at;
    g.d_lse = vector(out[1]);
    if (given) g.d_logp = vector(out[0]);
    if (entropy) g.d_entropy = vector(out[2]);
    out[5].unsafeGetTensorImpl()->set_sizes_contiguous({rows, 2});
    if (top) {
        out[3] = new_tensor(h, {rows, top}, at::kFloat);
        out[4] = new_tensor(h, {rows, top}, at::kLong);
    }
    g.d_top = top ? static_cast<float*>(out[3].data_ptr()) : nullptr;
    g.d_index = top ? static_cast<int64_t*>(out[4].data_ptr()) : nullptr;
    check(shifter_log_probs_layout(g.rows, g.cols, g.top, &g.work_bytes), Py_None);
    const Work work(a[7], g.work_bytes);
    g.d_work = work.p;
    check(shifter_log_probs(h.ctx, &g), a[0]);     // with the interpreter's lock: calls of several launches have the same workspace
    Owned all(PyTuple_New(6));
    for (int i = 0; i < 6; ++i) {
        if (!out[i].defined()) {
            Py_INCREF(Py_None);
            PyTuple_SET_ITEM(all.p, i, Py_None);
        } else {
            PyTuple_SET_ITEM(all.p, i, THPVariable_Wrap(i != 4 ? tied(std::move(out[i]), tx, at::Tensor(), "log_probs") : std::move(out[i])));
        }
    }
    return all.release();
}

// ctx, device, x, target, norm, g_logp, g_lse, entropy, g_entropy, scale, out -> dx
PyObject* log_probs_grad(PyObject* const* a) {
    const Handle h = handle_of(a);
    const at::Tensor& tx = tensor_of(a[2], "x");
    if (!is_none(a[10])) {
        constant(tx, "x");
        for (int i : {5, 6, 8})
            if (!is_none(a[i])) constant(tensor_of(a[i], "a gradient"), "a gradient");
    }
    const Rows x = rows_of(h, tx, "x");
    shifter_log_probs_grad_args g{};
    g.d_x = x.p;
    g.ld_x = x.ld;
    g.rows = x.rows;
    g.cols = x.cols;
    g.dtype = x.dtype;
    if (!is_none(a[3])) g.d_target = numbers_of(h, a[3], x.rows, "target");
    const at::Tensor& norm = tensor_of(a[4], "norm");
    TORCH_CHECK_VALUE(norm.scalar_type() == at::kFloat && norm.dim() == 2 && (uint64_t)norm.size(0) == x.rows && norm.size(1) == 2 &&
                      norm.is_contiguous(), "norm must be a contiguous float32 tensor of ", x.rows, " rows of 2");
    here(h, norm, "norm");
    g.d_norm = static_cast<const float*>(norm.data_ptr());
    if (!is_none(a[5])) g.d_g_logp = vector_of(h, a[5], x.rows, "g_logp");
    if (!is_none(a[6])) g.d_g_lse = vector_of(h, a[6], x.rows, "g_lse");
    if (!is_none(a[8])) {
        TORCH_CHECK_VALUE(!is_none(a[7]), "g_entropy without entropy");
        g.d_entropy = vector_of(h, a[7], x.rows, "entropy");
        g.d_g_entropy = vector_of(h, a[8], x.rows, "g_entropy");
    }
    TORCH_CHECK_VALUE(!g.d_g_logp || g.d_target || x.rows == 0, "g_logp without target");
    g.scale = number_of(a[9]);
    at::Tensor dx;
    if (is_none(a[10])) {
        dx = new_rows(h, x.rows, x.cols, tx.scalar_type());
    } else {
        dx = tensor_of(a[10], "out");
        constant(dx, "out");
        same(dx, x.rows, x.cols, tx.scalar_type(), "out");
    }
    const Rows r = rows_of(h, dx, "out");
    g.d_dx = r.p;
    g.ld_dx = r.ld;
    enqueue(a[0], [&] { return shifter_log_probs_grad(h.ctx, &g); });
    if (is_none(a[10])) {
        dx = tied(std::move(dx), tx, is_none(a[5]) ? at::Tensor() : tensor_of(a[5], "g_logp"), "log_probs_grad");
        for (int i : {6, 8})
            if (!is_none(a[i])) dx = tied(std::move(dx), tensor_of(a[i], "a gradient"), at::Tensor(), "log_probs_grad");
    }
    return wrap(a[10], std::move(dx));
}

// The items of a list or tuple.
struct Items {
    Owned seq;
    Items(PyObject* o, const char* what) : seq(PySequence_Fast(o, what)) {}
    Py_ssize_t size() const { return PySequence_Fast_GET_SIZE(seq.p); }
    PyObject* operator[](Py_ssize_t i) const { return PySequence_Fast_GET_ITEM(seq.p, i); }
};

// Whether both, of one shape and without gaps, have their elements in the same order: the strides of dimensions of one element say nothing.
bool in_order(const at::Tensor& a, const at::Tensor& b) {
    if (a.numel() < 2) return true;
    for (int64_t i = 0; i < a.dim(); ++i)
        if (a.size(i) != 1 && a.stride(i) != b.stride(i)) return false;
    return true;
}

// ctx, device, grads, masks, max_norm, out, room -> norm.  max_norm None: the norm alone.
PyObject* grad_norm(PyObject* const* a) {
    const Handle h = handle_of(a);
    const bool clip = !is_none(a[4]);
    const float max_norm = clip ? number_of(a[4]) : 0.0f;
    const Items grads(a[2], "grads must be a list of tensors");
    const Items masks(is_none(a[3]) ? a[2] : a[3], "masks must be a list");
    const Items out(is_none(a[5]) ? a[2] : a[5], "out must be a list of tensors");
    const Py_ssize_t n = grads.size();
    TORCH_CHECK_VALUE(masks.size() == n && out.size() == n, "masks and out must have an entry for each of grads");
    TORCH_CHECK_VALUE(!clip || max_norm >= 0.0f, "max_norm must not be negative");
    std::vector<shifter_grad> list((size_t)n);
    for (Py_ssize_t i = 0; i < n; ++i) {
        const at::Tensor& g = tensor_of(grads[i], "a gradient");
        const int code = g.layout() == at::kStrided ? code_of(g.scalar_type()) : -1;
        TORCH_CHECK_VALUE(code >= 0, "gradient ", i, " must be fp32, bf16 or fp16");
        TORCH_CHECK_VALUE(g.is_non_overlapping_and_dense(), "gradient ", i, " has gaps between its elements");
        constant(g, "a gradient");
        here(h, g, "a gradient");
        shifter_grad& e = list[(size_t)i];
        e = shifter_grad{g.data_ptr(), nullptr, nullptr, (uint64_t)g.numel(), code};
        auto alike = [&](const at::Tensor& t, at::ScalarType type, const char* what) {
            TORCH_CHECK_VALUE(t.layout() == at::kStrided && t.scalar_type() == type && t.sizes() == g.sizes() && in_order(g, t), what, " ", i, " must be ", type,
                              " of its gradient's shape and layout in memory");
            here(h, t, what);
            return t.data_ptr();
        };
        if (!is_none(a[3]) && !is_none(masks[i])) e.d_mask = static_cast<const uint8_t*>(alike(tensor_of(masks[i], "a mask"), at::kByte, "mask"));
        if (!clip) continue;
        const at::Tensor& t = tensor_of(out[i], "out");
        constant(t, "out");
        e.d_out = alike(t, g.scalar_type(), "out");
    }
    uint64_t need = 0;
    check(shifter_grad_norm_layout((uint64_t)n, &need), Py_None);
    const Work work(a[6], need);
    at::Tensor norm = new_tensor(h, {}, at::kFloat);
    float* p = static_cast<float*>(norm.data_ptr());
    // with the interpreter's lock: the launches share the handle's workspace, and another thread's stay out from between them
    check(clip ? shifter_clip_grad_norm(h.ctx, list.data(), (uint64_t)n, max_norm, p, work.p, need)
               : shifter_grad_norm(h.ctx, list.data(), (uint64_t)n, p, work.p, need), a[0]);
    if (clip)
        for (Py_ssize_t i = 0; i < n; ++i) written(tensor_of(out[i], "out"));
    return THPVariable_Wrap(std::move(norm));
}

// The adapters of a call, and x: elements of their type, or an 8-bit matrix.
struct Adapted {
    at::ScalarType type;
    int dtype;
    const void *x, *a, *b;
    uint64_t ld_x, m, n, k, rank, adapters;
    const float *q_scale = nullptr, *scale = nullptr;
    const int64_t* which;
    Adapted(const Handle& h, PyObject* ox, PyObject* oa, PyObject* ob, PyObject* owhich, PyObject* oscale) {
        const at::Tensor &ta = tensor_of(oa, "a"), &tb = tensor_of(ob, "b");
        type = ta.scalar_type();
        dtype = code_of(type);
        TORCH_CHECK_VALUE(dtype >= 0 && ta.dim() == 3 && ta.is_contiguous(), "a must be a contiguous fp32, bf16 or fp16 tensor of adapters, rank, columns of x");
        adapters = (uint64_t)ta.size(0);
        rank = (uint64_t)ta.size(1);
        k = (uint64_t)ta.size(2);
        TORCH_CHECK_VALUE(tb.dim() == 3 && tb.scalar_type() == type && tb.is_contiguous() && (uint64_t)tb.size(0) == adapters &&
                          (uint64_t)tb.size(2) == rank, "b must be a contiguous tensor of adapters, columns of y, rank, of a's type");
        n = (uint64_t)tb.size(1);
        here(h, ta, "a");
        here(h, tb, "b");
        a = ta.data_ptr();
        b = tb.data_ptr();
        if (THPVariable_Check(ox)) {
            const at::Tensor& tx = THPVariable_Unpack(ox);
            TORCH_CHECK_VALUE(tx.scalar_type() == type, "x must have a's type, or be a Q8Matrix");
            const Rows r = rows_of(h, tx, "x");
            TORCH_CHECK_VALUE(r.cols == k, "x must have a's columns");
            x = r.p;
            ld_x = r.ld;
            m = r.rows;
        } else {
            const Codes c = codes_of(h, ox, "x");
            TORCH_CHECK_VALUE(c.cols == k, "x must have a's columns");
            x = c.q;
            ld_x = c.ld;
            m = c.rows;
            q_scale = c.scale;
        }
        which = numbers_of(h, owhich, m, "which");
        if (!is_none(oscale)) scale = vector_of(h, oscale, adapters, "scale");
    }
    template <typename Args>
    void put(Args& g) const {
        g.d_x = x; g.ld_x = ld_x; g.d_q_scale = q_scale; g.m = m; g.n = n; g.k = k; g.rank = rank; g.adapters = adapters;
        g.d_a = a; g.d_b = b; g.d_which = which; g.d_scale = scale; g.dtype = dtype;
    }
};

// A float32 matrix without gaps.
float* numbers32_of(const Handle& h, PyObject* o, uint64_t rows, uint64_t cols, const char* what) {
    const at::Tensor& t = tensor_of(o, what);
    same(t, rows, cols, at::kFloat, what);
    TORCH_CHECK_VALUE(t.is_contiguous(), what, " must be contiguous");
    here(h, t, what);
    return static_cast<float*>(t.data_ptr());
}

// ctx, device, y, x, a, b, which, scale, out, down, room -> out
PyObject* adapters(PyObject* const* a) {
    const Handle h = handle_of(a);
    const at::Tensor& ty = tensor_of(a[2], "y");
    const int given[] = {2, 3, 4, 5, 7};           // elements that may need a gradient
    if (!is_none(a[8]) || !is_none(a[9]))
        for (int i : given)
            if (THPVariable_Check(a[i])) constant(THPVariable_Unpack(a[i]), "an operand");
    const Adapted s(h, a[3], a[4], a[5], a[6], a[7]);
    same(ty, s.m, s.n, ty.scalar_type(), "y");
    const Rows y = rows_of(h, ty, "y");
    shifter_adapters_args g{};
    s.put(g);
    g.d_y = y.p;
    g.ld_y = y.ld;
    g.y_dtype = y.dtype;
    at::Tensor out;
    if (is_none(a[8])) {
        out = new_rows(h, s.m, s.n, ty.scalar_type());
    } else {
        out = tensor_of(a[8], "out");
        constant(out, "out");
        same(out, s.m, s.n, ty.scalar_type(), "out");
    }
    const Rows r = rows_of(h, out, "out");
    g.d_out = r.p;
    g.ld_out = r.ld;
    if (!is_none(a[9])) {
        constant(tensor_of(a[9], "down"), "down");
        g.d_down = numbers32_of(h, a[9], s.m, s.rank, "down");
    }
    check(shifter_adapters_layout(s.m, s.n, s.k, s.rank, s.adapters, &g.work_bytes), Py_None);
    const Work work(a[10], g.work_bytes);
    g.d_work = work.p;
    // with the interpreter's lock: the launches share the handle's workspace
    check(shifter_adapters(h.ctx, &g), a[0]);
    if (!is_none(a[9])) written(tensor_of(a[9], "down"));
    if (is_none(a[8]))
        for (int i : given)
            if (THPVariable_Check(a[i])) out = tied(std::move(out), THPVariable_Unpack(a[i]), at::Tensor(), "adapters");
    return wrap(a[8], std::move(out));
}

// ctx, device, g, x, a, b, which, scale, down, dx wanted, room -> (dx, da, db)
PyObject* adapters_grad(PyObject* const* a) {
    const Handle h = handle_of(a);
    const at::Tensor& tg = tensor_of(a[2], "g");
    const Adapted s(h, a[3], a[4], a[5], a[6], a[7]);
    same(tg, s.m, s.n, s.type, "g");
    const Rows r = rows_of(h, tg, "g");
    shifter_adapters_grad_args g{};
    s.put(g);
    g.d_g = r.p;
    g.ld_g = r.ld;
    if (!is_none(a[8])) g.d_down = numbers32_of(h, a[8], s.m, s.rank, "down");
    at::Tensor out[3];
    if (truth(a[9])) {
        out[0] = new_rows(h, s.m, s.k, s.type);
        g.d_dx = out[0].data_ptr();
        g.ld_dx = s.k;
    }
    out[1] = new_tensor(h, {(int64_t)s.adapters, (int64_t)s.rank, (int64_t)s.k}, at::kFloat);
    out[2] = new_tensor(h, {(int64_t)s.adapters, (int64_t)s.n, (int64_t)s.rank}, at::kFloat);
    g.d_da = static_cast<float*>(out[1].data_ptr());
    g.d_db = static_cast<float*>(out[2].data_ptr());
    check(shifter_adapters_grad_layout(s.m, s.n, s.k, s.rank, s.adapters, s.dtype, &g.work_bytes), Py_None);
    const Work work(a[10], g.work_bytes);
    g.d_work = work.p;
    check(shifter_adapters_grad(h.ctx, &g), a[0]);         // with the interpreter's lock, as above
    Owned all(PyTuple_New(3));
    for (int i = 0; i < 3; ++i) {
        if (!out[i].defined()) {
            Py_INCREF(Py_None);
            PyTuple_SET_ITEM(all.p, i, Py_None);
            continue;
        }
        for (int j : {2, 3, 4, 5, 7, 8})
            if (THPVariable_Check(a[j])) out[i] = tied(std::move(out[i]), THPVariable_Unpack(a[j]), at::Tensor(), "adapters_grad");
        PyTuple_SET_ITEM(all.p, i, THPVariable_Wrap(std::move(out[i])));
    }
    return all.release();
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
                         Q8_ENTRY(matmul, 8), Q8_ENTRY(weight_grad, 9), Q8_ENTRY(log_probs, 8), Q8_ENTRY(log_probs_grad, 11),
                         Q8_ENTRY(grad_norm, 7), Q8_ENTRY(adapters, 11), Q8_ENTRY(adapters_grad, 11), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_q8", "The 8-bit operators' calls; see q8.py.", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__q8() {
    struct { PyObject** at; const char* name; } const names[] = {{&g_q, "q"}, {&g_scale, "scale"}, {&g_rows, "rows"}, {&g_cols, "cols"}, {&g_ld, "ld"}};
    for (const auto& n : names)
        if (!(*n.at = PyUnicode_InternFromString(n.name))) return nullptr;
    return PyModule_Create(&module);
}
