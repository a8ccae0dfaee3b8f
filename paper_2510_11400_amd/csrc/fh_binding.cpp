// The microscaled and layer norm calls as Python functions of tensors: checks of the arguments, allocation of the outputs, the current
// stream.  Every byte of a result comes from the library's kernels through its C ABI.
//
// The other calls are marshalled by ctypes in api.py.  These kernels take 3 to 10 us for small inputs, and ctypes' marshalling was what their
// callers waited for: quantising 17 x 768 values took the host 6.9 us a call from Python, 3.9 us compiled (of which the launch is 3.1); a product 7.6 and
// 4.2, a norm 10.4 and 5.1, its backward pass (two launches) 16.3 and 8.8; a training step of a layer of 8192 x 768 tokens took 162 us, and takes 96 to 102
// (its kernels 98) with the step of autograd compiled as well.
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/functions/basic_ops.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/hip/EmptyTensor.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>

#include "../../include/fedhybrid.h"

namespace {

PyObject* g_error;                       // FedHybridError(status)
PyObject* g_matrix;                      // MxMatrix(data, rows, cols)
PyObject *g_data, *g_rows, *g_cols, *g_cuda_stream, *g_nearest, *g_stochastic;     // interned names

// The interpreter's lock; autograd's threads come without it.
struct Inside {
    PyGILState_STATE state = PyGILState_Ensure();
    ~Inside() { PyGILState_Release(state); }
};
template <typename... A>
[[noreturn]] void raise(PyObject* type, const char* format, A... a)
{
    const Inside inside;
    PyErr_Format(type, format, a...);
    python_error e;
    e.persist();
    throw e;
}

// An owned reference.
struct Ref {
    PyObject* p;
    explicit Ref(PyObject* o) : p(o) { if (!o) throw python_error(); }
    Ref(const Ref&) = delete;
    Ref(Ref&& r) noexcept : p(r.p) { r.p = nullptr; }
    ~Ref() { Py_XDECREF(p); }
    PyObject* take() { PyObject* o = p; p = nullptr; return o; }
};
Ref attribute(PyObject* o, PyObject* name) { return Ref(PyObject_GetAttr(o, name)); }
PyObject* wrap(const at::Tensor& t) { return t.defined() ? THPVariable_Wrap(t) : Py_NewRef(Py_None); }

// The arguments are at::Tensor objects from here on; None where one may be left out gives an undefined tensor.
at::Tensor tensor(PyObject* o, const char* what)
{
    if (!THPVariable_Check(o)) raise(PyExc_TypeError, "%s must be a tensor (got %s)", what, Py_TYPE(o)->tp_name);
    return THPVariable_Unpack(o);
}
at::Tensor tensor_or_none(PyObject* o, const char* what) { return o == Py_None ? at::Tensor() : tensor(o, what); }

int dtype_code(at::ScalarType t)
{
    if (t == at::kFloat) return FH_F32;
    if (t == at::kBFloat16) return FH_BF16;
    raise(PyExc_TypeError, "unsupported dtype %s; expected float32 or bfloat16", c10::toString(t));
}
size_t size_of(int code) { return code == FH_F32 ? 4 : 2; }

at::ScalarType scalar_type(PyObject* o)
{
    if (!THPDtype_Check(o)) raise(PyExc_TypeError, "a dtype is wanted (got %s)", Py_TYPE(o)->tp_name);
    return reinterpret_cast<THPDtype*>(o)->scalar_type;
}

void on_device(const at::Tensor& t, c10::Device device, const char* what)
{
    if (t.device() != device)
        raise(PyExc_ValueError, "%s lives on %s, other tensors of the call on %s", what, t.device().str().c_str(), device.str().c_str());
}
void in_device_memory(const at::Tensor& t, const char* what)
{
    if (!t.is_cuda()) raise(PyExc_ValueError, "%s must live in device memory (got a %s tensor)", what, t.device().str().c_str());
}

// A matrix whose rows are contiguous.
struct Matrix {
    at::Tensor t;
    int64_t rows, cols, stride;
    int dtype;
    void* data() const { return t.data_ptr(); }
    size_t bytes() const { return rows > 0 && cols > 0 ? ((size_t)(rows - 1) * (size_t)stride + (size_t)cols) * size_of(dtype) : 0; }
    c10::Device device() const { return t.device(); }
};
Matrix matrix(at::Tensor t, const char* what)
{
    in_device_memory(t, what);
    if (t.dim() != 2) raise(PyExc_ValueError, "%s must have two dimensions (got %d)", what, (int)t.dim());
    Matrix m{std::move(t), 0, 0, 0, 0};
    m.rows = m.t.size(0);
    m.cols = m.t.size(1);
    if (m.t.stride(1) != 1 && m.cols > 1) raise(PyExc_ValueError, "the rows of %s must be contiguous", what);
    m.stride = m.rows <= 1 ? m.cols : m.t.stride(0);
    if (m.stride < m.cols) raise(PyExc_ValueError, "the rows of %s overlap", what);
    m.dtype = dtype_code(m.t.scalar_type());
    return m;
}
Matrix matrix(PyObject* o, const char* what) { return matrix(tensor(o, what), what); }

// n values, contiguous; null for an undefined tensor.
void* vector(const at::Tensor& t, int64_t n, c10::Device device, const char* what)
{
    if (!t.defined()) return nullptr;
    in_device_memory(t, what);
    on_device(t, device, what);
    if (t.dim() != 1 || t.size(0) != n || (n > 1 && t.stride(0) != 1)) raise(PyExc_ValueError, "%s must be a vector of %lld values", what, (long long)n);
    return t.data_ptr();
}

at::Tensor bytes(size_t n, c10::Device device)
{
    return at::Tensor(at::detail::empty_cuda({(int64_t)n}, at::kByte, device, std::nullopt));
}
at::Tensor values(int64_t n, at::ScalarType type, c10::Device device) { return at::Tensor(at::detail::empty_cuda({n}, type, device, std::nullopt)); }
// Two vectors of n values in one allocation.
struct Pair { at::Tensor first, second; };
Pair pair(int64_t n, at::ScalarType type, c10::Device device)
{
    Pair p{values(2 * n, type, device), at::Tensor()};
    p.second = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(p.first.storage()), p.first.key_set(), p.first.dtype());
    const int64_t step = 1;
    p.second.unsafeGetTensorImpl()->set_sizes_and_strides(at::IntArrayRef(n), at::IntArrayRef(step), n);
    p.first.unsafeGetTensorImpl()->set_sizes_contiguous(at::IntArrayRef(n));
    return p;
}
Matrix new_matrix(int64_t rows, int64_t cols, at::ScalarType type, c10::Device device)
{
    const int code = dtype_code(type);
    return Matrix{at::Tensor(at::detail::empty_cuda({rows, cols}, type, device, std::nullopt)), rows, cols, cols, code};
}
// `o`, which has to be like x, or a new matrix.
Matrix matrix_like(PyObject* o, const Matrix& x, const char* what)
{
    if (o == Py_None) return new_matrix(x.rows, x.cols, x.t.scalar_type(), x.device());
    Matrix m = matrix(o, what);
    if (m.rows != x.rows || m.cols != x.cols || m.dtype != x.dtype) raise(PyExc_ValueError, "%s must have the shape and the dtype of x", what);
    on_device(m.t, x.device(), what);
    return m;
}
// A caller's scratch buffer, or a new one of `need` bytes.
struct Work { at::Tensor t; void* p = nullptr; size_t n = 0; };
Work work(PyObject* given, size_t need, c10::Device device)
{
    Work w;
    w.t = tensor_or_none(given, "workspace");
    if (w.t.defined()) {
        in_device_memory(w.t, "workspace");
        if (!w.t.is_contiguous()) raise(PyExc_ValueError, "workspace must be contiguous");
        on_device(w.t, device, "workspace");
    } else if (need) {
        w.t = bytes(need, device);
    } else {
        return w;
    }
    w.p = w.t.data_ptr();
    w.n = w.t.nbytes();
    return w;
}

int rounding_of(PyObject* o)
{
    if (o == g_nearest) return FH_ROUND_NEAREST;
    if (o == g_stochastic) return FH_ROUND_STOCHASTIC;
    if (PyUnicode_Check(o)) {
        if (PyUnicode_Compare(o, g_nearest) == 0) return FH_ROUND_NEAREST;
        if (PyUnicode_Compare(o, g_stochastic) == 0) return FH_ROUND_STOCHASTIC;
    } else if (PyLong_Check(o)) {
        const long v = PyLong_AsLong(o);
        if (v == FH_ROUND_NEAREST || v == FH_ROUND_STOCHASTIC) return (int)v;
        PyErr_Clear();
    }
    PyErr_SetObject(PyExc_KeyError, o);
    throw python_error();
}
uint64_t u64(PyObject* o)
{
    const uint64_t v = PyLong_AsUnsignedLongLongMask(o);
    if (v == (uint64_t)-1 && PyErr_Occurred()) throw python_error();
    return v;
}
int64_t i64(PyObject* o)
{
    const int64_t v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw python_error();
    return v;
}
double f64(PyObject* o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw python_error();
    return v;
}
bool truth(PyObject* o)
{
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw python_error();
    return v != 0;
}

// The stream of a call as the current one, for the time of the call: what is allocated belongs to that stream, is written after all that
// the stream did with it before, and goes back to that stream's allocations, whether it is a workspace, what a layer keeps or
// a result.  Results are read on the stream that was current as well, as a rule: they are marked as in use there (lent()).
struct On {
    std::optional<c10::hip::HIPStream> before;
    On(PyObject* stream, c10::Device device)
    {
        if (stream == Py_None) return;
        const hipStream_t given = reinterpret_cast<hipStream_t>(u64(attribute(stream, g_cuda_stream).p));
        const c10::hip::HIPStream current = c10::hip::getCurrentHIPStream(device.index());
        if (current.stream() == given) return;
        c10::hip::setCurrentHIPStream(c10::hip::getStreamFromExternal(given, device.index()));
        before = current;
    }
    On(const On&) = delete;
    ~On() { if (before) c10::hip::setCurrentHIPStream(*before); }
    void lent(const at::Tensor& t) const { if (before && t.defined()) t.record_stream(as_recorded(*before)); }
    static c10::Stream as_recorded(const c10::hip::HIPStream& s) { return c10::Stream::unpack3(s.id(), s.device_index(), c10::DeviceType::CUDA); }
};

Ref wrapped_matrix(const at::Tensor& data, int64_t rows, int64_t cols)
{
    Ref d(THPVariable_Wrap(data)), r(PyLong_FromLongLong(rows)), c(PyLong_FromLongLong(cols));
    PyTypeObject* type = reinterpret_cast<PyTypeObject*>(g_matrix);      // filled here: its __init__ is interpreted, 0.1 us of a call
    Ref m(type->tp_alloc(type, 0));
    if (PyObject_SetAttr(m.p, g_data, d.p) < 0 || PyObject_SetAttr(m.p, g_rows, r.p) < 0 || PyObject_SetAttr(m.p, g_cols, c.p) < 0) throw python_error();
    return m;
}
template <typename... R>
PyObject* tuple(R&&... r)
{
    PyObject* t = PyTuple_New(sizeof...(r));
    if (!t) throw python_error();
    Py_ssize_t i = 0;
    (PyTuple_SET_ITEM(t, i++, r.take()), ...);
    return t;
}

// A stored matrix, MxMatrix in Python.
struct Stored { at::Tensor data; int64_t rows, cols; };
Stored stored(PyObject* o, const char* what)
{
    Stored s;
    s.data = tensor(attribute(o, g_data).p, what);
    s.rows = i64(attribute(o, g_rows).p);
    s.cols = i64(attribute(o, g_cols).p);
    in_device_memory(s.data, what);
    if (!s.data.is_contiguous()) raise(PyExc_ValueError, "%s must be contiguous", what);
    if (s.data.scalar_type() != at::kByte) raise(PyExc_TypeError, "%s holds %s, a stored matrix bytes", what, c10::toString(s.data.scalar_type()));
    return s;
}

// `device` as the current one, the interpreter's lock let go: for the time of a call.
struct Outside {
    c10::DeviceIndex before;
    PyThreadState* gil;
    explicit Outside(c10::DeviceIndex index) : before(c10::hip::current_device())
    {
        if (before != index) c10::hip::set_device(index);
        else before = -1;
        gil = PyGILState_Check() ? PyEval_SaveThread() : nullptr;
    }
    ~Outside()
    {
        if (gil) PyEval_RestoreThread(gil);
        if (before >= 0) c10::hip::set_device(before);
    }
};
template <typename F>
void enqueue(c10::Device device, F call)
{
    void* handle = c10::hip::getCurrentHIPStream(device.index()).stream();
    fh_status status;
    {
        const Outside outside(device.index());
        status = call(handle);
    }
    if (status == FH_OK) return;
    const Inside inside;
    Ref value(PyObject_CallFunction(g_error, "i", (int)status));
    PyErr_SetObject(g_error, value.p);
    python_error e;
    e.persist();
    throw e;
}

// What the forms of a stored matrix are asked for by.
struct Forms { bool rows, columns; };
Forms forms_of(PyObject* o)
{
    const char* s = PyUnicode_Check(o) ? PyUnicode_AsUTF8(o) : nullptr;
    if (s) {
        if (!strcmp(s, "rows")) return {true, false};
        if (!strcmp(s, "columns")) return {false, true};
        if (!strcmp(s, "both")) return {true, true};
    }
    PyErr_Clear();
    raise(PyExc_ValueError, "forms must be 'rows', 'columns' or 'both' (got %R)", o);
}
struct Stores {
    at::Tensor by_rows, by_columns;
    int64_t rows, cols;
    Stores(Forms f, int64_t r, int64_t c, c10::Device device) : rows(r), cols(c)
    {
        if (f.rows) by_rows = bytes(fh_mx_bytes(r, c), device);
        if (f.columns) by_columns = bytes(fh_mx_bytes(c, r), device);
    }
    void lent(const On& on) const
    {
        on.lent(by_rows);
        on.lent(by_columns);
    }
    static void* data(const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }
    static size_t size(const at::Tensor& t) { return t.defined() ? (size_t)t.numel() : 0; }
    Ref wrapped() const
    {
        if (!by_columns.defined()) return wrapped_matrix(by_rows, rows, cols);
        if (!by_rows.defined()) return wrapped_matrix(by_columns, cols, rows);
        return Ref(tuple(wrapped_matrix(by_rows, rows, cols), wrapped_matrix(by_columns, cols, rows)));
    }
};

void want(Py_ssize_t got, Py_ssize_t n)
{
    if (got != n) raise(PyExc_TypeError, "%d arguments are wanted (got %d)", (int)n, (int)got);
}
#define FH_ENTRY(NAME, COUNT)                                                          \
    PyObject* NAME(PyObject*, PyObject* const* a, Py_ssize_t n)                        \
    {                                                                                  \
        HANDLE_TH_ERRORS                                                               \
        want(n, COUNT);
#define FH_EXIT                                                                        \
        END_HANDLE_TH_ERRORS                                                           \
    }

// (x, forms, rounding, seed, tensor_id, stream)
FH_ENTRY(mx_quantize, 6)
    const Forms f = forms_of(a[1]);
    const Matrix x = matrix(a[0], "x");
    const int rounding = rounding_of(a[2]);
    const uint64_t seed = u64(a[3]), id = u64(a[4]);
    const On on(a[5], x.device());
    const Stores s(f, x.rows, x.cols, x.device());
    s.lent(on);
    enqueue(x.device(), [&](void* stream) {
        return fh_mx_quantize(x.data(), (fh_dtype)x.dtype, x.rows, x.cols, x.stride, rounding, seed, id, s.data(s.by_rows), s.size(s.by_rows),
                              s.data(s.by_columns), s.size(s.by_columns), stream);
    });
    return s.wrapped().take();
FH_EXIT

// (matrix, out_dtype, out, stream)
FH_ENTRY(mx_dequantize, 4)
    const Stored m = stored(a[0], "the stored matrix");
    const c10::Device device = m.data.device();
    const On on(a[3], device);
    const Matrix out = a[2] == Py_None ? new_matrix(m.rows, m.cols, scalar_type(a[1]), device) : matrix(a[2], "out");
    if (out.rows != m.rows || out.cols != m.cols)
        raise(PyExc_ValueError, "out is %lld x %lld, the matrix %lld x %lld", (long long)out.rows, (long long)out.cols, (long long)m.rows, (long long)m.cols);
    on_device(out.t, device, "out");
    if (a[2] == Py_None) on.lent(out.t);
    enqueue(device, [&](void* stream) {
        return fh_mx_dequantize(m.data.data_ptr(), (size_t)m.data.numel(), m.rows, m.cols, (fh_dtype)out.dtype, out.data(), out.stride, out.bytes(), stream);
    });
    return wrap(out.t);
FH_EXIT

// (a, b, bias, out_dtype, out, workspace, stream)
FH_ENTRY(mx_matmul, 7)
    const Stored x = stored(a[0], "a"), y = stored(a[1], "b");
    const at::Tensor bias = tensor_or_none(a[2], "bias");
    const c10::Device device = x.data.device();
    if (x.cols != y.cols) raise(PyExc_ValueError, "a has %lld columns, b %lld", (long long)x.cols, (long long)y.cols);
    on_device(y.data, device, "b");
    const On on(a[6], device);
    const Matrix out = a[4] == Py_None ? new_matrix(x.rows, y.rows, scalar_type(a[3]), device) : matrix(a[4], "out");
    if (out.rows != x.rows || out.cols != y.rows)
        raise(PyExc_ValueError, "out is %lld x %lld, the product %lld x %lld", (long long)out.rows, (long long)out.cols, (long long)x.rows, (long long)y.rows);
    on_device(out.t, device, "out");
    if (a[4] == Py_None) on.lent(out.t);
    const Work w = work(a[5], fh_mx_matmul_workspace_bytes(x.rows, y.rows, x.cols), device);
    const fh_mx_product p = {x.data.data_ptr(), (size_t)x.data.numel(), y.data.data_ptr(), (size_t)y.data.numel(), x.rows, y.rows, x.cols,
                             vector(bias, y.rows, device, "bias"), bias.defined() ? dtype_code(bias.scalar_type()) : FH_F32, out.dtype, out.data(),
                             out.stride, out.bytes(), w.p, w.n, 0};
    enqueue(device, [&](void* stream) { return fh_mx_matmul(&p, stream); });
    return wrap(out.t);
FH_EXIT

// A norm's weight and bias.
struct Parameters {
    at::Tensor weight, bias;
    void *w, *b;
    int dtype;
    Parameters(PyObject* wo, PyObject* bo, int64_t cols, c10::Device device) : weight(tensor_or_none(wo, "weight")), bias(tensor_or_none(bo, "bias"))
    {
        if (weight.defined() && bias.defined() && weight.scalar_type() != bias.scalar_type())
            raise(PyExc_TypeError, "weight and bias have different dtypes (%s, %s)", c10::toString(weight.scalar_type()), c10::toString(bias.scalar_type()));
        w = vector(weight, cols, device, "weight");
        b = vector(bias, cols, device, "bias");
        dtype = weight.defined() ? dtype_code(weight.scalar_type()) : bias.defined() ? dtype_code(bias.scalar_type()) : FH_F32;
    }
};

// (x, weight, bias, eps, out, stream)
FH_ENTRY(layer_norm, 6)
    const Matrix x = matrix(a[0], "x");
    const Parameters p(a[1], a[2], x.cols, x.device());
    const float eps = (float)f64(a[3]);
    const On on(a[5], x.device());
    const Matrix y = matrix_like(a[4], x, "out");
    const Pair stats = pair(x.rows, at::kFloat, x.device());
    if (a[4] == Py_None) on.lent(y.t);
    on.lent(stats.first);
    enqueue(x.device(), [&](void* stream) {
        return fh_layer_norm(x.data(), (fh_dtype)x.dtype, x.rows, x.cols, x.stride, p.w, p.b, (fh_dtype)p.dtype, eps, y.data(), y.stride, y.bytes(),
                             stats.first.data_ptr(), stats.second.data_ptr(), stream);
    });
    return tuple(Ref(wrap(y.t)), Ref(wrap(stats.first)), Ref(wrap(stats.second)));
FH_EXIT

// (x, weight, bias, eps, forms, rounding, seed, tensor_id, stream)
FH_ENTRY(layer_norm_mx, 9)
    const Matrix x = matrix(a[0], "x");
    const Parameters p(a[1], a[2], x.cols, x.device());
    const float eps = (float)f64(a[3]);
    const Forms f = forms_of(a[4]);
    const int rounding = rounding_of(a[5]);
    const uint64_t seed = u64(a[6]), id = u64(a[7]);
    const On on(a[8], x.device());
    const Stores s(f, x.rows, x.cols, x.device());
    const Pair stats = pair(x.rows, at::kFloat, x.device());
    s.lent(on);
    on.lent(stats.first);
    enqueue(x.device(), [&](void* stream) {
        return fh_layer_norm_mx(x.data(), (fh_dtype)x.dtype, x.rows, x.cols, x.stride, p.w, p.b, (fh_dtype)p.dtype, eps, rounding, seed, id,
                                s.data(s.by_rows), s.size(s.by_rows), s.data(s.by_columns), s.size(s.by_columns), stats.first.data_ptr(), stats.second.data_ptr(), stream);
    });
    return tuple(s.wrapped(), Ref(wrap(stats.first)), Ref(wrap(stats.second)));
FH_EXIT

// (dy, x, mean, rstd, weight, sums, dx, workspace, stream, the sums' dtype or None)
FH_ENTRY(layer_norm_backward, 10)
    const Matrix x = matrix(a[1], "x"), dy = matrix(a[0], "dy");
    const c10::Device device = x.device();
    if (dy.rows != x.rows || dy.cols != x.cols || dy.dtype != x.dtype) raise(PyExc_ValueError, "dy must have the shape and the dtype of x");
    on_device(dy.t, device, "dy");
    const at::Tensor mean = tensor(a[2], "mean"), rstd = tensor(a[3], "rstd"), weight = tensor_or_none(a[4], "weight");
    if (mean.scalar_type() != at::kFloat || rstd.scalar_type() != at::kFloat) raise(PyExc_TypeError, "mean and rstd must be float32");
    void *mean_at = vector(mean, x.rows, device, "mean"), *rstd_at = vector(rstd, x.rows, device, "rstd"), *weight_at = vector(weight, x.cols, device, "weight");
    const bool sums = truth(a[5]);
    const On on(a[8], device);
    const Matrix dx = matrix_like(a[6], x, "dx");
    if (a[6] == Py_None) on.lent(dx.t);
    const at::ScalarType type = a[9] != Py_None ? scalar_type(a[9]) : weight.defined() ? weight.scalar_type() : x.t.scalar_type();
    if (weight.defined() && type != weight.scalar_type())
        raise(PyExc_TypeError, "the sums are of the weight's dtype, %s, not of %s", c10::toString(weight.scalar_type()), c10::toString(type));
    const int p_dtype = dtype_code(type);
    Pair sum;
    Work w;
    if (sums) {
        sum = pair(x.cols, type, device);
        on.lent(sum.first);
        w = work(a[7], fh_layer_norm_backward_workspace_bytes(x.rows, x.cols), device);
    }
    const fh_norm_backward b = {dy.data(), x.data(), dy.stride, x.stride, mean_at, rstd_at, weight_at, x.rows, x.cols, x.dtype, p_dtype, dx.data(), dx.stride,
                                dx.bytes(), sums ? sum.first.data_ptr() : nullptr, sums ? sum.second.data_ptr() : nullptr, w.p, w.n};
    enqueue(device, [&](void* stream) { return fh_layer_norm_backward(&b, stream); });
    return tuple(Ref(wrap(dx.t)), Ref(wrap(sum.first)), Ref(wrap(sum.second)));
FH_EXIT

// ---- a linear layer's two halves ----------------------------------------------------------------
struct Layer {
    bool norm;
    float eps;
    bool input, weight, bias;                                             // what gradients are wanted of
    int rounding;
    uint64_t seed, id;
    bool wide;                                                            // the gradient of a norm's output in fp32
    int32_t needs() const { return (input ? FH_MX_NEEDS_INPUT : 0) | (weight ? FH_MX_NEEDS_WEIGHT : 0); }
};
struct Sizes { size_t kept, forward, backward; };
Sizes sizes_of(const fh_mx_layer& l)                                      // of a layer that the call itself will refuse: nothing
{
    Sizes s = {};
    if (fh_mx_layer_sizes(&l, &s.kept, &s.forward, &s.backward) != FH_OK) return {};
    return s;
}

struct Forward { at::Tensor y, kept; };
Forward forward_of(const Layer& layer, const Matrix& x, const Matrix& weight, const at::Tensor& bias, const at::Tensor& norm_weight, const at::Tensor& norm_bias)
{
    const c10::Device device = x.device();
    if (weight.cols != x.cols) raise(PyExc_ValueError, "x has %lld features, weight takes %lld", (long long)x.cols, (long long)weight.cols);
    on_device(weight.t, device, "weight");
    for (const at::Tensor* t : {&bias, &norm_weight, &norm_bias})
        if (t->defined() && t->scalar_type() != weight.t.scalar_type())
            raise(PyExc_TypeError, "the parameters of one layer are of one dtype, as its weight: %s", c10::toString(weight.t.scalar_type()));
    fh_mx_layer l = {};
    l.tokens = x.rows; l.features = x.cols; l.out_features = weight.rows;
    l.dtype = x.dtype; l.p_dtype = weight.dtype; l.norm = layer.norm;
    l.needs = l.kept_for = layer.needs();
    l.eps = layer.eps;
    l.x = x.data(); l.x_stride = x.stride; l.weight = weight.data(); l.weight_stride = weight.stride; l.dy_stride = weight.rows;
    l.norm_weight = vector(norm_weight, x.cols, device, "norm_weight");
    l.norm_bias = vector(norm_bias, x.cols, device, "norm_bias");
    l.bias = vector(bias, weight.rows, device, "bias");
    const Sizes sizes = sizes_of(l);
    Forward f;
    f.y = new_matrix(x.rows, weight.rows, x.t.scalar_type(), device).t;
    l.y = f.y.data_ptr();
    if (l.needs) {
        f.kept = bytes(sizes.kept, device);
        l.kept = f.kept.data_ptr(); l.kept_cap = (size_t)f.kept.numel();
    }
    const Work w = work(Py_None, sizes.forward, device);
    l.scratch = w.p; l.scratch_cap = w.n;
    enqueue(device, [&](void* s) { return fh_mx_layer_forward(&l, s); });
    return f;
}

struct Backward { at::Tensor dx, dweight, dbias; Pair dnorm; };
Backward backward_of(const Layer& layer, const Matrix& dy, const at::Tensor& x_again, const at::Tensor& norm_weight, const at::Tensor& kept, int64_t features,
                     at::ScalarType p_type, int32_t kept_for)
{
    const c10::Device device = dy.device();
    if (kept.defined()) {
        in_device_memory(kept, "kept");
        on_device(kept, device, "kept");
        if (kept.scalar_type() != at::kByte || !kept.is_contiguous()) raise(PyExc_ValueError, "what the forward call kept has changed");
    }
    const at::ScalarType type = dy.t.scalar_type();
    fh_mx_layer l = {};
    l.tokens = dy.rows; l.features = features; l.out_features = dy.cols;
    l.dtype = dy.dtype; l.p_dtype = dtype_code(p_type); l.norm = layer.norm;
    l.needs = layer.needs();
    l.kept_for = kept_for;
    l.eps = layer.eps;
    l.rounding = layer.rounding; l.seed = layer.seed; l.tensor_id = layer.id; l.wide_gradient = layer.wide;
    l.dy = dy.data(); l.dy_stride = dy.stride; l.x_stride = l.weight_stride = features;
    if (kept.defined()) { l.kept = kept.data_ptr(); l.kept_cap = kept.nbytes(); }
    Backward b;
    Matrix x{};
    if (layer.weight) {
        b.dweight = new_matrix(l.out_features, features, p_type, device).t;
        l.dweight = b.dweight.data_ptr();
    }
    if (layer.bias) {
        b.dbias = values(l.out_features, p_type, device);
        l.dbias = b.dbias.data_ptr();
    }
    if (layer.input) {
        b.dx = new_matrix(l.tokens, features, type, device).t;
        l.dx = b.dx.data_ptr();
        if (layer.norm) {
            if (!x_again.defined()) raise(PyExc_ValueError, "with a norm the backward call takes x again");
            x = matrix(x_again, "x");
            if (x.rows != l.tokens || x.cols != features || x.dtype != l.dtype) raise(PyExc_ValueError, "x must have the shape and the dtype of the forward call's");
            on_device(x.t, device, "x");
            l.x = x.data(); l.x_stride = x.stride;
            if (norm_weight.defined() && norm_weight.scalar_type() != p_type)      // it is read as the parameters' type
                raise(PyExc_TypeError, "norm_weight is of %s, the layer's parameters of %s", c10::toString(norm_weight.scalar_type()), c10::toString(p_type));
            l.norm_weight = vector(norm_weight, features, device, "norm_weight");
            b.dnorm = pair(features, p_type, device);
            l.dnorm_weight = b.dnorm.first.data_ptr(); l.dnorm_bias = b.dnorm.second.data_ptr();
        }
    }
    const Work w = work(Py_None, sizes_of(l).backward, device);
    l.scratch = w.p; l.scratch_cap = w.n;
    enqueue(device, [&](void* s) { return fh_mx_layer_backward(&l, s); });
    return b;
}

// (x, weight, bias, norm, norm_weight, norm_bias, eps, needs_input, needs_weight, stream) -> (y, kept)
FH_ENTRY(layer_forward, 10)
    const Layer layer = {truth(a[3]), (float)f64(a[6]), truth(a[7]), truth(a[8]), false, FH_ROUND_NEAREST, 0, 0, false};
    const Matrix x = matrix(a[0], "x");
    const On on(a[9], x.device());
    const Forward f = forward_of(layer, x, matrix(a[1], "weight"), tensor_or_none(a[2], "bias"), tensor_or_none(a[4], "norm_weight"), tensor_or_none(a[5], "norm_bias"));
    on.lent(f.y);
    return tuple(Ref(wrap(f.y)), Ref(wrap(f.kept)));
FH_EXIT

// (dy, x, norm_weight, kept, features, p_dtype, norm, eps, needs_input, needs_weight, needs_bias, rounding, seed, tensor_id, wide_gradient,
//  the forward call's needs, stream) -> (dx, dweight, dnorm_weight, dnorm_bias, dbias)
FH_ENTRY(layer_backward, 17)
    const Layer layer = {truth(a[6]), (float)f64(a[7]), truth(a[8]), truth(a[9]), truth(a[10]), rounding_of(a[11]), u64(a[12]), u64(a[13]), truth(a[14])};
    const Matrix dy = matrix(a[0], "dy");
    const at::Tensor kept = tensor_or_none(a[3], "kept");
    const On on(a[16], dy.device());
    const Backward b = backward_of(layer, dy, tensor_or_none(a[1], "x"), tensor_or_none(a[2], "norm_weight"), kept, i64(a[4]), scalar_type(a[5]),
                                   (int32_t)i64(a[15]));
    // it is of the stream that the forward call went through, and may be dropped before this one is through with it
    if (kept.defined()) kept.record_stream(On::as_recorded(c10::hip::getCurrentHIPStream(dy.device().index())));
    for (const at::Tensor* t : {&b.dx, &b.dweight, &b.dnorm.first, &b.dbias}) on.lent(*t);
    return tuple(Ref(wrap(b.dx)), Ref(wrap(b.dweight)), Ref(wrap(b.dnorm.first)), Ref(wrap(b.dnorm.second)), Ref(wrap(b.dbias)));
FH_EXIT

// ---- the same as a step of autograd -------------------------------------------------------------
// x as a matrix of its last dimension, its rows contiguous and apart (an expanded gradient's are not).
at::Tensor rows_of(const at::Tensor& x)
{
    const at::Tensor m = x.dim() == 2 ? x : x.reshape({-1, x.size(-1)});
    return m.stride(1) == 1 && m.stride(0) >= m.size(1) ? m : m.contiguous();
}

// y's rows in the order of x's.
at::Tensor shaped(const at::Tensor& y, const at::Tensor& x)
{
    if (x.dim() == 2) return y;
    std::vector<int64_t> shape = x.sizes().vec();
    shape.back() = y.size(1);
    return y.view(shape);
}

struct Pass : torch::CustomClassHolder {                                  // from one half to the other, but for what is saved as a variable
    Layer layer;
    bool x, norm_weight, norm_bias;                                       // whose gradients are wanted, beside the layer's
    std::vector<int64_t> shape;
    int64_t features;
    at::ScalarType p_type;
};

struct Linear : torch::autograd::Function<Linear> {
    using Context = torch::autograd::AutogradContext;
    static at::Tensor forward(Context* ctx, const at::Tensor& x, const std::optional<at::Tensor>& norm_weight, const std::optional<at::Tensor>& norm_bias,
                              const at::Tensor& weight, const std::optional<at::Tensor>& bias, const c10::intrusive_ptr<Pass>& pass)
    {
        const at::Tensor m = rows_of(x);
        const Forward f = forward_of(pass->layer, matrix(m, "x"), matrix(weight, "weight"), bias.value_or(at::Tensor()), norm_weight.value_or(at::Tensor()),
                               norm_bias.value_or(at::Tensor()));
        pass->features = m.size(1);
        // Saved as variables are, so that the backward pass frees what was kept and checkpointing drops it; one row of bytes, which hooks for
        // activations leave as it is.
        if (f.kept.defined() && pass->layer.norm && pass->layer.input) ctx->save_for_backward({f.kept.unsqueeze(0), m, norm_weight.value_or(at::Tensor())});
        else if (f.kept.defined()) ctx->save_for_backward({f.kept.unsqueeze(0)});
        ctx->saved_data.emplace("pass", c10::IValue::make_capsule(pass));
        return shaped(f.y, x);
    }
    static torch::autograd::variable_list backward(Context* ctx, const torch::autograd::variable_list& given)
    {
        const auto pass = c10::static_intrusive_pointer_cast<Pass>(ctx->saved_data.at("pass").toCapsule());
        const bool again = at::GradMode::is_enabled() && given[0].requires_grad();
        torch::autograd::variable_list grads(6);
        {
            const at::AutoGradMode off(false);
            const at::Tensor dy = rows_of(given[0]);
            const auto saved = ctx->get_saved_variables();
            const auto from = [&](size_t i) { return i < saved.size() ? saved[i] : at::Tensor(); };
            const Backward b = backward_of(pass->layer, matrix(dy, "dy"), from(1), from(2), from(0), pass->features, pass->p_type,
                                           pass->layer.needs());
            if (pass->x) grads[0] = b.dx.view(pass->shape);
            if (pass->norm_weight) grads[1] = b.dnorm.first;
            if (pass->norm_bias) grads[2] = b.dnorm.second;
            grads[3] = b.dweight;
            grads[4] = b.dbias;
        }
        if (!again) return grads;
        for (at::Tensor& g : grads)                                       // leaves of a graph that ends in an error
            if (g.defined()) g = g.detach().set_requires_grad(true);
        return torch::autograd::DelayedError("a linear layer in microscaled form is differentiated once", (int64_t)grads.size()).apply(std::move(grads));
    }
};

// Forward-mode derivatives: a tangent that went no further would be read as a derivative of zero.
void no_tangent(const at::Tensor& t, const char* what)
{
    if (t.defined() && t._fw_grad(/*level=*/0).defined()) raise(PyExc_NotImplementedError, "%s carries a tangent; the microscaled layers have no forward-mode derivative", what);
}

// (tensors): refused where one carries a tangent
PyObject* refuse_tangents(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    for (Py_ssize_t i = 0; i < n; ++i) no_tangent(tensor_or_none(a[i], "x"), "an input");
    Py_RETURN_NONE;
    END_HANDLE_TH_ERRORS
}

// (x, norm_weight, norm_bias, weight, bias, eps or None where there is no norm, rounding, seed, tensor_id) -> y
FH_ENTRY(mx_linear, 9)
    const at::Tensor x = tensor(a[0], "x"), norm_weight = tensor_or_none(a[1], "norm_weight"), norm_bias = tensor_or_none(a[2], "norm_bias"),
                     weight = tensor(a[3], "weight"), bias = tensor_or_none(a[4], "bias");
    no_tangent(x, "x"); no_tangent(norm_weight, "norm_weight"); no_tangent(norm_bias, "norm_bias"); no_tangent(weight, "weight"); no_tangent(bias, "bias");
    in_device_memory(x, "x");
    if (x.dim() == 0) raise(PyExc_ValueError, "x must have a dimension");
    const auto pass = c10::make_intrusive<Pass>();
    const bool norm = a[5] != Py_None, grad = at::GradMode::is_enabled();
    const auto wanted = [&](const at::Tensor& t) { return grad && t.defined() && t.requires_grad(); };
    pass->x = wanted(x); pass->norm_weight = wanted(norm_weight); pass->norm_bias = wanted(norm_bias);
    pass->layer = {norm, norm ? (float)f64(a[5]) : 0.0f, pass->x || pass->norm_weight || pass->norm_bias, wanted(weight), wanted(bias),
                   rounding_of(a[6]), u64(a[7]), u64(a[8]), true};
    pass->p_type = weight.scalar_type();
    pass->shape = x.sizes().vec();
    at::Tensor y;
    if (pass->layer.input || pass->layer.weight || pass->layer.bias) {
        const auto some = [](const at::Tensor& t) { return t.defined() ? std::optional<at::Tensor>(t) : std::nullopt; };
        y = Linear::apply(x, some(norm_weight), some(norm_bias), weight, some(bias), pass);
    } else {
        y = shaped(forward_of(pass->layer, matrix(rows_of(x), "x"), matrix(weight, "weight"), bias, norm_weight, norm_bias).y, x);
    }
    return wrap(y);
FH_EXIT

// (FedHybridError, MxMatrix): the classes that results and errors are of.
FH_ENTRY(use, 2)
    Py_XSETREF(g_error, Py_NewRef(a[0]));
    Py_XSETREF(g_matrix, Py_NewRef(a[1]));
    Py_RETURN_NONE;
FH_EXIT

#define FH_METHOD(NAME) {#NAME, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(NAME)), METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {FH_METHOD(mx_quantize), FH_METHOD(mx_dequantize), FH_METHOD(mx_matmul), FH_METHOD(layer_norm), FH_METHOD(layer_norm_mx),
                           FH_METHOD(layer_norm_backward), FH_METHOD(layer_forward), FH_METHOD(layer_backward), FH_METHOD(mx_linear), FH_METHOD(refuse_tangents),
                           FH_METHOD(use), {}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_fh_binding", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fh_binding()
{
    struct { PyObject** to; const char* name; } names[] = {{&g_data, "data"}, {&g_rows, "rows"}, {&g_cols, "cols"}, {&g_cuda_stream, "cuda_stream"},
                                                           {&g_nearest, "nearest"}, {&g_stochastic, "stochastic"}};
    for (auto& n : names)
        if (!(*n.to = PyUnicode_InternFromString(n.name))) return nullptr;
    return PyModule_Create(&g_module);
}
