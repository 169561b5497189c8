// The microscaled-format calls of molgrid.py in their common form (dense rows, new results), marshalled in C++:
// a kernel on a few thousand rows runs for 3 to 10 us, and the same checks and allocations take as long in
// Python.  Tensors come in as Python objects, their checks and the results' allocation happen here, and the
// C ABI's function does the rest.  Every function returns None where a call is not of that form (strided,
// wrong, on another device): molgrid.py then goes its own way, which handles it or says what is wrong with it.
// An int is the library's error code.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/core/impl/LocalDispatchKeySet.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>

#include "../../include/molgrid_hip.h"

namespace {

decltype(&mg_mx_pack) pack_fn;
decltype(&mg_mx_unpack) unpack_fn;
decltype(&mg_mx8_weight_gradient_workspace) gradient_workspace_fn;
decltype(&mg_mx8_weight_gradient) gradient_fn;
decltype(&mg_mx4_product) product_fn;
decltype(&mg_mx4_linear_workspace) linear_workspace_fn;
decltype(&mg_mx4_linear) linear_fn;

struct NotPlain {};                     // a call of another form

void plain(bool ok)
{
    if (!ok) throw NotPlain();
}

const at::Tensor &tensor(PyObject *o)
{
    plain(THPVariable_CheckExact(o) || THPVariable_Check(o));
    return THPVariable_Unpack(o);
}

int64_t integer(PyObject *o)
{
    plain(PyLong_Check(o));
    const int64_t v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        throw NotPlain();
    }
    return v;
}

// a dense tensor on the device of the call
const at::Tensor &dense(PyObject *o, int64_t dev)
{
    const at::Tensor &t = tensor(o);
    plain(t.is_cuda() && t.get_device() == dev && t.layout() == at::kStrided && t.is_contiguous() && !t.is_neg());
    return t;
}

int number(at::ScalarType t)
{
    switch (t) {
    case at::kFloat: return MG_F32;
    case at::kHalf: return MG_F16;
    case at::kBFloat16: return MG_BF16;
    default: throw NotPlain();
    }
}

at::ScalarType scalar(int64_t n)
{
    plain(n >= MG_F32 && n <= MG_BF16);
    return n == MG_F32 ? at::kFloat : n == MG_F16 ? at::kHalf : at::kBFloat16;
}

at::Tensor make(const at::Tensor &like, at::IntArrayRef shape, at::ScalarType type)
{
    return at::empty(shape, like.options().dtype(type).requires_grad(false));
}

// Shape, codes and scales of a tensor in a microscaled format.
struct Packed {
    c10::SmallVector<int64_t, 6> shape;
    int64_t rows, cols;
    uint8_t *codes, *scales;
    const at::Tensor *like;
};

void rows_of(at::IntArrayRef shape, int64_t &rows, int64_t &cols)
{
    plain(!shape.empty());
    rows = 1;
    for (size_t i = 0; i + 1 < shape.size(); ++i) rows *= shape[i];
    cols = shape.back();
    plain(rows >= 1 && cols >= 1);
}

int64_t code_pitch(int64_t format, int64_t cols) { return (cols + 31) / 32 * (format == MG_MX_E2M1 ? 16 : 32); }
int64_t scale_pitch(int64_t cols) { return ((cols + 31) / 32 + 3) / 4 * 4; }

Packed packed(PyObject *codes, PyObject *scales, PyObject *shape, int64_t format, int64_t dev)
{
    Packed p;
    plain(PyTuple_CheckExact(shape));
    for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(shape); ++i) p.shape.push_back(integer(PyTuple_GET_ITEM(shape, i)));
    rows_of(p.shape, p.rows, p.cols);
    const at::Tensor &c = dense(codes, dev), &s = dense(scales, dev);
    plain(c.scalar_type() == at::kByte && s.scalar_type() == at::kByte && c.dim() == 2 && s.dim() == 2);
    plain(c.size(0) == p.rows && c.size(1) == code_pitch(format, p.cols));
    plain(s.size(0) == p.rows && s.size(1) == scale_pitch(p.cols));
    p.codes = (uint8_t *)c.data_ptr();
    p.scales = (uint8_t *)s.data_ptr();
    p.like = &c;
    return p;
}

const float *optional_floats(PyObject *o, int64_t n, int64_t dev)
{
    if (o == Py_None) return nullptr;
    const at::Tensor &t = dense(o, dev);
    plain(t.scalar_type() == at::kFloat && t.dim() == 1 && t.size(0) == n);
    return (const float *)t.data_ptr();
}

PyObject *result(int code, at::Tensor &&t) { return code == MG_OK ? THPVariable_Wrap(std::move(t)) : PyLong_FromLong(code); }

PyObject *result(int code, at::Tensor &&a, at::Tensor &&b)
{
    if (code != MG_OK) return PyLong_FromLong(code);
    PyObject *pair = PyTuple_New(2);
    if (!pair) return nullptr;
    PyTuple_SET_ITEM(pair, 0, THPVariable_Wrap(std::move(a)));
    PyTuple_SET_ITEM(pair, 1, THPVariable_Wrap(std::move(b)));
    return pair;
}

// (x, format, device, stream) -> (codes, scales)
PyObject *pack(PyObject *const *a, Py_ssize_t n)
{
    plain(n == 4);
    const int64_t format = integer(a[1]), dev = integer(a[2]);
    const at::Tensor &x = dense(a[0], dev);
    const int type = number(x.scalar_type());
    int64_t rows, cols;
    rows_of(x.sizes(), rows, cols);
    at::Tensor codes = make(x, {rows, code_pitch(format, cols)}, at::kByte), scales = make(x, {rows, scale_pitch(cols)}, at::kByte);
    const int rc = pack_fn((int)format, type, rows, cols, x.data_ptr(), cols, (uint8_t *)codes.data_ptr(),
                           (uint8_t *)scales.data_ptr(), (void *)integer(a[3]));
    return result(rc, std::move(codes), std::move(scales));
}

// (codes, scales, shape, format, number type, device, stream) -> tensor
PyObject *unpack(PyObject *const *a, Py_ssize_t n)
{
    plain(n == 7);
    const int64_t format = integer(a[3]), type = integer(a[4]), dev = integer(a[5]);
    const Packed p = packed(a[0], a[1], a[2], format, dev);
    at::Tensor x = make(*p.like, p.shape, scalar(type));
    const int rc = unpack_fn((int)format, (int)type, p.rows, p.cols, p.codes, p.scales, x.data_ptr(), p.cols, (void *)integer(a[6]));
    return result(rc, std::move(x));
}

// (grad, codes, scales, shape, format, natoms or None, device, stream) -> (grad_weight, grad_bias)
PyObject *gradient(PyObject *const *a, Py_ssize_t n)
{
    plain(n == 8);
    const int64_t format = integer(a[4]), dev = integer(a[6]);
    const at::Tensor &grad = dense(a[0], dev);
    const int type = number(grad.scalar_type());
    const Packed p = packed(a[1], a[2], a[3], format, dev);
    plain(grad.dim() == (int64_t)p.shape.size());
    for (size_t i = 0; i + 1 < p.shape.size(); ++i) plain(grad.size(i) == p.shape[i]);
    const int64_t T = grad.size(-1), B = p.shape.size() == 3 ? p.shape[0] : 1, N = p.rows / B;
    plain(T >= 1 && T < INT32_MAX && B < INT32_MAX && N < INT32_MAX && p.cols < INT32_MAX);
    const int32_t *natoms = nullptr;
    if (a[5] != Py_None) {
        const at::Tensor &t = dense(a[5], dev);
        plain(t.scalar_type() == at::kInt && t.dim() == 1 && p.shape.size() == 3 && t.size(0) == B);
        natoms = (const int32_t *)t.data_ptr();
    }
    size_t bytes = 0;
    int rc = gradient_workspace_fn((int)B, (int)N, (int)T, (int)p.cols, &bytes);
    if (rc != MG_OK) return PyLong_FromLong(rc);
    at::Tensor weight = make(grad, {T, p.cols}, at::kFloat), bias = make(grad, {T}, at::kFloat), ws;
    if (bytes) ws = make(grad, {(int64_t)bytes}, at::kByte);
    rc = gradient_fn((int)format, type, (int)B, (int)N, (int)T, (int)p.cols, grad.data_ptr(), T, p.codes, p.scales, natoms,
                     (float *)weight.data_ptr(), (float *)bias.data_ptr(), bytes ? ws.data_ptr() : nullptr, bytes,
                     (void *)integer(a[7]));
    return result(rc, std::move(weight), std::move(bias));
}

// (codes, scales, shape of a; codes, scales, shape of b; bias or None, number type, device, stream) -> tensor
PyObject *product(PyObject *const *a, Py_ssize_t n)
{
    plain(n == 10);
    const int64_t type = integer(a[7]), dev = integer(a[8]);
    Packed x = packed(a[0], a[1], a[2], MG_MX_E2M1, dev);
    const Packed w = packed(a[3], a[4], a[5], MG_MX_E2M1, dev);
    plain(x.cols == w.cols && x.rows < INT32_MAX && w.rows < INT32_MAX && x.cols < INT32_MAX);
    const float *bias = optional_floats(a[6], w.rows, dev);
    x.shape.back() = w.rows;
    at::Tensor out = make(*x.like, x.shape, scalar(type));
    const int rc = product_fn((int)type, (int)x.rows, (int)w.rows, (int)w.cols, x.codes, x.scales, w.codes, w.scales, bias,
                              out.data_ptr(), w.rows, (void *)integer(a[9]));
    return result(rc, std::move(out));
}

// (x; codes, scales, shape of the weight; bias or None, device, stream) -> tensor
PyObject *linear(PyObject *const *a, Py_ssize_t n)
{
    plain(n == 7);
    const int64_t dev = integer(a[5]);
    const at::Tensor &x = dense(a[0], dev);
    const int type = number(x.scalar_type());
    const Packed w = packed(a[1], a[2], a[3], MG_MX_E2M1, dev);
    int64_t rows, cols;
    rows_of(x.sizes(), rows, cols);
    plain(cols == w.cols && rows < INT32_MAX && w.rows < INT32_MAX && cols < INT32_MAX);
    const float *bias = optional_floats(a[4], w.rows, dev);
    size_t bytes = 0;
    int rc = linear_workspace_fn((int)rows, (int)w.rows, (int)cols, &bytes);
    if (rc != MG_OK) return PyLong_FromLong(rc);
    c10::SmallVector<int64_t, 6> shape(x.sizes().begin(), x.sizes().end());
    shape.back() = w.rows;
    at::Tensor out = make(x, shape, x.scalar_type()), ws;
    if (bytes) ws = make(x, {(int64_t)bytes}, at::kByte);
    rc = linear_fn(type, (int)rows, (int)w.rows, (int)cols, x.data_ptr(), cols, w.codes, w.scales, bias, out.data_ptr(), w.rows,
                   bytes ? ws.data_ptr() : nullptr, bytes, (void *)integer(a[6]));
    return result(rc, std::move(out));
}

// torch's own exception for it
void raise_out_of_memory(const char *what)
{
    PyObject *torch = PyImport_ImportModule("torch");
    PyObject *type = torch ? PyObject_GetAttrString(torch, "OutOfMemoryError") : nullptr;
    PyErr_Clear();
    PyErr_SetString(type ? type : PyExc_RuntimeError, what);
    Py_XDECREF(type);
    Py_XDECREF(torch);
}

template <PyObject *(*F)(PyObject *const *, Py_ssize_t)>
PyObject *guarded(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    try {
        plain(linear_fn != nullptr);
        const at::AutoDispatchBelowADInplaceOrView below;      // results carry no history: no need to look for any
        return F(args, n);
    } catch (const NotPlain &) {
        Py_RETURN_NONE;
    } catch (const c10::OutOfMemoryError &e) {
        raise_out_of_memory(e.what_without_backtrace());
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
    }
    return nullptr;
}

// the addresses of the loaded library's functions, in the order above
PyObject *bind(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    void *p[7];
    if (n != 7) {
        PyErr_SetString(PyExc_TypeError, "bind takes seven addresses");
        return nullptr;
    }
    for (int i = 0; i < 7; ++i) {
        p[i] = PyLong_AsVoidPtr(a[i]);
        if (PyErr_Occurred()) return nullptr;
    }
    pack_fn = (decltype(pack_fn))p[0];
    unpack_fn = (decltype(unpack_fn))p[1];
    gradient_workspace_fn = (decltype(gradient_workspace_fn))p[2];
    gradient_fn = (decltype(gradient_fn))p[3];
    product_fn = (decltype(product_fn))p[4];
    linear_workspace_fn = (decltype(linear_workspace_fn))p[5];
    linear_fn = (decltype(linear_fn))p[6];
    Py_RETURN_NONE;
}

#define MG_METHOD(f) {#f, (PyCFunction)(void (*)())guarded<f>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {MG_METHOD(pack), MG_METHOD(unpack), MG_METHOD(gradient), MG_METHOD(product), MG_METHOD(linear),
                         {"bind", (PyCFunction)(void (*)())bind, METH_FASTCALL, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&module); }
