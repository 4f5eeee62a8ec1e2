// The common calls of ops.py in compiled form: the tensors' checks, the
// outputs and the call into libember without the interpreter in between.  A
// small call is bound by the host.  Host time per call on the Grace cores, this
// form against the interpreter with ctypes: the norm of one row 4.4 us against
// 13, in 8 bits 5.7 against 15, its backward pass 6.9 against 17, the 8-bit
// product 3.9 against 12, clipping twelve tensors 6.7 against 19; about 3 us
// of each are the launch, and the rest mostly torch's allocator.
//
// Each function takes the device index and, where it needs them, the
// workspace's address and size and the status block's address, then the
// operator's arguments; it returns the outputs, a status (an int) if libember
// refused the call, or None where the arguments are not the common case (other
// types, devices or strides, a device that is not the current one, a workspace
// that is too small).  ops.py then
// takes its own path, which grows the workspace or names what is wrong.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/empty_strided.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <c10/util/Exception.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstring>
#include <vector>

#include "ember.h"

namespace {

using at::Tensor;

struct Lib {
    decltype(&ember_rmsnorm) rmsnorm;
    decltype(&ember_rmsnorm_quant) rmsnorm_quant;
    decltype(&ember_rmsnorm_backward_workspace_bytes) back_bytes;
    decltype(&ember_rmsnorm_backward) back;
    decltype(&ember_dequantize_rows) dequantize;
    decltype(&ember_matmul_quant_workspace_bytes) matmul_bytes;
    decltype(&ember_matmul_quant) matmul;
    decltype(&ember_softmax_loss_workspace_bytes) loss_bytes;
    decltype(&ember_softmax_loss) loss;
    decltype(&ember_clip_workspace_bytes) clip_bytes;
    decltype(&ember_clip_grads) clip;
    decltype(&ember_grad_norm) norm;
} lib;

constexpr int kInt8 = 100;  // beside ember_wdtype

int type_of(const Tensor &t)
{
    switch (t.scalar_type()) {
    case at::kFloat: return EMBER_F32;
    case at::kBFloat16: return EMBER_BF16;
    case at::kChar: return kInt8;
    default: return -1;
    }
}
at::ScalarType scalar(int type) { return type == EMBER_BF16 ? at::kBFloat16 : at::kFloat; }
bool is_float(int type) { return type == EMBER_F32 || type == EMBER_BF16; }

// A tensor argument as a matrix with unit stride along rows that do not overlap.
struct Mat {
    void *p = nullptr;
    int64_t ld = 0, rows = 0, cols = 0;
    int type = EMBER_F32;
};
bool matrix(PyObject *o, int64_t index, Mat &m)
{
    if (!THPVariable_Check(o))
        return false;
    const Tensor &t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.get_device() != index || t.dim() != 2)
        return false;
    m.rows = t.size(0);
    m.cols = t.size(1);
    m.ld = t.stride(0);
    m.type = type_of(t);
    m.p = t.data_ptr();
    return m.cols > 0 && t.stride(1) == 1 && m.ld >= m.cols && m.type >= 0;
}
bool like(const Mat &a, const Mat &b, int type) { return a.rows == b.rows && a.cols == b.cols && a.type == type; }

// A contiguous vector of n values; its scalar type.
bool vector(PyObject *o, int64_t index, int64_t n, void *&p, at::ScalarType &type)
{
    if (!THPVariable_Check(o))
        return false;
    const Tensor &t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.get_device() != index || t.dim() != 1 || t.size(0) != n || !t.is_contiguous())
        return false;
    p = t.data_ptr();
    type = t.scalar_type();
    return true;
}
bool floats(PyObject *o, int64_t index, int64_t n, void *&p)
{
    at::ScalarType type;
    return vector(o, index, n, p, type) && type == at::kFloat;
}
bool gain_of(PyObject *o, int64_t index, int64_t D, void *&p, int &type)
{
    p = nullptr;
    type = EMBER_F32;
    if (o == Py_None)
        return true;
    at::ScalarType s;
    if (!vector(o, index, D, p, s) || (s != at::kFloat && s != at::kBFloat16))
        return false;
    type = s == at::kBFloat16 ? EMBER_BF16 : EMBER_F32;
    return true;
}

at::TensorOptions on(int64_t index, at::ScalarType type)
{
    return at::TensorOptions().dtype(type).device(at::Device(at::kCUDA, (c10::DeviceIndex)index));
}
void *stream_of(int64_t index) { return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)index).stream(); }

// An output: the argument, if it is like `m` and of `type`, or a new matrix.
bool output(PyObject *o, int64_t index, const Mat &m, int type, Mat &out, PyObject *&keep)
{
    if (o == Py_None) {
        Tensor t = at::empty({m.rows, m.cols}, on(index, scalar(type)));
        out.p = t.data_ptr();
        out.ld = m.cols;
        keep = THPVariable_Wrap(std::move(t));
        return true;
    }
    if (!matrix(o, index, out) || !like(out, m, type))
        return false;
    Py_INCREF(o);
    keep = o;
    return true;
}

// References that are given up unless they are returned.
struct Refs {
    PyObject *r[4] = {nullptr, nullptr, nullptr, nullptr};
    ~Refs()
    {
        for (PyObject *o : r)
            Py_XDECREF(o);
    }
    PyObject *take(int k)
    {
        PyObject *o = r[k];
        r[k] = nullptr;
        if (o)
            return o;
        Py_INCREF(Py_None);
        return Py_None;
    }
};

PyObject *tuple2(Refs &r)
{
    PyObject *a = r.take(0), *b = r.take(1);
    return Py_BuildValue("(NN)", a, b);
}
PyObject *tuple3(Refs &r)
{
    PyObject *a = r.take(0), *b = r.take(1), *c = r.take(2);
    return Py_BuildValue("(NNN)", a, b, c);
}

#define COMMON(condition)   \
    do {                    \
        if (!(condition))   \
            Py_RETURN_NONE; \
    } while (0)
// Without the interpreter's lock: the call takes C values alone.
#define LAUNCHED(call)                         \
    do {                                       \
        void *const stream = stream_of(index); \
        ember_status st_;                      \
        Py_BEGIN_ALLOW_THREADS st_ = (call);   \
        Py_END_ALLOW_THREADS                   \
        if (st_ != EMBER_OK)                   \
            return PyLong_FromLong((long)st_); \
    } while (0)

struct Residual {
    Mat r, h;
};
bool residual_of(PyObject *res, PyObject *out, int64_t index, const Mat &x, Residual &q, PyObject *&keep)
{
    if (res == Py_None)
        return out == Py_None;
    return matrix(res, index, q.r) && is_float(q.r.type) && like(q.r, x, q.r.type) &&
           output(out, index, x, q.r.type, q.h, keep);
}

// (index, x, gain, residual, eps, out, residual_out) -> (y, h)
PyObject *rmsnorm(PyObject *const *a)
{
    const int64_t index = PyLong_AsLongLong(a[0]);
    Mat x, y;
    Residual q;
    void *gain;
    int gtype;
    Refs refs;
    COMMON(PyFloat_Check(a[4]) && matrix(a[1], index, x) && is_float(x.type) && gain_of(a[2], index, x.cols, gain, gtype) &&
           residual_of(a[3], a[6], index, x, q, refs.r[1]) && output(a[5], index, x, x.type, y, refs.r[0]));
    const float eps = (float)PyFloat_AS_DOUBLE(a[4]);
    LAUNCHED(lib.rmsnorm(x.p, x.ld, (ember_wdtype)x.type, q.r.p, q.r.ld, (ember_wdtype)q.r.type, gain,
                         (ember_wdtype)gtype, x.rows, x.cols, eps, q.h.p, q.h.ld, y.p, y.ld,
                         stream));
    return tuple2(refs);
}

// (index, x, gain, residual, eps, residual_out) -> (q, scales, h)
PyObject *rmsnorm_quant(PyObject *const *a)
{
    const int64_t index = PyLong_AsLongLong(a[0]);
    Mat x;
    Residual q;
    void *gain;
    int gtype;
    Refs refs;
    COMMON(PyFloat_Check(a[4]) && matrix(a[1], index, x) && is_float(x.type) && gain_of(a[2], index, x.cols, gain, gtype) &&
           residual_of(a[3], a[5], index, x, q, refs.r[2]));
    const int64_t ld = (x.cols + 15) / 16 * 16;
    Tensor v = at::empty({x.rows, ld}, on(index, at::kChar)), s = at::empty({x.rows}, on(index, at::kFloat));
    const float eps = (float)PyFloat_AS_DOUBLE(a[4]);
    LAUNCHED(lib.rmsnorm_quant(x.p, x.ld, (ember_wdtype)x.type, q.r.p, q.r.ld, (ember_wdtype)q.r.type, gain,
                               (ember_wdtype)gtype, x.rows, x.cols, eps, q.h.p, q.h.ld,
                               static_cast<int8_t *>(v.data_ptr()), ld, static_cast<float *>(s.data_ptr()),
                               stream));
    refs.r[0] = THPVariable_Wrap(ld == x.cols ? v : v.narrow(1, 0, x.cols));
    refs.r[1] = THPVariable_Wrap(std::move(s));
    return tuple3(refs);
}

// (index, workspace, bytes, dy, h, gain, eps, dres, out) -> (dx, dgain)
PyObject *rmsnorm_backward(PyObject *const *a)
{
    const int64_t index = PyLong_AsLongLong(a[0]);
    const size_t bytes = (size_t)PyLong_AsLongLong(a[2]);
    Mat dy, h, dres, dx;
    void *gain;
    int gtype;
    Refs refs;
    COMMON(PyFloat_Check(a[6]) && matrix(a[4], index, h) && is_float(h.type) && matrix(a[3], index, dy) &&
           like(dy, h, h.type) && gain_of(a[5], index, h.cols, gain, gtype) &&
           (a[7] == Py_None || (matrix(a[7], index, dres) && like(dres, h, h.type))));
    COMMON(lib.back_bytes(h.rows, h.cols) <= bytes && output(a[8], index, h, h.type, dx, refs.r[0]));
    Tensor g = at::empty({h.cols}, on(index, at::kFloat));
    const float eps = (float)PyFloat_AS_DOUBLE(a[6]);
    void *work = (void *)PyLong_AsLongLong(a[1]);
    LAUNCHED(lib.back(dy.p, dy.ld, h.p, h.ld, dres.p, dres.ld, (ember_wdtype)h.type, gain, (ember_wdtype)gtype, h.rows,
                      h.cols, eps, dx.p, dx.ld, static_cast<float *>(g.data_ptr()),
                      work, bytes, stream));
    refs.r[1] = THPVariable_Wrap(std::move(g));
    return tuple2(refs);
}

// (index, q, scales, type, out) -> y
PyObject *dequantize_rows(PyObject *const *a)
{
    const int64_t index = PyLong_AsLongLong(a[0]);
    const int type = (int)PyLong_AsLong(a[3]);
    Mat q, y;
    void *s;
    Refs refs;
    COMMON(is_float(type) && matrix(a[1], index, q) && q.type == kInt8 && floats(a[2], index, q.rows, s) &&
           output(a[4], index, q, type, y, refs.r[0]));
    LAUNCHED(lib.dequantize(static_cast<int8_t *>(q.p), q.ld, static_cast<float *>(s), q.rows, q.cols, y.p, y.ld,
                            (ember_wdtype)type, stream));
    return refs.take(0);
}

// (index, workspace, bytes, status, xq, xs, wq, ws, type, out) -> logits
PyObject *matmul_quant(PyObject *const *a)
{
    const int64_t index = PyLong_AsLongLong(a[0]);
    const size_t bytes = (size_t)PyLong_AsLongLong(a[2]);
    const int type = (int)PyLong_AsLong(a[8]);
    Mat x, w, o;
    void *xs, *ws;
    Refs refs;
    COMMON(is_float(type) && matrix(a[4], index, x) && x.type == kInt8 && matrix(a[6], index, w) && w.type == kInt8 && x.cols == w.cols &&
           floats(a[5], index, x.rows, xs) && floats(a[7], index, w.rows, ws) && w.rows > 0);
    Mat shape;
    shape.rows = x.rows;
    shape.cols = w.rows;
    COMMON(lib.matmul_bytes(x.rows, w.rows, x.cols) <= bytes && output(a[9], index, shape, type, o, refs.r[0]));
    void *work = (void *)PyLong_AsLongLong(a[1]);
    unsigned *status = (unsigned *)PyLong_AsLongLong(a[3]);
    LAUNCHED(lib.matmul(static_cast<int8_t *>(x.p), x.ld, static_cast<float *>(xs), static_cast<int8_t *>(w.p), w.ld,
                        static_cast<float *>(ws), x.rows, w.rows, x.cols, o.p, o.ld, (ember_wdtype)type,
                        work, bytes, status, stream));
    return refs.take(0);
}

// (index, workspace, bytes, status, logits, targets, weights, ignore, mean,
// type (-1: no gradient; others are not the common case), out) -> (loss, nll, dlogits)
PyObject *softmax_loss(PyObject *const *a)
{
    const int64_t index = PyLong_AsLongLong(a[0]);
    const size_t bytes = (size_t)PyLong_AsLongLong(a[2]);
    const int type = (int)PyLong_AsLong(a[9]);
    Mat z, d;
    void *y, *w = nullptr;
    at::ScalarType yt;
    Refs refs;
    COMMON(matrix(a[4], index, z) && is_float(z.type) && vector(a[5], index, z.rows, y, yt) &&
           (yt == at::kLong || yt == at::kInt) && (a[6] == Py_None || floats(a[6], index, z.rows, w)) &&
           (type == -1 || is_float(type)) && lib.loss_bytes(z.rows) <= bytes);
    const long long ignore = PyLong_AsLongLong(a[7]);
    if (ignore == -1 && PyErr_Occurred())
        return nullptr;
    if (type >= 0) {
        // rows of the gradient at the same places of their 16-byte units as the logits'
        const int64_t ld = z.ld < z.cols + 64 ? z.ld : (z.cols + 7) / 8 * 8;
        if (a[10] == Py_None && ld != z.cols) {
            Tensor t = at::empty_strided({z.rows, z.cols}, {ld, 1}, on(index, scalar(type)));
            d.p = t.data_ptr();
            d.ld = ld;
            refs.r[2] = THPVariable_Wrap(std::move(t));
        } else
            COMMON(output(a[10], index, z, type, d, refs.r[2]));
    }
    Tensor loss = at::empty({}, on(index, at::kFloat)), nll = at::empty({z.rows}, on(index, at::kFloat));
    const int mean = PyObject_IsTrue(a[8]);
    void *work = (void *)PyLong_AsLongLong(a[1]);
    unsigned *status = (unsigned *)PyLong_AsLongLong(a[3]);
    LAUNCHED(lib.loss(z.p, z.ld, (ember_wdtype)z.type, y, yt == at::kLong ? EMBER_I64 : EMBER_I32,
                      static_cast<float *>(w), ignore, mean, z.rows, z.cols,
                      static_cast<float *>(loss.data_ptr()), static_cast<float *>(nll.data_ptr()), d.p, d.ld,
                      (ember_wdtype)(type >= 0 ? type : EMBER_F32), work, bytes, status, stream));
    refs.r[0] = THPVariable_Wrap(std::move(loss));
    refs.r[1] = THPVariable_Wrap(std::move(nll));
    return tuple3(refs);
}

// grad_norm: (index, workspace, bytes, gradients) -> norm
// clip_grads: (index, workspace, bytes, gradients, max_norm, eps, out) -> norm
// The gradients and outputs are lists.
template <bool SCALE>
PyObject *clip(PyObject *const *a)
{
    const int64_t index = PyLong_AsLongLong(a[0]);
    const size_t bytes = (size_t)PyLong_AsLongLong(a[2]);
    PyObject *outs = SCALE ? a[6] : Py_None;
    COMMON(PyList_Check(a[3]) &&
           (outs == Py_None || (PyList_Check(outs) && PyList_GET_SIZE(outs) == PyList_GET_SIZE(a[3]))));
    if constexpr (SCALE)
        COMMON(PyFloat_Check(a[4]) && PyFloat_Check(a[5]));
    const Py_ssize_t n = PyList_GET_SIZE(a[3]);
    COMMON(n < (1 << 24) && lib.clip_bytes((int)n) <= bytes);
    std::vector<void *> in(n), out(n);
    std::vector<int64_t> numel(n);
    std::vector<int> types(n);
    for (Py_ssize_t k = 0; k < n; ++k) {
        PyObject *o = PyList_GET_ITEM(a[3], k);
        COMMON(THPVariable_Check(o));
        const Tensor &t = THPVariable_Unpack(o);
        types[k] = type_of(t);
        COMMON(t.is_cuda() && t.get_device() == index && t.is_contiguous() && is_float(types[k]));
        in[k] = out[k] = t.data_ptr();
        numel[k] = t.numel();
        if (outs != Py_None) {
            PyObject *p = PyList_GET_ITEM(outs, k);
            COMMON(THPVariable_Check(p));
            const Tensor &u = THPVariable_Unpack(p);
            COMMON(u.is_cuda() && u.get_device() == index && u.is_contiguous() && u.scalar_type() == t.scalar_type() &&
                   u.sizes() == t.sizes());
            out[k] = u.data_ptr();
        }
    }
    Tensor norm = at::empty({}, on(index, at::kFloat));
    float *np = static_cast<float *>(norm.data_ptr());
    void *ws = (void *)PyLong_AsLongLong(a[1]);
    if constexpr (SCALE) {
        const float max_norm = (float)PyFloat_AS_DOUBLE(a[4]), eps = (float)PyFloat_AS_DOUBLE(a[5]);
        LAUNCHED(lib.clip((int)n, in.data(), out.data(), numel.data(), types.data(), max_norm, eps, np, ws, bytes,
                          stream));
    } else
        LAUNCHED(lib.norm((int)n, in.data(), numel.data(), types.data(), np, ws, bytes, stream));
    return THPVariable_Wrap(std::move(norm));
}

template <PyObject *(*F)(PyObject *const *), Py_ssize_t N>
PyObject *entry(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != N) {
        PyErr_Format(PyExc_TypeError, "%zd arguments, not %zd", N, n);
        return nullptr;
    }
    try {
        // libember launches on the current device: another one's call is left to
        // the module, which makes it current (about 0.03 us here, 0.25 there)
        c10::DeviceIndex current;
        if (c10::cuda::GetDevice(&current) != cudaSuccess || current != PyLong_AsLongLong(args[0]))
            Py_RETURN_NONE;
        return F(args);
    } catch (const c10::OutOfMemoryError &) {
        Py_RETURN_NONE;  // before the launch; the module's own path raises torch's exception
    } catch (const std::exception &e) {
        if (!PyErr_Occurred())
            PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        if (!PyErr_Occurred())
            PyErr_SetString(PyExc_RuntimeError, "unknown exception");
    }
    return nullptr;
}

// (addresses of the functions of `lib`, in order)
PyObject *bind(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    void *p[sizeof(Lib) / sizeof(void *)];
    if (n != (Py_ssize_t)(sizeof(p) / sizeof(p[0]))) {
        PyErr_SetString(PyExc_TypeError, "wrong number of functions");
        return nullptr;
    }
    for (Py_ssize_t k = 0; k < n; ++k)
        p[k] = PyLong_AsVoidPtr(args[k]);
    if (PyErr_Occurred())
        return nullptr;
    memcpy(&lib, p, sizeof(lib));
    Py_RETURN_NONE;
}

template <typename F>
PyCFunction fast(F f) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)); }

PyMethodDef methods[] = {
    {"bind", fast(&bind), METH_FASTCALL, nullptr},
    {"rmsnorm", fast(&entry<rmsnorm, 7>), METH_FASTCALL, nullptr},
    {"rmsnorm_quant", fast(&entry<rmsnorm_quant, 6>), METH_FASTCALL, nullptr},
    {"rmsnorm_backward", fast(&entry<rmsnorm_backward, 9>), METH_FASTCALL, nullptr},
    {"dequantize_rows", fast(&entry<dequantize_rows, 5>), METH_FASTCALL, nullptr},
    {"matmul_quant", fast(&entry<matmul_quant, 10>), METH_FASTCALL, nullptr},
    {"softmax_loss", fast(&entry<softmax_loss, 11>), METH_FASTCALL, nullptr},
    {"grad_norm", fast(&entry<clip<false>, 4>), METH_FASTCALL, nullptr},
    {"clip_grads", fast(&entry<clip<true>, 7>), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_ops_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__ops_binding() { return PyModule_Create(&module); }
