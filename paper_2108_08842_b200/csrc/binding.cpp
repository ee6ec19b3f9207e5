// The Python side of the client's training step (the entry points of include/eden.h from
// eden_linear on): argument checks, outputs and the argument blocks, over torch's tensors.
// In C++ because a single token's layer takes 5 us on the GPU and marshalling the same
// arguments through ctypes took 5 us more than that.  It computes nothing.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <cstring>
#include <string>

#include <ATen/ATen.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/eden.h"

namespace {

struct Refused {};                                   // a Python error is set

struct Native {
    eden_ctx* ctx;
    int device;
    cudaStream_t raw;
    c10::Stream stream;
};

struct Library {
    int (*linear)(eden_ctx*, const eden_linear_args*);
    int (*save)(eden_ctx*, const eden_checkpoint_args*);
    int (*restore)(eden_ctx*, const eden_checkpoint_args*);
    int (*act_backward)(eden_ctx*, const eden_act_backward_args*);
    int (*input_grad)(eden_ctx*, const eden_linear_input_grad_args*);
    int (*weight_grad)(eden_ctx*, const eden_linear_weight_grad_args*);
} lib;
PyObject *error_type = nullptr, *checkpoint_type = nullptr;

[[noreturn]] void refuse(const std::string& what)
{
    PyErr_SetString(PyExc_ValueError, ("eden: " + what).c_str());
    throw Refused();
}

std::string described(const at::Tensor& t)
{
    std::string s = std::string(c10::toString(t.scalar_type())) + " [";
    for (int64_t i = 0; i < t.dim(); ++i) s += (i ? ", " : "") + std::to_string(t.size(i));
    return s + "] on " + t.device().str();
}

Native* native_of(PyObject* o)
{
    Native* n = (Native*)PyCapsule_GetPointer(o, "eden.native");
    if (!n) throw Refused();
    return n;
}

bool given(PyObject* o) { return o != Py_None; }
bool left_out(PyObject* o) { return o == Py_False; }   // outputs that a call can do without

const at::Tensor& tensor_of(PyObject* o, const char* name)
{
    if (!THPVariable_Check(o)) refuse(std::string(name) + " has to be a tensor");
    return THPVariable_Unpack(o);
}

const at::Tensor& matrix_of(PyObject* o, const char* name)
{
    const at::Tensor& t = tensor_of(o, name);
    if (t.dim() != 2) refuse(std::string(name) + " has to be a matrix");
    return t;
}

// address and row stride of a CUDA matrix with contiguous rows
struct Matrix {
    void* data = nullptr;
    uint64_t stride = 0;
    Matrix() {}
    Matrix(const Native* n, const at::Tensor& t, const char* name, int64_t rows, int64_t cols, at::ScalarType type)
    {
        if (t.dim() != 2 || t.scalar_type() != type || t.size(0) != rows || t.size(1) != cols || !t.is_cuda() || t.get_device() != n->device)
            refuse(std::string(name) + " has to be " + c10::toString(type) + " [" + std::to_string(rows) + ", " + std::to_string(cols) +
                   "] on cuda:" + std::to_string(n->device) + ", got " + described(t));
        if (cols > 1 && t.stride(1) != 1) refuse(std::string("the rows of ") + name + " have to be contiguous");
        if (rows > 1 && t.stride(0) < cols) refuse(std::string("the rows of ") + name + " overlap");
        data = t.data_ptr();
        stride = (uint64_t)(rows > 1 ? t.stride(0) : cols);
    }
};

void* vector_of(const Native* n, PyObject* o, const char* name, int64_t count, at::ScalarType type)
{
    const at::Tensor& t = tensor_of(o, name);
    if (t.dim() != 1 || t.scalar_type() != type || t.size(0) != count || !t.is_cuda() || t.get_device() != n->device ||
        (count > 1 && t.stride(0) != 1))
        refuse(std::string(name) + " has to be a contiguous " + c10::toString(type) + " [" + std::to_string(count) + "] on cuda:" +
               std::to_string(n->device) + ", got " + described(t));
    return t.data_ptr();
}

int64_t groups_of(int64_t n) { return (n + EDEN_CHECKPOINT_GROUP - 1) / EDEN_CHECKPOINT_GROUP; }

struct Checkpoint {
    at::Tensor codes, exps;
    Matrix c, e;
};

Checkpoint checkpoint_of(const Native* n, PyObject* o, const char* name, int64_t rows, int64_t cols)
{
    if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 2) refuse(std::string(name) + " has to be a pair of codes and exponents");
    Checkpoint c;
    c.codes = tensor_of(PyTuple_GET_ITEM(o, 0), name);
    c.exps = tensor_of(PyTuple_GET_ITEM(o, 1), name);
    c.c = Matrix(n, c.codes, (std::string("the codes of ") + name).c_str(), rows, cols, at::kChar);
    c.e = Matrix(n, c.exps, (std::string("the exponents of ") + name).c_str(), rows, groups_of(cols), at::kByte);
    return c;
}

int32_t type_of(const at::Tensor& t, bool with_fp32, const char* name)
{
    switch (t.scalar_type()) {
        case at::kBFloat16: return EDEN_TYPE_BF16;
        case at::kHalf: return EDEN_TYPE_FP16;
        case at::kFloat:
            if (with_fp32) return EDEN_TYPE_FP32;
        default: refuse(std::string(name) + " has to be bf16" + (with_fp32 ? ", fp16 or fp32" : " or fp16") + ", got " + described(t));
    }
}

int32_t name_of(PyObject* o, const char* what, const char* const* names, int count)
{
    const char* s = PyUnicode_Check(o) ? PyUnicode_AsUTF8(o) : nullptr;
    if (s)
        for (int i = 0; i < count; ++i)
            if (std::strcmp(s, names[i]) == 0) return i;
    PyErr_Clear();
    std::string all;
    for (int i = 0; i < count; ++i) all += std::string(i ? ", " : "") + names[i];
    refuse(std::string(what) + " is not one of " + all);
}

const char* const kActs[] = {"none", "relu", "gelu", "gelu_tanh", "silu"};
const char* const kSaves[] = {"none", "pre", "out"};
int32_t act_of(PyObject* o) { return name_of(o, "act", kActs, 5); }

bool flag_of(PyObject* o)
{
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw Refused();
    return v != 0;
}

bool on_own_stream(const Native* n) { return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)n->device).stream() == n->raw; }

// an output, made on the context's stream whichever stream is current
at::Tensor fresh(const Native* n, at::IntArrayRef sizes, at::ScalarType type)
{
    const auto options = at::TensorOptions().dtype(type).device(at::kCUDA, (c10::DeviceIndex)n->device);
    if (on_own_stream(n)) return at::empty(sizes, options);
    c10::cuda::CUDAStreamGuard guard(c10::cuda::CUDAStream(n->stream));
    return at::empty(sizes, options);
}

// The call's result is in.  Where another stream is current, the tensors' memory stays until the
// context's stream is done with them.
void done(const Native* n, int rc, std::initializer_list<const at::Tensor*> used)
{
    if (rc != 0) {
        PyObject* code = PyLong_FromLong(rc);
        PyErr_SetObject(error_type, code);
        Py_XDECREF(code);
        throw Refused();
    }
    if (!on_own_stream(n))
        for (const at::Tensor* t : used)
            if (t && t->defined()) t->record_stream(n->stream);
}

PyObject* again(PyObject* o)
{
    Py_INCREF(o);
    return o;
}

PyObject* wrapped(const at::Tensor& t) { return THPVariable_Wrap(t); }

// what a call returns for an output
PyObject* returned(PyObject* o, const at::Tensor& made) { return left_out(o) ? again(Py_None) : given(o) ? again(o) : wrapped(made); }

PyObject* pair(PyObject* a, PyObject* b)             // takes both references
{
    PyObject* t = a && b ? PyTuple_Pack(2, a, b) : nullptr;
    Py_XDECREF(a);
    Py_XDECREF(b);
    return t;
}

PyObject* wrapped_checkpoint(const Checkpoint& c)
{
    PyObject *codes = wrapped(c.codes), *exps = wrapped(c.exps);
    PyObject* r = codes && exps ? PyObject_CallFunctionObjArgs(checkpoint_type, codes, exps, nullptr) : nullptr;
    Py_XDECREF(codes);
    Py_XDECREF(exps);
    return r;
}

Checkpoint fresh_checkpoint(const Native* n, int64_t rows, int64_t cols)
{
    Checkpoint c;
    c.codes = fresh(n, {rows, cols}, at::kChar);
    c.exps = fresh(n, {rows, groups_of(cols)}, at::kByte);
    c.c.data = c.codes.data_ptr();
    c.c.stride = (uint64_t)cols;
    c.e.data = c.exps.data_ptr();
    c.e.stride = (uint64_t)groups_of(cols);
    return c;
}

// No C++ exception leaves a function that Python calls.
template <typename F>
PyObject* called(Py_ssize_t got, Py_ssize_t wanted, F&& f)
{
    if (got != wanted) {
        PyErr_Format(PyExc_TypeError, "eden: %zd arguments, got %zd", wanted, got);
        return nullptr;
    }
    try {
        return f();
    } catch (const Refused&) {
        return nullptr;
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// (native, x, weight, bias, act, residual, out, save, saved)
PyObject* linear(PyObject*, PyObject* const* v, Py_ssize_t count)
{
    return called(count, 9, [&]() -> PyObject* {
        const Native* n = native_of(v[0]);
        const at::Tensor &x = matrix_of(v[1], "x"), &weight = matrix_of(v[2], "weight");
        const int64_t m = x.size(0), k = x.size(1), cols = weight.size(0);
        const at::ScalarType t = x.scalar_type();
        eden_linear_args a;
        std::memset(&a, 0, sizeof(a));
        a.type = type_of(x, false, "x");
        a.act = act_of(v[4]);
        a.save = name_of(v[7], "save", kSaves, 3);
        if (!a.save && given(v[8])) refuse("saved is given, but nothing is saved (save is none)");
        const Matrix mx(n, x, "x", m, k, t), mw(n, weight, "weight", cols, k, t);
        a.x = mx.data; a.x_stride = mx.stride;
        a.weight = mw.data; a.weight_stride = mw.stride;
        if (given(v[3])) a.bias = vector_of(n, v[3], "bias", cols, t);
        at::Tensor residual, out = given(v[6]) ? matrix_of(v[6], "out") : fresh(n, {m, cols}, t);
        if (given(v[5])) {
            residual = matrix_of(v[5], "residual");
            const Matrix r(n, residual, "residual", m, cols, t);
            a.residual = r.data; a.residual_stride = r.stride;
        }
        const Matrix mo(n, out, "out", m, cols, t);
        a.y = mo.data; a.y_stride = mo.stride;
        Checkpoint c;
        if (a.save) {
            c = given(v[8]) ? checkpoint_of(n, v[8], "saved", m, cols) : fresh_checkpoint(n, m, cols);
            a.saved = (int8_t*)c.c.data; a.saved_stride = c.c.stride;
            a.saved_exp = (uint8_t*)c.e.data; a.saved_exp_stride = c.e.stride;
        }
        a.m = (uint64_t)m; a.n = (uint64_t)cols; a.k = (uint64_t)k;
        done(n, lib.linear(n->ctx, &a), {&x, &weight, given(v[3]) ? &THPVariable_Unpack(v[3]) : nullptr, &residual, &out, &c.codes, &c.exps});
        PyObject* y = given(v[6]) ? again(v[6]) : wrapped(out);
        return a.save ? pair(y, given(v[8]) ? again(v[8]) : wrapped_checkpoint(c)) : y;
    });
}

// (native, m, n)
PyObject* checkpoint_empty(PyObject*, PyObject* const* v, Py_ssize_t count)
{
    return called(count, 3, [&]() -> PyObject* {
        const int64_t m = PyLong_AsLongLong(v[1]), n = PyLong_AsLongLong(v[2]);
        if (PyErr_Occurred()) throw Refused();
        if (m < 0 || n < 0) refuse("a checkpoint has no negative sizes");
        return wrapped_checkpoint(fresh_checkpoint(native_of(v[0]), m, n));
    });
}

// (native, x, out)
PyObject* checkpoint_save(PyObject*, PyObject* const* v, Py_ssize_t count)
{
    return called(count, 3, [&]() -> PyObject* {
        const Native* n = native_of(v[0]);
        const at::Tensor& x = matrix_of(v[1], "x");
        const int64_t m = x.size(0), cols = x.size(1);
        const int32_t type = type_of(x, true, "x");
        const Matrix mx(n, x, "x", m, cols, x.scalar_type());
        const Checkpoint c = given(v[2]) ? checkpoint_of(n, v[2], "out", m, cols) : fresh_checkpoint(n, m, cols);
        const eden_checkpoint_args a{mx.data, mx.stride, (int8_t*)c.c.data, c.c.stride, (uint8_t*)c.e.data, c.e.stride, (uint64_t)m, (uint64_t)cols, type, 0};
        done(n, lib.save(n->ctx, &a), {&x, &c.codes, &c.exps});
        return given(v[2]) ? again(v[2]) : wrapped_checkpoint(c);
    });
}

// (native, saved, dtype, out)
PyObject* checkpoint_restore(PyObject*, PyObject* const* v, Py_ssize_t count)
{
    return called(count, 4, [&]() -> PyObject* {
        const Native* n = native_of(v[0]);
        if (!THPDtype_Check(v[2])) refuse("a checkpoint is restored to a dtype");
        const at::ScalarType t = ((THPDtype*)v[2])->scalar_type;
        if (t != at::kBFloat16 && t != at::kHalf && t != at::kFloat) refuse("a checkpoint is restored to bf16, fp16 or fp32");
        if (!PyTuple_Check(v[1]) || PyTuple_GET_SIZE(v[1]) != 2) refuse("saved has to be a pair of codes and exponents");
        const at::Tensor& codes = matrix_of(PyTuple_GET_ITEM(v[1], 0), "the codes of saved");
        const int64_t m = codes.size(0), cols = codes.size(1);
        const Checkpoint c = checkpoint_of(n, v[1], "saved", m, cols);
        const at::Tensor out = given(v[3]) ? matrix_of(v[3], "out") : fresh(n, {m, cols}, t);
        const Matrix mo(n, out, "out", m, cols, t);
        const eden_checkpoint_args a{mo.data, mo.stride, (int8_t*)c.c.data, c.c.stride, (uint8_t*)c.e.data, c.e.stride, (uint64_t)m, (uint64_t)cols,
                                     type_of(out, true, "out"), 0};
        done(n, lib.restore(n->ctx, &a), {&out, &c.codes, &c.exps});
        return given(v[3]) ? again(v[3]) : wrapped(out);
    });
}

// fp32 sums over a matrix's columns: the given vector, or a fresh one that nothing is added to
at::Tensor sums_of(const Native* n, PyObject* o, const char* name, int64_t cols, bool accumulate)
{
    if (given(o)) {
        vector_of(n, o, name, cols, at::kFloat);
        return THPVariable_Unpack(o);
    }
    if (accumulate) refuse(std::string("accumulate needs a ") + name + " to add to");
    return fresh(n, {cols}, at::kFloat);
}

// (native, dy, pre, act, out, bias_grad, accumulate)
PyObject* act_backward(PyObject*, PyObject* const* v, Py_ssize_t count)
{
    return called(count, 7, [&]() -> PyObject* {
        const Native* n = native_of(v[0]);
        const at::Tensor& dy = matrix_of(v[1], "dy");
        const int64_t m = dy.size(0), cols = dy.size(1);
        const at::ScalarType t = dy.scalar_type();
        eden_act_backward_args a;
        std::memset(&a, 0, sizeof(a));
        a.type = type_of(dy, false, "dy");
        a.act = act_of(v[3]);
        a.accumulate = flag_of(v[6]);
        const Matrix md(n, dy, "dy", m, cols, t);
        a.dy = md.data; a.dy_stride = md.stride;
        Checkpoint pre;
        if (given(v[2])) pre = checkpoint_of(n, v[2], "pre", m, cols);
        if (a.act) {
            if (!given(v[2])) refuse("the slope of an activation needs its pre-activation");
            a.pre = (const int8_t*)pre.c.data; a.pre_stride = pre.c.stride;
            a.pre_exp = (const uint8_t*)pre.e.data; a.pre_exp_stride = pre.e.stride;
        }
        if (left_out(v[4]) && left_out(v[5])) refuse("out and bias_grad are both left out");
        at::Tensor out, sums;
        if (!left_out(v[4])) {
            out = given(v[4]) ? matrix_of(v[4], "out") : fresh(n, {m, cols}, t);
            const Matrix mo(n, out, "out", m, cols, t);
            a.dz = mo.data; a.dz_stride = mo.stride;
        }
        if (left_out(v[5]) && a.accumulate) refuse("accumulate needs a bias_grad to add to");
        if (!left_out(v[5])) {
            sums = sums_of(n, v[5], "bias_grad", cols, a.accumulate);
            a.bias_grad = (float*)sums.data_ptr();
        }
        a.m = (uint64_t)m; a.n = (uint64_t)cols;
        done(n, lib.act_backward(n->ctx, &a), {&dy, &pre.codes, &pre.exps, &out, &sums});
        return pair(returned(v[4], out), returned(v[5], sums));
    });
}

// (native, dz, weight, residual, pre, act, out, bias_grad, accumulate)
PyObject* input_grad(PyObject*, PyObject* const* v, Py_ssize_t count)
{
    return called(count, 9, [&]() -> PyObject* {
        const Native* n = native_of(v[0]);
        const at::Tensor &dz = matrix_of(v[1], "dz"), &weight = matrix_of(v[2], "weight");
        const int64_t m = dz.size(0), cols = dz.size(1), k = weight.size(1);
        const at::ScalarType t = dz.scalar_type();
        eden_linear_input_grad_args a;
        std::memset(&a, 0, sizeof(a));
        a.type = type_of(dz, false, "dz");
        a.act = act_of(v[5]);
        a.accumulate = flag_of(v[8]);
        const Matrix md(n, dz, "dz", m, cols, t), mw(n, weight, "weight", cols, k, t);
        a.dz = md.data; a.dz_stride = md.stride;
        a.weight = mw.data; a.weight_stride = mw.stride;
        at::Tensor residual;
        if (given(v[3])) {
            residual = matrix_of(v[3], "residual");
            const Matrix r(n, residual, "residual", m, k, t);
            a.residual = r.data; a.residual_stride = r.stride;
        }
        Checkpoint pre;
        if (given(v[4])) pre = checkpoint_of(n, v[4], "pre", m, k);
        if (a.act) {
            if (!given(v[4])) refuse("the slope of an activation needs its pre-activation");
            a.pre = (const int8_t*)pre.c.data; a.pre_stride = pre.c.stride;
            a.pre_exp = (const uint8_t*)pre.e.data; a.pre_exp_stride = pre.e.stride;
        }
        const at::Tensor out = given(v[6]) ? matrix_of(v[6], "out") : fresh(n, {m, k}, t);
        const Matrix mo(n, out, "out", m, k, t);
        a.dx = mo.data; a.dx_stride = mo.stride;
        at::Tensor sums;
        const bool summed = !left_out(v[7]) && (given(v[4]) || given(v[7]) || a.accumulate);
        if (left_out(v[7]) && a.accumulate) refuse("accumulate needs a bias_grad to add to");
        if (summed) {
            sums = sums_of(n, v[7], "bias_grad", k, a.accumulate);
            a.bias_grad = (float*)sums.data_ptr();
        }
        a.m = (uint64_t)m; a.n = (uint64_t)cols; a.k = (uint64_t)k;
        done(n, lib.input_grad(n->ctx, &a), {&dz, &weight, &residual, &pre.codes, &pre.exps, &out, &sums});
        PyObject* dx = given(v[6]) ? again(v[6]) : wrapped(out);
        return summed ? pair(dx, given(v[7]) ? again(v[7]) : wrapped(sums)) : dx;
    });
}

// (native, dz, x, out, accumulate)
PyObject* weight_grad(PyObject*, PyObject* const* v, Py_ssize_t count)
{
    return called(count, 5, [&]() -> PyObject* {
        const Native* n = native_of(v[0]);
        const at::Tensor& dz = matrix_of(v[1], "dz");
        const int64_t m = dz.size(0), cols = dz.size(1);
        const at::ScalarType t = dz.scalar_type();
        eden_linear_weight_grad_args a;
        std::memset(&a, 0, sizeof(a));
        a.type = type_of(dz, false, "dz");
        a.accumulate = flag_of(v[4]);
        const Matrix md(n, dz, "dz", m, cols, t);
        a.dz = md.data; a.dz_stride = md.stride;
        at::Tensor x;
        Checkpoint held;
        int64_t k;
        if (THPVariable_Check(v[2])) {
            x = matrix_of(v[2], "x");
            k = x.size(1);
            const Matrix mx(n, x, "x", m, k, t);
            a.x = mx.data; a.x_stride = mx.stride;
        } else {
            if (!PyTuple_Check(v[2]) || PyTuple_GET_SIZE(v[2]) != 2) refuse("x has to be a tensor or a pair of codes and exponents");
            k = matrix_of(PyTuple_GET_ITEM(v[2], 0), "the codes of x").size(1);
            held = checkpoint_of(n, v[2], "x", m, k);
            a.codes = (const int8_t*)held.c.data; a.codes_stride = held.c.stride;
            a.exps = (const uint8_t*)held.e.data; a.exps_stride = held.e.stride;
        }
        if (a.accumulate && !given(v[3])) refuse("accumulate needs an out to add to");
        const at::Tensor out = given(v[3]) ? matrix_of(v[3], "out") : fresh(n, {cols, k}, at::kFloat);
        const Matrix mo(n, out, "out", cols, k, at::kFloat);
        a.weight_grad = (float*)mo.data; a.weight_grad_stride = mo.stride;
        a.m = (uint64_t)m; a.n = (uint64_t)cols; a.k = (uint64_t)k;
        done(n, lib.weight_grad(n->ctx, &a), {&dz, &x, &held.codes, &held.exps, &out});
        return given(v[3]) ? again(v[3]) : wrapped(out);
    });
}

// (context, device, stream, stream's id, device index and device type) -> handle
PyObject* native(PyObject*, PyObject* const* v, Py_ssize_t count)
{
    return called(count, 6, [&]() -> PyObject* {
        long long f[6];
        for (int i = 0; i < 6; ++i) f[i] = (long long)PyLong_AsUnsignedLongLongMask(v[i]);
        if (PyErr_Occurred()) throw Refused();
        Native* n = new Native{(eden_ctx*)f[0], (int)f[1], (cudaStream_t)f[2], c10::Stream::unpack3(f[3], (c10::DeviceIndex)f[4], (c10::DeviceType)f[5])};
        PyObject* o = PyCapsule_New(n, "eden.native", [](PyObject* c) { delete (Native*)PyCapsule_GetPointer(c, "eden.native"); });
        if (!o) delete n;
        return o;
    });
}

// (handle): its calls are refused from now on
PyObject* close_native(PyObject*, PyObject* const* v, Py_ssize_t count)
{
    return called(count, 1, [&]() -> PyObject* {
        native_of(v[0])->ctx = nullptr;
        Py_RETURN_NONE;
    });
}

// (the six entry points' addresses in the order of Library, EdenError, Checkpoint)
PyObject* bind(PyObject*, PyObject* const* v, Py_ssize_t count)
{
    return called(count, 8, [&]() -> PyObject* {
        void* f[6];
        for (int i = 0; i < 6; ++i) f[i] = PyLong_AsVoidPtr(v[i]);
        if (PyErr_Occurred()) throw Refused();
        std::memcpy(&lib, f, sizeof(lib));
        Py_XDECREF(error_type);
        Py_XDECREF(checkpoint_type);
        error_type = again(v[6]);
        checkpoint_type = again(v[7]);
        Py_RETURN_NONE;
    });
}

#define EDEN_METHOD(name, function) {name, (PyCFunction)(void (*)())(function), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {EDEN_METHOD("bind", bind),
                         EDEN_METHOD("native", native),
                         EDEN_METHOD("close", close_native),
                         EDEN_METHOD("linear", linear),
                         EDEN_METHOD("checkpoint_empty", checkpoint_empty),
                         EDEN_METHOD("checkpoint_save", checkpoint_save),
                         EDEN_METHOD("checkpoint_restore", checkpoint_restore),
                         EDEN_METHOD("act_backward", act_backward),
                         EDEN_METHOD("input_grad", input_grad),
                         EDEN_METHOD("weight_grad", weight_grad),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// `built_for`: the torch and the Python whose interfaces this was compiled against
PyMODINIT_FUNC PyInit__binding(void)
{
    PyObject* module = PyModule_Create(&module_def);
    if (module && PyModule_AddStringConstant(module, "built_for", EDEN_BUILT_FOR) != 0) Py_CLEAR(module);
    return module;
}
