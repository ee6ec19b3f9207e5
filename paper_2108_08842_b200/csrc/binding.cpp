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
    int (*join)(eden_ctx*, const eden_block_join_args*);
    int (*join_backward)(eden_ctx*, const eden_block_join_backward_args*);
    int (*mx4_quantize)(eden_ctx*, const eden_mx4_quantize_args*);
    int (*mx4_restore)(eden_ctx*, const eden_mx4_restore_args*);
    int (*mx4_linear)(eden_ctx*, const eden_mx4_linear_args*);
    int (*mx4_input_grad)(eden_ctx*, const eden_mx4_linear_input_grad_args*);
    int (*mx4_weight_grad)(eden_ctx*, const eden_mx4_linear_weight_grad_args*);
} lib;
constexpr int kCalls = sizeof(Library) / sizeof(void*);
PyObject *error_type = nullptr, *checkpoint_type = nullptr, *mx4_type = nullptr;

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

// ---- what joins the blocks ----------------------------------------------------------------
const char* const kNorms[] = {"none", "rms", "layer"};

double number_of(PyObject* o, const char* name)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) {
        PyErr_Clear();
        refuse(std::string(name) + " has to be a number");
    }
    return v;
}

uint64_t count_of(PyObject* o, const char* name)
{
    const unsigned long long v = PyLong_Check(o) ? PyLong_AsUnsignedLongLong(o) : (unsigned long long)-1;
    if (!PyLong_Check(o) || PyErr_Occurred()) {
        PyErr_Clear();
        refuse(std::string(name) + " has to be a whole number from 0 to 2^64 - 1");
    }
    return v;
}

// a norm (weight, bias, kind, eps), or None; the names of it and of its parts
struct NormNames {
    const char *norm, *weight, *bias, *kind, *eps;
};
constexpr NormNames kAfterNames{"after", "the weight of after", "the bias of after", "the kind of after", "eps of after"};
constexpr NormNames kBeforeNames{"before", "the weight of before", "the bias of before", "the kind of before", "eps of before"};

eden_norm norm_of(const Native* n, PyObject* o, const NormNames& names, int64_t cols, at::ScalarType t)
{
    eden_norm r;
    std::memset(&r, 0, sizeof(r));
    if (!given(o)) return r;
    if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 4) refuse(std::string(names.norm) + " has to be a Norm");
    if (given(PyTuple_GET_ITEM(o, 0))) r.weight = vector_of(n, PyTuple_GET_ITEM(o, 0), names.weight, cols, t);
    if (given(PyTuple_GET_ITEM(o, 1))) r.bias = vector_of(n, PyTuple_GET_ITEM(o, 1), names.bias, cols, t);
    r.kind = name_of(PyTuple_GET_ITEM(o, 2), names.kind, kNorms, 3);
    r.eps = (float)number_of(PyTuple_GET_ITEM(o, 3), names.eps);
    if (!(r.eps >= 0.f) || r.eps > 1e30f) refuse(std::string(names.eps) + " has to be a finite number from 0 on");
    if (r.kind == EDEN_NORM_NONE) r.weight = r.bias = nullptr;
    return r;
}

eden_drop drop_of(const Native* n, PyObject* rate, PyObject* seed, PyObject* first_row)
{
    eden_drop d;
    std::memset(&d, 0, sizeof(d));
    d.rate = number_of(rate, "drop");
    if (!(d.rate >= 0.0 && d.rate <= 1.0)) refuse("drop has to be from 0 to 1");
    d.first_row = count_of(first_row, "first_row");
    if (THPVariable_Check(seed)) {
        const at::Tensor& t = THPVariable_Unpack(seed);
        if (t.scalar_type() != at::kLong || t.numel() != 1 || !t.is_cuda() || t.get_device() != n->device)
            refuse("seed has to be a whole number, or one int64 on cuda:" + std::to_string(n->device) + ", got " + described(t));
        d.seed_at = (const uint64_t*)t.data_ptr();
    } else {
        d.seed = count_of(seed, "seed");
    }
    return d;
}

// a gate: one value per column, or a matrix
const void* gate_of(const Native* n, PyObject* o, int64_t rows, int64_t cols, at::ScalarType t, uint64_t* stride, int32_t* per_value)
{
    *stride = 0;
    *per_value = 0;
    if (!given(o)) return nullptr;
    const at::Tensor& gate = tensor_of(o, "gate");
    if (gate.dim() != 2) return vector_of(n, o, "gate", cols, t);
    const Matrix m(n, gate, "gate", rows, cols, t);
    *stride = m.stride;
    *per_value = 1;
    return m.data;
}

const at::Tensor* tensor_in(PyObject* o) { return THPVariable_Check(o) ? &THPVariable_Unpack(o) : nullptr; }
const at::Tensor* tensor_in(PyObject* o, int i) { return PyTuple_Check(o) && PyTuple_GET_SIZE(o) > i ? tensor_in(PyTuple_GET_ITEM(o, i)) : nullptr; }

float* stats_of(const Native* n, PyObject* o, const char* name, int64_t rows)
{
    const at::Tensor& t = tensor_of(o, name);
    if (t.dim() != 2 || t.scalar_type() != at::kFloat || t.size(0) != rows || t.size(1) != 2 || !t.is_cuda() || t.get_device() != n->device || !t.is_contiguous())
        refuse(std::string(name) + " has to be a contiguous Float [" + std::to_string(rows) + ", 2] on cuda:" + std::to_string(n->device) + ", got " + described(t));
    if ((uintptr_t)t.data_ptr() & 7) refuse(std::string(name) + " has to start on 8 bytes");
    return (float*)t.data_ptr();
}

// (native, h, residual, after, before, gate, scale, drop, seed, first_row, out, normed, stats)
//   -> (x, y, after_stats, before_stats)
PyObject* join(PyObject*, PyObject* const* v, Py_ssize_t count)
{
    return called(count, 13, [&]() -> PyObject* {
        const Native* n = native_of(v[0]);
        const at::Tensor& h = matrix_of(v[1], "h");
        const int64_t m = h.size(0), cols = h.size(1);
        const at::ScalarType t = h.scalar_type();
        eden_block_join_args a;
        std::memset(&a, 0, sizeof(a));
        a.type = type_of(h, false, "h");
        const Matrix mh(n, h, "h", m, cols, t);
        a.h = mh.data; a.h_stride = mh.stride;
        a.after = norm_of(n, v[3], kAfterNames, cols, t);
        a.before = norm_of(n, v[4], kBeforeNames, cols, t);
        a.gate = gate_of(n, v[5], m, cols, t, &a.gate_stride, &a.gate_per_value);
        a.scale = (float)number_of(v[6], "scale");
        a.drop = drop_of(n, v[7], v[8], v[9]);
        at::Tensor residual, x, y, after_stats, before_stats;
        if (given(v[2])) {
            residual = matrix_of(v[2], "residual");
            const Matrix r(n, residual, "residual", m, cols, t);
            a.residual = r.data; a.residual_stride = r.stride;
        }
        if (!left_out(v[10])) {
            x = given(v[10]) ? matrix_of(v[10], "out") : fresh(n, {m, cols}, t);
            const Matrix mx(n, x, "out", m, cols, t);
            a.x = mx.data; a.x_stride = mx.stride;
        } else if (!a.before.kind) {
            refuse("out is left out, and there is no norm before");
        }
        if (a.before.kind) {
            if (left_out(v[11])) refuse("normed cannot be left out of a call with a norm before");
            y = given(v[11]) ? matrix_of(v[11], "normed") : fresh(n, {m, cols}, t);
            const Matrix my(n, y, "normed", m, cols, t);
            a.y = my.data; a.y_stride = my.stride;
        } else if (given(v[11]) && !left_out(v[11])) {
            refuse("normed is given, but there is no norm before");
        }
        if (flag_of(v[12])) {
            if (a.after.kind) a.after_stats = (float*)(after_stats = fresh(n, {m, 2}, at::kFloat)).data_ptr();
            if (a.before.kind) a.before_stats = (float*)(before_stats = fresh(n, {m, 2}, at::kFloat)).data_ptr();
        }
        a.m = (uint64_t)m; a.n = (uint64_t)cols;
        done(n, lib.join(n->ctx, &a), {&h, &residual, &x, &y, &after_stats, &before_stats, tensor_in(v[3], 0), tensor_in(v[3], 1), tensor_in(v[4], 0),
                                       tensor_in(v[4], 1), tensor_in(v[5]), tensor_in(v[8])});
        PyObject* r = PyTuple_New(4);
        if (!r) return nullptr;
        PyTuple_SET_ITEM(r, 0, returned(v[10], x));
        PyTuple_SET_ITEM(r, 1, !a.before.kind ? again(Py_None) : given(v[11]) ? again(v[11]) : wrapped(y));
        PyTuple_SET_ITEM(r, 2, after_stats.defined() ? wrapped(after_stats) : again(Py_None));
        PyTuple_SET_ITEM(r, 3, before_stats.defined() ? wrapped(before_stats) : again(Py_None));
        return r;
    });
}

// an activation that was kept: a matrix of type t, or a checkpoint
eden_kept kept_of(const Native* n, PyObject* o, const char* name, int64_t rows, int64_t cols, at::ScalarType t)
{
    eden_kept k;
    std::memset(&k, 0, sizeof(k));
    if (THPVariable_Check(o)) {
        const Matrix m(n, THPVariable_Unpack(o), name, rows, cols, t);
        k.data = m.data; k.stride = m.stride;
    } else {
        const Checkpoint c = checkpoint_of(n, o, name, rows, cols);
        k.codes = (const int8_t*)c.c.data; k.codes_stride = c.c.stride;
        k.exps = (const uint8_t*)c.e.data; k.exps_stride = c.e.stride;
    }
    return k;
}

// (native, dx, dy, h, x, after_stats, before_stats, after, before, gate, scale, drop, seed, first_row, residual, out, gate_grad,
//  after_weight_grad, after_bias_grad, before_weight_grad, before_bias_grad, accumulate)
//   -> (residual, h, gate, after weight, after bias, before weight, before bias)
PyObject* join_backward(PyObject*, PyObject* const* v, Py_ssize_t count)
{
    return called(count, 22, [&]() -> PyObject* {
        const Native* n = native_of(v[0]);
        if (!given(v[1]) && !given(v[2])) refuse("dx and dy are both left out");
        const at::Tensor& leading = given(v[1]) ? matrix_of(v[1], "dx") : matrix_of(v[2], "dy");
        const int64_t m = leading.size(0), cols = leading.size(1);
        const at::ScalarType t = leading.scalar_type();
        eden_block_join_backward_args a;
        std::memset(&a, 0, sizeof(a));
        a.type = type_of(leading, false, given(v[1]) ? "dx" : "dy");
        a.after = norm_of(n, v[7], kAfterNames, cols, t);
        a.before = norm_of(n, v[8], kBeforeNames, cols, t);
        a.gate = gate_of(n, v[9], m, cols, t, &a.gate_stride, &a.gate_per_value);
        a.scale = (float)number_of(v[10], "scale");
        a.drop = drop_of(n, v[11], v[12], v[13]);
        a.accumulate = flag_of(v[21]);
        if (given(v[1])) {
            const Matrix d(n, leading, "dx", m, cols, t);
            a.dx = d.data; a.dx_stride = d.stride;
        }
        if (given(v[2])) {
            if (!a.before.kind) refuse("dy is given, but there is no norm before");
            const Matrix d(n, matrix_of(v[2], "dy"), "dy", m, cols, t);
            a.dy = d.data; a.dy_stride = d.stride;
        } else if (a.before.kind) {
            refuse("a norm before needs its gradient dy");
        }
        if (a.before.kind) {
            if (!given(v[4])) refuse("the gradient of the norm before needs x");
            a.x = kept_of(n, v[4], "x", m, cols, t);
            a.before_stats = stats_of(n, v[6], "before_stats", m);
        }
        if (a.after.kind || a.gate) {
            if (!given(v[3])) refuse("the gradients of a norm after and of a gate need h");
            a.h = kept_of(n, v[3], "h", m, cols, t);
        }
        if (a.after.kind) a.after_stats = stats_of(n, v[5], "after_stats", m);
        auto matrix = [&](PyObject* o, const char* name, at::Tensor& made, void*& data, uint64_t& stride) {
            if (left_out(o)) return;
            made = given(o) ? matrix_of(o, name) : fresh(n, {m, cols}, t);
            const Matrix d(n, made, name, m, cols, t);
            data = d.data; stride = d.stride;
        };
        at::Tensor residual, dh, gate, sums[4];
        matrix(v[14], "residual", residual, a.d_residual, a.d_residual_stride);
        matrix(v[15], "out", dh, a.dh, a.dh_stride);
        if (!a.gate && given(v[16]) && !left_out(v[16])) refuse("gate_grad is given, but there is no gate");
        auto vector = [&](PyObject* o, const char* name, bool wanted, bool there, at::Tensor& made, float*& data) {
            if (left_out(o)) return;
            if (given(o) && !there) refuse(std::string(name) + " is given, but there is nothing that it is the gradient of");
            if (!given(o) && !wanted) return;
            made = sums_of(n, o, name, cols, a.accumulate);
            data = (float*)made.data_ptr();
        };
        if (a.gate && a.gate_per_value) matrix(v[16], "gate_grad", gate, a.d_gate, a.d_gate_stride);
        else if (a.gate) vector(v[16], "gate_grad", true, true, gate, a.gate_sum);
        vector(v[17], "after_weight_grad", a.after.weight != nullptr, a.after.kind != 0, sums[0], a.after_weight_grad);
        vector(v[18], "after_bias_grad", a.after.bias != nullptr, a.after.kind != 0, sums[1], a.after_bias_grad);
        vector(v[19], "before_weight_grad", a.before.weight != nullptr, a.before.kind != 0, sums[2], a.before_weight_grad);
        vector(v[20], "before_bias_grad", a.before.bias != nullptr, a.before.kind != 0, sums[3], a.before_bias_grad);
        a.m = (uint64_t)m; a.n = (uint64_t)cols;
        done(n, lib.join_backward(n->ctx, &a),
             {tensor_in(v[1]), tensor_in(v[2]), tensor_in(v[3]), tensor_in(v[3], 0), tensor_in(v[3], 1), tensor_in(v[4]), tensor_in(v[4], 0), tensor_in(v[4], 1),
              tensor_in(v[5]), tensor_in(v[6]), tensor_in(v[7], 0), tensor_in(v[7], 1), tensor_in(v[8], 0), tensor_in(v[8], 1), tensor_in(v[9]), tensor_in(v[12]),
              &residual, &dh, &gate, &sums[0], &sums[1], &sums[2], &sums[3]});
        const at::Tensor* const made[7] = {&residual, &dh, &gate, &sums[0], &sums[1], &sums[2], &sums[3]};
        PyObject* r = PyTuple_New(7);
        if (!r) return nullptr;
        for (int i = 0; i < 7; ++i) {
            PyObject* const o = v[14 + i];
            PyTuple_SET_ITEM(r, i, !made[i]->defined() ? again(Py_None) : given(o) ? again(o) : wrapped(*made[i]));
        }
        return r;
    });
}

// ---- 4 bits -------------------------------------------------------------------------------
int64_t tiles_of(int64_t n, int64_t tile) { return (n + tile - 1) / tile; }

struct Mx4 {
    at::Tensor codes, exps;
    int64_t features = 0;
    eden_mx4 view() const { return {(uint8_t*)codes.data_ptr(), (uint64_t)(codes.size(0) > 1 ? codes.stride(0) : codes.size(1)), (uint8_t*)exps.data_ptr()}; }
};

bool is_mx4(PyObject* o) { return PyTuple_Check(o) && PyTuple_GET_SIZE(o) == 3; }

// rows or features below 0: any
Mx4 mx4_of(const Native* n, PyObject* o, const char* name, int64_t rows, int64_t features)
{
    if (!is_mx4(o)) refuse(std::string(name) + " has to be an Mx4");
    Mx4 q;
    q.codes = tensor_of(PyTuple_GET_ITEM(o, 0), name);
    q.exps = tensor_of(PyTuple_GET_ITEM(o, 1), name);
    q.features = PyLong_Check(PyTuple_GET_ITEM(o, 2)) ? PyLong_AsLongLong(PyTuple_GET_ITEM(o, 2)) : -1;
    if (PyErr_Occurred() || q.features < 1 || q.features > 0x7FFFFFFF) {
        PyErr_Clear();
        refuse(std::string("the features of ") + name + " have to be a whole number from 1 on");
    }
    if (q.codes.dim() != 2 || (features >= 0 && q.features != features) || (rows >= 0 && q.codes.size(0) != rows))
        refuse(std::string(name) + " has to hold [" + (rows >= 0 ? std::to_string(rows) : "rows") + ", " + (features >= 0 ? std::to_string(features) : "features") +
               "] values, got features " + std::to_string(q.features) + " and codes " + described(q.codes));
    const Matrix codes(n, q.codes, name, q.codes.size(0), groups_of(q.features) * 16, at::kByte);
    if ((uintptr_t)codes.data & 15 || codes.stride & 15) refuse(std::string("the rows of the codes of ") + name + " have to start on 16 bytes");
    const int64_t across = tiles_of(q.codes.size(0), 128), along = tiles_of(q.features, 256);
    if (q.exps.dim() != 3 || q.exps.scalar_type() != at::kByte || q.exps.size(0) != across || q.exps.size(1) != along || q.exps.size(2) != 1024 || !q.exps.is_cuda() ||
        q.exps.get_device() != n->device || !q.exps.is_contiguous() || (uintptr_t)q.exps.data_ptr() & 15)
        refuse(std::string("the exponents of ") + name + " have to be contiguous Byte [" + std::to_string(across) + ", " + std::to_string(along) + ", 1024] on cuda:" +
               std::to_string(n->device) + " and 16 bytes, got " + described(q.exps));
    return q;
}

Mx4 fresh_mx4(const Native* n, int64_t rows, int64_t features)
{
    Mx4 q;
    q.codes = fresh(n, {rows, groups_of(features) * 16}, at::kByte);
    q.exps = fresh(n, {tiles_of(rows, 128), tiles_of(features, 256), 1024}, at::kByte);
    q.features = features;
    return q;
}

PyObject* wrapped_mx4(const Mx4& q)
{
    PyObject *codes = wrapped(q.codes), *exps = wrapped(q.exps), *features = PyLong_FromLongLong(q.features);
    PyObject* r = codes && exps && features ? PyObject_CallFunctionObjArgs(mx4_type, codes, exps, features, nullptr) : nullptr;
    Py_XDECREF(codes);
    Py_XDECREF(exps);
    Py_XDECREF(features);
    return r;
}

// (native, rows, features)
PyObject* mx4_empty(PyObject*, PyObject* const* v, Py_ssize_t count)
{
    return called(count, 3, [&]() -> PyObject* {
        const int64_t m = PyLong_AsLongLong(v[1]), n = PyLong_AsLongLong(v[2]);
        if (PyErr_Occurred()) throw Refused();
        if (m < 0 || n < 1) refuse("an Mx4 has rows from 0 and features from 1 on");
        return wrapped_mx4(fresh_mx4(native_of(v[0]), m, n));
    });
}

// (native, x, rows, columns): each an Mx4, None (made) or False (left out)
PyObject* mx4_quantize(PyObject*, PyObject* const* v, Py_ssize_t count)
{
    return called(count, 4, [&]() -> PyObject* {
        const Native* n = native_of(v[0]);
        const at::Tensor& x = matrix_of(v[1], "x");
        const int64_t m = x.size(0), cols = x.size(1);
        eden_mx4_quantize_args a;
        std::memset(&a, 0, sizeof(a));
        a.type = type_of(x, true, "x");
        const Matrix mx(n, x, "x", m, cols, x.scalar_type());
        a.x = mx.data; a.x_stride = mx.stride;
        if (cols < 1) refuse("x has no features");
        if (!left_out(v[3]) && m < 1) refuse("the columns of a matrix without rows have no groups");
        Mx4 rows, columns;
        if (!left_out(v[2])) {
            rows = given(v[2]) ? mx4_of(n, v[2], "out", m, cols) : fresh_mx4(n, m, cols);
            a.rows = rows.view();
        }
        if (!left_out(v[3])) {
            columns = given(v[3]) ? mx4_of(n, v[3], "out", cols, m) : fresh_mx4(n, cols, m);
            a.columns = columns.view();
        }
        a.m = (uint64_t)m; a.n = (uint64_t)cols;
        if (m > 0) done(n, lib.mx4_quantize(n->ctx, &a), {&x, &rows.codes, &rows.exps, &columns.codes, &columns.exps});
        auto result = [&](PyObject* o, const Mx4& q) { return given(o) ? again(o) : wrapped_mx4(q); };
        if (left_out(v[3])) return result(v[2], rows);
        if (left_out(v[2])) return result(v[3], columns);
        return pair(result(v[2], rows), result(v[3], columns));
    });
}

at::ScalarType scalar_of(PyObject* o, const char* what, bool with_fp32)
{
    if (!THPDtype_Check(o)) refuse(std::string(what) + " has to be a dtype");
    const at::ScalarType t = ((THPDtype*)o)->scalar_type;
    if (t != at::kBFloat16 && t != at::kHalf && !(with_fp32 && t == at::kFloat)) refuse(std::string(what) + " has to be bf16" + (with_fp32 ? ", fp16 or fp32" : " or fp16"));
    return t;
}

// (native, q, dtype, out)
PyObject* mx4_restore(PyObject*, PyObject* const* v, Py_ssize_t count)
{
    return called(count, 4, [&]() -> PyObject* {
        const Native* n = native_of(v[0]);
        const at::ScalarType t = scalar_of(v[2], "dtype", true);
        const Mx4 q = mx4_of(n, v[1], "q", -1, -1);
        const int64_t m = q.codes.size(0);
        const at::Tensor out = given(v[3]) ? matrix_of(v[3], "out") : fresh(n, {m, q.features}, t);
        const Matrix mo(n, out, "out", m, q.features, t);
        const eden_mx4_restore_args a{mo.data, mo.stride, q.view(), (uint64_t)m, (uint64_t)q.features, type_of(out, true, "out"), 0};
        if (m > 0) done(n, lib.mx4_restore(n->ctx, &a), {&out, &q.codes, &q.exps});
        return given(v[3]) ? again(v[3]) : wrapped(out);
    });
}

// An operand [m, k]: a matrix of a 16-bit type, or an Mx4, whose product has the given type, else
// that of the first tensor that the call brings, else bf16.
struct Operand4 {
    at::Tensor matrix;
    Matrix view;
    Mx4 held;
    int64_t m, k;
    at::ScalarType t;
    Operand4(const Native* n, PyObject* o, const char* name, PyObject* dtype, std::initializer_list<PyObject*> brought)
    {
        if (THPVariable_Check(o)) {
            matrix = matrix_of(o, name);
            m = matrix.size(0);
            k = matrix.size(1);
            t = matrix.scalar_type();
            type_of(matrix, false, name);
            if (given(dtype) && scalar_of(dtype, "dtype", false) != t) refuse(std::string("dtype is another one than that of ") + name);
            view = Matrix(n, matrix, name, m, k, t);
        } else {
            held = mx4_of(n, o, name, -1, -1);
            m = held.codes.size(0);
            k = held.features;
            t = at::kBFloat16;
            for (PyObject* b : brought)
                if (const at::Tensor* tensor = tensor_in(b)) {
                    t = tensor->scalar_type() == at::kHalf ? at::kHalf : at::kBFloat16;
                    break;
                }
            if (given(dtype)) t = scalar_of(dtype, "dtype", false);
        }
    }
};

// (native, x, weight, bias, act, residual, out, save, saved, dtype)
PyObject* mx4_linear(PyObject*, PyObject* const* v, Py_ssize_t count)
{
    return called(count, 10, [&]() -> PyObject* {
        const Native* n = native_of(v[0]);
        eden_mx4_linear_args a;
        std::memset(&a, 0, sizeof(a));
        const Operand4 x(n, v[1], "x", v[9], {v[6], v[5], v[3]});
        const Mx4 weight = mx4_of(n, v[2], "weight", -1, x.k);
        const int64_t m = x.m, cols = weight.codes.size(0);
        const at::ScalarType t = x.t;
        a.type = t == at::kBFloat16 ? EDEN_TYPE_BF16 : EDEN_TYPE_FP16;
        a.act = act_of(v[4]);
        a.save = name_of(v[7], "save", kSaves, 3);
        if (!a.save && given(v[8])) refuse("saved is given, but nothing is saved (save is none)");
        if (x.matrix.defined()) a.x = x.view.data, a.x_stride = x.view.stride;
        else a.held = x.held.view();
        a.weight = weight.view();
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
        a.m = (uint64_t)m; a.n = (uint64_t)cols; a.k = (uint64_t)x.k;
        done(n, lib.mx4_linear(n->ctx, &a), {&x.matrix, &x.held.codes, &x.held.exps, &weight.codes, &weight.exps, tensor_in(v[3]), &residual, &out, &c.codes, &c.exps});
        PyObject* y = given(v[6]) ? again(v[6]) : wrapped(out);
        return a.save ? pair(y, given(v[8]) ? again(v[8]) : wrapped_checkpoint(c)) : y;
    });
}

// (native, dz, weight_t, residual, pre, act, out, bias_grad, accumulate, dtype)
PyObject* mx4_input_grad(PyObject*, PyObject* const* v, Py_ssize_t count)
{
    return called(count, 10, [&]() -> PyObject* {
        const Native* n = native_of(v[0]);
        eden_mx4_linear_input_grad_args a;
        std::memset(&a, 0, sizeof(a));
        const Operand4 dz(n, v[1], "dz", v[9], {v[6], v[3]});
        const Mx4 weight = mx4_of(n, v[2], "weight_t", -1, dz.k);
        const int64_t m = dz.m, k = weight.codes.size(0);
        const at::ScalarType t = dz.t;
        a.type = t == at::kBFloat16 ? EDEN_TYPE_BF16 : EDEN_TYPE_FP16;
        a.act = act_of(v[5]);
        a.accumulate = flag_of(v[8]);
        if (dz.matrix.defined()) a.dz = dz.view.data, a.dz_stride = dz.view.stride;
        else a.held = dz.held.view();
        a.weight_t = weight.view();
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
        a.m = (uint64_t)m; a.n = (uint64_t)dz.k; a.k = (uint64_t)k;
        done(n, lib.mx4_input_grad(n->ctx, &a), {&dz.matrix, &dz.held.codes, &dz.held.exps, &weight.codes, &weight.exps, &residual, &pre.codes, &pre.exps, &out, &sums});
        PyObject* dx = given(v[6]) ? again(v[6]) : wrapped(out);
        return summed ? pair(dx, given(v[7]) ? again(v[7]) : wrapped(sums)) : dx;
    });
}

// (native, dz_t, x_t, out, accumulate)
PyObject* mx4_weight_grad(PyObject*, PyObject* const* v, Py_ssize_t count)
{
    return called(count, 5, [&]() -> PyObject* {
        const Native* n = native_of(v[0]);
        eden_mx4_linear_weight_grad_args a;
        std::memset(&a, 0, sizeof(a));
        a.accumulate = flag_of(v[4]);
        const Mx4 dz = mx4_of(n, v[1], "dz_t", -1, -1), x = mx4_of(n, v[2], "x_t", -1, dz.features);
        const int64_t cols = dz.codes.size(0), k = x.codes.size(0);
        a.dz_t = dz.view();
        a.x_t = x.view();
        if (a.accumulate && !given(v[3])) refuse("accumulate needs an out to add to");
        const at::Tensor out = given(v[3]) ? matrix_of(v[3], "out") : fresh(n, {cols, k}, at::kFloat);
        const Matrix mo(n, out, "out", cols, k, at::kFloat);
        a.weight_grad = (float*)mo.data; a.weight_grad_stride = mo.stride;
        a.m = (uint64_t)dz.features; a.n = (uint64_t)cols; a.k = (uint64_t)k;
        done(n, lib.mx4_weight_grad(n->ctx, &a), {&dz.codes, &dz.exps, &x.codes, &x.exps, &out});
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

// (the entry points' addresses in the order of Library, EdenError, Checkpoint, Mx4)
PyObject* bind(PyObject*, PyObject* const* v, Py_ssize_t count)
{
    return called(count, kCalls + 3, [&]() -> PyObject* {
        void* f[kCalls];
        for (int i = 0; i < kCalls; ++i) f[i] = PyLong_AsVoidPtr(v[i]);
        if (PyErr_Occurred()) throw Refused();
        std::memcpy(&lib, f, sizeof(lib));
        PyObject** const types[3] = {&error_type, &checkpoint_type, &mx4_type};
        for (int i = 0; i < 3; ++i) {
            Py_XDECREF(*types[i]);
            *types[i] = again(v[kCalls + i]);
        }
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
                         EDEN_METHOD("join", join),
                         EDEN_METHOD("join_backward", join_backward),
                         EDEN_METHOD("mx4_empty", mx4_empty),
                         EDEN_METHOD("mx4_quantize", mx4_quantize),
                         EDEN_METHOD("mx4_restore", mx4_restore),
                         EDEN_METHOD("mx4_linear", mx4_linear),
                         EDEN_METHOD("mx4_input_grad", mx4_input_grad),
                         EDEN_METHOD("mx4_weight_grad", mx4_weight_grad),
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
