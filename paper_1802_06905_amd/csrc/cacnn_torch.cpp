// The usual call of the binding in native code: contiguous device tensors of the right element sizes (feed-forward operators: matrices of the right shapes).
// Asking a tensor for its address, length, element size and layout, and torch for its current stream, through the interpreter took 1.1 of a small
// call's 5.2 us; the launch itself takes 2.9 (a quantisation of one token 7.7 and 3.8 us a call).  Everything else (other operands, wrong sizes, errors) is left to the binding: -1 says that nothing was tried.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/cacnn.h"
#include "cacnn_internal.h"

namespace {

using ConvFn = int (*)(const void* problem, int dtype, const void* image, int64_t image_elems, const void* filter, int64_t filter_elems,
                       void* out, int64_t out_elems, void* stream);
using PoolFn = int (*)(const void* problem, int dtype, int mode, const void* image, int64_t image_elems, void* out, int64_t out_elems, void* stream);

using QuantizeFn = decltype(&cacnn_quantize);
using MatmulFn = decltype(&cacnn_matmul_scaled);
using GatedFn = decltype(&cacnn_gated_forward);
using GatedScaledFn = decltype(&cacnn_gated_forward_scaled);
using GatedBackwardFn = decltype(&cacnn_gated_backward);

constexpr Py_ssize_t kProblemBytes = 9 * 8;
PyTypeObject* g_problem = nullptr;   // the binding's Problem, a ctypes structure
ConvFn g_conv = nullptr;
PoolFn g_pool = nullptr;
QuantizeFn g_quantize = nullptr;
MatmulFn g_matmul = nullptr;
GatedFn g_gated = nullptr;
GatedScaledFn g_gated_scaled = nullptr;
GatedBackwardFn g_gated_backward = nullptr;

PyObject* not_tried() { return PyLong_FromLong(-1); }

bool small_int(PyObject* o, int* value) {
    if (!PyLong_CheckExact(o)) return false;
    int overflow = 0;
    const long v = PyLong_AsLongAndOverflow(o, &overflow);
    *value = (int)v;
    return !overflow && v == (long)*value;
}

// None: torch's current stream of the current device; else a raw handle
bool stream_of(PyObject* o, void** stream) {
    if (o == Py_None) {
        *stream = (void*)c10::hip::getCurrentHIPStream().stream();
        return true;
    }
    if (!PyLong_CheckExact(o)) return false;
    *stream = PyLong_AsVoidPtr(o);
    if (*stream || !PyErr_Occurred()) return true;
    PyErr_Clear();
    return false;
}

// a contiguous device tensor of torch's own class with elements of `size` bytes
const at::Tensor* usual(PyObject* o, int64_t size) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    return t.is_cuda() && t.element_size() == size && t.is_contiguous() ? &t : nullptr;
}

// the structure's bytes (they belong to the object, which the caller's arguments keep)
const void* problem_of(PyObject* o) {
    if (Py_TYPE(o) != g_problem) return nullptr;
    Py_buffer view;
    if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) {
        PyErr_Clear();
        return nullptr;
    }
    const void* p = view.len == kProblemBytes ? view.buf : nullptr;
    PyBuffer_Release(&view);
    return p;
}

// conv(problem, dtype, image, filter, out, stream)
PyObject* conv(PyObject*, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    int dtype = 0;
    void* stream = nullptr;
    if (n != 6 || !g_conv || !small_int(args[1], &dtype) || (dtype != 0 && dtype != 1)) return not_tried();
    const int64_t size = dtype == 0 ? 4 : 2;
    const void* const problem = problem_of(args[0]);
    const at::Tensor* const image = usual(args[2], size);
    const at::Tensor* const filter = usual(args[3], size);
    const at::Tensor* const out = usual(args[4], 4);
    if (!problem || !image || !filter || !out || out->scalar_type() != at::kFloat || !stream_of(args[5], &stream)) return not_tried();
    const void *pi = image->data_ptr(), *pf = filter->data_ptr();
    void* const po = out->data_ptr();
    const int64_t ni = image->numel(), nf = filter->numel(), no = out->numel();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = g_conv(problem, dtype, pi, ni, pf, nf, po, no, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
    END_HANDLE_TH_ERRORS
}

// pool(problem, dtype, mode, image, out, stream)
PyObject* pool(PyObject*, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    int dtype = 0, mode = 0;
    void* stream = nullptr;
    if (n != 6 || !g_pool || !small_int(args[1], &dtype) || !small_int(args[2], &mode) || (dtype != 0 && dtype != 1)) return not_tried();
    const void* const problem = problem_of(args[0]);
    const at::Tensor* const image = usual(args[3], dtype == 0 ? 4 : 2);
    const at::Tensor* const out = usual(args[4], 4);
    if (!problem || !image || !out || out->scalar_type() != at::kFloat || !stream_of(args[5], &stream)) return not_tried();
    const void* const pi = image->data_ptr();
    void* const po = out->data_ptr();
    const int64_t ni = image->numel(), no = out->numel();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = g_pool(problem, dtype, mode, pi, ni, po, no, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
    END_HANDLE_TH_ERRORS
}

// ---- feed-forward operators: a problem that is a tuple of integers, matrices of exactly its sizes on the current device, rows of adjacent elements
struct Feed {
    bool usual = true;
    int device = -1;               // (asked for a first device tensor only: there may be no GPU)
    int64_t size[4] = {0, 0, 0, 0};

    Feed(PyObject* problem, Py_ssize_t sizes) {
        usual = PyTuple_CheckExact(problem) && PyTuple_GET_SIZE(problem) == sizes;
        for (Py_ssize_t i = 0; usual && i < sizes; ++i) {
            int v = 0;
            usual = small_int(PyTuple_GET_ITEM(problem, i), &v);
            size[i] = v;
        }
        usual = usual && size[0] >= 1;
    }
    // the address of a matrix; its row stride (that of the array it goes with) in *ld, nullptr: rows that follow one another
    void* take(PyObject* o, at::ScalarType type, int64_t rows, int64_t cols, int64_t* ld) {
        if (!usual || !(usual = THPVariable_CheckExact(o))) return nullptr;
        const at::Tensor& t = THPVariable_Unpack(o);
        const bool bytes = type == at::kByte && t.scalar_type() == at::kFloat8_e4m3fn;
        if (!(usual = t.is_cuda())) return nullptr;
        if (device < 0) device = c10::hip::current_device();
        usual = t.get_device() == device && (t.scalar_type() == type || bytes) && t.dim() == 2 && t.size(0) == rows && t.size(1) == cols &&
                (cols == 1 || t.stride(1) == 1);
        if (!usual) return nullptr;
        const int64_t stride = rows > 1 ? t.stride(0) : cols;
        usual = stride >= cols && (ld ? *ld == 0 || *ld == stride : stride == cols);
        if (ld) *ld = stride;
        return t.data_ptr();
    }
    void* take_or_none(PyObject* o, at::ScalarType type, int64_t rows, int64_t cols, int64_t* ld) {
        return o == Py_None ? nullptr : take(o, type, rows, cols, ld);
    }
    bool type_of(PyObject* o, int* code, at::ScalarType* type) {
        usual = usual && small_int(o, code) && (*code == 0 || *code == 1);
        *type = usual && *code == 0 ? at::kFloat : at::kBFloat16;
        return usual;
    }
};

int64_t blocks_of(int64_t n) { return (n + 127) / 128; }

// quantize(problem, dtype, x, q, scale, stream)
PyObject* quantize(PyObject*, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 6 || !g_quantize) return not_tried();
    Feed f(args[0], 3);
    int dtype = 0;
    at::ScalarType type;
    void* stream = nullptr;
    if (!f.type_of(args[1], &dtype, &type) || (f.size[2] != 1 && f.size[2] != 128)) return not_tried();
    cacnn_quantize_problem p = {f.size[0], f.size[1], f.size[2], 0, 0};
    const void* const x = f.take(args[2], type, p.T, p.C, &p.ld_x);
    void* const q = f.take(args[3], at::kByte, p.T, p.C, &p.ld_q);
    float* const scale = (float*)f.take(args[4], at::kFloat, (p.T + p.block_rows - 1) / p.block_rows, blocks_of(p.C), nullptr);
    if (!f.usual || !stream_of(args[5], &stream)) return not_tried();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = g_quantize(&p, dtype, x, q, scale, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
    END_HANDLE_TH_ERRORS
}

// matmul_scaled(problem, x, x_scale, w, w_scale, out_dtype, out, stream)
PyObject* matmul_scaled(PyObject*, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 8 || !g_matmul) return not_tried();
    Feed f(args[0], 3);
    int dtype = 0;
    at::ScalarType type;
    void* stream = nullptr;
    if (!f.type_of(args[5], &dtype, &type)) return not_tried();
    cacnn_matmul_problem p = {f.size[0], f.size[1], f.size[2], 0, 0, 0};
    const void* const x = f.take(args[1], at::kByte, p.T, p.C, &p.ld_x);
    const float* const xs = (const float*)f.take(args[2], at::kFloat, p.T, blocks_of(p.C), nullptr);
    const void* const w = f.take(args[3], at::kByte, p.K, p.C, &p.ld_w);
    const float* const ws = (const float*)f.take(args[4], at::kFloat, blocks_of(p.K), blocks_of(p.C), nullptr);
    void* const out = f.take(args[6], type, p.T, p.K, &p.ld_out);
    if (!f.usual || !stream_of(args[7], &stream)) return not_tried();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = g_matmul(&p, x, xs, w, ws, dtype, out, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
    END_HANDLE_TH_ERRORS
}

// gated_forward(problem, dtype, x, w_gate, w_up, out, gate, up, stream)
PyObject* gated_forward(PyObject*, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 9 || !g_gated) return not_tried();
    Feed f(args[0], 4);
    int dtype = 0;
    at::ScalarType type;
    void* stream = nullptr;
    if (!f.type_of(args[1], &dtype, &type)) return not_tried();
    cacnn_gated_problem p = {f.size[0], f.size[1], f.size[2], f.size[3], 0, 0, 0, 0, 0, 0};
    const void* const x = f.take(args[2], type, p.T, p.C, &p.ld_x);
    const void* const wg = f.take(args[3], type, p.F, p.C, &p.ld_w);
    const void* const wu = f.take(args[4], type, p.F, p.C, &p.ld_w);
    void* const out = f.take(args[5], type, p.T, p.F, &p.ld_out);
    void* const gate = f.take_or_none(args[6], type, p.T, p.F, &p.ld_pre);
    void* const up = f.take_or_none(args[7], type, p.T, p.F, &p.ld_pre);
    if (!f.usual || !stream_of(args[8], &stream)) return not_tried();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = g_gated(&p, dtype, x, wg, wu, out, gate, up, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
    END_HANDLE_TH_ERRORS
}

// gated_forward_scaled(problem, x, x_scale, w_gate, w_gate_scale, w_up, w_up_scale, out_dtype, out, stream)
PyObject* gated_forward_scaled(PyObject*, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 10 || !g_gated_scaled) return not_tried();
    Feed f(args[0], 4);
    int dtype = 0;
    at::ScalarType type;
    void* stream = nullptr;
    if (!f.type_of(args[7], &dtype, &type)) return not_tried();
    cacnn_gated_problem p = {f.size[0], f.size[1], f.size[2], f.size[3], 0, 0, 0, 0, 0, 0};
    const int64_t blocks = blocks_of(p.C);
    const void* const x = f.take(args[1], at::kByte, p.T, p.C, &p.ld_x);
    const float* const xs = (const float*)f.take(args[2], at::kFloat, p.T, blocks, nullptr);
    const void* const wg = f.take(args[3], at::kByte, p.F, p.C, &p.ld_w);
    const float* const gs = (const float*)f.take(args[4], at::kFloat, blocks_of(p.F), blocks, nullptr);
    const void* const wu = f.take(args[5], at::kByte, p.F, p.C, &p.ld_w);
    const float* const us = (const float*)f.take(args[6], at::kFloat, blocks_of(p.F), blocks, nullptr);
    void* const out = f.take(args[8], type, p.T, p.F, &p.ld_out);
    if (!f.usual || !stream_of(args[9], &stream)) return not_tried();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = g_gated_scaled(&p, x, xs, wg, gs, wu, us, dtype, out, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
    END_HANDLE_TH_ERRORS
}

// gated_backward(problem, dtype, x, w_gate, w_up, grad_out, grad_x, grad_w_gate, grad_w_up, workspace, gate, up, stream)
PyObject* gated_backward(PyObject*, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 13 || !g_gated_backward) return not_tried();
    Feed f(args[0], 4);
    int dtype = 0;
    at::ScalarType type;
    void* stream = nullptr;
    if (!f.type_of(args[1], &dtype, &type)) return not_tried();
    cacnn_gated_problem p = {f.size[0], f.size[1], f.size[2], f.size[3], 0, 0, 0, 0, 0, 0};
    const void* const x = f.take(args[2], type, p.T, p.C, &p.ld_x);
    const void* const wg = f.take(args[3], type, p.F, p.C, &p.ld_w);
    const void* const wu = f.take(args[4], type, p.F, p.C, &p.ld_w);
    const void* const grad_out = f.take(args[5], type, p.T, p.F, &p.ld_out);
    void* const grad_x = f.take_or_none(args[6], type, p.T, p.C, &p.ld_grad_x);
    void* const grad_wg = f.take_or_none(args[7], type, p.F, p.C, &p.ld_grad_w);
    void* const grad_wu = f.take_or_none(args[8], type, p.F, p.C, &p.ld_grad_w);
    const void* const gate = f.take_or_none(args[10], type, p.T, p.F, &p.ld_pre);
    const void* const up = f.take_or_none(args[11], type, p.T, p.F, &p.ld_pre);
    if (!f.usual || !THPVariable_CheckExact(args[9]) || !stream_of(args[12], &stream)) return not_tried();
    const at::Tensor& work = THPVariable_Unpack(args[9]);
    if (!work.is_cuda() || work.get_device() != f.device || !work.is_contiguous()) return not_tried();
    void* const workspace = work.data_ptr();
    const size_t bytes = (size_t)work.numel() * work.element_size();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = g_gated_backward(&p, dtype, x, wg, wu, gate, up, grad_out, grad_x, grad_wg, grad_wu, workspace, bytes, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
    END_HANDLE_TH_ERRORS
}

// setup(cacnn_internal_sized_interface(), size of Problem, Problem, addresses of cacnn_internal_conv_forward_sized,
// cacnn_internal_pool_forward_sized, cacnn_quantize, cacnn_matmul_scaled, cacnn_gated_forward, cacnn_gated_forward_scaled, cacnn_gated_backward); ImportError where the first two are not what this module was compiled for
PyObject* setup(PyObject*, PyObject* args) {
    PyObject *problem, *at[7];
    int interface = 0;
    Py_ssize_t size = 0;
    if (!PyArg_ParseTuple(args, "inO!OOOOOOO", &interface, &size, &PyType_Type, &problem, &at[0], &at[1], &at[2], &at[3], &at[4], &at[5], &at[6])) return nullptr;
    if (interface != cacnn::kSizedInterface || size != kProblemBytes) {
        PyErr_SetString(PyExc_ImportError, "_cacnn_torch was compiled for another version of the library");
        return nullptr;
    }
    void* f[7];
    for (int i = 0; i < 7; ++i) f[i] = PyLong_AsVoidPtr(at[i]);
    if (PyErr_Occurred()) return nullptr;
    Py_INCREF(problem);
    Py_XDECREF((PyObject*)g_problem);
    g_problem = (PyTypeObject*)problem;
    g_conv = (ConvFn)f[0];
    g_pool = (PoolFn)f[1];
    g_quantize = (QuantizeFn)f[2];
    g_matmul = (MatmulFn)f[3];
    g_gated = (GatedFn)f[4];
    g_gated_scaled = (GatedScaledFn)f[5];
    g_gated_backward = (GatedBackwardFn)f[6];
    Py_RETURN_NONE;
}

PyMethodDef g_methods[] = {
    {"conv", (PyCFunction)(void (*)(void))conv, METH_FASTCALL, nullptr},
    {"pool", (PyCFunction)(void (*)(void))pool, METH_FASTCALL, nullptr},
    {"quantize", (PyCFunction)(void (*)(void))quantize, METH_FASTCALL, nullptr},
    {"matmul_scaled", (PyCFunction)(void (*)(void))matmul_scaled, METH_FASTCALL, nullptr},
    {"gated_forward", (PyCFunction)(void (*)(void))gated_forward, METH_FASTCALL, nullptr},
    {"gated_forward_scaled", (PyCFunction)(void (*)(void))gated_forward_scaled, METH_FASTCALL, nullptr},
    {"gated_backward", (PyCFunction)(void (*)(void))gated_backward, METH_FASTCALL, nullptr},
    {"setup", setup, METH_VARARGS, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_cacnn_torch", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__cacnn_torch() { return PyModule_Create(&g_module); }
