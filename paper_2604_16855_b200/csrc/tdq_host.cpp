// The host side of the Python binding: takes torch tensors, checks the layout the C ABI assumes but cannot see,
// makes the outputs the caller did not pass and enqueues the call.
//
// One pass of a small layer is a few microseconds of GPU work, so what the host does per call decides its time:
// marshalled through ctypes a quantize_act + w4a4_linear pair took 27 us to issue (46 us with outputs and workspace
// made by the calls), of which the two calls into the library were about 11.  Here the tensors are read in C++: 5 to 8 us
// (8.5), two launches included.
//
// The functions take every argument by position (binding.py gives them names and defaults) and release the
// interpreter lock while the library works, as ctypes does.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/DynamicTypes.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <string>

#include "../../include/tdq.h"

namespace {

PyObject* g_tdq_error = nullptr;   // binding.TdqError, set once by the binding

struct Bad {                       // a Python exception to raise
    PyObject* type;
    std::string text;
};

const at::Tensor* opt_tensor(PyObject* o) {
    if (o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) throw Bad{PyExc_TypeError, std::string("expected a torch.Tensor, got ") + Py_TYPE(o)->tp_name};
    return &THPVariable_Unpack(o);
}
const at::Tensor& tensor(PyObject* o) {
    const at::Tensor* t = opt_tensor(o);
    if (!t) throw Bad{PyExc_TypeError, "expected a torch.Tensor, got None"};
    return *t;
}
std::string dtype_name(at::ScalarType s) { return std::string("torch.") + torch::getTHPDtype(s)->name; }

void need_cuda(std::initializer_list<const at::Tensor*> ts) {
    for (const at::Tensor* t : ts)
        if (t && !t->is_cuda()) throw Bad{PyExc_ValueError, "tdq runs on CUDA tensors only; there is no CPU path"};
}
tdq_dtype dtype_id(const at::Tensor& t) {
    switch (t.scalar_type()) {
        case at::kFloat: return TDQ_F32;
        case at::kBFloat16: return TDQ_BF16;
        case at::kHalf: return TDQ_F16;   // the library refuses it where a call does not take it
        default: throw Bad{PyExc_TypeError, "tdq takes float32, bfloat16 or (where the call says so) float16 tensors, got " + dtype_name(t.scalar_type())};
    }
}
at::ScalarType dtype_arg(PyObject* o) {
    if (!THPDtype_Check(o)) throw Bad{PyExc_TypeError, "out_dtype must be a torch.dtype"};
    return reinterpret_cast<THPDtype*>(o)->scalar_type;
}

// One operand of the linear layer: type, contiguity and the device all operands share.
void check_operand(const char* name, const at::Tensor* t, at::ScalarType want, const at::Tensor*& first) {
    if (!t) return;
    if (t->scalar_type() != want)
        throw Bad{PyExc_TypeError, std::string(name) + " must be " + dtype_name(want) + ", got " + dtype_name(t->scalar_type())};
    if (!t->is_contiguous()) throw Bad{PyExc_ValueError, std::string(name) + " must be contiguous"};
    if (!first) first = t;
    else if (t->device() != first->device())
        throw Bad{PyExc_ValueError, std::string(name) + " is on " + t->device().str() + ", the other operands on " + first->device().str()};
}
// y may have a row pitch but its columns must be adjacent
void check_y(const at::Tensor& y, const at::Tensor* first) {
    if (y.dim() != 2 || (y.size(1) > 1 && y.stride(1) != 1))
        throw Bad{PyExc_ValueError, "y must be a matrix whose columns are adjacent in memory"};
    if (first && y.device() != first->device())
        throw Bad{PyExc_ValueError, "y is on " + y.device().str() + ", the operands on " + first->device().str()};
}

tdq_act_params params_arg(PyObject* o) {
    tdq_act_params p;
    if (o == Py_None) {
        tdq_default_act_params(&p);
        return p;
    }
    Py_buffer b;   // a ctypes structure exposes its bytes
    if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) {
        PyErr_Clear();
        throw Bad{PyExc_TypeError, "params must be an ActParams"};
    }
    const bool fits = b.len == (Py_ssize_t)sizeof p;
    if (fits) memcpy(&p, b.buf, sizeof p);
    PyBuffer_Release(&b);
    if (!fits) throw Bad{PyExc_TypeError, "params must be an ActParams"};
    return p;
}
int64_t int_arg(PyObject* o) {
    PyObject* i = PyNumber_Index(o);
    if (!i) throw python_error();
    const int64_t v = PyLong_AsLongLong(i);
    Py_DECREF(i);
    if (v == -1 && PyErr_Occurred()) throw python_error();
    return v;
}

bool truth(PyObject* o) {
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw python_error();
    return v != 0;
}
double float_arg(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw python_error();
    return v;
}

template <typename T = void>
T* ptr(const at::Tensor* t) { return t ? reinterpret_cast<T*>(t->data_ptr()) : nullptr; }
template <typename T = void>
T* ptr(const at::Tensor& t) { return reinterpret_cast<T*>(t.data_ptr()); }
void* stream_of(const at::Tensor& t) { return c10::cuda::getCurrentCUDAStream(t.device().index()).stream(); }

void check(tdq_status st, const char* where) {
    if (st == TDQ_OK) return;
    PyObject* e = PyObject_CallFunction(g_tdq_error, "is", (int)st, where);
    if (e) {
        PyErr_SetObject(g_tdq_error, e);
        Py_DECREF(e);
    }
    throw python_error();
}
// Runs a library call without the interpreter lock, on the device of `on`.
template <typename F>
tdq_status call(const at::Tensor& on, F&& f) {
    pybind11::gil_scoped_release release;
    c10::cuda::CUDAGuard guard(on.device());
    return f(stream_of(on));
}

PyObject* tuple2(const at::Tensor& a, const at::Tensor& b) {
    PyObject* pa = THPVariable_Wrap(a);
    PyObject* pb = pa ? THPVariable_Wrap(b) : nullptr;
    PyObject* t = pb ? PyTuple_Pack(2, pa, pb) : nullptr;
    Py_XDECREF(pa);
    Py_XDECREF(pb);
    return t;
}
// Straight to the caching allocator: the dispatcher's share of at::empty is half of its time, and a small layer whose
// outputs the calls make allocates four times.
at::Tensor new_like(const at::Tensor& on, at::IntArrayRef sizes, at::ScalarType s) {
    return at::Tensor(at::detail::empty_cuda(sizes, s, on.device(), c10::nullopt));
}
// The caller's workspace, or one from the caching allocator for the length of the call (given back to the stream's pool, so
// whatever the stream runs next is ordered behind its use).  Every linear call writes what it reads of the workspace, so
// nothing has to be cleared.
struct Workspace {
    at::DataPtr own;
    void* ptr;
    size_t bytes;
    Workspace(const at::Tensor* given, const at::Tensor& on, int64_t M, int64_t I_pad, int64_t O, int64_t g) {
        if (given) {
            ptr = given->data_ptr();
            bytes = (size_t)given->numel();
        } else {
            c10::cuda::CUDAGuard guard(on.device());
            bytes = tdq_linear_workspace_bytes(M, I_pad, O, (int32_t)g);
            own = c10::cuda::CUDACachingAllocator::get()->allocate(bytes);
            ptr = own.get();
        }
    }
};
at::Tensor workspace_for(const at::Tensor& on, int64_t M, int64_t I_pad, int64_t O, int64_t g) {
    return new_like(on, {(int64_t)tdq_linear_workspace_bytes(M, I_pad, O, (int32_t)g)}, at::kByte);
}

// quantize_act(x, params, codes, scale, offset)
PyObject* quantize_act(PyObject* const* a) {
    const at::Tensor& x = tensor(a[0]);
    need_cuda({&x});
    const tdq_act_params p = params_arg(a[1]);
    const int64_t C = x.size(-1);
    const at::Tensor x2 = x.dim() == 2 ? x : x.reshape({-1, C});
    if (x2.stride(-1) != 1) throw Bad{PyExc_ValueError, "the channel axis must be contiguous"};
    const int64_t M = x2.size(0), g = p.group_size;
    if (g == 0) throw Bad{PyExc_ZeroDivisionError, "group_size is 0"};
    const int64_t K = (C + g - 1) / g;
    const at::Tensor *oc = opt_tensor(a[2]), *os = opt_tensor(a[3]), *oo = opt_tensor(a[4]);
    const at::Tensor codes = oc ? *oc : new_like(x, {M, K * g / 2}, at::kByte);
    const at::Tensor scale = os ? *os : new_like(x, {M, K}, at::kFloat);
    if (M > 0) {   // an empty tensor has no device pointer to pass
        const tdq_dtype dt = dtype_id(x2);
        check(call(x, [&](void* st) {
                  return tdq_quantize_act(ptr(x2), dt, 1, M, C, M > 1 ? x2.stride(0) : C, &p, ptr<uint8_t>(codes), ptr<float>(scale),
                                          ptr<float>(oo), st);
              }), "tdq_quantize_act");
    }
    return tuple2(codes, scale);
}

// quantize_act_fixed(x, radius, g, codes, scale, offset)
PyObject* quantize_act_fixed(PyObject* const* a) {
    const at::Tensor& x = tensor(a[0]);
    const at::Tensor *oc = opt_tensor(a[3]), *os = opt_tensor(a[4]), *oo = opt_tensor(a[5]);
    need_cuda({&x, oc, os, oo});
    const double radius = PyFloat_AsDouble(a[1]);
    if (radius == -1.0 && PyErr_Occurred()) throw python_error();
    const int64_t g = int_arg(a[2]), C = x.size(-1);
    if (g == 0) throw Bad{PyExc_ZeroDivisionError, "group size is 0"};
    const at::Tensor x2 = x.dim() == 2 ? x : x.reshape({-1, C});
    const int64_t M = x2.size(0);
    const at::Tensor codes = oc ? *oc : new_like(x, {M, C / 2}, at::kByte);
    const at::Tensor scale = os ? *os : new_like(x, {M, std::max<int64_t>(C / g, 1)}, at::kFloat);
    const tdq_dtype dt = dtype_id(x2);
    check(call(x, [&](void* st) {
              return tdq_quantize_act_fixed(ptr(x2), dt, 1, M, C, M > 1 ? x2.stride(0) : C, (int32_t)g, (float)radius, ptr<uint8_t>(codes),
                                            ptr<float>(scale), ptr<float>(oo), st);
          }), "tdq_quantize_act_fixed");
    return tuple2(codes, scale);
}

// quantize_act_nchw(x, params, codes, scale, offset)
PyObject* quantize_act_nchw(PyObject* const* a) {
    const at::Tensor& x = tensor(a[0]);
    const at::Tensor *oc = opt_tensor(a[2]), *os = opt_tensor(a[3]), *oo = opt_tensor(a[4]);
    need_cuda({&x, oc, os, oo});
    const tdq_act_params p = params_arg(a[1]);
    if (x.dim() != 4 || !x.is_contiguous()) throw Bad{PyExc_ValueError, "x must be a contiguous [B, C, H, W] tensor"};
    const int64_t B = x.size(0), C = x.size(1), H = x.size(2), W = x.size(3), M = B * H * W;
    const at::Tensor codes = oc ? *oc : new_like(x, {M, C / 2}, at::kByte);
    const at::Tensor scale = os ? *os : new_like(x, {M, std::max<int64_t>(C / 32, 1)}, at::kFloat);
    const tdq_dtype dt = dtype_id(x);
    check(call(x, [&](void* st) {
              return tdq_quantize_act_nchw(ptr(x), dt, B, C, H, W, &p, ptr<uint8_t>(codes), ptr<float>(scale), ptr<float>(oo), st);
          }), "tdq_quantize_act_nchw");
    return tuple2(codes, scale);
}

// quantize_weight(w, pad_to, wcodes, wscale)
PyObject* quantize_weight(PyObject* const* a) {
    const at::Tensor& w0 = tensor(a[0]);
    need_cuda({&w0});
    const at::Tensor w = w0.contiguous();
    if (w.dim() != 2) throw Bad{PyExc_ValueError, "w must be a matrix [O, I]"};
    const int64_t O = w.size(0), I = w.size(1), pad = int_arg(a[1]);
    if (pad == 0) throw Bad{PyExc_ZeroDivisionError, "pad_to is 0"};
    const int64_t I_pad = (I + pad - 1) / pad * pad;
    const at::Tensor *oc = opt_tensor(a[2]), *os = opt_tensor(a[3]);
    const at::Tensor codes = oc ? *oc : new_like(w, {O, I_pad / 2}, at::kByte);
    const at::Tensor scale = os ? *os : new_like(w, {O}, at::kFloat);
    const tdq_dtype dt = dtype_id(w);
    check(call(w, [&](void* st) {
              return tdq_quantize_weight(ptr(w), dt, O, I, (int32_t)pad, ptr<uint8_t>(codes), ptr<float>(scale), st);
          }), "tdq_quantize_weight");
    return tuple2(codes, scale);
}

// w4a4_linear(xcodes, xscale, wcodes, wscale, bias, g, out_dtype, y, acc_debug, workspace, pow2)
PyObject* w4a4_linear(PyObject* const* a) {
    const at::Tensor &xc = tensor(a[0]), &xs = tensor(a[1]), &wc = tensor(a[2]), &ws = tensor(a[3]);
    const at::Tensor* bias = opt_tensor(a[4]);
    need_cuda({&xc, &xs, &wc, &ws, bias});
    const int64_t g = int_arg(a[5]);
    const at::Tensor *oy = opt_tensor(a[7]), *acc = opt_tensor(a[8]), *ow = opt_tensor(a[9]);
    const bool pow2 = a[10] == Py_True;
    if (xc.dim() != 2) throw Bad{PyExc_ValueError, "xcodes must be a matrix"};
    if (wc.dim() < 1) throw Bad{PyExc_ValueError, "wcodes must be a matrix"};
    const int64_t M = xc.size(0), I_pad = 2 * xc.size(1), O = wc.size(0);
    const at::Tensor y = oy ? *oy : new_like(xc, {M, O}, dtype_arg(a[6]));
    const at::Tensor* first = nullptr;
    check_operand("xcodes", &xc, at::kByte, first);
    check_operand("xscale", &xs, at::kFloat, first);
    check_operand("wcodes", &wc, at::kByte, first);
    check_operand("wscale", &ws, at::kFloat, first);
    check_operand("bias", bias, at::kFloat, first);
    check_operand("workspace", ow, at::kByte, first);
    check_operand("acc_debug", acc, at::kInt, first);
    check_y(y, first);
    const tdq_dtype dt = dtype_id(y);
    const Workspace workspace(ow, xc, M, I_pad, O, g);
    const int64_t y_stride = M > 0 ? y.stride(0) : O;
    check(call(xc, [&](void* st) {
              if (pow2)
                  return tdq_w4a4_linear_pow2(ptr<uint8_t>(xc), ptr<float>(xs), ptr<uint8_t>(wc), ptr<float>(ws), ptr<float>(bias), M, I_pad,
                                              O, (int32_t)g, ptr(y), dt, y_stride, workspace.ptr, workspace.bytes, st);
              return tdq_w4a4_linear(ptr<uint8_t>(xc), ptr<float>(xs), ptr<uint8_t>(wc), ptr<float>(ws), ptr<float>(bias), M, I_pad, O,
                                     (int32_t)g, ptr(y), dt, y_stride, ptr<int32_t>(acc), workspace.ptr, workspace.bytes, st);
          }), pow2 ? "tdq_w4a4_linear_pow2" : "tdq_w4a4_linear");
    return THPVariable_Wrap(y);
}

// w4a4_linear_static(xcodes, xscale, wcodes, wscale, bias, g, y, wait)
PyObject* w4a4_linear_static(PyObject* const* a) {
    const at::Tensor &xc = tensor(a[0]), &xs = tensor(a[1]), &wc = tensor(a[2]), &ws = tensor(a[3]), &y = tensor(a[6]);
    const at::Tensor* bias = opt_tensor(a[4]);
    need_cuda({&xc, &xs, &wc, &ws, bias, &y});
    const int64_t g = int_arg(a[5]);
    const int wait = PyObject_IsTrue(a[7]);
    if (wait < 0) throw python_error();
    if (xc.dim() != 2) throw Bad{PyExc_ValueError, "xcodes must be a matrix"};
    if (wc.dim() < 1) throw Bad{PyExc_ValueError, "wcodes must be a matrix"};
    const int64_t M = xc.size(0), O = wc.size(0);
    const at::Tensor* first = nullptr;
    check_operand("xcodes", &xc, at::kByte, first);
    check_operand("xscale", &xs, at::kFloat, first);
    check_operand("wcodes", &wc, at::kByte, first);
    check_operand("wscale", &ws, at::kFloat, first);
    check_operand("bias", bias, at::kFloat, first);
    check_y(y, first);
    const tdq_dtype dt = dtype_id(y);
    check(call(xc, [&](void* st) {
              return tdq_w4a4_linear_static(ptr<uint8_t>(xc), ptr<float>(xs), ptr<uint8_t>(wc), ptr<float>(ws), ptr<float>(bias), M,
                                            2 * xc.size(1), O, (int32_t)g, ptr(y), dt, M > 0 ? y.stride(0) : O, wait, st);
          }), "tdq_w4a4_linear_static");
    Py_INCREF(a[6]);
    return a[6];
}

// quant_linear_fused(x, wcodes, wscale, bias, params, out_dtype, y, workspace)
PyObject* quant_linear_fused(PyObject* const* a) {
    const at::Tensor &x = tensor(a[0]), &wc = tensor(a[1]), &ws = tensor(a[2]);
    const at::Tensor *bias = opt_tensor(a[3]), *oy = opt_tensor(a[6]), *ow = opt_tensor(a[7]);
    need_cuda({&x, &wc, &ws, bias});
    const tdq_act_params p = params_arg(a[4]);
    const int64_t C = x.size(-1);
    const at::Tensor x2 = x.dim() == 2 ? x : x.reshape({-1, C});
    if (wc.dim() != 2) throw Bad{PyExc_ValueError, "wcodes must be a matrix"};
    const int64_t M = x2.size(0), O = wc.size(0);
    const at::Tensor y = oy ? *oy : new_like(x, {M, O}, dtype_arg(a[5]));
    if (C > 1 && x2.stride(1) != 1) throw Bad{PyExc_ValueError, "the channels of x must be adjacent in memory"};
    const at::Tensor* first = nullptr;
    check_operand("wcodes", &wc, at::kByte, first);
    check_operand("wscale", &ws, at::kFloat, first);
    check_operand("bias", bias, at::kFloat, first);
    check_operand("workspace", ow, at::kByte, first);
    check_y(y, first);
    if (x2.device() != first->device())
        throw Bad{PyExc_ValueError, "x is on " + x2.device().str() + ", the weights on " + first->device().str()};
    const tdq_dtype xdt = dtype_id(x2), ydt = dtype_id(y);
    const Workspace workspace(ow, x, M, wc.size(1) * 2, O, p.group_size);
    check(call(x, [&](void* st) {
              return tdq_quant_linear_fused(ptr(x2), xdt, 1, M, C, M > 1 ? x2.stride(0) : C, &p, ptr<uint8_t>(wc), ptr<float>(ws),
                                            ptr<float>(bias), O, ptr(y), ydt, y.stride(0), workspace.ptr, workspace.bytes, st);
          }), "tdq_quant_linear_fused");
    return THPVariable_Wrap(y);
}

// quant_linear_host(x_host, wcodes, wscale, bias, params, out_dtype, y_host)  ->  (y_host, buffers)
PyObject* quant_linear_host(PyObject* const* a) {
    const at::Tensor &x = tensor(a[0]), &wc = tensor(a[1]), &ws = tensor(a[2]);
    const at::Tensor *bias = opt_tensor(a[3]), *oy = opt_tensor(a[6]);
    need_cuda({&wc, &ws, bias});
    const tdq_act_params p = params_arg(a[4]);
    if (x.dim() != 2) throw Bad{PyExc_ValueError, "x_host must be a matrix"};
    const int64_t M = x.size(0), C = x.size(1), O = wc.size(0), g = p.group_size;
    if (g == 0) throw Bad{PyExc_ZeroDivisionError, "group_size is 0"};
    const int64_t K = (C + g - 1) / g, I_pad = K * g;
    const at::ScalarType yt = dtype_arg(a[5]);
    const at::Tensor x_dev = new_like(wc, {M, C}, x.scalar_type()), codes = new_like(wc, {M, I_pad / 2}, at::kByte);
    const at::Tensor scale = new_like(wc, {M, K}, at::kFloat), y_dev = new_like(wc, {M, O}, yt);
    const at::Tensor y = oy ? *oy : at::empty({M, O}, at::TensorOptions().dtype(yt)).pin_memory();
    const at::Tensor workspace = workspace_for(wc, M, I_pad, O, g);
    const tdq_dtype xdt = dtype_id(x), ydt = dtype_id(y);
    check(call(wc, [&](void* st) {
              return tdq_quant_linear_host(ptr(x), xdt, 1, M, C, &p, ptr<uint8_t>(wc), ptr<float>(ws), ptr<float>(bias), O, ptr(y), ydt,
                                           ptr(x_dev), ptr<uint8_t>(codes), ptr<float>(scale), ptr(y_dev), ptr(workspace),
                                           (size_t)workspace.numel(), st);
          }), "tdq_quant_linear_host");
    PyObject* bufs = PyTuple_New(5);
    if (!bufs) return nullptr;
    const at::Tensor* keep[5] = {&workspace, &x_dev, &codes, &scale, &y_dev};
    for (int i = 0; i < 5; ++i) PyTuple_SET_ITEM(bufs, i, THPVariable_Wrap(*keep[i]));
    PyObject* py = THPVariable_Wrap(y);
    PyObject* t = PyTuple_Pack(2, py, bufs);
    Py_DECREF(py);
    Py_DECREF(bufs);
    return t;
}

// ---------------------------------------------------------------------------------------------- 8-bit floating point layer

// A tensor that the caller passed for an output or operand: type, sizes, contiguity, device.
void check_tensor(const char* name, const at::Tensor& t, std::initializer_list<at::ScalarType> types, at::IntArrayRef sizes, const at::Tensor& on) {
    bool fits = false;
    for (at::ScalarType s : types) fits = fits || t.scalar_type() == s;
    if (!fits) throw Bad{PyExc_TypeError, std::string(name) + " must be " + dtype_name(*types.begin()) + ", got " + dtype_name(t.scalar_type())};
    if (t.sizes() != sizes) {
        std::string want, got;
        for (int64_t n : sizes) want += (want.empty() ? "" : ", ") + std::to_string(n);
        for (int64_t n : t.sizes()) got += (got.empty() ? "" : ", ") + std::to_string(n);
        throw Bad{PyExc_ValueError, std::string(name) + " must be of size [" + want + "], got [" + got + "]"};
    }
    if (!t.is_contiguous()) throw Bad{PyExc_ValueError, std::string(name) + " must be contiguous"};
    if (t.device() != on.device()) throw Bad{PyExc_ValueError, std::string(name) + " is on " + t.device().str() + ", not on " + on.device().str()};
}
constexpr int64_t kFp8Block = 128;
int64_t fp8_blocks(int64_t n) { return (n + kFp8Block - 1) / kFp8Block; }

// quantize_act_fp8(x, codes, scale, pow2)
PyObject* quantize_act_fp8(PyObject* const* a) {
    const at::Tensor& x = tensor(a[0]);
    const at::Tensor *oc = opt_tensor(a[1]), *os = opt_tensor(a[2]);
    const bool pow2 = truth(a[3]);
    need_cuda({&x, oc, os});
    if (x.dim() < 1 || x.size(-1) < 1) throw Bad{PyExc_ValueError, "x must have channels"};
    const int64_t C = x.size(-1), K = fp8_blocks(C);
    const at::Tensor x2 = x.dim() == 2 ? x : x.reshape({x.numel() / C, C});
    const int64_t M = x2.size(0);
    if (C > 1 && M > 0 && x2.stride(1) != 1) throw Bad{PyExc_ValueError, "the channel axis must be contiguous"};
    const tdq_dtype dt = dtype_id(x2);
    if (oc) check_tensor("codes", *oc, {at::kFloat8_e4m3fn, at::kByte}, {M, K * kFp8Block}, x);
    if (os) check_tensor("scale", *os, {at::kFloat}, {M, K}, x);
    const at::Tensor codes = oc ? *oc : new_like(x, {M, K * kFp8Block}, at::kFloat8_e4m3fn);
    const at::Tensor scale = os ? *os : new_like(x, {M, K}, at::kFloat);
    check(call(x, [&](void* st) {
              return (pow2 ? tdq_quantize_act_fp8_pow2 : tdq_quantize_act_fp8)(ptr(x2), dt, 1, M, C, M > 1 ? x2.stride(0) : C, ptr<uint8_t>(codes),
                                                                               ptr<float>(scale), st);
          }), pow2 ? "tdq_quantize_act_fp8_pow2" : "tdq_quantize_act_fp8");
    return tuple2(codes, scale);
}

// quantize_weight_fp8(w, wcodes, wscale)
PyObject* quantize_weight_fp8(PyObject* const* a) {
    const at::Tensor& w0 = tensor(a[0]);
    const at::Tensor *oc = opt_tensor(a[1]), *os = opt_tensor(a[2]);
    need_cuda({&w0, oc, os});
    if (w0.dim() != 2 || w0.size(1) < 1) throw Bad{PyExc_ValueError, "w must be a matrix [O, I]"};
    const at::Tensor w = w0.contiguous();
    const int64_t O = w.size(0), I = w.size(1), K = fp8_blocks(I), T = fp8_blocks(O);
    const tdq_dtype dt = dtype_id(w);
    if (oc) check_tensor("wcodes", *oc, {at::kFloat8_e4m3fn, at::kByte}, {O, K * kFp8Block}, w);
    if (os) check_tensor("wscale", *os, {at::kFloat}, {T, K}, w);
    const at::Tensor codes = oc ? *oc : new_like(w, {O, K * kFp8Block}, at::kFloat8_e4m3fn);
    const at::Tensor scale = os ? *os : new_like(w, {T, K}, at::kFloat);
    check(call(w, [&](void* st) {
              return tdq_quantize_weight_fp8(ptr(w), dt, O, I, ptr<uint8_t>(codes), ptr<float>(scale), st);
          }), "tdq_quantize_weight_fp8");
    return tuple2(codes, scale);
}

// fp8_linear(xcodes, xscale, wcodes, wscale, bias, out_dtype, y, workspace, activation, residual, pre)
PyObject* fp8_linear(PyObject* const* a) {
    const at::Tensor &xc = tensor(a[0]), &xs = tensor(a[1]), &wc = tensor(a[2]), &ws = tensor(a[3]);
    const at::Tensor *bias = opt_tensor(a[4]), *oy = opt_tensor(a[6]), *ow = opt_tensor(a[7]), *res = opt_tensor(a[9]), *pre = opt_tensor(a[10]);
    need_cuda({&xc, &xs, &wc, &ws, bias, oy, ow, res, pre});
    tdq_fp8_epilogue e = {};
    e.activation = (int32_t)int_arg(a[8]);
    if (xc.dim() != 2 || wc.dim() != 2) throw Bad{PyExc_ValueError, "xcodes and wcodes must be matrices"};
    const int64_t M = xc.size(0), I_pad = xc.size(1), O = wc.size(0), K = I_pad / kFp8Block;
    if (I_pad < 1 || I_pad % kFp8Block) throw Bad{PyExc_ValueError, "the codes' rows must be a multiple of 128 long"};
    check_tensor("xcodes", xc, {at::kFloat8_e4m3fn, at::kByte}, {M, I_pad}, xc);
    check_tensor("xscale", xs, {at::kFloat}, {M, K}, xc);
    check_tensor("wcodes", wc, {at::kFloat8_e4m3fn, at::kByte}, {O, I_pad}, xc);
    check_tensor("wscale", ws, {at::kFloat}, {fp8_blocks(O), K}, xc);
    if (bias) check_tensor("bias", *bias, {at::kFloat}, {O}, xc);
    if (ow) check_tensor("workspace", *ow, {at::kByte}, ow->sizes(), xc);
    const at::Tensor y = oy ? *oy : new_like(xc, {M, O}, dtype_arg(a[5]));
    check_y(y, &xc);
    if (y.size(0) != M || y.size(1) != O) throw Bad{PyExc_ValueError, "y must be of size [" + std::to_string(M) + ", " + std::to_string(O) + "]"};
    const tdq_dtype dt = dtype_id(y);
    const auto beside = [&](const char* name, const at::Tensor& t) {   // a matrix like y
        if (t.scalar_type() != y.scalar_type()) throw Bad{PyExc_TypeError, std::string(name) + " must be " + dtype_name(y.scalar_type()) + ", got " + dtype_name(t.scalar_type())};
        if (t.sizes() != y.sizes() || (O > 1 && t.stride(1) != 1) || t.device() != y.device())
            throw Bad{PyExc_ValueError, std::string(name) + " must be of y's size and device, its columns adjacent in memory"};
        return M > 1 ? t.stride(0) : O;
    };
    if (res) { e.residual = ptr(res); e.residual_row_stride = beside("residual", *res); }
    if (pre) { e.pre = ptr(pre); e.pre_row_stride = beside("pre", *pre); }
    at::DataPtr own;
    void* wsp = ow ? ow->data_ptr() : nullptr;
    size_t wsp_bytes = ow ? (size_t)ow->numel() : 0;
    if (!ow) {
        c10::cuda::CUDAGuard guard(xc.device());
        wsp_bytes = tdq_fp8_linear_workspace_bytes(M, I_pad, O);
        own = c10::cuda::CUDACachingAllocator::get()->allocate(wsp_bytes);
        wsp = own.get();
    }
    if (e.activation != TDQ_ACT_NONE || res || pre)
        check(call(xc, [&](void* st) {
                  return tdq_fp8_linear_epilogue(ptr<uint8_t>(xc), ptr<float>(xs), ptr<uint8_t>(wc), ptr<float>(ws), ptr<float>(bias), M, I_pad, O, &e, ptr(y), dt,
                                                 M > 1 ? y.stride(0) : O, wsp, wsp_bytes, st);
              }), "tdq_fp8_linear_epilogue");
    else
        check(call(xc, [&](void* st) {
                  return tdq_fp8_linear(ptr<uint8_t>(xc), ptr<float>(xs), ptr<uint8_t>(wc), ptr<float>(ws), ptr<float>(bias), M, I_pad, O, ptr(y), dt,
                                        M > 1 ? y.stride(0) : O, wsp, wsp_bytes, st);
              }), "tdq_fp8_linear");
    return THPVariable_Wrap(y);
}

// One side of the rotation: the strides of x and out, both [M, H, D].
tdq_rope_heads rope_side(const char* name, const at::Tensor& x, const at::Tensor& out, const at::Tensor* weight, int64_t M, int64_t D) {
    const int64_t H = x.size(1);
    const auto last = [&](const at::Tensor& t) { return D == 1 || t.numel() == 0 || t.stride(2) == 1; };
    if (!last(x) || !last(out)) throw Bad{PyExc_ValueError, std::string("the channels of ") + name + " must be adjacent in memory"};
    if (weight) check_tensor((std::string(name) + "_weight").c_str(), *weight, {at::kFloat}, {D}, x);
    return {ptr(x), ptr(out), ptr<float>(weight), H, M > 1 ? x.stride(0) : 0, H > 1 ? x.stride(1) : 0, M > 1 ? out.stride(0) : 0, H > 1 ? out.stride(1) : 0};
}

// qk_norm_rope(q, k, positions, freq, axis, q_weight, k_weight, eps, adjacent, q_out, k_out)  ->  (q_out, k_out)
PyObject* qk_norm_rope(PyObject* const* a) {
    const at::Tensor &q = tensor(a[0]), &pos = tensor(a[2]), &freq = tensor(a[3]), &axis = tensor(a[4]);
    const at::Tensor *k = opt_tensor(a[1]), *qw = opt_tensor(a[5]), *kw = opt_tensor(a[6]), *oq = opt_tensor(a[9]), *ok = opt_tensor(a[10]);
    need_cuda({&q, k, &pos, &freq, &axis, qw, kw, oq, ok});
    if (q.dim() != 3 || (k && k->dim() != 3)) throw Bad{PyExc_ValueError, "q and k must be [M, heads, head_dim]"};
    const int64_t M = q.size(0), D = q.size(2);
    if (k && (k->size(0) != M || k->size(2) != D || k->scalar_type() != q.scalar_type() || k->device() != q.device()))
        throw Bad{PyExc_ValueError, "k must agree with q in tokens, head size, type and device"};
    if (!k && (kw || ok)) throw Bad{PyExc_ValueError, "k_weight and k_out need k"};
    const tdq_dtype dt = dtype_id(q);
    tdq_rope_params p = {};
    if (D > INT32_MAX) throw Bad{PyExc_ValueError, "head_dim is out of range"};
    p.head_dim = (int32_t)D;
    check_tensor("freq", freq, {at::kDouble}, {freq.numel()}, q);
    check_tensor("axis", axis, {at::kInt}, {freq.numel()}, q);
    if (2 * freq.numel() > D) throw Bad{PyExc_ValueError, "the table has more pairs than half of head_dim"};
    p.rotary_dim = (int32_t)(2 * freq.numel());
    if (pos.dim() < 1 || pos.dim() > 2) throw Bad{PyExc_ValueError, "positions must be [M, axes] or [M]"};
    const int64_t axes = pos.dim() == 2 ? pos.size(1) : 1;
    if (pos.dim() == 2) check_tensor("positions", pos, {at::kLong}, {M, axes}, q);
    else check_tensor("positions", pos, {at::kLong}, {M}, q);
    if (axes > INT32_MAX) throw Bad{PyExc_ValueError, "positions have too many axes"};
    p.n_axes = (int32_t)axes;
    if (a[7] != Py_None) {
        const double eps = PyFloat_AsDouble(a[7]);
        if (eps == -1.0 && PyErr_Occurred()) throw python_error();
        p.eps = (float)eps;
        p.flags |= TDQ_ROPE_NORM;
    } else if (qw || kw) {
        throw Bad{PyExc_ValueError, "weights need the norm: eps is None"};
    }
    const int adjacent = PyObject_IsTrue(a[8]);
    if (adjacent < 0) throw python_error();
    if (adjacent) p.flags |= TDQ_ROPE_ADJACENT;
    const auto out_of = [&](const char* name, const at::Tensor& x, const at::Tensor* o) {
        if (!o) return new_like(x, x.sizes(), x.scalar_type());
        if (o->sizes() != x.sizes() || o->scalar_type() != x.scalar_type() || o->device() != x.device())
            throw Bad{PyExc_ValueError, std::string(name) + " must agree with its input in sizes, type and device"};
        return *o;
    };
    const at::Tensor q_out = out_of("q_out", q, oq);
    const at::Tensor k_out = k ? out_of("k_out", *k, ok) : at::Tensor();
    const tdq_rope_heads hq = rope_side("q", q, q_out, qw, M, D);
    tdq_rope_heads hk = {};
    if (k) hk = rope_side("k", *k, k_out, kw, M, D);
    check(call(q, [&](void* st) {
              return tdq_qk_norm_rope(&hq, k ? &hk : nullptr, dt, M, &p, ptr<int64_t>(pos), ptr<double>(freq), ptr<int32_t>(axis), st);
          }), "tdq_qk_norm_rope");
    if (k) return tuple2(q_out, k_out);
    PyObject* pq = THPVariable_Wrap(q_out);
    PyObject* t = pq ? PyTuple_Pack(2, pq, Py_None) : nullptr;
    Py_XDECREF(pq);
    return t;
}

// The rows of a [..., C] tensor: M of them, `stride` elements apart, channels adjacent.
struct Rows {
    at::Tensor t;          // keeps a copy alive where the rows had to be brought together
    int64_t M, C, stride;
    void* p() const { return t.data_ptr(); }
};
Rows rows_of(const char* name, const at::Tensor& t, bool may_copy) {
    if (t.dim() < 1 || t.size(-1) < 1) throw Bad{PyExc_ValueError, std::string(name) + " must have channels"};
    const int64_t C = t.size(-1), M = t.numel() / C;
    if (!may_copy && t.dim() != 2 && !t.is_contiguous()) throw Bad{PyExc_ValueError, std::string(name) + " must be a matrix or contiguous"};
    const at::Tensor r = t.dim() == 2 ? t : t.reshape({M, C});
    if (C > 1 && M > 0 && r.stride(1) != 1) throw Bad{PyExc_ValueError, std::string(name) + ": the channel axis must be contiguous"};
    return {r, M, C, M > 1 ? r.stride(0) : C};
}
// a tensor whose rows go with those of x: as many, as long, of its type and device
Rows rows_like(const char* name, const at::Tensor& t, const Rows& x, bool may_copy) {
    if (t.device() != x.t.device()) throw Bad{PyExc_ValueError, std::string(name) + " is on " + t.device().str() + ", not on " + x.t.device().str()};
    if (t.scalar_type() != x.t.scalar_type()) throw Bad{PyExc_TypeError, std::string(name) + " must be " + dtype_name(x.t.scalar_type()) + ", got " + dtype_name(t.scalar_type())};
    const Rows r = rows_of(name, t, may_copy);
    if (r.M != x.M || r.C != x.C)
        throw Bad{PyExc_ValueError, std::string(name) + " must have " + std::to_string(x.M) + " rows of " + std::to_string(x.C) + " channels"};
    return r;
}
at::Tensor vector_of(const char* name, const at::Tensor* given, int64_t n, const at::Tensor& on) {
    if (given) check_tensor(name, *given, {at::kFloat}, {n}, on);
    return given ? *given : new_like(on, {n}, at::kFloat);
}
PyObject* tuple_of(std::initializer_list<at::Tensor> ts) {
    PyObject* t = PyTuple_New((Py_ssize_t)ts.size());
    Py_ssize_t i = 0;
    for (const at::Tensor& v : ts) {
        if (!t) break;
        PyObject* o = v.defined() ? THPVariable_Wrap(v) : Py_NewRef(Py_None);
        if (!o) {
            Py_DECREF(t);
            return nullptr;
        }
        PyTuple_SET_ITEM(t, i++, o);
    }
    return t;
}
// The caller's workspace, or one from the caching allocator for the length of the call.
struct Scratch {
    at::DataPtr own;
    void* p = nullptr;
    size_t bytes = 0;
    template <typename F>
    Scratch(const at::Tensor* given, const at::Tensor& on, F&& size) {
        if (given) {
            check_tensor("workspace", *given, {at::kByte}, given->sizes(), on);
            p = given->data_ptr();
            bytes = (size_t)given->numel();
            return;
        }
        c10::cuda::CUDAGuard guard(on.device());
        bytes = size();
        if (!bytes) return;
        own = c10::cuda::CUDACachingAllocator::get()->allocate(bytes);
        p = own.get();
    }
};

// layer_norm(x, weight, bias, eps, y, mean, rstd)  ->  (y, mean, rstd)
PyObject* layer_norm(PyObject* const* a) {
    const at::Tensor& x0 = tensor(a[0]);
    const at::Tensor *w = opt_tensor(a[1]), *b = opt_tensor(a[2]), *oy = opt_tensor(a[4]), *om = opt_tensor(a[5]), *orr = opt_tensor(a[6]);
    need_cuda({&x0, w, b, oy, om, orr});
    const double eps = float_arg(a[3]);
    const Rows x = rows_of("x", x0, true);
    const tdq_dtype dt = dtype_id(x0);
    if (w) check_tensor("weight", *w, {at::kFloat}, {x.C}, x0);
    if (b) check_tensor("bias", *b, {at::kFloat}, {x.C}, x0);
    const at::Tensor out = oy ? *oy : new_like(x0, x0.sizes(), x0.scalar_type());
    const Rows y = rows_like("y", out, x, false);
    const at::Tensor mean = vector_of("mean", om, x.M, x0), rstd = vector_of("rstd", orr, x.M, x0);
    if (x.M > 0)
        check(call(x0, [&](void* st) {
                  return tdq_layer_norm(x.p(), dt, x.M, x.C, x.stride, ptr<float>(w), ptr<float>(b), (float)eps, 0, y.p(), y.stride, nullptr, nullptr,
                                        ptr<float>(mean), ptr<float>(rstd), st);
              }), "tdq_layer_norm");
    return tuple_of({out, mean, rstd});
}

// layer_norm_fp8(x, weight, bias, eps, pow2, codes, scale, mean, rstd)  ->  (codes, scale, mean, rstd)
PyObject* layer_norm_fp8(PyObject* const* a) {
    const at::Tensor& x0 = tensor(a[0]);
    const at::Tensor *w = opt_tensor(a[1]), *b = opt_tensor(a[2]), *oc = opt_tensor(a[5]), *os = opt_tensor(a[6]), *om = opt_tensor(a[7]), *orr = opt_tensor(a[8]);
    need_cuda({&x0, w, b, oc, os, om, orr});
    const double eps = float_arg(a[3]);
    const bool pow2 = truth(a[4]);
    const Rows x = rows_of("x", x0, true);
    const tdq_dtype dt = dtype_id(x0);
    const int64_t K = fp8_blocks(x.C);
    if (w) check_tensor("weight", *w, {at::kFloat}, {x.C}, x0);
    if (b) check_tensor("bias", *b, {at::kFloat}, {x.C}, x0);
    if (oc) check_tensor("codes", *oc, {at::kFloat8_e4m3fn, at::kByte}, {x.M, K * kFp8Block}, x0);
    if (os) check_tensor("scale", *os, {at::kFloat}, {x.M, K}, x0);
    const at::Tensor codes = oc ? *oc : new_like(x0, {x.M, K * kFp8Block}, at::kFloat8_e4m3fn);
    const at::Tensor scale = os ? *os : new_like(x0, {x.M, K}, at::kFloat);
    const at::Tensor mean = vector_of("mean", om, x.M, x0), rstd = vector_of("rstd", orr, x.M, x0);
    if (x.M > 0)
        check(call(x0, [&](void* st) {
                  return tdq_layer_norm(x.p(), dt, x.M, x.C, x.stride, ptr<float>(w), ptr<float>(b), (float)eps, pow2 ? TDQ_NORM_POW2 : 0u, nullptr, 0,
                                        ptr<uint8_t>(codes), ptr<float>(scale), ptr<float>(mean), ptr<float>(rstd), st);
              }), "tdq_layer_norm");
    return tuple_of({codes, scale, mean, rstd});
}

// layer_norm_backward(dy, x, mean, rstd, weight, add, dx, dweight, dbias, workspace)  ->  (dx, dweight, dbias)
PyObject* layer_norm_backward(PyObject* const* a) {
    const at::Tensor &dy0 = tensor(a[0]), &x0 = tensor(a[1]), &mean = tensor(a[2]), &rstd = tensor(a[3]);
    const at::Tensor *w = opt_tensor(a[4]), *add0 = opt_tensor(a[5]), *odx = opt_tensor(a[6]), *odw = opt_tensor(a[7]), *odb = opt_tensor(a[8]), *ow = opt_tensor(a[9]);
    need_cuda({&dy0, &x0, &mean, &rstd, w, add0, odx, odw, odb, ow});
    const Rows x = rows_of("x", x0, true);
    const tdq_dtype dt = dtype_id(x0);
    const Rows dy = rows_like("dy", dy0, x, true);
    Rows add = {};
    if (add0) add = rows_like("add", *add0, x, true);
    check_tensor("mean", mean, {at::kFloat}, {x.M}, x0);
    check_tensor("rstd", rstd, {at::kFloat}, {x.M}, x0);
    if (w) check_tensor("weight", *w, {at::kFloat}, {x.C}, x0);
    const at::Tensor out = odx ? *odx : new_like(x0, x0.sizes(), x0.scalar_type());
    const Rows dx = rows_like("dx", out, x, false);
    const at::Tensor dw = vector_of("dweight", odw, x.C, x0), db = vector_of("dbias", odb, x.C, x0);
    const Scratch ws(ow, x0, [&] { return tdq_layer_norm_backward_workspace_bytes(x.M, x.C); });
    check(call(x0, [&](void* st) {
              return tdq_layer_norm_backward(dy.p(), dy.stride, x.p(), x.stride, dt, x.M, x.C, ptr<float>(mean), ptr<float>(rstd), ptr<float>(w),
                                             add0 ? add.p() : nullptr, add.stride, dx.p(), dx.stride, ptr<float>(dw), ptr<float>(db), ws.p, ws.bytes, st);
          }), "tdq_layer_norm_backward");
    return tuple_of({out, dw, db});
}

// fp8_weight_grad(dy, xcodes, xscale, cin, out_dtype, bias, dw, db, workspace)  ->  (dw, db or None)
PyObject* fp8_weight_grad(PyObject* const* a) {
    const at::Tensor &dy0 = tensor(a[0]), &xc = tensor(a[1]), &xs = tensor(a[2]);
    const at::Tensor *odw = opt_tensor(a[6]), *odb = opt_tensor(a[7]), *ow = opt_tensor(a[8]);
    need_cuda({&dy0, &xc, &xs, odw, odb, ow});
    const Rows dy = rows_of("dy", dy0, true);
    const tdq_dtype dt = dtype_id(dy0);
    const int64_t I = int_arg(a[3]), M = dy.M, O = dy.C;
    if (I < 1) throw Bad{PyExc_ValueError, "cin must be positive"};
    const int64_t K = fp8_blocks(I);
    check_tensor("xcodes", xc, {at::kFloat8_e4m3fn, at::kByte}, {M, K * kFp8Block}, dy0);
    check_tensor("xscale", xs, {at::kFloat}, {M, K}, dy0);
    const at::Tensor dw = odw ? *odw : new_like(dy0, {O, I}, dtype_arg(a[4]));
    if (dw.dim() != 2 || dw.size(0) != O || dw.size(1) != I || (I > 1 && dw.stride(1) != 1))
        throw Bad{PyExc_ValueError, "dw must be of size [" + std::to_string(O) + ", " + std::to_string(I) + "], its columns adjacent in memory"};
    if (dw.device() != dy0.device()) throw Bad{PyExc_ValueError, "dw is on " + dw.device().str() + ", not on " + dy0.device().str()};
    const tdq_dtype wt = dtype_id(dw);
    const bool bias = truth(a[5]);
    if (!bias && odb) throw Bad{PyExc_ValueError, "db was given and bias is False"};
    const at::Tensor db = bias ? vector_of("db", odb, O, dy0) : at::Tensor();
    const Scratch ws(ow, dy0, [&] { return tdq_fp8_weight_grad_workspace_bytes(dy.p(), dt, dy.stride, M, O, I); });
    check(call(dy0, [&](void* st) {
              return tdq_fp8_weight_grad(dy.p(), dt, dy.stride, ptr<uint8_t>(xc), ptr<float>(xs), M, O, I, ptr(dw), wt, O > 1 ? dw.stride(0) : I,
                                         bias ? ptr<float>(db) : nullptr, ws.p, ws.bytes, st);
          }), "tdq_fp8_weight_grad");
    return tuple_of({dw, db});
}

// activation_backward_fp8(dh, zcodes, zscale, activation, dz)
PyObject* activation_backward_fp8(PyObject* const* a) {
    const at::Tensor &dh0 = tensor(a[0]), &zc = tensor(a[1]), &zs = tensor(a[2]);
    const at::Tensor* odz = opt_tensor(a[4]);
    need_cuda({&dh0, &zc, &zs, odz});
    const Rows dh = rows_of("dh", dh0, true);
    const tdq_dtype dt = dtype_id(dh0);
    const int64_t act = int_arg(a[3]), K = fp8_blocks(dh.C);
    check_tensor("zcodes", zc, {at::kFloat8_e4m3fn, at::kByte}, {dh.M, K * kFp8Block}, dh0);
    check_tensor("zscale", zs, {at::kFloat}, {dh.M, K}, dh0);
    const at::Tensor out = odz ? *odz : new_like(dh0, dh0.sizes(), dh0.scalar_type());
    const Rows dz = rows_like("dz", out, dh, false);
    check(call(dh0, [&](void* st) {
              return tdq_activation_backward_fp8(dh.p(), dt, dh.M, dh.C, dh.stride, ptr<uint8_t>(zc), ptr<float>(zs), (int32_t)act, dz.p(), dz.stride, st);
          }), "tdq_activation_backward_fp8");
    return THPVariable_Wrap(out);
}

// Argument count, and C++ exceptions as Python ones.
template <PyObject* (*F)(PyObject* const*), int N>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != N) {
        PyErr_Format(PyExc_TypeError, "expected %d arguments, got %zd", N, n);
        return nullptr;
    }
    try {
        return F(args);
    } catch (const Bad& b) {
        PyErr_SetString(b.type, b.text.c_str());
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

PyObject* set_error_class(PyObject*, PyObject* cls) {
    Py_INCREF(cls);
    Py_XSETREF(g_tdq_error, cls);
    Py_RETURN_NONE;
}

#define TDQ_ENTRY(NAME, N) {#NAME, (PyCFunction)(void (*)(void))entry<NAME, N>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    TDQ_ENTRY(quantize_act, 5), TDQ_ENTRY(quantize_act_fixed, 6), TDQ_ENTRY(quantize_act_nchw, 5), TDQ_ENTRY(quantize_weight, 4),
    TDQ_ENTRY(w4a4_linear, 11), TDQ_ENTRY(w4a4_linear_static, 8), TDQ_ENTRY(quant_linear_fused, 8), TDQ_ENTRY(quant_linear_host, 7),
    TDQ_ENTRY(quantize_act_fp8, 4), TDQ_ENTRY(quantize_weight_fp8, 3), TDQ_ENTRY(fp8_linear, 11), TDQ_ENTRY(qk_norm_rope, 11),
    TDQ_ENTRY(layer_norm, 7), TDQ_ENTRY(layer_norm_fp8, 9), TDQ_ENTRY(layer_norm_backward, 10),
    TDQ_ENTRY(fp8_weight_grad, 9), TDQ_ENTRY(activation_backward_fp8, 5),
    {"set_error_class", set_error_class, METH_O, nullptr}, {nullptr, nullptr, 0, nullptr}};
#undef TDQ_ENTRY

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tdq_host", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tdq_host(void) { return PyModule_Create(&module); }
