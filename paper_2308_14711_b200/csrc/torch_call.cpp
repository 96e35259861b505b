// The tensor-level calls of small launches for Python, as a CPython extension module: fff_forward_infer, the routing losses and
// fff_quantize_mx4.
//
// Checks of type, shape and contiguity, two allocations, the current stream's handle and the call cost 9.4 us of host time per
// forward when Python and ctypes make them, more than the kernel of a small batch takes (5 to 8.5 us); here they cost about
// half of that, and a batch of one image (197 tokens, D = 768) went from 9.6 us to the 8.6 us that its kernel takes.  The
// module computes nothing: it calls the library's functions, whose addresses it is given, with the tensors' addresses.  For arguments
// that it does not take as they are it returns None, and the caller's own checks then say what is wrong with them.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/EmptyTensor.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

namespace {

using ForwardInfer = int (*)(void*, const void*, void*, int32_t*, int64_t, void*);
using BalanceLoss = int (*)(void*, const float*, const int32_t*, const uint8_t*, float*, int32_t*, float*, int64_t, void*);
using BalanceBackward = int (*)(void*, const int32_t*, const uint8_t*, const int32_t*, const float*, float*, int64_t, void*);
using RoutingBackward = int (*)(void*, const float*, const float*, const int32_t*, const uint8_t*, const int32_t*, const float*, float*, int64_t,
                                void*);
using QuantizeMx4 = int (*)(const void*, int, int64_t, int64_t, uint8_t*, uint8_t*, void*, void*);
ForwardInfer g_forward = nullptr;
BalanceLoss g_balance_loss = nullptr;
BalanceBackward g_balance_backward = nullptr;
RoutingBackward g_routing_backward = nullptr;
QuantizeMx4 g_quantize_mx4 = nullptr;

bool matches(const at::Tensor& t, at::ScalarType type, int64_t rows, int64_t cols) {
    if (!t.is_cuda() || t.layout() != at::kStrided || t.scalar_type() != type || !t.is_contiguous()) return false;
    if (cols < 0) return t.dim() == 1 && t.size(0) == rows;
    return t.dim() == 2 && t.size(0) == rows && t.size(1) == cols;
}

// New tensors on the device of one, straight from the allocator where that device is the current one (at::empty finds its way there through the
// dispatcher: 0.4 us more each, of 6.0 us for fff_balance_loss with three of them).
// They are memory of the stream that writes them (its address is an argument, or None for the current one): memory of another stream may still be
// read there for whoever had it before.  The current stream, which may read them, is noted, so that they may be dropped at any time.
struct Fresh {
    const at::Tensor& like;
    const bool here, elsewhere;
    void* const stream;
    Fresh(const at::Tensor& t, PyObject* arg, void* st) : like(t), here(t.device().index() == c10::cuda::current_device()), elsewhere(arg != Py_None), stream(st) {}
    at::Tensor operator()(at::IntArrayRef sizes, at::ScalarType type) const {
        if (!elsewhere) return make(sizes, type);
        const auto device = like.device().index();
        const c10::cuda::CUDAStream current = c10::cuda::getCurrentCUDAStream(device);
        at::Tensor t;
        {
            c10::cuda::CUDAStreamGuard guard(c10::cuda::getStreamFromExternal(static_cast<cudaStream_t>(stream), device));
            t = at::empty(sizes, like.options().requires_grad(false).dtype(type));
        }
        c10::cuda::CUDACachingAllocator::recordStream(t.storage().data_ptr(), current);
        return t;
    }
private:
    at::Tensor make(at::IntArrayRef sizes, at::ScalarType type) const {
        if (!here) return at::empty(sizes, like.options().requires_grad(false).dtype(type));
        return at::Tensor(at::detail::empty_generic(sizes, c10::cuda::CUDACachingAllocator::get(), c10::DispatchKeySet(c10::DispatchKey::CUDA), type, {}));
    }
};

// set_addresses(forward_infer, balance_loss, balance_loss_backward, routing_backward, quantize_mx4)
PyObject* set_addresses(PyObject*, PyObject* const* args, Py_ssize_t n) {
    void* p[5];
    if (n != 5) return PyErr_SetString(PyExc_TypeError, "five addresses"), nullptr;
    for (int i = 0; i < 5; ++i) p[i] = PyLong_AsVoidPtr(args[i]);
    if (PyErr_Occurred()) return nullptr;
    g_forward = reinterpret_cast<ForwardInfer>(p[0]);
    g_balance_loss = reinterpret_cast<BalanceLoss>(p[1]);
    g_balance_backward = reinterpret_cast<BalanceBackward>(p[2]);
    g_routing_backward = reinterpret_cast<RoutingBackward>(p[3]);
    g_quantize_mx4 = reinterpret_cast<QuantizeMx4>(p[4]);
    Py_RETURN_NONE;
}

// An optional tensor argument: false if it is there and not what is wanted.  `p` is its address, or null.
template <typename T>
bool optional(PyObject* arg, at::ScalarType type, int64_t rows, int64_t cols, const T** p) {
    *p = nullptr;
    if (arg == Py_None) return true;
    if (!THPVariable_Check(arg) || !matches(THPVariable_Unpack(arg), type, rows, cols)) return false;
    *p = static_cast<const T*>(THPVariable_Unpack(arg).data_ptr());
    return true;
}
// A token mask: bool or uint8.
bool optional_mask(PyObject* arg, int64_t B, const uint8_t** p) {
    return optional(arg, at::kBool, B, -1, p) || optional(arg, at::kByte, B, -1, p);
}
// One float32 of any shape, or None.
bool optional_scalar(PyObject* arg, const float** p) {
    *p = nullptr;
    if (arg == Py_None) return true;
    if (!THPVariable_Check(arg)) return false;
    const at::Tensor& t = THPVariable_Unpack(arg);
    if (!t.is_cuda() || t.layout() != at::kStrided || t.scalar_type() != at::kFloat || t.numel() != 1) return false;
    *p = static_cast<const float*>(t.data_ptr());
    return true;
}
// The stream of an address argument, or the current one of the tensor's device.
void* stream_of(PyObject* arg, const at::Tensor& t) {
    return arg == Py_None ? (void*)c10::cuda::getCurrentCUDAStream(t.device().index()).stream() : PyLong_AsVoidPtr(arg);
}
// (status, tensors ..), undefined tensors as None.
PyObject* results(int status, std::initializer_list<at::Tensor> tensors) {
    PyObject* out = PyTuple_New(1 + (Py_ssize_t)tensors.size());
    PyObject* ps = out ? PyLong_FromLong(status) : nullptr;
    if (!ps) return Py_XDECREF(out), nullptr;
    PyTuple_SET_ITEM(out, 0, ps);
    Py_ssize_t i = 1;
    for (const at::Tensor& t : tensors) {
        PyObject* p = t.defined() ? THPVariable_Wrap(t) : (Py_INCREF(Py_None), Py_None);
        if (!p) return Py_DECREF(out), nullptr;
        PyTuple_SET_ITEM(out, i++, p);
    }
    return out;
}

// balance_loss(handle, n_leaves, mixture, leaf_idx, token_mask or None, stream address or None) -> (status, loss, counts, mean) or None
PyObject* balance_loss(PyObject*, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 6 || !g_balance_loss || !THPVariable_Check(args[2])) Py_RETURN_NONE;
    void* handle = args[0] == Py_None ? nullptr : PyLong_AsVoidPtr(args[0]);
    const int64_t L = PyLong_AsLongLong(args[1]);
    if (PyErr_Occurred()) return nullptr;
    const at::Tensor& mix = THPVariable_Unpack(args[2]);
    if (mix.dim() != 2 || !matches(mix, at::kFloat, mix.size(0), L)) Py_RETURN_NONE;
    const int64_t B = mix.size(0);
    const int32_t* leaf;
    const uint8_t* mask;
    if (args[3] == Py_None || !optional(args[3], at::kInt, B, -1, &leaf) || !optional_mask(args[4], B, &mask)) Py_RETURN_NONE;
    void* stream = stream_of(args[5], mix);
    if (PyErr_Occurred()) return nullptr;
    const Fresh fresh(mix, args[5], stream);
    at::Tensor loss = fresh({}, at::kFloat), counts = fresh({L}, at::kInt), mean = fresh({L}, at::kFloat);
    const float* mp = static_cast<const float*>(mix.data_ptr());
    float *lp = static_cast<float*>(loss.data_ptr()), *ep = static_cast<float*>(mean.data_ptr());
    int32_t* cp = static_cast<int32_t*>(counts.data_ptr());
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = g_balance_loss(handle, mp, leaf, mask, lp, cp, ep, B, stream);
    Py_END_ALLOW_THREADS
    return results(status, {loss, counts, mean});
    END_HANDLE_TH_ERRORS
}

// balance_loss_backward(handle, n_leaves, leaf_idx, counts, dloss, token_mask or None, stream address or None) -> (status, dmixture) or None
PyObject* balance_loss_backward(PyObject*, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 7 || !g_balance_backward || !THPVariable_Check(args[2]) || args[3] == Py_None || args[4] == Py_None) Py_RETURN_NONE;
    void* handle = args[0] == Py_None ? nullptr : PyLong_AsVoidPtr(args[0]);
    const int64_t L = PyLong_AsLongLong(args[1]);
    if (PyErr_Occurred()) return nullptr;
    const at::Tensor& leaves = THPVariable_Unpack(args[2]);
    if (leaves.dim() != 1) Py_RETURN_NONE;
    const int64_t B = leaves.size(0);
    const int32_t *leaf, *counts;
    const float* dloss;
    const uint8_t* mask;
    if (!optional(args[2], at::kInt, B, -1, &leaf) || !optional(args[3], at::kInt, L, -1, &counts) || !optional_scalar(args[4], &dloss) ||
        !optional_mask(args[5], B, &mask))
        Py_RETURN_NONE;
    void* stream = stream_of(args[6], leaves);
    if (PyErr_Occurred()) return nullptr;
    at::Tensor out = Fresh(leaves, args[6], stream)({B, L}, at::kFloat);
    float* op = static_cast<float*>(out.data_ptr());
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = g_balance_backward(handle, leaf, mask, counts, dloss, op, B, stream);
    Py_END_ALLOW_THREADS
    return results(status, {out});
    END_HANDLE_TH_ERRORS
}

// routing_backward(handle, n_leaves, mixture, dmixture, leaf_idx, counts, dloss, token_mask, stream address), all from dmixture on may be None
//   -> (status, dlogits) or None
PyObject* routing_backward(PyObject*, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 9 || !g_routing_backward || !THPVariable_Check(args[2])) Py_RETURN_NONE;
    void* handle = args[0] == Py_None ? nullptr : PyLong_AsVoidPtr(args[0]);
    const int64_t L = PyLong_AsLongLong(args[1]);
    if (PyErr_Occurred()) return nullptr;
    const at::Tensor& mix = THPVariable_Unpack(args[2]);
    if (mix.dim() != 2 || !matches(mix, at::kFloat, mix.size(0), L)) Py_RETURN_NONE;
    const int64_t B = mix.size(0);
    const float *up, *dloss;
    const int32_t *leaf, *counts;
    const uint8_t* mask;
    if (!optional(args[3], at::kFloat, B, L, &up) || !optional(args[4], at::kInt, B, -1, &leaf) || !optional(args[5], at::kInt, L, -1, &counts) ||
        !optional_scalar(args[6], &dloss) || !optional_mask(args[7], B, &mask))
        Py_RETURN_NONE;
    void* stream = stream_of(args[8], mix);
    if (PyErr_Occurred()) return nullptr;
    at::Tensor out = Fresh(mix, args[8], stream)({B, L - 1}, at::kFloat);
    const float* mp = static_cast<const float*>(mix.data_ptr());
    float* op = static_cast<float*>(out.data_ptr());
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = g_routing_backward(handle, mp, up, leaf, mask, counts, dloss, op, B, stream);
    Py_END_ALLOW_THREADS
    return results(status, {out});
    END_HANDLE_TH_ERRORS
}

// quantize_mx4(w, want_values, stream address or None) -> (status, codes, scales, values or None) or None (w on another device too)
PyObject* quantize_mx4(PyObject*, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 3 || !g_quantize_mx4 || !THPVariable_Check(args[0])) Py_RETURN_NONE;
    const at::Tensor& w = THPVariable_Unpack(args[0]);
    if (!w.is_cuda() || w.layout() != at::kStrided || !w.is_contiguous() || w.dim() < 1 ||
        (w.scalar_type() != at::kFloat && w.scalar_type() != at::kBFloat16) || w.device().index() != c10::cuda::current_device())
        Py_RETURN_NONE;
    const int want = PyObject_IsTrue(args[1]);
    void* stream = stream_of(args[2], w);
    if (want < 0 || PyErr_Occurred()) return nullptr;
    const int64_t cols = w.size(w.dim() - 1), rows = cols > 0 ? w.numel() / cols : 0;
    const Fresh fresh(w, args[2], stream);
    at::DimVector shape(w.sizes().begin(), w.sizes().end());
    shape.back() = (cols + 1) / 2;
    at::Tensor codes = fresh(shape, at::kByte);
    shape.back() = (cols + 31) / 32;
    at::Tensor scales = fresh(shape, at::kByte), values;
    if (want) values = fresh(w.sizes(), w.scalar_type());
    const void* wp = w.data_ptr();
    uint8_t *cp = static_cast<uint8_t*>(codes.data_ptr()), *sp = static_cast<uint8_t*>(scales.data_ptr());
    void* vp = want ? values.data_ptr() : nullptr;
    const int dtype = w.scalar_type() == at::kFloat ? 0 : 1;
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = g_quantize_mx4(wp, dtype, rows, cols, cp, sp, vp, stream);
    Py_END_ALLOW_THREADS
    return results(status, {codes, scales, values});
    END_HANDLE_TH_ERRORS
}

// forward(handle, D, O, is_bf16, x, y or None, leaf_idx or None, want_leaf_idx, stream address or None)
//   -> (status, y, leaf_idx or None), or None when the arguments are not what the call takes
// (A tensor may answer any question about itself with an exception, a Python one from a subclass's dispatch among them: all of
// it stands between the macros that turn C++ exceptions into Python errors, each into the type that torch raises for it.)
PyObject* forward(PyObject*, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 9 || !g_forward || !THPVariable_Check(args[4])) Py_RETURN_NONE;
    void* handle = args[0] == Py_None ? nullptr : PyLong_AsVoidPtr(args[0]);
    const int64_t D = PyLong_AsLongLong(args[1]), O = PyLong_AsLongLong(args[2]);
    const bool bf16 = PyObject_IsTrue(args[3]) == 1, want_leaf = PyObject_IsTrue(args[7]) == 1;
    if (PyErr_Occurred()) return nullptr;
    const at::ScalarType type = bf16 ? at::kBFloat16 : at::kFloat;
    const at::Tensor& x = THPVariable_Unpack(args[4]);
    if (x.dim() != 2 || !matches(x, type, x.size(0), D)) Py_RETURN_NONE;
    const int64_t B = x.size(0);
    if (args[5] != Py_None && (!THPVariable_Check(args[5]) || !matches(THPVariable_Unpack(args[5]), type, B, O))) Py_RETURN_NONE;
    if (args[6] != Py_None && (!THPVariable_Check(args[6]) || !matches(THPVariable_Unpack(args[6]), at::kInt, B, -1))) Py_RETURN_NONE;
    at::Tensor y, leaf;
    void* stream = nullptr;
    if (args[8] == Py_None) stream = c10::cuda::getCurrentCUDAStream().stream();
    else stream = PyLong_AsVoidPtr(args[8]);
    if (PyErr_Occurred()) return nullptr;
    if (args[5] != Py_None) y = THPVariable_Unpack(args[5]);
    else y = Fresh(x, args[8], stream)({B, O}, type);
    if (args[6] != Py_None) leaf = THPVariable_Unpack(args[6]);
    else if (want_leaf) leaf = Fresh(x, args[8], stream)({B}, at::kInt);
    const void* xp = x.data_ptr();
    void* yp = y.data_ptr();
    int32_t* lp = leaf.defined() ? static_cast<int32_t*>(leaf.data_ptr()) : nullptr;
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = g_forward(handle, xp, yp, lp, B, stream);
    Py_END_ALLOW_THREADS
    PyObject* py = args[5] != Py_None ? (Py_INCREF(args[5]), args[5]) : THPVariable_Wrap(std::move(y));
    PyObject* pl = args[6] != Py_None   ? (Py_INCREF(args[6]), args[6])
                   : leaf.defined()     ? THPVariable_Wrap(std::move(leaf))
                                        : (Py_INCREF(Py_None), Py_None);
    PyObject* ps = PyLong_FromLong(status);
    PyObject* out = py && pl && ps ? PyTuple_New(3) : nullptr;
    if (!out) {
        Py_XDECREF(py); Py_XDECREF(pl); Py_XDECREF(ps);
        return nullptr;
    }
    PyTuple_SET_ITEM(out, 0, ps);
    PyTuple_SET_ITEM(out, 1, py);
    PyTuple_SET_ITEM(out, 2, pl);
    return out;
    END_HANDLE_TH_ERRORS
}

PyMethodDef kMethods[] = {
    {"set_addresses", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(set_addresses)), METH_FASTCALL, "Addresses of the library's functions."},
    {"balance_loss", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(balance_loss)), METH_FASTCALL, "Tensor-level fff_balance_loss."},
    {"balance_loss_backward", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(balance_loss_backward)), METH_FASTCALL,
     "Tensor-level fff_balance_loss_backward."},
    {"routing_backward", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(routing_backward)), METH_FASTCALL,
     "Tensor-level fff_routing_backward."},
    {"quantize_mx4", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(quantize_mx4)), METH_FASTCALL, "Tensor-level fff_quantize_mx4."},
    {"forward", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(forward)), METH_FASTCALL, "Tensor-level fff_forward_infer."},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "torch_call", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_torch_call() { return PyModule_Create(&kModule); }
