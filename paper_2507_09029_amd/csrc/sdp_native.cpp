// The library's per-step calls for Python (module _sdp_native): the C functions of sdp.h, with tensors where they take
// device pointers.  A call checks every tensor (contiguous, on the GPU, of the expected type; TypeError otherwise) and
// passes its address; integers pass as they are.  The GIL is released around the call.  Returns the status.
//
// Through ctypes a worker's MLP forward or backward costs the host about 9 us, most of it in marshalling 20 arguments,
// which is more than the fp32 kernels of a small step take on the GPU (four workers of 256 tokens, 10 calls and 18 launches:
// 139 us a step then, 101 this way).
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include <tuple>
#include <type_traits>
#include <utility>

#include "sdp.h"

namespace {

// A pointer parameter: its name in messages and what it points to: 'a' the type given by the call's dtype argument,
// 'i' int32, 'f' float32, 't' int32 or int64, 'v' float32 or bfloat16, 'w' bytes, 'z' as 'a' but a
// matrix whose rows may lie apart (the caller passes their distance), in capitals where None stands for a null pointer; 0 for parameters
// passed as they are (numbers, workspace and stream addresses).
// For calls that state their shapes: d0, d1 are the places of the integer arguments that are the tensor's sizes (kOne: size 1), ld that of
// the distance of its rows.
constexpr signed char kAny = -1, kOne = -2;
struct Param {
    const char* name = nullptr;
    char kind = 0;
    signed char d0 = kAny, d1 = kAny, ld = kAny;
};

// whether argument i has the shape that p states, in every call with such a statement before any tensor is looked at otherwise
bool shape_fits(PyObject* const* args, size_t i, const Param& p) {
    if (p.d0 == kAny || args[i] == Py_None || !THPVariable_Check(args[i])) return true;
    const at::Tensor& t = THPVariable_Unpack(args[i]);
    auto size = [&](signed char d) { return d == kOne ? 1LL : PyLong_AsLongLong(args[d]); };
    const long long n0 = size(p.d0), n1 = p.d1 == kAny ? 0 : size(p.d1);
    if (t.dim() != (p.d1 == kAny ? 1 : 2) || t.size(0) != n0 || (p.d1 != kAny && t.size(1) != n1)) {
        if (p.d1 == kAny) PyErr_Format(PyExc_ValueError, "%s: expected shape (%lld,)", p.name, n0);
        else PyErr_Format(PyExc_ValueError, "%s: expected shape (%lld, %lld)", p.name, n0, n1);
        return false;
    }
    if (p.ld != kAny && n0 > 1 && t.stride(0) != size(p.ld)) {
        PyErr_Format(PyExc_ValueError, "%s: expected rows %lld values apart (the strides of Z)", p.name, size(p.ld));
        return false;
    }
    return true;
}

bool type_error(const Param& p, c10::ScalarType t) {
    const char* n = t == c10::kFloat ? "torch.float32" : t == c10::kBFloat16 ? "torch.bfloat16" : t == c10::kByte ? "torch.uint8" : "torch.int32";
    PyErr_Format(PyExc_TypeError, "%s: expected a contiguous %s tensor on the GPU", p.name, n);
    return false;
}

// `device`: where every tensor has to be, -1 = anywhere
template <class A>
bool take(PyObject* o, const Param& p, c10::ScalarType act, int device, A& out) {
    if constexpr (std::is_pointer_v<A>) {
        if (p.kind == 0) {
            out = (A)PyLong_AsVoidPtr(o);
            return !PyErr_Occurred();
        }
        const bool optional = p.kind >= 'A' && p.kind <= 'Z';
        const char kind = optional ? (char)(p.kind - 'A' + 'a') : p.kind;
        if (optional && o == Py_None) {
            out = nullptr;
            return true;
        }
        c10::ScalarType want = kind == 'f' || kind == 'v' ? c10::kFloat : kind == 'i' || kind == 't' ? c10::kInt : kind == 'w' ? c10::kByte : act;
        if (!THPVariable_Check(o)) return type_error(p, want);
        const at::Tensor& t = THPVariable_Unpack(o);
        if (kind == 't' && t.scalar_type() == c10::kLong) want = c10::kLong;
        if (kind == 'v' && t.scalar_type() == c10::kBFloat16) want = c10::kBFloat16;
        const bool rows_apart = kind == 'z' && t.dim() == 2 && (t.size(1) <= 1 || t.stride(1) == 1);
        if (!t.is_cuda() || !(rows_apart || t.is_contiguous()) || t.scalar_type() != want) return type_error(p, want);
        if (device >= 0 && t.get_device() != device) {
            PyErr_Format(PyExc_ValueError, "%s: on cuda:%d, but the current device is cuda:%d", p.name, (int)t.get_device(), device);
            return false;
        }
        out = (A)t.data_ptr();
        return true;
    } else if constexpr (std::is_floating_point_v<A>) {
        out = (A)PyFloat_AsDouble(o);
        return !PyErr_Occurred();
    } else if constexpr (std::is_unsigned_v<A>) {
        out = (A)PyLong_AsUnsignedLongLong(o);
        return !PyErr_Occurred();
    } else {
        const long long v = PyLong_AsLongLong(o);
        if (v == -1 && PyErr_Occurred()) return false;
        if (v != (long long)(A)v) {
            PyErr_SetString(PyExc_OverflowError, "integer argument out of range");
            return false;
        }
        out = (A)v;
        return true;
    }
}

template <class... A, size_t... I>
PyObject* call(int (*fn)(A...), const Param* params, int dtype_at, PyObject* const* args, Py_ssize_t n, std::index_sequence<I...>,
               int device = -1) {
    if (n != (Py_ssize_t)sizeof...(A)) {
        PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", (Py_ssize_t)sizeof...(A), n);
        return nullptr;
    }
    const long dtype = PyLong_AsLong(args[dtype_at]);
    if (dtype == -1 && PyErr_Occurred()) return nullptr;
    const c10::ScalarType act = dtype == SDP_F32 ? c10::kFloat : c10::kBFloat16;
    std::tuple<A...> v;
    int rc = 0;
    try {
        if (!(shape_fits(args, I, params[I]) && ...)) return nullptr;
        if (!(take(args[I], params[I], act, device, std::get<I>(v)) && ...)) return nullptr;
    } catch (const std::exception& e) { // a tensor without storage
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
    Py_BEGIN_ALLOW_THREADS
    rc = std::apply(fn, v);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

#define SDP_ENTRY(py, fn, dtype_at, ...)                                                                     \
    const Param py##_params[] = {__VA_ARGS__};                                                               \
    template <class... A>                                                                                    \
    PyObject* py##_call(int (*f)(A...), PyObject* const* args, Py_ssize_t n) {                               \
        static_assert(sizeof(py##_params) / sizeof(Param) == sizeof...(A), "one entry per parameter");       \
        return call(f, py##_params, dtype_at, args, n, std::index_sequence_for<A...>{});                     \
    }                                                                                                        \
    PyObject* py(PyObject*, PyObject* const* args, Py_ssize_t n) { return py##_call(&fn, args, n); }

// the same for calls whose first argument is the current device, where every tensor has to be
#define SDP_ENTRY_HERE(py, fn, dtype_at, ...)                                                                \
    const Param py##_params[] = {__VA_ARGS__};                                                               \
    template <class... A>                                                                                    \
    PyObject* py##_call(int (*f)(A...), PyObject* const* args, Py_ssize_t n) {                               \
        static_assert(sizeof(py##_params) / sizeof(Param) == sizeof...(A), "one entry per parameter");       \
        const long device = n > 0 ? PyLong_AsLong(args[0]) : 0;                                              \
        if (device == -1 && PyErr_Occurred()) return nullptr;                                                \
        return call(f, py##_params, dtype_at, args + 1, n - 1, std::index_sequence_for<A...>{}, (int)device); \
    }                                                                                                        \
    PyObject* py(PyObject*, PyObject* const* args, Py_ssize_t n) { return py##_call(&fn, args, n); }

SDP_ENTRY(mlp_fwd, sdp_masked_mlp_fwd, 1, {}, {}, {}, {}, {}, {}, {"X", 'a'}, {"W1", 'a'}, {"W3", 'a'}, {"W2T", 'a'},
          {"idx_k", 'I'}, {"Y", 'a'}, {"G_save", 'a'}, {"U_save", 'a'}, {}, {}, {})
SDP_ENTRY(mlp_bwd, sdp_masked_mlp_bwd, 1, {}, {}, {}, {}, {}, {}, {"X", 'a'}, {"dY", 'a'}, {"W1", 'a'}, {"W3", 'a'},
          {"W2T", 'a'}, {"idx_k", 'i'}, {"G_save", 'a'}, {"U_save", 'a'}, {"dX", 'a'}, {"dW1", 'a'}, {"dW3", 'a'}, {"dW2T", 'a'},
          {}, {}, {}, {})
SDP_ENTRY(attn_fwd, sdp_masked_attn_fwd, 1, {}, {}, {}, {}, {}, {}, {}, {}, {"X", 'a'}, {"Wqkv", 'a'}, {"WoT", 'a'},
          {"head_idx_k", 'I'}, {"Y", 'a'}, {"QKV_save", 'a'}, {"O_save", 'a'}, {"LSE_save", 'f'}, {}, {}, {})
SDP_ENTRY(attn_bwd, sdp_masked_attn_bwd, 1, {}, {}, {}, {}, {}, {}, {}, {}, {"X", 'a'}, {"dY", 'a'}, {"Wqkv", 'a'},
          {"WoT", 'a'}, {"head_idx_k", 'i'}, {"QKV_save", 'a'}, {"O_save", 'a'}, {"LSE_save", 'f'}, {"dX", 'a'}, {"dWqkv", 'a'},
          {"dWoT", 'a'}, {}, {}, {}, {})
SDP_ENTRY(block_fwd, sdp_block_fwd, 2, {}, {}, {}, {}, {}, {}, {}, {}, {}, {"X", 'a'}, {"Wqkv", 'a'}, {"WoT", 'a'},
          {"W1", 'a'}, {"W3", 'a'}, {"W2T", 'a'}, {"Y", 'a'}, {"Hm_save", 'a'}, {"QKV_save", 'a'}, {"O_save", 'a'},
          {"LSE_save", 'f'}, {"G_save", 'a'}, {"U_save", 'a'}, {}, {}, {})
SDP_ENTRY(block_bwd, sdp_block_bwd, 3, {}, {}, {}, {}, {}, {}, {}, {}, {}, {}, {"X", 'a'}, {"dY", 'a'}, {"Wqkv", 'a'},
          {"WoT", 'a'}, {"W1", 'a'}, {"W3", 'a'}, {"W2T", 'a'}, {"Hm_save", 'a'}, {"QKV_save", 'a'}, {"O_save", 'a'},
          {"LSE_save", 'f'}, {"G_save", 'a'}, {"U_save", 'a'}, {"dX", 'a'}, {"dW", 'A'}, {"dW", 'A'}, {"dW", 'A'}, {"dW", 'A'},
          {"dW", 'A'}, {}, {}, {})

SDP_ENTRY_HERE(norm_fwd, sdp_norm_fwd, 1, {}, {}, {}, {}, {}, {"X", 'a', 2, 3}, {"residual", 'A', 2, 3}, {"gamma", 'a', 3}, {"beta", 'A', 3},
               {"H", 'A', 2, 3}, {"Y", 'a', 2, 3}, {"mean", 'F', 2}, {"rstd", 'f', 2}, {})
SDP_ENTRY_HERE(norm_bwd, sdp_norm_bwd, 1, {}, {}, {}, {}, {"H", 'a', 2, 3}, {"dY", 'a', 2, 3}, {"dH", 'A', 2, 3}, {"gamma", 'a', 3}, {"mean", 'F', 2},
               {"rstd", 'f', 2}, {"dX", 'a', 2, 3}, {"dgamma", 'A', 3}, {"dbeta", 'A', 3}, {"ws", 'W'}, {}, {})
SDP_ENTRY_HERE(embed_fwd, sdp_embed_fwd, 0, {}, {}, {}, {}, {}, {}, {"E", 'a', 3, 4}, {"ids", 't', 2}, {"Y", 'a', 2, 4}, {})
SDP_ENTRY_HERE(embed_bwd, sdp_embed_bwd, 0, {}, {}, {}, {}, {}, {}, {"dY", 'a', 2, 4}, {"ids", 't', 2}, {"dE", 'a', 3, 4}, {"ws", 'w'}, {}, {})
SDP_ENTRY_HERE(token_loss, sdp_token_loss, 0, {}, {}, {}, {}, {}, {}, {"Z", 'z', 2, 3, 4}, {"labels", 't', 2}, {"scale_dev", 'F', kOne}, {"nll", 'f', 2},
               {"lse", 'F', 2}, {"dZ", 'Z', 2, 3, 4}, {"loss", 'F', kOne}, {})
SDP_ENTRY_HERE(distill_loss, sdp_distill_loss, 0, {}, {}, {}, {}, {}, {}, {}, {}, {}, {"Z", 'z', 3, 4, 6}, {"ids", 't', 3, 5}, {"top", 'v', 3, 5},
               {"top_lse", 'F', 3}, {"scale_dev", 'F', kOne}, {"kl", 'f', 3}, {"lse", 'F', 3}, {"dZ", 'Z', 3, 4, 6}, {"loss", 'F', kOne}, {})
SDP_ENTRY_HERE(head_loss, sdp_head_loss, 0, {}, {}, {}, {}, {}, {}, {"X", 'a', 2, 4}, {"W", 'a', 3, 4}, {"labels", 't', 2}, {"scale_dev", 'F', kOne},
               {"nll", 'f', 2}, {"lse", 'F', 2}, {"dX", 'A', 2, 4}, {"dW", 'A', 3, 4}, {"loss", 'F', kOne}, {"ws", 'w'}, {}, {})
SDP_ENTRY_HERE(head_distill, sdp_head_distill, 0, {}, {}, {}, {}, {}, {}, {}, {}, {}, {"X", 'a', 3, 5}, {"W", 'a', 4, 5}, {"ids", 't', 3, 6},
               {"top", 'v', 3, 6}, {"top_lse", 'F', 3}, {"scale_dev", 'F', kOne}, {"kl", 'f', 3}, {"lse", 'F', 3}, {"dX", 'A', 3, 5}, {"dW", 'A', 4, 5},
               {"loss", 'F', kOne}, {"ws", 'w'}, {}, {})
SDP_ENTRY_HERE(label_scale, sdp_label_scale, 0, {}, {}, {}, {"labels", 't'}, {"scale", 'f', kOne}, {})

#define SDP_METHOD(py) {#py, (PyCFunction)(void (*)(void))py, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {SDP_METHOD(mlp_fwd),   SDP_METHOD(mlp_bwd),   SDP_METHOD(attn_fwd), SDP_METHOD(attn_bwd),
                         SDP_METHOD(block_fwd), SDP_METHOD(block_bwd),
                         SDP_METHOD(norm_fwd),  SDP_METHOD(norm_bwd),  SDP_METHOD(embed_fwd), SDP_METHOD(embed_bwd),
                         SDP_METHOD(token_loss), SDP_METHOD(label_scale),
                         SDP_METHOD(distill_loss), SDP_METHOD(head_loss), SDP_METHOD(head_distill), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_sdp_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

} // namespace

PyMODINIT_FUNC PyInit__sdp_native() {
    PyObject* m = PyModule_Create(&module);
    // the C++ interface of one torch build: binding.py compares
    if (m && PyModule_AddStringConstant(m, "torch_version", SDP_TORCH_VERSION) < 0) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
