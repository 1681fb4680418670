// The per-call half of the Python binding: argument checks, device pointers and the current stream of the hot entry points, in
// native code.  Through ctypes a grouped call cost about 17 microseconds of interpreter time (argument arrays, type checks,
// stream lookup), more than the GPU needs for it at decode; here it is well under two.  The functions return the library's
// status; bwla.py turns it into an exception.  The library's entry points are handed over as addresses (`bind`), so that
// whichever build of the library the process has loaded is the one that is called.  As through ctypes, other threads run while the
// library works, and what PyTorch throws (a tensor without memory of its own, a stream of a device that is not there) becomes a Python
// exception.
#include <algorithm>

#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "bwla.h"

namespace {

struct Entry {
    decltype(&bwla_w1ax_linear_group) group;
    decltype(&bwla_w1ax_linear) linear;
    decltype(&bwla_layer_w1a16_linear) a16;
    decltype(&bwla_pack_signs) pack;
    decltype(&bwla_fp4_quantize_rows) fp4_quantize;
    decltype(&bwla_fp4_expand_rows) fp4_expand;
    decltype(&bwla_fp4_gemm_codes) fp4_gemm;
    decltype(&bwla_fp4_layer_linear) fp4_linear;
} entry;

PyObject *name_handle, *name_fp4, *name_n, *name_k;      // of a layer: "_h" or "_fp4", its handle as an integer; "N", "K"

const char* dtype_name(at::ScalarType t) {
    return t == at::kBFloat16 ? "torch.bfloat16" : t == at::kFloat ? "torch.float32" : t == at::kInt ? "torch.int32" : t == at::kByte ? "torch.uint8" : "another type";
}

// The tensor behind `o` when it is a CUDA tensor of this type (and number of dimensions), else NULL with TypeError set.
const at::Tensor* need(PyObject* o, at::ScalarType type, const char* name, int ndim) {
    const at::Tensor* t = THPVariable_Check(o) ? &THPVariable_Unpack(o) : nullptr;
    if (!t || !t->is_cuda() || t->scalar_type() != type || (ndim > 0 && t->dim() != ndim)) {
        if (ndim > 0) PyErr_Format(PyExc_TypeError, "%s: expected a CUDA tensor of %s with %d dims", name, dtype_name(type), ndim);
        else PyErr_Format(PyExc_TypeError, "%s: expected a CUDA tensor of %s", name, dtype_name(type));
        return nullptr;
    }
    if (t->numel() > 0 && t->stride(-1) != 1) {
        PyErr_Format(PyExc_TypeError, "%s: innermost dimension must be contiguous", name);
        return nullptr;
    }
    return t;
}
const at::Tensor* tensor(PyObject* o, const char* name) {
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "%s: expected a tensor", name);
        return nullptr;
    }
    return &THPVariable_Unpack(o);
}
void* stream() { return (void*)c10::cuda::getCurrentCUDAStream().stream(); }
// The layer's handle, NULL when it has been destroyed (the library refuses that); false with an exception set for other objects.
bool handle_of(PyObject* layer, const bwla_layer** out) {
    PyObject* h = PyObject_GetAttr(layer, name_handle);
    if (!h) return false;
    *out = h == Py_None ? nullptr : (const bwla_layer*)PyLong_AsVoidPtr(h);
    Py_DECREF(h);
    return !PyErr_Occurred();
}
bool size_of(PyObject* layer, PyObject* name, int64_t* out) {
    PyObject* v = PyObject_GetAttr(layer, name);
    if (!v) return false;
    *out = PyLong_AsLongLong(v);
    Py_DECREF(v);
    return !PyErr_Occurred();
}
// The library's call, with the interpreter free for other threads.
template <typename F, typename... A>
PyObject* unlocked(F entry_point, A... args) {
    int st;
    Py_BEGIN_ALLOW_THREADS
    st = entry_point(args...);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
}
struct Ref {
    PyObject* o;
    explicit Ref(PyObject* p) : o(p) {}
    ~Ref() { Py_XDECREF(o); }
    Ref(const Ref&) = delete;
    Ref(Ref&& other) noexcept : o(other.o) { other.o = nullptr; }
};

// group(layers, x, outs, workspace) -> status
PyObject* call_group(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    if (nargs != 4) { PyErr_SetString(PyExc_TypeError, "group(layers, x, outs, workspace)"); return nullptr; }
    const at::Tensor* x = need(args[1], at::kBFloat16, "x", 2);
    if (!x || PyObject_Size(args[0]) < 0 || PyObject_Size(args[2]) < 0) return nullptr;
    Ref layers(PySequence_Fast(args[0], "layers: expected a sequence")), outs(PySequence_Fast(args[2], "outs: expected a sequence"));
    if (!layers.o || !outs.o) return nullptr;
    constexpr Py_ssize_t kMost = 4;                   // what the library takes
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(layers.o), n_out = PySequence_Fast_GET_SIZE(outs.o);
    const int64_t M = x->size(0);
    const bwla_layer* h[kMost] = {};
    void* o[kMost] = {};                              // (fewer outputs than layers: the library refuses the missing ones)
    int64_t ldo[kMost] = {};
    for (Py_ssize_t i = 0; i < n_out; ++i) {
        const at::Tensor* t = need(PySequence_Fast_GET_ITEM(outs.o, i), at::kBFloat16, "out", 2);
        if (!t) return nullptr;
        if (i >= n) { PyErr_SetString(PyExc_IndexError, "more outputs than layers"); return nullptr; }
        if (i < kMost) { o[i] = t->data_ptr(); ldo[i] = t->stride(0); }
    }
    for (Py_ssize_t i = 0; i < n; ++i) {
        PyObject* layer = PySequence_Fast_GET_ITEM(layers.o, i);
        const bwla_layer* handle = nullptr;
        if (!handle_of(layer, &handle)) return nullptr;
        if (i >= kMost) continue;
        h[i] = handle;
        if (M == 0 && i < n_out && !size_of(layer, name_n, &ldo[i])) return nullptr;
    }
    const at::Tensor* ws = tensor(args[3], "workspace");
    if (!ws) return nullptr;
    return unlocked(entry.group, h, (int)n, (const void*)x->data_ptr(), M, M > 0 ? x->stride(0) : x->size(1), (void* const*)o, (const int64_t*)ldo,
                    ws->data_ptr(), (size_t)ws->numel(), stream());
    END_HANDLE_TH_ERRORS
}

// a16(layer, x, out, workspace) -> status
PyObject* call_a16(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    if (nargs != 4) { PyErr_SetString(PyExc_TypeError, "a16(layer, x, out, workspace)"); return nullptr; }
    const at::Tensor *x = need(args[1], at::kBFloat16, "x", 2), *out, *ws;
    if (!x || !(out = need(args[2], at::kBFloat16, "out", 2)) || !(ws = tensor(args[3], "workspace"))) return nullptr;
    const bwla_layer* h = nullptr;
    if (!handle_of(args[0], &h)) return nullptr;
    const int64_t M = x->size(0);
    int64_t ldx = x->stride(0), ldo = out->stride(0);
    if (M == 0 && (!size_of(args[0], name_k, &ldx) || !size_of(args[0], name_n, &ldo))) return nullptr;
    return unlocked(entry.a16, h, (const void*)x->data_ptr(), M, ldx, out->data_ptr(), ldo, ws->data_ptr(), (size_t)ws->numel(), stream());
    END_HANDLE_TH_ERRORS
}

// linear(x, P1, P2, bits, packed, alpha, U, V, mu, out, workspace) -> status; U, V, mu may be None
PyObject* call_linear(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    if (nargs != 11) { PyErr_SetString(PyExc_TypeError, "linear: eleven arguments"); return nullptr; }
    const at::Tensor *x = need(args[0], at::kBFloat16, "x", 2), *packed, *alpha, *U = nullptr, *V = nullptr, *mu = nullptr, *P1, *P2, *out, *ws;
    if (!x || !(packed = need(args[4], at::kInt, "packed", 2)) || !(alpha = need(args[5], at::kFloat, "alpha", 1))) return nullptr;
    const int64_t M = x->size(0), K = x->size(1), N = packed->size(0);
    int64_t r = 0;
    if (args[6] != Py_None) {
        if (!(U = need(args[6], at::kBFloat16, "U", 2)) || !(V = need(args[7], at::kBFloat16, "V", 2))) return nullptr;
        r = U->size(1);
        if (!U->is_contiguous() || !V->is_contiguous() || V->size(0) != r || V->size(1) != K || U->size(0) != N) {
            PyErr_SetString(PyExc_TypeError, "U must be contiguous [N][r] and V contiguous [r][K]");
            return nullptr;
        }
    }
    if (args[8] != Py_None && !(mu = need(args[8], at::kFloat, "mu", 1))) return nullptr;
    if (!(P1 = tensor(args[1], "P1")) || !(P2 = tensor(args[2], "P2"))) return nullptr;
    if (!packed->is_contiguous() || !P1->is_contiguous() || !P2->is_contiguous()) {
        PyErr_SetString(PyExc_TypeError, "packed, P1 and P2 must be contiguous");
        return nullptr;
    }
    if (!(out = need(args[9], at::kBFloat16, "out", 2)) || !(ws = tensor(args[10], "workspace"))) return nullptr;
    const long bits = PyLong_AsLong(args[3]);
    if (bits == -1 && PyErr_Occurred()) return nullptr;
    return unlocked(entry.linear, (const void*)x->data_ptr(), M, K, M > 0 ? x->stride(0) : K, (const float*)P1->data_ptr(), (int)P1->size(0),
                    (const float*)P2->data_ptr(), (int)P2->size(0), (int)bits, (const uint32_t*)packed->data_ptr(), (const float*)alpha->data_ptr(),
                    mu ? (const float*)mu->data_ptr() : nullptr, U ? (const void*)U->data_ptr() : nullptr, V ? (const void*)V->data_ptr() : nullptr, (int)r,
                    out->data_ptr(), N, M > 0 ? out->stride(0) : N, ws->data_ptr(), (size_t)ws->numel(), stream());
    END_HANDLE_TH_ERRORS
}

// pack(w, packed) -> status
PyObject* call_pack(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    if (nargs != 2) { PyErr_SetString(PyExc_TypeError, "pack(w, packed)"); return nullptr; }
    const at::Tensor* w = tensor(args[0], "w");
    if (!w) return nullptr;
    if (w->scalar_type() != at::kFloat && w->scalar_type() != at::kBFloat16) { PyErr_SetString(PyExc_TypeError, "w must be fp32 or bf16"); return nullptr; }
    const at::Tensor* packed;
    if (!need(args[0], w->scalar_type(), "w", 2) || !(packed = need(args[1], at::kInt, "packed", 2))) return nullptr;
    const int64_t N = w->size(0), K = w->size(1);
    return unlocked(entry.pack, (const void*)w->data_ptr(), w->scalar_type() == at::kFloat ? BWLA_DTYPE_F32 : BWLA_DTYPE_BF16, N, K,
                    N > 0 ? w->stride(0) : K, (uint32_t*)packed->data_ptr(), stream());
    END_HANDLE_TH_ERRORS
}

// ---- microscaled 4-bit rows: codes [rows][K/2], scale tiles, row scales (or None) ----
struct Fp4Rows {
    int64_t rows = 0, K = 0;
    void *codes = nullptr, *scales = nullptr, *row_scales = nullptr;
};
// The library works on the current device: tensors of another one are refused.
bool here(const at::Tensor& t, const char* name) {
    if (t.is_cuda() && t.device().index() == c10::cuda::current_device()) return true;
    PyErr_Format(PyExc_TypeError, "%s: expected a tensor of the current CUDA device", name);
    return false;
}
// Elements from a row to the next; of a single row, whose stride may be anything, at least its length.
int64_t row_stride(const at::Tensor& t) { return t.size(0) > 1 ? t.stride(0) : std::max(t.size(0) == 1 ? t.stride(0) : 0, t.size(1)); }
// A workspace: one piece of memory of the current device.
const at::Tensor* workspace(PyObject* o) {
    const at::Tensor* t = tensor(o, "workspace");
    if (!t || !here(*t, "workspace")) return nullptr;
    if (!t->is_contiguous()) { PyErr_SetString(PyExc_TypeError, "workspace: expected a contiguous tensor"); return nullptr; }
    return t;
}
// tensors that are long enough for their rows: the library sees pointers only
bool fp4_rows(PyObject* codes, PyObject* scales, PyObject* row_scales, int format, const char* names[3], Fp4Rows* out) {
    const at::Tensor *c = need(codes, at::kByte, names[0], 2), *s, *r = nullptr;
    if (!c || !(s = need(scales, at::kByte, names[1], 1)) || (row_scales != Py_None && !(r = need(row_scales, at::kFloat, names[2], 1)))) return false;
    out->rows = c->size(0);
    out->K = 2 * c->size(1);
    const int64_t block = format == BWLA_FP4_NV ? 16 : 32;
    if (!c->is_contiguous() || s->numel() < (out->rows + 127) / 128 * ((out->K / block + 3) / 4) * 512 || (r && r->numel() < out->rows)) {
        PyErr_Format(PyExc_TypeError, "%s must be contiguous, %s and %s long enough for its rows", names[0], names[1], names[2]);
        return false;
    }
    if (!here(*c, names[0]) || !here(*s, names[1]) || (r && !here(*r, names[2]))) return false;
    out->codes = c->data_ptr();
    out->scales = s->data_ptr();
    out->row_scales = r ? r->data_ptr() : nullptr;
    return true;
}
bool fp4_format(PyObject* o, int* format) {
    const long v = PyLong_AsLong(o);
    if (v == -1 && PyErr_Occurred()) return false;
    *format = v == BWLA_FP4_MX || v == BWLA_FP4_NV ? (int)v : -1;      // (what is neither is refused by the library)
    return true;
}
int float_dtype(const at::Tensor& t) {
    return t.scalar_type() == at::kFloat ? BWLA_DTYPE_F32 : t.scalar_type() == at::kBFloat16 ? BWLA_DTYPE_BF16 : t.scalar_type() == at::kHalf ? BWLA_DTYPE_F16 : -1;
}

// What a call returns: the status where it is not 0, else its outputs.
PyObject* fp4_result(PyObject* status, PyObject* outputs) {
    if (!status || !outputs) { Py_XDECREF(status); Py_XDECREF(outputs); return nullptr; }
    if (PyLong_AsLong(status) != 0) { Py_DECREF(outputs); return status; }
    Py_DECREF(status);
    return outputs;
}
// (without the dispatcher, which takes longer than the allocator)
Ref fp4_new(at::IntArrayRef sizes, at::ScalarType type, const at::Tensor& like) {
    return Ref(THPVariable_Wrap(at::detail::empty_cuda(sizes, type, like.device(), std::nullopt)));
}

// fp4_quantize(x, format, codes, scales, row_scales) -> (codes, scales, row_scales), those that are None made here, or status
PyObject* call_fp4_quantize(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    if (nargs != 5) { PyErr_SetString(PyExc_TypeError, "fp4_quantize(x, format, codes, scales, row_scales)"); return nullptr; }
    static const char* names[3] = {"codes", "scales", "row_scales"};
    const at::Tensor* x = tensor(args[0], "x");
    int format;
    Fp4Rows q;
    if (!x) return nullptr;
    if (float_dtype(*x) < 0) { PyErr_SetString(PyExc_TypeError, "x must be fp32, bf16 or fp16"); return nullptr; }
    if (!need(args[0], x->scalar_type(), "x", 2) || !here(*x, "x") || !fp4_format(args[1], &format)) return nullptr;
    const int64_t M = x->size(0), K = x->size(1);
    const Ref codes = args[2] != Py_None ? Ref(Py_NewRef(args[2])) : fp4_new({M, K / 2}, at::kByte, *x);
    const Ref scales = args[3] != Py_None ? Ref(Py_NewRef(args[3])) : fp4_new({(M + 127) / 128 * ((K / (format == BWLA_FP4_NV ? 16 : 32) + 3) / 4) * 512}, at::kByte, *x);
    const Ref rows = args[4] != Py_None || format != BWLA_FP4_NV ? Ref(Py_NewRef(args[4])) : fp4_new({M}, at::kFloat, *x);
    if (!codes.o || !scales.o || !rows.o || !fp4_rows(codes.o, scales.o, rows.o, format, names, &q)) return nullptr;
    if (q.rows != M || q.K != K / 2 * 2) { PyErr_SetString(PyExc_TypeError, "codes must be [M][K/2] for x of [M][K]"); return nullptr; }
    return fp4_result(unlocked(entry.fp4_quantize, (const void*)x->data_ptr(), float_dtype(*x), M, K, row_stride(*x), format, (uint8_t*)q.codes,
                               (uint8_t*)q.scales, (float*)q.row_scales, stream()),
                      PyTuple_Pack(3, codes.o, scales.o, rows.o));
    END_HANDLE_TH_ERRORS
}

// fp4_expand(codes, scales, row_scales, format, out) -> out, or status; out: a tensor, or 0 (bf16) or 1 (fp32) for a new one
PyObject* call_fp4_expand(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    if (nargs != 5) { PyErr_SetString(PyExc_TypeError, "fp4_expand(codes, scales, row_scales, format, out)"); return nullptr; }
    static const char* names[3] = {"codes", "scales", "row_scales"};
    int format;
    Fp4Rows q;
    if (!fp4_format(args[3], &format) || !fp4_rows(args[0], args[1], args[2], format, names, &q)) return nullptr;
    const Ref made = PyLong_Check(args[4]) ? fp4_new({q.rows, q.K}, PyLong_AsLong(args[4]) ? at::kFloat : at::kBFloat16, THPVariable_Unpack(args[0])) : Ref(Py_NewRef(args[4]));
    const at::Tensor* out = made.o ? tensor(made.o, "out") : nullptr;
    if (!out) return nullptr;
    if (float_dtype(*out) != BWLA_DTYPE_F32 && float_dtype(*out) != BWLA_DTYPE_BF16) { PyErr_SetString(PyExc_TypeError, "out must be fp32 or bf16"); return nullptr; }
    if (!need(made.o, out->scalar_type(), "out", 2) || !here(*out, "out")) return nullptr;
    if (out->size(0) != q.rows || out->size(1) != q.K) { PyErr_SetString(PyExc_TypeError, "out must be [M][K] for codes of [M][K/2]"); return nullptr; }
    return fp4_result(unlocked(entry.fp4_expand, (const uint8_t*)q.codes, (const uint8_t*)q.scales, (const float*)q.row_scales, q.rows, q.K, format,
                               out->data_ptr(), float_dtype(*out), row_stride(*out), stream()),
                      Py_NewRef(made.o));
    END_HANDLE_TH_ERRORS
}

// fp4_gemm(a_codes, a_scales, a_rows, w_codes, w_scales, w_rows, format, out, workspace) -> out (made here where it is None), or status
PyObject* call_fp4_gemm(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    if (nargs != 9) { PyErr_SetString(PyExc_TypeError, "fp4_gemm: nine arguments"); return nullptr; }
    static const char *a_names[3] = {"a_codes", "a_scales", "a_rows"}, *w_names[3] = {"w_codes", "w_scales", "w_rows"};
    int format;
    Fp4Rows a, w;
    const at::Tensor *out, *ws;
    if (!fp4_format(args[6], &format) || !fp4_rows(args[0], args[1], args[2], format, a_names, &a) || !fp4_rows(args[3], args[4], args[5], format, w_names, &w))
        return nullptr;
    const Ref made = args[7] != Py_None ? Ref(Py_NewRef(args[7])) : fp4_new({a.rows, w.rows}, at::kBFloat16, THPVariable_Unpack(args[0]));
    if (!made.o || !(out = need(made.o, at::kBFloat16, "out", 2)) || !here(*out, "out") || !(ws = workspace(args[8])))
        return nullptr;
    if (a.K != w.K || out->size(0) != a.rows || out->size(1) != w.rows) {
        PyErr_SetString(PyExc_TypeError, "a_codes [M][K/2], w_codes [N][K/2] and out [M][N] do not fit");
        return nullptr;
    }
    return fp4_result(unlocked(entry.fp4_gemm, (const uint8_t*)a.codes, (const uint8_t*)a.scales, (const float*)a.row_scales, a.rows, a.K, (const uint8_t*)w.codes,
                               (const uint8_t*)w.scales, (const float*)w.row_scales, w.rows, format, out->data_ptr(), row_stride(*out),
                               ws->data_ptr(), (size_t)ws->nbytes(), stream()),
                      Py_NewRef(made.o));
    END_HANDLE_TH_ERRORS
}

// fp4_linear(layer, x, out, workspace) -> out (made here where it is None), or status
PyObject* call_fp4_linear(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    if (nargs != 4) { PyErr_SetString(PyExc_TypeError, "fp4_linear(layer, x, out, workspace)"); return nullptr; }
    const at::Tensor *x = need(args[1], at::kBFloat16, "x", 2), *out, *ws;
    if (!x || !here(*x, "x") || !(ws = workspace(args[3]))) return nullptr;
    const Ref h(PyObject_GetAttr(args[0], name_fp4));
    if (!h.o) return nullptr;
    const bwla_fp4_layer* layer = h.o == Py_None ? nullptr : (const bwla_fp4_layer*)PyLong_AsVoidPtr(h.o);
    int64_t K, N;
    if (PyErr_Occurred() || !size_of(args[0], name_k, &K) || !size_of(args[0], name_n, &N)) return nullptr;
    const int64_t M = x->size(0);
    const Ref made = args[2] != Py_None ? Ref(Py_NewRef(args[2])) : fp4_new({M, N}, at::kBFloat16, *x);
    if (!made.o || !(out = need(made.o, at::kBFloat16, "out", 2)) || !here(*out, "out")) return nullptr;
    if (x->size(1) != K || out->size(0) != M || out->size(1) != N) { PyErr_SetString(PyExc_TypeError, "x must be [M][K] and out [M][N] of the layer"); return nullptr; }
    return fp4_result(unlocked(entry.fp4_linear, layer, (const void*)x->data_ptr(), M, row_stride(*x), out->data_ptr(), row_stride(*out),
                               ws->data_ptr(), (size_t)ws->nbytes(), stream()),
                      Py_NewRef(made.o));
    END_HANDLE_TH_ERRORS
}

bool addresses(PyObject* const* args, void* (&p)[4]) {
    for (int i = 0; i < 4; ++i) {
        p[i] = PyLong_AsVoidPtr(args[i]);
        if (!p[i]) { if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "bind: null address"); return false; }
    }
    return true;
}
// bind_fp4(quantize, expand, gemm, linear): as bind
PyObject* bind_fp4(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    if (nargs != 4) { PyErr_SetString(PyExc_TypeError, "bind_fp4: four addresses"); return nullptr; }
    void* p[4];
    if (!addresses(args, p)) return nullptr;
    entry.fp4_quantize = (decltype(entry.fp4_quantize))p[0];
    entry.fp4_expand = (decltype(entry.fp4_expand))p[1];
    entry.fp4_gemm = (decltype(entry.fp4_gemm))p[2];
    entry.fp4_linear = (decltype(entry.fp4_linear))p[3];
    Py_RETURN_NONE;
}

// bind(group, linear, a16, pack): the library's entry points as addresses
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    if (nargs != 4) { PyErr_SetString(PyExc_TypeError, "bind: four addresses"); return nullptr; }
    void* p[4];
    if (!addresses(args, p)) return nullptr;
    entry.group = (decltype(entry.group))p[0];
    entry.linear = (decltype(entry.linear))p[1];
    entry.a16 = (decltype(entry.a16))p[2];
    entry.pack = (decltype(entry.pack))p[3];
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"bind", (PyCFunction)(void (*)(void))bind, METH_FASTCALL, nullptr},
    {"bind_fp4", (PyCFunction)(void (*)(void))bind_fp4, METH_FASTCALL, nullptr},
    {"fp4_quantize", (PyCFunction)(void (*)(void))call_fp4_quantize, METH_FASTCALL, nullptr},
    {"fp4_expand", (PyCFunction)(void (*)(void))call_fp4_expand, METH_FASTCALL, nullptr},
    {"fp4_gemm", (PyCFunction)(void (*)(void))call_fp4_gemm, METH_FASTCALL, nullptr},
    {"fp4_linear", (PyCFunction)(void (*)(void))call_fp4_linear, METH_FASTCALL, nullptr},
    {"group", (PyCFunction)(void (*)(void))call_group, METH_FASTCALL, nullptr},
    {"a16", (PyCFunction)(void (*)(void))call_a16, METH_FASTCALL, nullptr},
    {"linear", (PyCFunction)(void (*)(void))call_linear, METH_FASTCALL, nullptr},
    {"pack", (PyCFunction)(void (*)(void))call_pack, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls(void) {
    name_handle = PyUnicode_InternFromString("_h");
    name_fp4 = PyUnicode_InternFromString("_fp4");
    name_n = PyUnicode_InternFromString("N");
    name_k = PyUnicode_InternFromString("K");
    return name_handle && name_fp4 && name_n && name_k ? PyModule_Create(&module_def) : nullptr;
}
