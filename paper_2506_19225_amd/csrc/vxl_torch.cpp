// The hot entry points of include/vxl.h as Python functions over torch tensors: argument marshalling only.
// A small call is bound by the host: through ctypes, seven tensors asked for is_cuda, is_contiguous and data_ptr and
// thirteen arguments converted took 2.5 of the 9.0 us that a generated token's call took to submit, which is 6.5 so (two
// launches); the four calls of a prompt of 576 tokens 25.7 -> 17.1, a question's three on 16k tokens 22.5 -> 16.2.
//
// Arguments in the order of the C functions, without the sizes, which are read off the tensors; last the stream, which
// vxl._stream makes a handle of when all others are found good.  What an argument may be goes by its position alone (the
// kinds at each function below): an object of another kind is refused, never taken for an address.  The result is the
// vxl_status.
#include <Python.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <exception>
#include <initializer_list>

#include "vxl.h"

namespace {

// The functions of the library that vxl.lib() loaded, as setup() is given them: linked against it, the binding of a second
// copy in the process called the first copy's library, and one of another path than its own was never called.
#define VXL_PATH(X)                                                                                               \
    X(chunk_prefill) X(chunk_score_topk) X(chunk_score_topk_mass) X(gather_bilevel_kv) X(pool_sparse_kv)          \
    X(gather_bilevel_kv_pooled) X(bilevel_decode) X(bilevel_decode_inplace) X(kvq_write) X(kvq_read)              \
    X(gather_bilevel_kvq) X(bilevel_decode_kvq) X(rotate) X(mixed_append) X(mixed_attend) X(mixed_evict)

// Of one module object: a vxl.py that is loaded twice has two.
struct State {
    PyObject *desc_type, *handle_type, *stream_of, *cache_type;
    PyObject *rows, *scales, *format;                         // names of a cache's attributes
    PyObject *rotary_type, *rule_type, *device_of;
    PyObject *freqs, *slopes, *arg;                           // names of a rotary's and a rule's attributes
#define VXL_DECLARE(name) decltype(&vxl_##name) name;
    VXL_PATH(VXL_DECLARE)
};

// Kinds of an argument: a layout's c_void_p (or a number or None, the library's to refuse); the descriptor; a quantised cache
// (its tensors as they are at the call, and its format) or None, a null pointer; a tensor (its
// data pointer; a contiguous CUDA tensor or AssertionError) or None, a null pointer; a number.  Python does not pass
// kNumel, the number of elements of the tensor before it (0 for None), kCount, the same but -1 for None, and size(i, d), dimension d of
// its argument i.
// The calls on rotary positions and growing sets hold their tensors to more: of the descriptor's type, float32 or int32 (the workspace: of
// any), on one device, the current one; beside them a rotary or a rule, or None, a null pointer.
enum Kind { kLayout, kDesc, kCache, kTensor, kInt, kRotary, kRule, kOfDesc, kFloats, kInts, kWorkspace, kNumel, kCount, kSize };
constexpr int size(int arg, int dim) { return kSize | arg << 8 | dim << 16; }

// A number that an object answers with (a new reference, or null where it raised).
bool take(PyObject* r, long long* out) {
    if (!r) return false;
    *out = (long long)PyLong_AsUnsignedLongLongMask(r);
    Py_DECREF(r);
    return !PyErr_Occurred();
}

// Pointer of an object that is not a torch.Tensor but answers like one.
bool like_tensor(PyObject* o, long long* out) {
    PyObject* cuda = PyObject_GetAttrString(o, "is_cuda");
    if (!cuda) return false;
    int ok = PyObject_IsTrue(cuda);
    Py_DECREF(cuda);
    PyObject* r = ok > 0 ? PyObject_CallMethod(o, "is_contiguous", nullptr) : nullptr;
    if (ok < 0 || (ok > 0 && !r)) return false;
    if (r) {
        ok = PyObject_IsTrue(r);
        Py_DECREF(r);
        if (ok < 0) return false;
    }
    if (!ok) {
        PyErr_SetString(PyExc_AssertionError, "device tensors must be contiguous CUDA tensors");
        return false;
    }
    return take(PyObject_CallMethod(o, "data_ptr", nullptr), out);
}

bool size_of(PyObject* o, int d, long long* out) {
    if (THPVariable_Check(o)) {
        const at::Tensor& t = THPVariable_Unpack(o);
        if (d >= t.dim()) { PyErr_SetString(PyExc_IndexError, "tuple index out of range"); return false; }
        *out = t.size(d);
        return true;
    }
    PyObject* shape = PyObject_GetAttrString(o, "shape");
    if (!shape) return false;
    PyObject* r = PySequence_GetItem(shape, d);
    Py_DECREF(shape);
    return take(r, out);
}

bool numel_of(PyObject* o, long long* out) {
    if (o == Py_None) { *out = 0; return true; }
    if (THPVariable_Check(o)) { *out = THPVariable_Unpack(o).numel(); return true; }
    return take(PyObject_CallMethod(o, "numel", nullptr), out);
}

// The memory of a ctypes object.
bool memory_of(PyObject* o, void** out) {
    Py_buffer view;
    if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) < 0) return false;
    *out = view.buf;
    PyBuffer_Release(&view);                                  // (the object, which the caller holds, owns it)
    return true;
}

bool refuse(PyObject* o, const char* what) {
    PyErr_Format(PyExc_TypeError, "%s expected, not '%.100s'", what, Py_TYPE(o)->tp_name);
    return false;
}

bool int_of(PyObject* o, long long* out) {
    if (!PyLong_Check(o)) return refuse(o, "a number");
    *out = (long long)PyLong_AsUnsignedLongLongMask(o);
    return !PyErr_Occurred();
}

bool tensor_of(PyObject* o, long long* out) {
    if (o == Py_None) { *out = 0; return true; }
    if (!THPVariable_Check(o)) return like_tensor(o, out);
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || !t.is_contiguous()) {
        PyErr_SetString(PyExc_AssertionError, "device tensors must be contiguous CUDA tensors");
        return false;
    }
    *out = (long long)t.data_ptr();
    return true;
}

bool desc_of(const State& st, PyObject* o, long long* out) {
    void* p = nullptr;
    if (!PyObject_TypeCheck(o, (PyTypeObject*)st.desc_type)) return refuse(o, "a descriptor");
    if (!memory_of(o, &p)) return false;
    *out = (long long)p;
    return true;
}

bool layout_of(const State& st, PyObject* o, long long* out) {
    void* p = nullptr;
    if (o == Py_None) { *out = 0; return true; }
    if (PyLong_Check(o)) return int_of(o, out);
    if (!PyObject_TypeCheck(o, (PyTypeObject*)st.handle_type)) return refuse(o, "a layout's handle");
    if (!memory_of(o, &p)) return false;
    *out = (long long)*(void**)p;
    return true;
}

// A quantised cache for the library, and the heads that its tensors are of.
struct CacheArg {
    vxl_kvq_cache c;
    long long n_kv_heads, head_dim;
};

// What a call keeps until it returns: the place of the next argument, the caches given, references to their tensors; a rotary, a
// rule; the descriptor, and the device of the tensors that are held to one.
struct Frame {
    int next = 0, n_caches = 0, n_held = 0;
    CacheArg caches[2];
    vxl_rotary rotary;
    vxl_score_rule rule;
    const vxl_attn_desc* desc = nullptr;
    int device = -1;
    PyObject* held[4];
    ~Frame() { while (n_held > 0) Py_DECREF(held[--n_held]); }
};

// Pointer and dimensions of a cache's tensor: four, of uint8.
bool bytes_of(Frame& f, PyObject* cache, PyObject* name, long long* p, long long (&dims)[4]) {
    PyObject* t = PyObject_GetAttr(cache, name);
    if (!t) return false;
    f.held[f.n_held++] = t;
    if (!tensor_of(t, p)) return false;
    bool ok = t != Py_None;
    if (ok && THPVariable_Check(t)) {
        const at::Tensor& x = THPVariable_Unpack(t);
        ok = x.scalar_type() == at::kByte && x.dim() == 4;
        for (int d = 0; ok && d < 4; ++d) dims[d] = x.size(d);
    } else if (ok) {
        PyObject *type = PyObject_GetAttrString(t, "dtype"), *shape = type ? PyObject_GetAttrString(t, "shape") : nullptr;
        ok = shape && THPDtype_Check(type) && ((THPDtype*)type)->scalar_type == at::kByte && PySequence_Size(shape) == 4;
        Py_XDECREF(type);
        Py_XDECREF(shape);
        for (int d = 0; ok && d < 4; ++d) ok = size_of(t, d, &dims[d]);
    }
    if (!ok && !PyErr_Occurred()) PyErr_Format(PyExc_ValueError, "the %U of a quantised cache are a uint8 tensor of four dimensions", name);
    return ok;
}

bool cache_of(const State& st, Frame& f, PyObject* o, long long* out) {
    if (o == Py_None) { *out = 0; return true; }
    if (!st.cache_type || !PyObject_TypeCheck(o, (PyTypeObject*)st.cache_type)) return refuse(o, "a quantised cache");
    long long rows, scales, r[4], s[4], format;
    PyObject* code = PyObject_GetAttr(o, st.format);
    const bool known = code && int_of(code, &format);
    Py_XDECREF(code);
    if (!known || !bytes_of(f, o, st.rows, &rows, r) || !bytes_of(f, o, st.scales, &scales, s)) return false;
    if (r[0] != s[0] || r[1] != s[1] || r[2] != 2 || s[2] != 2 || r[3] != s[3] * (format == VXL_KVQ_FP4 ? 16 : 32)) {
        PyErr_SetString(PyExc_ValueError, "the rows and the scales of a quantised cache do not fit each other");
        return false;
    }
    CacheArg& c = f.caches[f.n_caches++];
    c = {{(void*)rows, (void*)scales, (int32_t)std::clamp<long long>(format, -1, INT32_MAX), (int32_t)std::min<long long>(r[1], INT32_MAX)},
         r[0], s[3] * 32};
    *out = (long long)&c;
    return true;
}

// Pointer of a tensor on the device of the others, or null for None.
bool placed_of(Frame& f, PyObject* o, long long* out) {
    if (!tensor_of(o, out)) return false;
    if (!THPVariable_Check(o)) return true;
    const int device = THPVariable_Unpack(o).device().index();
    if (f.device >= 0 && device != f.device) { PyErr_SetString(PyExc_ValueError, "the tensors are on several devices"); return false; }
    f.device = device;
    return true;
}

// The same for one of this type.
bool typed_of(Frame& f, PyObject* o, at::ScalarType type, const char* name, long long* out) {
    if (!placed_of(f, o, out) || o == Py_None) return !PyErr_Occurred();
    bool ok;
    if (THPVariable_Check(o)) {
        ok = THPVariable_Unpack(o).scalar_type() == type;
    } else {
        PyObject* dtype = PyObject_GetAttrString(o, "dtype");
        if (!dtype) return false;
        ok = THPDtype_Check(dtype) && ((THPDtype*)dtype)->scalar_type == type;
        Py_DECREF(dtype);
    }
    if (!ok) PyErr_Format(PyExc_ValueError, "a %s tensor expected", name);
    return ok;
}

bool data_of(Frame& f, PyObject* o, long long* out) {
    const bool f32 = f.desc && f.desc->dtype == VXL_F32;
    return typed_of(f, o, f32 ? at::kFloat : at::kBFloat16, f32 ? "float32" : "bfloat16", out);
}

// The struct of a rotary or a rule, copied, and the pointer and size of its tensor as they are at the call.
template <typename S>
bool struct_of(const State& st, Frame& f, PyObject* o, PyObject* type, PyObject* name, at::ScalarType of, const char* of_name, S* to,
               long long* tensor, long long* numel) {
    if (!type || !PyObject_TypeCheck(o, (PyTypeObject*)type)) return refuse(o, name == st.freqs ? "a Rotary" : "a ScoreRule");
    PyObject* arg = PyObject_GetAttr(o, st.arg);
    void* p = nullptr;
    const bool ok = arg && memory_of(arg, &p);
    if (ok) *to = *(const S*)p;
    Py_XDECREF(arg);
    if (!ok) return false;
    PyObject* t = PyObject_GetAttr(o, name);
    if (!t) return false;
    f.held[f.n_held++] = t;
    return typed_of(f, t, of, of_name, tensor) && numel_of(t, numel);
}

bool rotary_of(const State& st, Frame& f, PyObject* o, long long* out) {
    if (o == Py_None) { *out = 0; return true; }
    long long freqs, n;
    if (!struct_of(st, f, o, st.rotary_type, st.freqs, at::kDouble, "float64", &f.rotary, &freqs, &n)) return false;
    f.rotary.freqs = (const double*)freqs;
    if (2 * n != f.rotary.rotary_dim) { PyErr_SetString(PyExc_ValueError, "the frequencies of a rotary have changed their number"); return false; }
    *out = (long long)&f.rotary;
    return true;
}

bool rule_of(const State& st, Frame& f, PyObject* o, long long* out) {
    if (o == Py_None) { *out = 0; return true; }
    long long slopes, n;
    if (!struct_of(st, f, o, st.rule_type, st.slopes, at::kFloat, "float32", &f.rule, &slopes, &n)) return false;
    f.rule.slopes = (const float*)slopes;
    if (f.held[f.n_held - 1] != Py_None && f.desc && n != f.desc->n_q_heads) { PyErr_SetString(PyExc_ValueError, "a slope per query head expected"); return false; }
    *out = (long long)&f.rule;
    return true;
}

constexpr bool passed(int kind) { return kind < kNumel; }

// The argument of this kind: the next of Python's, or a number read off one.
template <int KIND>
bool convert(const State& st, PyObject* const* args, Frame& f, long long* out) {
    int* const next = &f.next;
    if constexpr ((KIND & 255) == kSize) return size_of(args[KIND >> 8 & 255], KIND >> 16, out);
    else if constexpr (KIND == kNumel) return numel_of(args[*next - 1], out);
    else if constexpr (KIND == kCount) return args[*next - 1] == Py_None ? (*out = -1, true) : numel_of(args[*next - 1], out);
    else if constexpr (KIND == kLayout) return layout_of(st, args[(*next)++], out);
    else if constexpr (KIND == kDesc) {
        if (!desc_of(st, args[(*next)++], out)) return false;
        f.desc = (const vxl_attn_desc*)*out;
        return true;
    } else if constexpr (KIND == kRotary) return rotary_of(st, f, args[(*next)++], out);
    else if constexpr (KIND == kRule) return rule_of(st, f, args[(*next)++], out);
    else if constexpr (KIND == kOfDesc) return data_of(f, args[(*next)++], out);
    else if constexpr (KIND == kFloats) return typed_of(f, args[(*next)++], at::kFloat, "float32", out);
    else if constexpr (KIND == kWorkspace) return placed_of(f, args[(*next)++], out);
    else if constexpr (KIND == kInts) return typed_of(f, args[(*next)++], at::kInt, "int32", out);
    else if constexpr (KIND == kCache) return cache_of(st, f, args[(*next)++], out);
    else if constexpr (KIND == kTensor) return tensor_of(args[(*next)++], out);
    else return int_of(args[(*next)++], out);
}

// f over the library's functions, the arguments of these kinds and the stream.
template <int... KINDS, typename F>
PyObject* call(PyObject* self, PyObject* const* args, Py_ssize_t n, F f) {
    const State& st = *(const State*)PyModule_GetState(self);
    constexpr int given = (passed(KINDS) + ...) + 1;
    if (n != given) { PyErr_Format(PyExc_TypeError, "%d arguments expected, %zd given", given, n); return nullptr; }
    if (!st.desc_type) { PyErr_SetString(PyExc_RuntimeError, "setup() has not been called"); return nullptr; }
    long long a[sizeof...(KINDS) + 1], *out = a;
    Frame frame;
    try {
        if (!(convert<KINDS>(st, args, frame, out++) && ...)) return nullptr;
    } catch (const std::exception& e) {                       // (a tensor without memory)
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
    if (frame.device >= 0) {
        long long current;
        if (!take(PyObject_CallNoArgs(st.device_of), &current)) return nullptr;
        if (current != frame.device) { PyErr_SetString(PyExc_ValueError, "the tensors are on another device than the current one"); return nullptr; }
    }
    PyObject* s = PyObject_CallFunctionObjArgs(st.stream_of, args[n - 1], nullptr);
    if (!s) return nullptr;
    *out = s == Py_None ? 0 : (long long)PyLong_AsUnsignedLongLongMask(s);
    Py_DECREF(s);
    if (PyErr_Occurred()) return nullptr;
    vxl_status status;
    Py_BEGIN_ALLOW_THREADS
    status = f(st, a);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

template <typename T> T* ptr(long long a) { return (T*)a; }
const vxl_layout* lay(long long a) { return (const vxl_layout*)a; }
const vxl_attn_desc* desc(long long a) { return (const vxl_attn_desc*)a; }
const vxl_kvq_cache* cache(long long a) { return a ? &((const CacheArg*)a)->c : nullptr; }

// Whether a cache (null: there is none) has the descriptor's heads.
bool of_heads(const vxl_attn_desc* d, long long a) {
    const CacheArg* c = (const CacheArg*)a;
    return !c || (c->n_kv_heads == d->n_kv_heads && c->head_dim == d->head_dim);
}

bool in_32_bits(long long n) { return n == (int32_t)n; }

// Whether a tensor of so many elements holds the rows that a call takes off it, by the descriptor's layout.
bool holds(const vxl_attn_desc* d, long long n_rows, long long numel) {
    if (n_rows <= 0) return true;                             // (for the library to refuse, or nothing to do)
    const __int128 rows = n_rows, head = d->kv_stride_head ? d->kv_stride_head : rows * d->head_dim, tok = d->kv_stride_tok ? d->kv_stride_tok : d->head_dim;
    return (d->n_kv_heads - 1) * head + (rows - 1) * tok + d->head_dim <= numel;
}

PyObject* chunk_prefill(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    return call<kLayout, kDesc, kTensor, kTensor, kTensor, kTensor, kTensor, kTensor, kNumel>(
        self, args, n, [](const State& lib, const long long* a) {
        return lib.chunk_prefill(lay(a[0]), desc(a[1]), ptr<void>(a[2]), ptr<void>(a[3]), ptr<void>(a[4]), ptr<void>(a[5]),
                                 ptr<float>(a[6]), ptr<void>(a[7]), (size_t)a[8], (vxl_stream)a[9]);
    });
}
PyObject* chunk_score_topk(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    return call<kLayout, kDesc, kTensor, size(2, 0), size(2, 1), kTensor, kInt, kTensor, kInt, kTensor, kTensor, kTensor, kTensor,
                kNumel>(
        self, args, n, [](const State& lib, const long long* a) {
        return lib.chunk_score_topk(lay(a[0]), desc(a[1]), ptr<void>(a[2]), (int32_t)a[3], (int32_t)a[4], ptr<void>(a[5]),
                                    (int32_t)a[6], ptr<float>(a[7]), (int32_t)a[8], ptr<int32_t>(a[9]), ptr<uint8_t>(a[10]),
                                    ptr<float>(a[11]), ptr<void>(a[12]), (size_t)a[13], (vxl_stream)a[14]);
    });
}
PyObject* chunk_score_topk_mass(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    return call<kLayout, kDesc, kTensor, size(2, 0), size(2, 1), kTensor, kInt, kTensor, kTensor, kTensor, kTensor, kNumel>(
        self, args, n, [](const State& lib, const long long* a) {
        return lib.chunk_score_topk_mass(lay(a[0]), desc(a[1]), ptr<void>(a[2]), (int32_t)a[3], (int32_t)a[4], ptr<void>(a[5]),
                                         (int32_t)a[6], ptr<int32_t>(a[7]), ptr<uint8_t>(a[8]), ptr<float>(a[9]),
                                         ptr<void>(a[10]), (size_t)a[11], (vxl_stream)a[12]);
    });
}
PyObject* gather_bilevel_kv(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    return call<kLayout, kDesc, kTensor, kTensor, kTensor, size(5, 0), kTensor, kTensor, size(5, 2), kTensor, kTensor>(
        self, args, n, [](const State& lib, const long long* a) {
        return lib.gather_bilevel_kv(lay(a[0]), desc(a[1]), ptr<void>(a[2]), ptr<void>(a[3]), ptr<uint8_t>(a[4]), (int32_t)a[5],
                                     ptr<void>(a[6]), ptr<void>(a[7]), (int32_t)a[8], ptr<int32_t>(a[9]), ptr<int32_t>(a[10]),
                                     (vxl_stream)a[11]);
    });
}
PyObject* pool_sparse_kv(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    return call<kLayout, kDesc, kTensor, kTensor, kTensor, kTensor>(
        self, args, n, [](const State& lib, const long long* a) {
        return lib.pool_sparse_kv(lay(a[0]), desc(a[1]), ptr<void>(a[2]), ptr<void>(a[3]), ptr<void>(a[4]), ptr<void>(a[5]),
                                  (vxl_stream)a[6]);
    });
}
PyObject* gather_bilevel_kv_pooled(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    return call<kLayout, kDesc, kTensor, kTensor, kTensor, kTensor, kTensor, size(7, 0), kTensor, kTensor, size(7, 2), kTensor, kTensor>(
        self, args, n, [](const State& lib, const long long* a) {
        return lib.gather_bilevel_kv_pooled(lay(a[0]), desc(a[1]), ptr<void>(a[2]), ptr<void>(a[3]), ptr<void>(a[4]),
                                            ptr<void>(a[5]), ptr<uint8_t>(a[6]), (int32_t)a[7], ptr<void>(a[8]), ptr<void>(a[9]),
                                            (int32_t)a[10], ptr<int32_t>(a[11]), ptr<int32_t>(a[12]), (vxl_stream)a[13]);
    });
}
PyObject* bilevel_decode(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    return call<kDesc, kTensor, size(1, 0), size(1, 1), kTensor, kTensor, size(2, 2), kTensor, kTensor, kTensor, kTensor, kNumel>(
        self, args, n, [](const State& lib, const long long* a) {
        return lib.bilevel_decode(desc(a[0]), ptr<void>(a[1]), (int32_t)a[2], (int32_t)a[3], ptr<void>(a[4]), ptr<void>(a[5]),
                                  (int32_t)a[6], ptr<int32_t>(a[7]), ptr<void>(a[8]), ptr<float>(a[9]), ptr<void>(a[10]),
                                  (size_t)a[11], (vxl_stream)a[12]);
    });
}
PyObject* bilevel_decode_inplace(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    return call<kLayout, kDesc, kTensor, size(2, 0), size(2, 1), kTensor, kTensor, kTensor, kTensor, kTensor, kInt, kInt, kTensor,
                kTensor, kTensor, kTensor, kNumel>(
        self, args, n, [](const State& lib, const long long* a) {
        return lib.bilevel_decode_inplace(lay(a[0]), desc(a[1]), ptr<void>(a[2]), (int32_t)a[3], (int32_t)a[4], ptr<void>(a[5]),
                                          ptr<void>(a[6]), ptr<void>(a[7]), ptr<void>(a[8]), ptr<uint8_t>(a[9]), (int32_t)a[10],
                                          (int32_t)a[11], ptr<void>(a[12]), ptr<float>(a[13]), ptr<int32_t>(a[14]),
                                          ptr<void>(a[15]), (size_t)a[16], (vxl_stream)a[17]);
    });
}
PyObject* kvq_write(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    return call<kDesc, kTensor, kNumel, kTensor, kNumel, kInt, kCache, kInt>(self, args, n, [](const State& lib, const long long* a) {
        if (!in_32_bits(a[5]) || !in_32_bits(a[7]) || !holds(desc(a[0]), a[5], a[2]) || !holds(desc(a[0]), a[5], a[4]) || !of_heads(desc(a[0]), a[6])) return VXL_ERR_INVALID_ARG;
        return lib.kvq_write(desc(a[0]), ptr<void>(a[1]), ptr<void>(a[3]), (int32_t)a[5], cache(a[6]), (int32_t)a[7], (vxl_stream)a[8]);
    });
}
PyObject* kvq_read(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    return call<kDesc, kCache, kInt, kInt, kTensor, kNumel, kTensor, kNumel>(self, args, n, [](const State& lib, const long long* a) {
        if (!in_32_bits(a[2]) || !in_32_bits(a[3]) || !holds(desc(a[0]), a[3], a[5]) || !holds(desc(a[0]), a[3], a[7]) || !of_heads(desc(a[0]), a[1])) return VXL_ERR_INVALID_ARG;
        return lib.kvq_read(desc(a[0]), cache(a[1]), (int32_t)a[2], (int32_t)a[3], ptr<void>(a[4]), ptr<void>(a[6]), (vxl_stream)a[8]);
    });
}
PyObject* gather_bilevel_kvq(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    return call<kLayout, kDesc, kCache, kCache, kTensor, size(5, 0), kTensor, kTensor, size(5, 2), kTensor, kTensor>(
        self, args, n, [](const State& lib, const long long* a) {
        if (!of_heads(desc(a[1]), a[2]) || !of_heads(desc(a[1]), a[3])) return VXL_ERR_INVALID_ARG;
        return lib.gather_bilevel_kvq(lay(a[0]), desc(a[1]), cache(a[2]), cache(a[3]), ptr<uint8_t>(a[4]), (int32_t)a[5], ptr<void>(a[6]),
                                      ptr<void>(a[7]), (int32_t)a[8], ptr<int32_t>(a[9]), ptr<int32_t>(a[10]), (vxl_stream)a[11]);
    });
}
PyObject* bilevel_decode_kvq(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    return call<kLayout, kDesc, kTensor, size(2, 0), size(2, 1), kCache, kCache, kTensor, kInt, kInt, kTensor, kTensor, kTensor,
                kTensor, kNumel>(
        self, args, n, [](const State& lib, const long long* a) {
        if (!of_heads(desc(a[1]), a[5]) || !of_heads(desc(a[1]), a[6])) return VXL_ERR_INVALID_ARG;
        return lib.bilevel_decode_kvq(lay(a[0]), desc(a[1]), ptr<void>(a[2]), (int32_t)a[3], (int32_t)a[4], cache(a[5]), cache(a[6]),
                                      ptr<uint8_t>(a[7]), (int32_t)a[8], (int32_t)a[9], ptr<void>(a[10]), ptr<float>(a[11]),
                                      ptr<int32_t>(a[12]), ptr<void>(a[13]), (size_t)a[14], (vxl_stream)a[15]);
    });
}

// Whether a tensor (-1 elements: there is none) has as many elements as the call takes off it.
bool has(long long numel, std::initializer_list<long long> dims) {
    __int128 n = 1;
    for (long long x : dims) n *= x;
    return numel < 0 || n == numel;
}
// Whether one of queries or keys holds the rows of n tokens, by the descriptor's layout.  Without strides heads lie n tokens apart, so that several
// of them in a tensor of more tokens would be taken for rows of others.
bool holds_rows(const vxl_attn_desc* d, long long n, long long numel, bool queries) {
    vxl_attn_desc x = *d;
    if (queries) {
        x.n_kv_heads = d->n_q_heads;
        x.kv_stride_head = d->q_stride_head;
        x.kv_stride_tok = d->q_stride_tok;
    }
    if (!x.kv_stride_head && x.n_kv_heads > 1) return (__int128)x.n_kv_heads * n * x.head_dim == numel;
    return holds(&x, n, numel);
}

PyObject* rotate(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    return call<kDesc, kRotary, kInts, kNumel, kOfDesc, kNumel, kOfDesc, kNumel, kOfDesc, kNumel, kOfDesc, kNumel>(
        self, args, n, [&](const State& lib, const long long* a) {
        const long long tokens = a[3];
        if (args[2] == Py_None || !in_32_bits(tokens)) return VXL_ERR_INVALID_ARG;          // (no positions are not positions of no tokens)
        for (int i : {4, 6, 8, 10})
            if (args[i / 2 + 1] != Py_None && !holds_rows(desc(a[0]), tokens, a[i + 1], i == 4 || i == 8)) return VXL_ERR_INVALID_ARG;
        return lib.rotate(desc(a[0]), ptr<vxl_rotary>(a[1]), ptr<int32_t>(a[2]), (int32_t)tokens, ptr<void>(a[4]), ptr<void>(a[6]),
                          ptr<void>(a[8]), ptr<void>(a[10]), (vxl_stream)a[12]);
    });
}
// (batch and new tokens: of positions; rows: of kmix)
PyObject* mixed_append(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    return call<kDesc, kRotary, kInts, size(2, 0), size(2, 1), kOfDesc, kCount, kOfDesc, kCount, kOfDesc, kCount, kOfDesc, kCount, kOfDesc, kCount,
                kOfDesc, kCount, size(7, 2), kInts, kCount, kInts, kCount, kFloats, kCount>(
        self, args, n, [](const State& lib, const long long* a) {
        const vxl_attn_desc* d = desc(a[0]);
        const long long batch = a[3], tokens = a[4], cap = a[17], hkv = d->n_kv_heads;
        if (!in_32_bits(batch) || !in_32_bits(tokens) || !in_32_bits(batch * tokens) || !in_32_bits(cap)) return VXL_ERR_INVALID_ARG;
        for (int i : {5, 7, 9})
            if (!holds_rows(d, batch * tokens, a[i + 1], i == 5)) return VXL_ERR_INVALID_ARG;
        if (!has(a[12], {batch, tokens, d->n_q_heads, d->head_dim}) || !has(a[14], {batch, hkv, cap, d->head_dim}) ||
            !has(a[16], {batch, hkv, cap, d->head_dim}) || !has(a[19], {batch}) || !has(a[21], {batch, hkv, cap}) || !has(a[23], {batch, hkv, cap}))
            return VXL_ERR_INVALID_ARG;
        return lib.mixed_append(d, ptr<vxl_rotary>(a[1]), ptr<int32_t>(a[2]), (int32_t)batch, (int32_t)tokens, ptr<void>(a[5]), ptr<void>(a[7]),
                                ptr<void>(a[9]), ptr<void>(a[11]), ptr<void>(a[13]), ptr<void>(a[15]), (int32_t)cap, ptr<int32_t>(a[18]),
                                ptr<int32_t>(a[20]), ptr<float>(a[22]), (vxl_stream)a[24]);
    });
}
// (batch and tokens: of qd; rows: of kmix)
PyObject* mixed_attend(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    return call<kDesc, kRule, kOfDesc, size(2, 0), size(2, 1), kCount, kInts, kCount, kOfDesc, size(4, 2), kCount, kOfDesc, kCount, kInts, kCount,
                kInts, kCount, kOfDesc, kCount, kFloats, kCount, kFloats, kCount, kFloats, kCount, kWorkspace, kNumel>(
        self, args, n, [](const State& lib, const long long* a) {
        const vxl_attn_desc* d = desc(a[0]);
        const long long batch = a[3], tokens = a[4], cap = a[9], hkv = d->n_kv_heads, hq = d->n_q_heads;
        if (!in_32_bits(batch) || !in_32_bits(tokens) || !in_32_bits(cap)) return VXL_ERR_INVALID_ARG;
        if (!has(a[5], {batch, tokens, hq, d->head_dim}) || !has(a[7], {batch, tokens}) || !has(a[10], {batch, hkv, cap, d->head_dim}) ||
            !has(a[12], {batch, hkv, cap, d->head_dim}) || !has(a[14], {batch}) || !has(a[16], {batch, hkv, cap}) ||
            !has(a[18], {batch, tokens, hq, d->head_dim}) || !has(a[20], {batch, tokens, hq}) || !has(a[22], {batch, hkv, cap}) ||
            !has(a[24], {batch, hkv, cap}))
            return VXL_ERR_INVALID_ARG;
        return lib.mixed_attend(d, ptr<vxl_score_rule>(a[1]), ptr<void>(a[2]), ptr<int32_t>(a[6]), (int32_t)batch, (int32_t)tokens, ptr<void>(a[8]),
                                ptr<void>(a[11]), (int32_t)cap, ptr<int32_t>(a[13]), ptr<int32_t>(a[15]), ptr<void>(a[17]), ptr<float>(a[19]),
                                ptr<float>(a[21]), ptr<float>(a[23]), ptr<void>(a[25]), (size_t)a[26], (vxl_stream)a[27]);
    });
}
// (batch and rows: of kmix; rows of the result: of kout)
PyObject* mixed_evict(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    return call<kDesc, kOfDesc, size(1, 0), size(1, 2), kCount, kOfDesc, kCount, kInts, kCount, kFloats, kCount, kInts, kCount, kInts, kCount, kInt,
                kInt, kInt, kOfDesc, size(10, 2), kCount, kOfDesc, kCount, kFloats, kCount, kInts, kCount, kInts, kCount, kWorkspace, kNumel>(
        self, args, n, [](const State& lib, const long long* a) {
        const vxl_attn_desc* d = desc(a[0]);
        const long long batch = a[2], cap = a[3], to = a[19], hkv = d->n_kv_heads, dim = d->head_dim;
        for (long long x : {batch, cap, to, a[15], a[16], a[17]})
            if (!in_32_bits(x)) return VXL_ERR_INVALID_ARG;
        if (!has(a[4], {batch, hkv, cap, dim}) || !has(a[6], {batch, hkv, cap, dim}) || !has(a[8], {batch}) || !has(a[10], {batch, hkv, cap}) ||
            !has(a[12], {batch, hkv, cap}) || !has(a[14], {batch}) || !has(a[20], {batch, hkv, to, dim}) || !has(a[22], {batch, hkv, to, dim}) ||
            !has(a[24], {batch, hkv, to}) || !has(a[26], {batch, hkv, to}) || !has(a[28], {batch}))
            return VXL_ERR_INVALID_ARG;
        return lib.mixed_evict(d, ptr<void>(a[1]), ptr<void>(a[5]), (int32_t)cap, ptr<int32_t>(a[7]), ptr<float>(a[9]), ptr<int32_t>(a[11]),
                               ptr<int32_t>(a[13]), (int32_t)batch, (int32_t)a[15], (int32_t)a[16], (int32_t)a[17], ptr<void>(a[18]), ptr<void>(a[21]),
                               (int32_t)to, ptr<float>(a[23]), ptr<int32_t>(a[25]), ptr<int32_t>(a[27]), ptr<void>(a[29]), (size_t)a[30],
                               (vxl_stream)a[31]);
    });
}
// setup(type of the descriptor, type of a layout's handle, vxl._stream, the addresses of VXL_PATH)
PyObject* setup(PyObject* self, PyObject* const* args, Py_ssize_t n) {
#define VXL_COUNT(name) + 1
    if (n != 3 VXL_PATH(VXL_COUNT) || !PyType_Check(args[0]) || !PyType_Check(args[1]) || !PyCallable_Check(args[2])) {
        PyErr_SetString(PyExc_TypeError, "two types, a function and the library's addresses expected");
        return nullptr;
    }
    for (int i = 3; i < n; ++i)
        if (!PyLong_Check(args[i]) || !PyLong_AsVoidPtr(args[i])) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "an address expected");
            return nullptr;
        }
    State& st = *(State*)PyModule_GetState(self);
    int i = 3;
#define VXL_TAKE(name) st.name = (decltype(st.name))PyLong_AsVoidPtr(args[i++]);
    VXL_PATH(VXL_TAKE)
    PyObject** to[] = {&st.desc_type, &st.handle_type, &st.stream_of};
    for (int j = 0; j < 3; ++j) {
        Py_INCREF(args[j]);
        Py_XSETREF(*to[j], args[j]);
    }
    Py_RETURN_NONE;
}
// setup_cache(type of a quantised cache)
PyObject* setup_cache(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    if (n != 1 || !PyType_Check(args[0])) { PyErr_SetString(PyExc_TypeError, "a type expected"); return nullptr; }
    State& st = *(State*)PyModule_GetState(self);
    PyObject** const names[] = {&st.rows, &st.scales, &st.format};
    const char* const text[] = {"rows", "scales", "format"};
    for (int i = 0; i < 3; ++i)
        if (!*names[i] && !(*names[i] = PyUnicode_InternFromString(text[i]))) return nullptr;
    Py_INCREF(args[0]);
    Py_XSETREF(st.cache_type, args[0]);
    Py_RETURN_NONE;
}
// setup_mixed(type of a rotary, type of a rule, function that answers the current device's number)
PyObject* setup_mixed(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    if (n != 3 || !PyType_Check(args[0]) || !PyType_Check(args[1]) || !PyCallable_Check(args[2])) {
        PyErr_SetString(PyExc_TypeError, "two types and a function expected");
        return nullptr;
    }
    State& st = *(State*)PyModule_GetState(self);
    PyObject** const names[] = {&st.freqs, &st.slopes, &st.arg};
    const char* const text[] = {"freqs", "slopes", "arg"};
    for (int i = 0; i < 3; ++i)
        if (!*names[i] && !(*names[i] = PyUnicode_InternFromString(text[i]))) return nullptr;
    PyObject** to[] = {&st.rotary_type, &st.rule_type, &st.device_of};
    for (int i = 0; i < 3; ++i) {
        Py_INCREF(args[i]);
        Py_XSETREF(*to[i], args[i]);
    }
    Py_RETURN_NONE;
}

int traverse(PyObject* self, visitproc visit, void* arg) {
    const State* st = (const State*)PyModule_GetState(self);
    if (!st) return 0;
    Py_VISIT(st->desc_type);
    Py_VISIT(st->handle_type);
    Py_VISIT(st->cache_type);
    Py_VISIT(st->rotary_type);
    Py_VISIT(st->rule_type);
    Py_VISIT(st->device_of);
    Py_VISIT(st->stream_of);
    return 0;
}
int clear(PyObject* self) {
    State* st = (State*)PyModule_GetState(self);
    if (!st) return 0;
    Py_CLEAR(st->desc_type);
    Py_CLEAR(st->handle_type);
    Py_CLEAR(st->cache_type);
    Py_CLEAR(st->rows);
    Py_CLEAR(st->scales);
    Py_CLEAR(st->format);
    Py_CLEAR(st->stream_of);
    Py_CLEAR(st->rotary_type);
    Py_CLEAR(st->rule_type);
    Py_CLEAR(st->device_of);
    Py_CLEAR(st->freqs);
    Py_CLEAR(st->slopes);
    Py_CLEAR(st->arg);
    return 0;
}

int exec(PyObject* self) { return PyModule_AddStringConstant(self, "torch_version", VXL_TORCH_VERSION); }

#define VXL_METHOD(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr},
PyMethodDef methods[] = {VXL_METHOD(setup) VXL_METHOD(setup_cache) VXL_METHOD(setup_mixed) VXL_PATH(VXL_METHOD){nullptr, nullptr, 0, nullptr}};
PyModuleDef_Slot slots[] = {{Py_mod_exec, (void*)exec}, {0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_vxl_torch", nullptr, sizeof(State), methods, slots, traverse, clear, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__vxl_torch(void) { return PyModuleDef_Init(&module); }
