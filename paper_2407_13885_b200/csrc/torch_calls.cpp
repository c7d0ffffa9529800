// Native form of the tensor entry points in binding.py: checks the arguments, allocates the result, looks up the stream
// and calls the C ABI of libattnw.so.  No arithmetic of the method is here.
//
// Why it exists: a small call spends 3 to 13 us on the GPU, and the same steps in Python (argument checks, torch.empty,
// device context, current stream, ctypes marshalling) took 13 to 20 us, so the host was the bound of every small call.  Now 4.5 to 7 us: softmax_rows
// of 4096 x 1000 float32 back to back 13.4 -> 6.3 us (5.0 us on the GPU), one head of 256 keys 15.4 -> 12.3 us.
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <climits>
#include <cstdint>
#include <cstring>
#include <initializer_list>
#include <string>

#include "../../include/attnw.h"

namespace {

PyObject* g_error = nullptr;  // binding.AttnwError, handed over once by binding.py

// A tensor without storage (torch.func's wrappers) throws when it is asked for its address, so every entry point asks while it
// holds the interpreter's lock: HANDLE_TH_ERRORS needs the lock to turn the exception into a Python one.

// A CUDA tensor of the wanted type, contiguous and on the device of the call's first tensor (`like`; nullptr for that one itself, and
// its kernel would read another GPU's memory); nullptr with a Python exception set otherwise.
const at::Tensor* tensor_arg(PyObject* obj, const char* name, at::ScalarType type, const char* type_name, const at::Tensor* like) {
    if (!THPVariable_Check(obj) || !THPVariable_Unpack(obj).is_cuda()) {
        PyErr_Format(PyExc_TypeError, "%s must be a CUDA tensor", name);
        return nullptr;
    }
    const at::Tensor& t = THPVariable_Unpack(obj);
    if (t.scalar_type() != type) {
        PyErr_Format(PyExc_TypeError, "%s must have dtype %s, got %s", name, type_name, at::toString(t.scalar_type()));
        return nullptr;
    }
    if (!t.is_contiguous()) {
        PyErr_Format(PyExc_ValueError, "%s must be contiguous", name);
        return nullptr;
    }
    if (like && t.device() != like->device()) {
        PyErr_Format(PyExc_ValueError, "%s must be on %s like the other tensors, got %s", name, like->device().str().c_str(),
                     t.device().str().c_str());
        return nullptr;
    }
    return &t;
}

const at::Tensor* bf16_arg(PyObject* obj, const char* name, const at::Tensor* like) {
    return tensor_arg(obj, name, at::kBFloat16, "torch.bfloat16", like);
}

// The result: the caller's tensor `obj` (bfloat16, or also float32 where `f32_allowed`); none yet where it is None (new_on makes it).
bool output_arg(PyObject* obj, const char* name, at::IntArrayRef shape, bool f32_allowed, bool exact_type, const char* shape_text,
                const at::Tensor& like, at::Tensor* out) {
    if (obj == Py_None) return true;
    const bool f32 = f32_allowed && THPVariable_Check(obj) && THPVariable_Unpack(obj).scalar_type() == at::kFloat;
    if (exact_type || f32 || (THPVariable_Check(obj) && THPVariable_Unpack(obj).scalar_type() == at::kBFloat16)) {
        const at::Tensor* t = tensor_arg(obj, name, f32 ? at::kFloat : at::kBFloat16, f32 ? "torch.float32" : "torch.bfloat16", &like);
        if (!t) return false;
        if (t->sizes() == shape) {
            *out = *t;
            return true;
        }
    } else if (!THPVariable_Check(obj) || !THPVariable_Unpack(obj).is_cuda()) {
        PyErr_Format(PyExc_TypeError, "%s must be a CUDA tensor", name);
        return false;
    }
    PyErr_Format(PyExc_ValueError, "%s must be %s", name, shape_text);
    return false;
}

// Same meaning as in Python: None = torch's current stream of the device that is current.
bool stream_arg(PyObject* obj, void** out) {
    if (obj == Py_None) {
        *out = static_cast<void*>(c10::cuda::getCurrentCUDAStream().stream());
        return true;
    }
    *out = PyLong_AsVoidPtr(obj);
    return !PyErr_Occurred();
}

// New memory for a call on `stream`, which the device's current stream may use as well.  It comes from what belongs to that stream: a block of
// the current one's may still be in use there by work in front, and would go to other work there as soon as the result is dropped.
at::Tensor new_on(void* stream, at::IntArrayRef sizes, at::ScalarType type, const at::Tensor& like) {
    const auto options = like.options().dtype(type).requires_grad(false);
    const c10::cuda::CUDAStream current = c10::cuda::getCurrentCUDAStream(like.device().index());
    if (stream == static_cast<void*>(current.stream())) return at::empty(sizes, options);
    const c10::cuda::CUDAStreamGuard guard(c10::cuda::getStreamFromExternal(static_cast<cudaStream_t>(stream), like.device().index()));
    at::Tensor t = at::empty(sizes, options);
    t.record_stream(current);
    return t;
}

bool float_arg(PyObject* obj, float* out) {
    PyObject* f = PyNumber_Float(obj);
    if (!f) return false;
    *out = static_cast<float>(PyFloat_AS_DOUBLE(f));
    Py_DECREF(f);
    return true;
}

PyObject* failed(int code, const char* where) {
    PyObject* e = PyObject_CallFunction(g_error, "is", code, where);
    if (e) {
        PyErr_SetObject(g_error, e);
        Py_DECREF(e);
    }
    return nullptr;
}

bool count_is(Py_ssize_t n, Py_ssize_t want) {
    if (n != want) PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return n == want;
}

// None = torch's default type, as everywhere in torch.
bool is_float32(PyObject* dtype, bool* f32) {
    if (dtype == Py_None || THPDtype_Check(dtype)) {
        const at::ScalarType t = dtype == Py_None ? c10::get_default_dtype_as_scalartype() : reinterpret_cast<THPDtype*>(dtype)->scalar_type;
        *f32 = t == at::kFloat;
        if (*f32 || t == at::kBFloat16) return true;
    }
    PyErr_SetString(PyExc_ValueError, "out_dtype must be torch.bfloat16 or torch.float32");
    return false;
}

// attnw_fused(Q, K, scale, P, out_dtype, stream)
PyObject* py_attnw_fused(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!count_is(n, 6)) return nullptr;
    const at::Tensor *q, *k;
    if (!(q = bf16_arg(a[0], "Q", nullptr)) || !(k = bf16_arg(a[1], "K", q))) return nullptr;
    if (q->dim() != 4 || q->sizes() != k->sizes()) {
        PyErr_SetString(PyExc_ValueError, "Q and K must both be [B, H, N, d]");
        return nullptr;
    }
    const int64_t B = q->size(0), H = q->size(1), N = q->size(2), d = q->size(3);
    bool f32 = false;
    float scale;
    if ((a[3] == Py_None && !is_float32(a[4], &f32)) || !float_arg(a[2], &scale)) return nullptr;
    const void *q_ptr = q->data_ptr(), *k_ptr = k->data_ptr();
    at::Tensor p;
    if (!output_arg(a[3], "P", {B, H, N, N}, true, false, "[B, H, N, N] in bfloat16 or float32", *q, &p)) return nullptr;
    const c10::cuda::CUDAGuard guard(q->device());
    void* stream;
    if (!stream_arg(a[5], &stream)) return nullptr;
    if (!p.defined()) p = new_on(stream, {B, H, N, N}, f32 ? at::kFloat : at::kBFloat16, *q);
    const auto entry = p.scalar_type() == at::kBFloat16 ? attnw_fused : attnw_fused_f32;
    void* p_ptr = p.data_ptr();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = entry(q_ptr, k_ptr, p_ptr, static_cast<int>(B), static_cast<int>(H), static_cast<int>(N), static_cast<int>(d), scale, stream);
    Py_END_ALLOW_THREADS
    if (rc != ATTNW_OK) return failed(rc, "attnw_fused");
    if (a[3] != Py_None) return Py_NewRef(a[3]);
    return THPVariable_Wrap(std::move(p));
    END_HANDLE_TH_ERRORS
}

// attn_fused(Q, K, V, scale, O, stream)
PyObject* py_attn_fused(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!count_is(n, 6)) return nullptr;
    const at::Tensor *q, *k, *v;
    if (!(q = bf16_arg(a[0], "Q", nullptr)) || !(k = bf16_arg(a[1], "K", q)) || !(v = bf16_arg(a[2], "V", q))) return nullptr;
    if (q->dim() != 4 || q->sizes() != k->sizes() || q->sizes() != v->sizes()) {
        PyErr_SetString(PyExc_ValueError, "Q, K and V must all be [B, H, N, d]");
        return nullptr;
    }
    float scale;
    if (!float_arg(a[3], &scale)) return nullptr;
    const void *q_ptr = q->data_ptr(), *k_ptr = k->data_ptr(), *v_ptr = v->data_ptr();
    const int B = static_cast<int>(q->size(0)), H = static_cast<int>(q->size(1)), N = static_cast<int>(q->size(2)), d = static_cast<int>(q->size(3));
    at::Tensor o;
    if (!output_arg(a[4], "O", q->sizes(), false, true, "[B, H, N, d]", *q, &o)) return nullptr;
    const c10::cuda::CUDAGuard guard(q->device());
    void* stream;
    if (!stream_arg(a[5], &stream)) return nullptr;
    if (!o.defined()) o = new_on(stream, q->sizes(), at::kBFloat16, *q);
    void* o_ptr = o.data_ptr();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = attn_fused(q_ptr, k_ptr, v_ptr, o_ptr, B, H, N, d, scale, stream);
    Py_END_ALLOW_THREADS
    if (rc != ATTNW_OK) return failed(rc, "attn_fused");
    if (a[4] != Py_None) return Py_NewRef(a[4]);
    return THPVariable_Wrap(std::move(o));
    END_HANDLE_TH_ERRORS
}

// project_qk(X, Wq, Wk, Q, K, stream)
PyObject* py_project_qk(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!count_is(n, 6)) return nullptr;
    const at::Tensor *x, *wq, *wk;
    if (!(x = bf16_arg(a[0], "X", nullptr)) || !(wq = bf16_arg(a[1], "Wq", x)) || !(wk = bf16_arg(a[2], "Wk", x))) return nullptr;
    if (x->dim() != 3 || wq->dim() != 3 || wq->sizes() != wk->sizes() || wq->size(2) != x->size(2)) {
        PyErr_SetString(PyExc_ValueError, "X must be [B, N, d_model] and Wq, Wk [H, d, d_model]");
        return nullptr;
    }
    const int64_t B = x->size(0), N = x->size(1), d_model = x->size(2), H = wq->size(0), d = wq->size(1);
    const void *x_ptr = x->data_ptr(), *wq_ptr = wq->data_ptr(), *wk_ptr = wk->data_ptr();
    at::Tensor q, k;
    if (!output_arg(a[3], "Q", {B, H, N, d}, false, true, "[B, H, N, d]", *x, &q) ||
        !output_arg(a[4], "K", {B, H, N, d}, false, true, "[B, H, N, d]", *x, &k))
        return nullptr;
    const c10::cuda::CUDAGuard guard(x->device());
    void* stream;
    if (!stream_arg(a[5], &stream)) return nullptr;
    if (!q.defined()) q = new_on(stream, {B, H, N, d}, at::kBFloat16, *x);
    if (!k.defined()) k = new_on(stream, {B, H, N, d}, at::kBFloat16, *x);
    void *q_ptr = q.data_ptr(), *k_ptr = k.data_ptr();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = attnw_project_qk(x_ptr, wq_ptr, wk_ptr, q_ptr, k_ptr, static_cast<int>(B), static_cast<int>(N), static_cast<int>(d_model),
                          static_cast<int>(H), static_cast<int>(d), stream);
    Py_END_ALLOW_THREADS
    if (rc != ATTNW_OK) return failed(rc, "attnw_project_qk");
    PyObject* pq = a[3] != Py_None ? Py_NewRef(a[3]) : THPVariable_Wrap(std::move(q));
    PyObject* pk = a[4] != Py_None ? Py_NewRef(a[4]) : THPVariable_Wrap(std::move(k));
    PyObject* pair = pq && pk ? PyTuple_Pack(2, pq, pk) : nullptr;
    Py_XDECREF(pq);
    Py_XDECREF(pk);
    return pair;
    END_HANDLE_TH_ERRORS
}

// softmax_rows(S, P, out_dtype, stream)
PyObject* py_softmax_rows(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!count_is(n, 4)) return nullptr;
    const at::Tensor* s = tensor_arg(a[0], "S", at::kFloat, "torch.float32", nullptr);
    if (!s) return nullptr;
    if (s->dim() != 2) {
        PyErr_SetString(PyExc_ValueError, "S must be [rows, cols]");
        return nullptr;
    }
    bool f32 = false;
    if (a[1] == Py_None && !is_float32(a[2], &f32)) return nullptr;
    const long long rows = s->size(0), cols = s->size(1);
    const void* s_ptr = s->data_ptr();
    at::Tensor p;
    if (!output_arg(a[1], "P", s->sizes(), true, false, "[rows, cols] in bfloat16 or float32", *s, &p)) return nullptr;
    const c10::cuda::CUDAGuard guard(s->device());
    void* stream;
    if (!stream_arg(a[3], &stream)) return nullptr;
    if (!p.defined()) p = new_on(stream, s->sizes(), f32 ? at::kFloat : at::kBFloat16, *s);
    const auto entry = p.scalar_type() == at::kBFloat16 ? softmax_rows : softmax_rows_f32;
    void* p_ptr = p.data_ptr();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = entry(s_ptr, p_ptr, rows, cols, stream);
    Py_END_ALLOW_THREADS
    if (rc != ATTNW_OK) return failed(rc, "softmax_rows");
    if (a[1] != Py_None) return Py_NewRef(a[1]);
    return THPVariable_Wrap(std::move(p));
    END_HANDLE_TH_ERRORS
}

// ---- the paged cache ----------------------------------------------------------------------------------------------------------

bool value_error(const char* text) {
    PyErr_SetString(PyExc_ValueError, text);
    return false;
}

// As tensor_arg, but for strided tensors of `dim` dimensions whose last one is contiguous.
const at::Tensor* strided_arg(PyObject* obj, const char* name, at::ScalarType type, const char* type_name, int dim, const at::Tensor* like) {
    if (!THPVariable_Check(obj) || !THPVariable_Unpack(obj).is_cuda()) {
        PyErr_Format(PyExc_TypeError, "%s must be a CUDA tensor", name);
        return nullptr;
    }
    const at::Tensor& t = THPVariable_Unpack(obj);
    if (t.scalar_type() != type) {
        PyErr_Format(PyExc_TypeError, "%s must have dtype %s, got %s", name, type_name, at::toString(t.scalar_type()));
        return nullptr;
    }
    if (t.dim() != dim || (t.size(dim - 1) > 1 && t.stride(dim - 1) != 1)) {
        PyErr_Format(PyExc_ValueError, "%s must have %d dimensions, the last one contiguous", name, dim);
        return nullptr;
    }
    if (like && t.device() != like->device()) {
        PyErr_Format(PyExc_ValueError, "%s must be on %s like the other tensors, got %s", name, like->device().str().c_str(),
                     t.device().str().c_str());
        return nullptr;
    }
    return &t;
}

// A contiguous index or weight tensor of the given sizes (-1: any, written back).
const at::Tensor* plain_arg(PyObject* obj, const char* name, at::ScalarType type, const char* type_name, std::initializer_list<int64_t> sizes,
                            const at::Tensor* like) {
    const at::Tensor* t = tensor_arg(obj, name, type, type_name, like);
    if (!t) return nullptr;
    bool fits = t->dim() == static_cast<int64_t>(sizes.size());
    int i = 0;
    for (const int64_t n : sizes) {
        if (!fits) break;
        fits = n < 0 || t->size(i) == n;
        ++i;
    }
    if (!fits) {
        std::string want;
        for (const int64_t n : sizes) want += (want.empty() ? "" : ", ") + (n < 0 ? std::string("any") : std::to_string(n));
        PyErr_Format(PyExc_ValueError, "%s must be [%s]", name, want.c_str());
        return nullptr;
    }
    return t;
}
const at::Tensor* int_arg(PyObject* obj, const char* name, std::initializer_list<int64_t> sizes, const at::Tensor* like) {
    return plain_arg(obj, name, at::kInt, "torch.int32", sizes, like);
}
const at::Tensor* f32_arg(PyObject* obj, const char* name, std::initializer_list<int64_t> sizes, const at::Tensor* like) {
    return plain_arg(obj, name, at::kFloat, "torch.float32", sizes, like);
}

bool small(std::initializer_list<int64_t> sizes) {
    for (const int64_t n : sizes)
        if (n > INT_MAX) return value_error("a size is above 2^31 - 1");
    return true;
}

bool int_value(PyObject* obj, int* out) {
    const long v = PyLong_AsLong(obj);
    if (v == -1 && PyErr_Occurred()) return false;
    if (v < INT_MIN || v > INT_MAX) return value_error("a size is above 2^31 - 1");
    *out = static_cast<int>(v);
    return true;
}

bool layout_arg(PyObject* obj, int* out) {
    const char* s = PyUnicode_Check(obj) ? PyUnicode_AsUTF8(obj) : nullptr;
    if (s && !strcmp(s, "half")) {
        *out = 0;
        return true;
    }
    if (s && !strcmp(s, "interleaved")) {
        *out = 1;
        return true;
    }
    if (PyErr_Occurred()) return false;
    return value_error("layout must be \"half\" or \"interleaved\"");
}

// K_cache, V_cache, table and lengths at a[0 ... 3].
bool cache_arg(PyObject* const* a, attnw_cache* c, const at::Tensor** k_cache) {
    const at::Tensor *k, *v, *table, *lengths;
    if (!(k = bf16_arg(a[0], "K_cache", nullptr)) || !(v = bf16_arg(a[1], "V_cache", k))) return false;
    if (k->dim() != 4 || k->sizes() != v->sizes()) return value_error("K_cache and V_cache must both be [pages, kv_heads, page, d]");
    if (!(table = int_arg(a[2], "table", {-1, -1}, k)) || !(lengths = int_arg(a[3], "lengths", {table->size(0)}, k))) return false;
    if (!small({k->size(0), k->size(1), k->size(2), k->size(3), table->size(0), table->size(1)})) return false;
    c->K = k->data_ptr();
    c->V = v->data_ptr();
    c->table = static_cast<const int*>(table->data_ptr());
    c->lengths = static_cast<const int*>(lengths->data_ptr());
    c->pages = static_cast<int>(k->size(0));
    c->kv_heads = static_cast<int>(k->size(1));
    c->page = static_cast<int>(k->size(2));
    c->d = static_cast<int>(k->size(3));
    c->sequences = static_cast<int>(table->size(0));
    c->table_width = static_cast<int>(table->size(1));
    *k_cache = k;
    return true;
}

// Scratch memory of one call on `stream`: it belongs to that stream alone, so that whoever gets it next runs behind the call.
at::Tensor scratch(int64_t bytes, void* stream, const at::Tensor& like) {
    const c10::cuda::CUDAStreamGuard guard(c10::cuda::getStreamFromExternal(static_cast<cudaStream_t>(stream), like.device().index()));
    return at::empty({bytes}, like.options().dtype(at::kByte).requires_grad(false));
}

PyObject* given_or_new(PyObject* given, at::Tensor&& made) { return given != Py_None ? Py_NewRef(given) : THPVariable_Wrap(std::move(made)); }

// rope(X, positions, frequencies, layout, amplitude, inverse, out, stream)
PyObject* py_rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!count_is(n, 8)) return nullptr;
    const bool f32 = THPVariable_Check(a[0]) && THPVariable_Unpack(a[0]).scalar_type() == at::kFloat;
    const at::ScalarType type = f32 ? at::kFloat : at::kBFloat16;
    const char* type_name = f32 ? "torch.float32" : "torch.bfloat16";
    const at::Tensor *x, *positions, *frequencies;
    if (!(x = strided_arg(a[0], "X", type, type_name, 4, nullptr))) return nullptr;
    const int64_t B = x->size(0), H = x->size(1), N = x->size(2), d = x->size(3);
    if (!small({B, H, N, d})) return nullptr;
    if (!(positions = int_arg(a[1], "positions", {B, N}, x)) ||
        !(frequencies = plain_arg(a[2], "frequencies", at::kDouble, "torch.float64", {-1}, x)))
        return nullptr;
    if (!small({2 * frequencies->size(0)})) return nullptr;
    int layout;
    float amplitude;
    if (!layout_arg(a[3], &layout) || !float_arg(a[4], &amplitude)) return nullptr;
    const int inverse = PyObject_IsTrue(a[5]);
    if (inverse < 0) return nullptr;
    const void* x_ptr = x->data_ptr();
    const auto* p_ptr = static_cast<const int*>(positions->data_ptr());
    const auto* f_ptr = static_cast<const double*>(frequencies->data_ptr());
    at::Tensor y;
    if (a[6] != Py_None) {
        const at::Tensor* t = strided_arg(a[6], "out", type, type_name, 4, x);
        if (!t) return nullptr;
        if (t->sizes() != x->sizes()) {
            value_error("out must be [B, H, N, d] like X");
            return nullptr;
        }
        y = *t;
    }
    const c10::cuda::CUDAGuard guard(x->device());
    void* stream;
    if (!stream_arg(a[7], &stream)) return nullptr;
    if (!y.defined()) y = new_on(stream, x->sizes(), type, *x);
    const long long xs[3] = {x->stride(0), x->stride(1), x->stride(2)}, ys[3] = {y.stride(0), y.stride(1), y.stride(2)};
    const auto entry = f32 ? attnw_rope_f32 : attnw_rope;
    void* y_ptr = y.data_ptr();
    const int rotary = static_cast<int>(2 * frequencies->size(0));
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = entry(x_ptr, p_ptr, f_ptr, y_ptr, static_cast<int>(B), static_cast<int>(H), static_cast<int>(N), static_cast<int>(d), rotary, xs, ys, layout,
               inverse, amplitude, stream);
    Py_END_ALLOW_THREADS
    if (rc != ATTNW_OK) return failed(rc, "attnw_rope");
    return given_or_new(a[6], std::move(y));
    END_HANDLE_TH_ERRORS
}

// cache_append(K_cache, V_cache, table, lengths, starts, Q, K, V, positions, frequencies, layout, amplitude, Q_out, stream)
PyObject* py_cache_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!count_is(n, 14)) return nullptr;
    attnw_cache c;
    const at::Tensor *cache, *starts, *q = nullptr, *k, *v, *positions = nullptr, *frequencies = nullptr;
    if (!cache_arg(a, &c, &cache) || !(starts = int_arg(a[4], "starts", {c.sequences + int64_t{1}}, cache))) return nullptr;
    if (!(k = strided_arg(a[6], "K", at::kBFloat16, "torch.bfloat16", 3, cache)) || !(v = strided_arg(a[7], "V", at::kBFloat16, "torch.bfloat16", 3, cache)))
        return nullptr;
    if (k->sizes() != v->sizes() || k->size(1) != c.kv_heads || k->size(2) != c.d) {
        value_error("K and V must both be [tokens, kv_heads, d]");
        return nullptr;
    }
    const int64_t tokens = k->size(0);
    if (a[5] != Py_None) {
        if (!(q = strided_arg(a[5], "Q", at::kBFloat16, "torch.bfloat16", 3, cache))) return nullptr;
        if (q->size(0) != tokens || q->size(2) != c.d) {
            value_error("Q must be [tokens, heads, d]");
            return nullptr;
        }
    } else if (a[12] != Py_None) {
        value_error("Q_out needs Q");
        return nullptr;
    }
    if ((a[8] == Py_None) != (a[9] == Py_None)) {
        value_error("positions and frequencies come together");
        return nullptr;
    }
    if (a[8] != Py_None && (!(positions = int_arg(a[8], "positions", {tokens}, cache)) ||
                            !(frequencies = plain_arg(a[9], "frequencies", at::kDouble, "torch.float64", {-1}, cache))))
        return nullptr;
    const int64_t rotary = frequencies ? 2 * frequencies->size(0) : 0;
    if (!small({tokens, q ? q->size(1) : 0, rotary})) return nullptr;
    int layout;
    float amplitude;
    if (!layout_arg(a[10], &layout) || !float_arg(a[11], &amplitude)) return nullptr;
    const void *q_ptr = q ? q->data_ptr() : nullptr, *k_ptr = k->data_ptr(), *v_ptr = v->data_ptr();
    const auto* s_ptr = static_cast<const int*>(starts->data_ptr());
    const auto* p_ptr = positions ? static_cast<const int*>(positions->data_ptr()) : nullptr;
    const auto* f_ptr = frequencies ? static_cast<const double*>(frequencies->data_ptr()) : nullptr;
    at::Tensor out;
    if (q && a[12] != Py_None) {
        const at::Tensor* t = strided_arg(a[12], "Q_out", at::kBFloat16, "torch.bfloat16", 3, cache);
        if (!t) return nullptr;
        if (t->sizes() != q->sizes()) {
            value_error("Q_out must be [tokens, heads, d] like Q");
            return nullptr;
        }
        out = *t;
    }
    const c10::cuda::CUDAGuard guard(cache->device());
    void* stream;
    if (!stream_arg(a[13], &stream)) return nullptr;
    if (q && !out.defined()) out = new_on(stream, q->sizes(), at::kBFloat16, *q);
    const long long strides[8] = {q ? q->stride(0) : 0, q ? q->stride(1) : 0, k->stride(0), k->stride(1), v->stride(0), v->stride(1),
                                  q ? out.stride(0) : 0, q ? out.stride(1) : 0};
    void* o_ptr = q ? out.data_ptr() : nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = attnw_cache_append(&c, q_ptr, k_ptr, v_ptr, o_ptr, strides, s_ptr, p_ptr, f_ptr, static_cast<int>(tokens),
                            q ? static_cast<int>(q->size(1)) : 0, static_cast<int>(rotary), layout, amplitude, stream);
    Py_END_ALLOW_THREADS
    if (rc != ATTNW_OK) return failed(rc, "attnw_cache_append");
    if (!q) Py_RETURN_NONE;
    return given_or_new(a[12], std::move(out));
    END_HANDLE_TH_ERRORS
}

// attn_paged(K_cache, V_cache, table, lengths, starts, Q, scale, O, lse, mass, mass_out, stream)
PyObject* py_attn_paged(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!count_is(n, 12)) return nullptr;
    attnw_cache c;
    const at::Tensor *cache, *starts, *q, *lse = nullptr, *mass = nullptr;
    if (!cache_arg(a, &c, &cache) || !(starts = int_arg(a[4], "starts", {c.sequences + int64_t{1}}, cache))) return nullptr;
    if (!(q = strided_arg(a[5], "Q", at::kBFloat16, "torch.bfloat16", 3, cache))) return nullptr;
    if (q->size(2) != c.d) {
        value_error("Q must be [tokens, heads, d]");
        return nullptr;
    }
    const int64_t tokens = q->size(0), heads = q->size(1), capacity = int64_t{c.table_width} * c.page;
    if (!small({tokens, heads})) return nullptr;
    float scale;
    if (!float_arg(a[6], &scale)) return nullptr;
    if (a[8] != Py_None && !(lse = f32_arg(a[8], "lse", {tokens, heads}, cache))) return nullptr;
    if (a[9] != Py_None && !(mass = f32_arg(a[9], "mass", {c.sequences, c.kv_heads, capacity}, cache))) return nullptr;
    if (!mass && a[10] != Py_None) {
        value_error("mass_out needs mass");
        return nullptr;
    }
    const void* q_ptr = q->data_ptr();
    const auto* s_ptr = static_cast<const int*>(starts->data_ptr());
    float* lse_ptr = lse ? static_cast<float*>(lse->data_ptr()) : nullptr;
    const float* mass_ptr = mass ? static_cast<const float*>(mass->data_ptr()) : nullptr;
    at::Tensor o, mass_out;
    if (!output_arg(a[7], "O", q->sizes(), false, true, "[tokens, heads, d]", *q, &o)) return nullptr;
    if (mass && a[10] != Py_None) {
        const at::Tensor* t = f32_arg(a[10], "mass_out", {c.sequences, c.kv_heads, capacity}, cache);
        if (!t) return nullptr;
        mass_out = *t;
    }
    const c10::cuda::CUDAGuard guard(cache->device());
    void* stream;
    if (!stream_arg(a[11], &stream)) return nullptr;
    if (!o.defined()) o = new_on(stream, q->sizes(), at::kBFloat16, *q);
    if (mass && !mass_out.defined()) mass_out = new_on(stream, mass->sizes(), at::kFloat, *q);
    const long long strides[2] = {q->stride(0), q->stride(1)};
    const long long bytes = attn_paged_workspace(&c, static_cast<int>(tokens), static_cast<int>(heads), mass ? 1 : 0);
    at::Tensor workspace;
    if (bytes > 0) workspace = scratch(bytes, stream, *cache);
    void *o_ptr = o.data_ptr(), *w_ptr = bytes > 0 ? workspace.data_ptr() : nullptr;
    float* out_ptr = mass ? static_cast<float*>(mass_out.data_ptr()) : nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = attn_paged(&c, q_ptr, strides, s_ptr, o_ptr, lse_ptr, mass_ptr, out_ptr, w_ptr, bytes, static_cast<int>(tokens), static_cast<int>(heads), scale,
                    stream);
    Py_END_ALLOW_THREADS
    if (rc != ATTNW_OK) return failed(rc, "attn_paged");
    PyObject* po = given_or_new(a[7], std::move(o));
    if (!mass || !po) return po;
    PyObject* pm = given_or_new(a[10], std::move(mass_out));
    PyObject* pair = pm ? PyTuple_Pack(2, po, pm) : nullptr;
    Py_DECREF(po);
    Py_XDECREF(pm);
    return pair;
    END_HANDLE_TH_ERRORS
}

// cache_evict(K_cache, V_cache, table, lengths, mass, budget, recent, table_out, mass_out, stream)
PyObject* py_cache_evict(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!count_is(n, 10)) return nullptr;
    attnw_cache c;
    const at::Tensor *cache, *mass, *table_out = nullptr;
    if (!cache_arg(a, &c, &cache) || !(mass = f32_arg(a[4], "mass", {c.sequences, c.kv_heads, int64_t{c.table_width} * c.page}, cache))) return nullptr;
    int budget, recent;
    if (!int_value(a[5], &budget) || !int_value(a[6], &recent)) return nullptr;
    if (a[7] != Py_None && !(table_out = int_arg(a[7], "table_out", {c.sequences, -1}, cache))) return nullptr;
    const int64_t width = table_out ? table_out->size(1) : c.table_width, capacity = width * c.page;
    if (!small({width, capacity})) return nullptr;
    const float* mass_ptr = static_cast<const float*>(mass->data_ptr());
    const int* out_table = table_out ? static_cast<const int*>(table_out->data_ptr()) : nullptr;
    at::Tensor mass_out;
    if (a[8] != Py_None) {
        const at::Tensor* t = f32_arg(a[8], "mass_out", {c.sequences, c.kv_heads, capacity}, cache);
        if (!t) return nullptr;
        mass_out = *t;
    }
    const c10::cuda::CUDAGuard guard(cache->device());
    void* stream;
    if (!stream_arg(a[9], &stream)) return nullptr;
    if (!mass_out.defined()) mass_out = new_on(stream, {c.sequences, c.kv_heads, capacity}, at::kFloat, *cache);
    // (a budget that the call refuses, below 1 or more than the pages hold, gets no memory of its size)
    const at::Tensor kept = new_on(stream, {c.sequences, c.kv_heads, budget > 0 && budget <= capacity ? budget : 1}, at::kInt, *cache),
                     lengths_out = new_on(stream, {c.sequences}, at::kInt, *cache);
    float* out_ptr = static_cast<float*>(mass_out.data_ptr());
    int *kept_ptr = static_cast<int*>(kept.data_ptr()), *length_ptr = static_cast<int*>(lengths_out.data_ptr());
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = attnw_cache_evict(&c, out_table, static_cast<int>(width), mass_ptr, out_ptr, kept_ptr, length_ptr, budget, recent, stream);
    Py_END_ALLOW_THREADS
    if (rc != ATTNW_OK) return failed(rc, "attnw_cache_evict");
    PyObject *pk = THPVariable_Wrap(kept), *pl = THPVariable_Wrap(lengths_out), *pm = given_or_new(a[8], std::move(mass_out));
    PyObject* all = pk && pl && pm ? PyTuple_Pack(3, pk, pl, pm) : nullptr;
    Py_XDECREF(pk);
    Py_XDECREF(pl);
    Py_XDECREF(pm);
    return all;
    END_HANDLE_TH_ERRORS
}

PyObject* py_set_error(PyObject*, PyObject* type) {
    Py_XSETREF(g_error, Py_NewRef(type));
    Py_RETURN_NONE;
}

template <typename F>
PyCFunction fast(F f) {
    return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f));
}

PyMethodDef g_methods[] = {
    {"attnw_fused", fast(py_attnw_fused), METH_FASTCALL, "attnw_fused(Q, K, scale, P, out_dtype, stream)"},
    {"attn_fused", fast(py_attn_fused), METH_FASTCALL, "attn_fused(Q, K, V, scale, O, stream)"},
    {"project_qk", fast(py_project_qk), METH_FASTCALL, "project_qk(X, Wq, Wk, Q, K, stream)"},
    {"softmax_rows", fast(py_softmax_rows), METH_FASTCALL, "softmax_rows(S, P, out_dtype, stream)"},
    {"rope", fast(py_rope), METH_FASTCALL, "rope(X, positions, frequencies, layout, amplitude, inverse, out, stream)"},
    {"cache_append", fast(py_cache_append), METH_FASTCALL,
     "cache_append(K_cache, V_cache, table, lengths, starts, Q, K, V, positions, frequencies, layout, amplitude, Q_out, stream)"},
    {"attn_paged", fast(py_attn_paged), METH_FASTCALL,
     "attn_paged(K_cache, V_cache, table, lengths, starts, Q, scale, O, lse, mass, mass_out, stream)"},
    {"cache_evict", fast(py_cache_evict), METH_FASTCALL,
     "cache_evict(K_cache, V_cache, table, lengths, mass, budget, recent, table_out, mass_out, stream)"},
    {"set_error", py_set_error, METH_O, "the exception type for attnw status codes"},
    {nullptr, nullptr, 0, nullptr},
};
#ifndef ATTNW_BUILT_FOR
#error "build.py passes the torch and the Python that the module is built for and looks for them in it later"
#endif
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_attnw_torch", ATTNW_BUILT_FOR, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__attnw_torch() { return PyModule_Create(&g_module); }
