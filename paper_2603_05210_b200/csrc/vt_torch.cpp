// Argument marshalling of the decode step's calls: torch tensors in, C entry points of include/vt.h called, torch tensors out.
//
// What binding.py does for the other calls through ctypes, for the calls a decode step makes one after the other: their device work takes a few
// microseconds, and checking six tensors and making one in Python takes ten more.  Each function returns its output tensors, or the status as an
// int where the entry point refused.  TypeError and ValueError are raised here.
#include <Python.h>

#include <ATen/ops/empty.h>
#include <ATen/ops/empty_like.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/vt.h"

namespace {

struct Entry {
    decltype(&vt_rope) rope;
    decltype(&vt_rope_append) rope_append;
    decltype(&vt_tree_mask) tree_mask;
    decltype(&vt_tree_attention) tree_attention;
    decltype(&vt_tree_attention_workspace_bytes) tree_attention_workspace_bytes;
    decltype(&vt_verify_tokens) verify_tokens;
} entry;

bool refuse(PyObject* type, const char* name, const char* what) {
    PyErr_Format(type, "%s: %s", name, what);
    return false;
}
bool tensor(PyObject* o, const char* name, const at::Tensor** t) {
    if (!THPVariable_Check(o)) return refuse(PyExc_TypeError, name, "expected a tensor");
    *t = &THPVariable_Unpack(o);
    return true;
}
// On the current CUDA device (dev: -1 until the first tensor has been seen).
bool here(const at::Tensor& t, int* dev) {
    if (!t.is_cuda()) return false;
    if (*dev < 0) *dev = c10::cuda::current_device();
    return t.get_device() == *dev;
}

struct Heads {
    vt_heads h;
    int64_t n, heads, d;
};
bool describe(const at::Tensor& t, const char* name, int* dev, Heads* out) {
    if (t.scalar_type() != at::kBFloat16) return refuse(PyExc_TypeError, name, "expected torch.bfloat16");
    if (t.dim() != 3 || !here(t, dev) || (t.stride(2) != 1 && t.size(2) > 1 && t.size(0) > 0))
        return refuse(PyExc_ValueError, name, "expected [tokens, heads, D] with contiguous heads on the current CUDA device");
    out->n = t.size(0);
    out->heads = t.size(1);
    out->d = t.size(2);
    out->h.ptr = t.data_ptr();
    // the stride of one alone says nothing
    out->h.token_stride = out->n > 1 ? t.stride(0) : (out->heads > 0 ? out->heads : 1) * out->d;
    out->h.head_stride = out->heads > 1 ? t.stride(1) : out->d;
    if (out->n > INT32_MAX || out->heads > INT32_MAX || out->d > INT32_MAX) return refuse(PyExc_ValueError, name, "too large");
    return true;
}
bool heads(PyObject* o, const char* name, int* dev, Heads* out) {
    const at::Tensor* t;
    return tensor(o, name, &t) && describe(*t, name, dev, out);
}
// An output of the shape of `like`: the caller's, or a new one.
bool heads_out(PyObject* o, const char* name, const at::Tensor& like, int* dev, at::Tensor* t, Heads* out) {
    if (o == Py_None) {
        *t = at::empty_like(like, like.options(), at::MemoryFormat::Contiguous);
    } else {
        const at::Tensor* given;
        if (!tensor(o, name, &given)) return false;
        if (given->sizes() != like.sizes()) return refuse(PyExc_ValueError, name, "expected the shape of its input");
        *t = *given;
    }
    return describe(*t, name, dev, out);
}
// A contiguous vector of n entries (n < 0: any number).
bool vector(PyObject* o, const char* name, int64_t n, at::ScalarType type, int* dev, void** out, int64_t* length = nullptr) {
    const at::Tensor* t;
    if (!tensor(o, name, &t)) return false;
    if (t->scalar_type() != type || t->dim() != 1 || !here(*t, dev) || !t->is_contiguous() || (n >= 0 && t->size(0) != n)) {
        if (n >= 0) PyErr_Format(PyExc_ValueError, "%s: expected a contiguous %s vector of %lld on the current CUDA device", name,
                                 type == at::kInt ? "int32" : "float32", (long long)n);
        else PyErr_Format(PyExc_ValueError, "%s: expected a contiguous %s vector on the current CUDA device", name, type == at::kInt ? "int32" : "float32");
        return false;
    }
    *out = t->data_ptr();
    if (length) *length = t->size(0);
    return true;
}
bool given_or_new(PyObject* o, const char* name, at::IntArrayRef shape, at::ScalarType type, const at::Tensor& like, int* dev, at::Tensor* t) {
    if (o == Py_None) {
        *t = at::empty(shape, like.options().dtype(type));
        return true;
    }
    const at::Tensor* given;
    if (!tensor(o, name, &given)) return false;
    if (given->scalar_type() != type || !here(*given, dev) || !given->is_contiguous() || given->sizes() != shape)
        return refuse(PyExc_ValueError, name, "expected a contiguous output of the right shape and type on the current CUDA device");
    *t = *given;
    return true;
}
// float32 [N, vocabulary] with contiguous rows
bool rows(const at::Tensor& t, const char* name, int* dev) {
    if (t.scalar_type() != at::kFloat || t.dim() != 2 || !here(t, dev) || (t.stride(1) != 1 && t.size(1) > 1 && t.size(0) > 0) || t.size(0) > INT32_MAX ||
        t.size(1) > INT32_MAX)
        return refuse(PyExc_ValueError, name, "expected float32 [N, vocabulary] with contiguous rows on the current CUDA device");
    return true;
}
bool whole(PyObject* o, const char* name, int* out) {
    const long v = PyLong_AsLong(o);
    if (v == -1 && PyErr_Occurred()) return false;
    if (v < INT32_MIN || v > INT32_MAX) return refuse(PyExc_ValueError, name, "out of range");
    *out = (int)v;
    return true;
}
bool real(PyObject* o, float* out) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) return false;
    *out = (float)v;
    return true;
}
const vt_cache* cache_of(PyObject* o) { return reinterpret_cast<const vt_cache*>(PyLong_AsVoidPtr(o)); }
bool table_of(PyObject* o, int rot_dim, int* dev, const uint64_t** out) {
    const at::Tensor* t;
    if (!tensor(o, "rope", &t)) return false;
    if (!here(*t, dev)) return refuse(PyExc_ValueError, "rope", "its table lies on another device");
    if (t->scalar_type() != at::kLong || t->dim() != 1 || !t->is_contiguous() || t->size(0) != rot_dim / 2)
        return refuse(PyExc_ValueError, "rope", "its table is not one of rot_dim / 2 frequencies");
    *out = reinterpret_cast<const uint64_t*>(t->data_ptr());
    return true;
}
void* stream_of(int dev) { return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)dev).stream(); }
PyObject* status(vt_status s) { return PyLong_FromLong((long)s); }
bool count(Py_ssize_t got, Py_ssize_t want) {
    if (got == want) return true;
    PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, got);
    return false;
}

// (q, k or None, positions, table, rot_dim, amplitude, options, out_q or None, out_k or None) -> (out_q, out_k)
PyObject* rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    int dev = -1, rot = 0, options = 0;
    Heads q, k{}, qo, ko{};
    at::Tensor out_q, out_k;
    void* positions;
    const uint64_t* table;
    float amplitude;
    const bool with_k = n == 9 && a[1] != Py_None;
    if (!count(n, 9) || !heads(a[0], "q", &dev, &q) || !vector(a[2], "positions", q.n, at::kInt, &dev, &positions) || !whole(a[4], "rot_dim", &rot) ||
        !table_of(a[3], rot, &dev, &table) || !real(a[5], &amplitude) || !whole(a[6], "options", &options) ||
        !heads_out(a[7], "out_q", THPVariable_Unpack(a[0]), &dev, &out_q, &qo))
        return nullptr;
    if (with_k) {
        if (!heads(a[1], "k", &dev, &k)) return nullptr;
        if (k.n != q.n || k.d != q.d) { refuse(PyExc_ValueError, "q, k", "disagree on tokens or D"); return nullptr; }
        if (!heads_out(a[8], "out_k", THPVariable_Unpack(a[1]), &dev, &out_k, &ko)) return nullptr;
    } else if (a[8] != Py_None) {
        refuse(PyExc_ValueError, "out_k", "needs k");
        return nullptr;
    }
    void* stream = stream_of(dev);
    vt_status s;
    Py_BEGIN_ALLOW_THREADS
    s = entry.rope(&q.h, with_k ? &k.h : nullptr, (const int32_t*)positions, table, (int)q.n, (int)q.heads, with_k ? (int)k.heads : 0, (int)q.d, rot,
                   amplitude, options, &qo.h, with_k ? &ko.h : nullptr, stream);
    Py_END_ALLOW_THREADS
    if (s != VT_OK) return status(s);
    PyObject* pq = THPVariable_Wrap(out_q);
    PyObject* pk = with_k ? THPVariable_Wrap(out_k) : Py_NewRef(Py_None);
    return Py_BuildValue("(NN)", pq, pk);
    END_HANDLE_TH_ERRORS
}

// (q, k, v, positions, cu_tokens, cache's address, its device, table, rot_dim, amplitude, options, out_q or None) -> out_q
PyObject* rope_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    int dev = -1, rot = 0, options = 0, cache_dev = 0;
    Heads q, k, v, qo;
    at::Tensor out_q;
    void *positions, *cu;
    const uint64_t* table;
    float amplitude;
    if (!count(n, 12) || !heads(a[0], "q", &dev, &q) || !heads(a[1], "k", &dev, &k) || !heads(a[2], "v", &dev, &v) || !whole(a[6], "cache", &cache_dev))
        return nullptr;
    const vt_cache* c = cache_of(a[5]);
    if (!c) return nullptr;
    if (k.n != q.n || v.n != q.n || k.heads != c->heads || v.heads != k.heads || k.d != q.d || v.d != q.d || q.d != c->head_dim || cache_dev != dev) {
        PyErr_SetString(PyExc_ValueError, "q, k, v and the cache disagree on tokens, heads, D or device");
        return nullptr;
    }
    if (!vector(a[3], "positions", q.n, at::kInt, &dev, &positions) || !vector(a[4], "cu_tokens", (int64_t)c->B + 1, at::kInt, &dev, &cu) ||
        !whole(a[8], "rot_dim", &rot) || !table_of(a[7], rot, &dev, &table) || !real(a[9], &amplitude) || !whole(a[10], "options", &options) ||
        !heads_out(a[11], "out_q", THPVariable_Unpack(a[0]), &dev, &out_q, &qo))
        return nullptr;
    void* stream = stream_of(dev);
    vt_status s;
    Py_BEGIN_ALLOW_THREADS
    s = entry.rope_append(&q.h, &k.h, &v.h, (const int32_t*)positions, (const int32_t*)cu, table, (int)q.n, (int)q.heads, rot, amplitude, options, &qo.h,
                          c, stream);
    Py_END_ALLOW_THREADS
    return s == VT_OK ? THPVariable_Wrap(out_q) : status(s);
    END_HANDLE_TH_ERRORS
}

// (parents, cu_tokens, words, lens or None, mask or None, positions or None) -> (mask, positions)
PyObject* tree_mask(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    int dev = -1, words = 0;
    void *parents, *cu, *lens = nullptr;
    int64_t N = 0, B = 0;
    if (!count(n, 6) || !vector(a[0], "parents", -1, at::kInt, &dev, &parents, &N) || !vector(a[1], "cu_tokens", -1, at::kInt, &dev, &cu, &B) ||
        !whole(a[2], "max_tokens", &words) || (a[3] != Py_None && !vector(a[3], "lens", B - 1, at::kInt, &dev, &lens)))
        return nullptr;
    if (N > INT32_MAX || B > INT32_MAX || words < 0) { refuse(PyExc_ValueError, "parents, cu_tokens, max_tokens", "out of range"); return nullptr; }
    const at::Tensor& like = THPVariable_Unpack(a[0]);
    at::Tensor mask, positions;
    if (!given_or_new(a[4], "mask", {N, words}, at::kInt, like, &dev, &mask) || !given_or_new(a[5], "positions", {N}, at::kInt, like, &dev, &positions))
        return nullptr;
    void* stream = stream_of(dev);
    vt_status s;
    Py_BEGIN_ALLOW_THREADS
    s = entry.tree_mask((const int32_t*)parents, (const int32_t*)cu, (const int32_t*)lens, (int)N, (int)(B - 1), (int32_t*)mask.data_ptr(), words,
                        (int32_t*)positions.data_ptr(), stream);
    Py_END_ALLOW_THREADS
    if (s != VT_OK) return status(s);
    return Py_BuildValue("(NN)", THPVariable_Wrap(mask), THPVariable_Wrap(positions));
    END_HANDLE_TH_ERRORS
}

// (q, cu_tokens, cache's address, its device, mask or None, max_tokens, scale or None, out or None, lse or None, workspace or None) -> (out, lse)
PyObject* tree_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    int dev = -1, cache_dev = 0, max_tokens = 0, words = 0;
    Heads q, o;
    void* cu;
    if (!count(n, 10) || !heads(a[0], "q", &dev, &q) || !whole(a[3], "cache", &cache_dev) || !whole(a[5], "max_tokens", &max_tokens)) return nullptr;
    const vt_cache* c = cache_of(a[2]);
    if (!c) return nullptr;
    if (q.d != c->head_dim || cache_dev != dev) {
        PyErr_SetString(PyExc_ValueError, "q and the cache disagree on D or device");
        return nullptr;
    }
    if (!vector(a[1], "cu_tokens", (int64_t)c->B + 1, at::kInt, &dev, &cu)) return nullptr;
    const int32_t* mask = nullptr;
    if (a[4] != Py_None) {
        const at::Tensor* m;
        if (!tensor(a[4], "mask", &m)) return nullptr;
        if (m->scalar_type() != at::kInt || m->dim() != 2 || m->size(0) != q.n || !here(*m, &dev) || !m->is_contiguous() || m->size(1) < 1 || m->size(1) > INT32_MAX) {
            refuse(PyExc_ValueError, "mask", "expected a contiguous int32 tensor with a row of words per token on the current CUDA device");
            return nullptr;
        }
        mask = (const int32_t*)m->data_ptr();
        words = (int)m->size(1);
    }
    float scale = 0.0f;
    if (a[6] == Py_None) scale = (float)std::pow((double)q.d, -0.5);
    else if (!real(a[6], &scale)) return nullptr;
    const at::Tensor& like = THPVariable_Unpack(a[0]);
    at::Tensor out, lse, workspace;
    if (!heads_out(a[7], "out", like, &dev, &out, &o) || !given_or_new(a[8], "lse", {q.n, q.heads}, at::kFloat, like, &dev, &lse)) return nullptr;
    if (a[9] == Py_None) {
        const size_t bytes = entry.tree_attention_workspace_bytes((int)q.heads, c->heads, (int)q.d, max_tokens);
        workspace = at::empty({(int64_t)std::max<size_t>(bytes, 256)}, like.options().dtype(at::kByte));
    } else {
        const at::Tensor* w;
        if (!tensor(a[9], "workspace", &w)) return nullptr;
        if (!here(*w, &dev) || !w->is_contiguous()) {
            refuse(PyExc_ValueError, "workspace", "expected a contiguous tensor on the current CUDA device");
            return nullptr;
        }
        workspace = *w;
    }
    void* stream = stream_of(dev);
    vt_status s;
    Py_BEGIN_ALLOW_THREADS
    s = entry.tree_attention(&q.h, (const int32_t*)cu, c, mask, words, (int)q.n, (int)q.heads, max_tokens, scale, &o.h, (float*)lse.data_ptr(),
                             workspace.data_ptr(), (size_t)workspace.nbytes(), stream);
    Py_END_ALLOW_THREADS
    if (s != VT_OK) return status(s);
    return Py_BuildValue("(NN)", THPVariable_Wrap(out), THPVariable_Wrap(lse));
    END_HANDLE_TH_ERRORS
}

// (probs, tokens, parents, cu_tokens, u_accept, u_sample, max_tokens, draft_probs, draft_ids, d2t, n_accepted, path, out_tokens; the last six may
// be None) -> (n_accepted, path, out_tokens)
PyObject* verify_tokens(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    int dev = -1, max_tokens = 0;
    const at::Tensor *probs, *draft = nullptr;
    void *tokens, *parents, *cu, *ua, *us, *ids = nullptr, *d2t = nullptr;
    int64_t B = 0;
    if (!count(n, 13) || !tensor(a[0], "probs", &probs) || !rows(*probs, "probs", &dev) || !vector(a[5], "u_sample", -1, at::kFloat, &dev, &us, &B) ||
        !whole(a[6], "max_tokens", &max_tokens))
        return nullptr;
    const int64_t N = probs->size(0), V = probs->size(1);
    if (!vector(a[1], "tokens", N, at::kInt, &dev, &tokens) || !vector(a[2], "parents", N, at::kInt, &dev, &parents) ||
        !vector(a[3], "cu_tokens", B + 1, at::kInt, &dev, &cu) || !vector(a[4], "u_accept", N, at::kFloat, &dev, &ua))
        return nullptr;
    int64_t Vd = 0, ldq = 0;
    if (a[7] != Py_None) {
        if (!tensor(a[7], "draft_probs", &draft) || !rows(*draft, "draft_probs", &dev)) return nullptr;
        if (a[8] == Py_None || draft->size(0) != N || draft->size(1) < 1) {
            refuse(PyExc_ValueError, "draft_probs", "needs a row per token, and draft_ids");
            return nullptr;
        }
        Vd = draft->size(1);
        ldq = N > 1 ? draft->stride(0) : Vd;
        if (!vector(a[8], "draft_ids", N, at::kInt, &dev, &ids) || (a[9] != Py_None && !vector(a[9], "d2t", Vd, at::kInt, &dev, &d2t))) return nullptr;
    } else if (a[8] != Py_None || a[9] != Py_None) {
        refuse(PyExc_ValueError, "draft_ids, d2t", "need draft_probs");
        return nullptr;
    }
    const at::Tensor& like = THPVariable_Unpack(a[1]);
    const int64_t most = std::max(max_tokens, 0);
    at::Tensor n_out, path, out;
    if (!given_or_new(a[10], "n_accepted", {B}, at::kInt, like, &dev, &n_out) || !given_or_new(a[11], "path", {B, most}, at::kInt, like, &dev, &path) ||
        !given_or_new(a[12], "tokens", {B, most}, at::kInt, like, &dev, &out))
        return nullptr;
    if (B > INT32_MAX) { refuse(PyExc_ValueError, "u_sample", "too large"); return nullptr; }
    void* stream = stream_of(dev);
    vt_status s;
    Py_BEGIN_ALLOW_THREADS
    s = entry.verify_tokens((const float*)probs->data_ptr(), N > 1 ? probs->stride(0) : V, (const int32_t*)tokens, (const int32_t*)parents,
                            (const int32_t*)cu, (const float*)ua, (const float*)us, draft ? (const float*)draft->data_ptr() : nullptr, ldq,
                            (const int32_t*)ids, (const int32_t*)d2t, (int)N, (int)B, (int)V, (int)Vd, max_tokens, (int32_t*)n_out.data_ptr(),
                            (int32_t*)path.data_ptr(), (int32_t*)out.data_ptr(), stream);
    Py_END_ALLOW_THREADS
    if (s != VT_OK) return status(s);
    return Py_BuildValue("(NNN)", THPVariable_Wrap(n_out), THPVariable_Wrap(path), THPVariable_Wrap(out));
    END_HANDLE_TH_ERRORS
}

// (addresses of the six entry points, in the order of Entry)
PyObject* init(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!count(n, 6)) return nullptr;
    void* at[6];
    for (int i = 0; i < 6; ++i) {
        at[i] = PyLong_AsVoidPtr(a[i]);
        if (!at[i]) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "init: an entry point is missing");
            return nullptr;
        }
    }
    entry = {(decltype(entry.rope))at[0], (decltype(entry.rope_append))at[1], (decltype(entry.tree_mask))at[2], (decltype(entry.tree_attention))at[3],
             (decltype(entry.tree_attention_workspace_bytes))at[4], (decltype(entry.verify_tokens))at[5]};
    Py_RETURN_NONE;
}

#define VT_METHOD(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {VT_METHOD(init), VT_METHOD(rope), VT_METHOD(rope_append), VT_METHOD(tree_mask), VT_METHOD(tree_attention),
                         VT_METHOD(verify_tokens), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_vt_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__vt_torch() { return PyModule_Create(&module); }
