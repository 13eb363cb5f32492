// The per-call path of attn_fwd, gemm_lrelu, the cache's calls and the norms with rotation in native code: check the tensors, read their pointers and
// torch's current stream, call the library.  Done in Python the same steps take 6 us a call, more than
// the kernels of small problems (1 x 2 x 128 x 64 attention: 4.7 us), so back-to-back calls ran at the
// interpreter's pace.  The calls with more arguments took 14 to 30 us there (norms of 8 tokens, attention of one query
// over 1003 keys: 19.6 and 20.6 us a call, with kernels of 3.6 and 12).
//
// Only plain calls are served here: anything a check does not recognise (another device, layout, type,
// shape) returns kNotPlain and the caller takes the Python path, which names what is wrong.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <limits.h>

#include <ATen/core/Tensor.h>
#include <c10/hip/HIPCachingAllocator.h>
#include <c10/hip/HIPGraphsC10Utils.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/kv4.h"
#include "../../include/qk_rope.h"

namespace {

constexpr long kNotPlain = 1;  // library codes are 0 or negative

typedef int (*AttnFn)(const void*, const void*, const void*, void*, float*, int, int, int, int, int, float, int, void*);
typedef void* (*ScratchFn)(void*, long long);
typedef int (*GemmFn)(const void*, const void*, void*, int, int, int, float, int, void*, ScratchFn, void*);
typedef int (*CapturingFn)(void*);
AttnFn g_attn = nullptr;
GemmFn g_gemm = nullptr;
CapturingFn g_capturing = nullptr;
decltype(&kv4_append) g_kv4_append = nullptr;
decltype(&kv4_read) g_kv4_read = nullptr;
decltype(&kv4_attn) g_kv4_attn = nullptr;
decltype(&kv4_attn_workspace) g_kv4_attn_workspace = nullptr;
decltype(&qk_norm_rope) g_rope = nullptr;
decltype(&qk_norm_rope_bwd) g_rope_bwd = nullptr;
decltype(&qk_norm_rope_bwd_workspace) g_rope_bwd_workspace = nullptr;

// Whether torch's allocator has an address in a pool of its own: one that it opened for a graph that it records (or its user for tensors).  It looks
// through all segments, which a recording can wait for.
bool in_private_pool(const void* p) {
    for (const auto& s : c10::hip::HIPCachingAllocator::snapshot().segments)
        if ((size_t)p - s.address < s.total_size) return s.owner_private_pool_id.first || s.owner_private_pool_id.second;
    return false;
}

// Scratch memory of one call, from torch's caching allocator: it belongs to the stream the call runs on, so it
// may go back as soon as the kernels are enqueued (the next owner on that stream comes after them).  That holds
// where a handle is one queue and outlives its work: torch's current stream, but not a handle that only the
// caller knows, nor the per-thread stream, one handle for a queue of every thread.  No memory either
// on a device that is not the current one, or when there is none left, or while the stream is captured, unless `captured` and torch itself records: in its
// graph the memory comes from that graph's own pool and stays its, but a recording begun elsewhere would keep the address of memory that torch hands on at once.
// The call then does without.
class Workspace {
  public:
    Workspace(void* stream, int device, bool captured = false) : stream_(stream), device_(device), captured_(captured) {}
    // What the library calls if it has a use for the memory (without the interpreter's lock: torch takes it where its allocator needs it).
    static void* take(void* self, long long bytes) { return ((Workspace*)self)->take(bytes); }
    void* take(long long bytes) {
        try {
            if (stream_ != (void*)c10::hip::getCurrentHIPStream(device_).stream() || stream_ == (void*)hipStreamPerThread ||
                c10::hip::current_device() != device_)
                return nullptr;
            const bool capturing = g_capturing(stream_);
            if (capturing && !captured_) return nullptr;
            // A recording in another thread (in the default mode) forbids this thread the allocator's calls to the
            // device, and one such call would end it; they have nothing to do with it.
            const c10::hip::HIPStreamCaptureModeGuard beside(hipStreamCaptureModeRelaxed);
            p_ = c10::hip::HIPCachingAllocator::raw_alloc_with_stream((size_t)bytes, (hipStream_t)stream_);
            if (capturing && !in_private_pool(p_)) return nullptr;
        } catch (const std::exception&) {
            return nullptr;
        }
        return p_;
    }
    ~Workspace() {
        try {
            if (p_) c10::hip::HIPCachingAllocator::raw_delete(p_);
        } catch (const std::exception&) {
        }
    }
    Workspace(const Workspace&) = delete;
    Workspace& operator=(const Workspace&) = delete;

  private:
    void* stream_;
    int device_;
    bool captured_;
    void* p_ = nullptr;
};

const at::Tensor* plain_tensor(PyObject* o, int dim) {
    if (!THPVariable_Check(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.defined() || t.layout() != at::kStrided || !t.is_cuda() || t.dim() != dim || !t.is_contiguous()) return nullptr;
    for (int i = 0; i < dim; ++i)
        if (t.size(i) > INT_MAX) return nullptr;
    return &t;
}

int dtype_code(const at::Tensor& t) {  // the library's codes, the same for both entry points
    return t.scalar_type() == at::kHalf ? 0 : t.scalar_type() == at::kBFloat16 ? 1 : -1;
}

// `given`: None for torch's current stream of t's device, or an integer hipStream_t.
bool stream_of(PyObject* given, const at::Tensor& t, void** stream) {
    if (given == Py_None) {
        *stream = (void*)c10::hip::getCurrentHIPStream(t.device().index()).stream();
        return true;
    }
    if (!PyLong_CheckExact(given)) return false;
    *stream = PyLong_AsVoidPtr(given);
    return !PyErr_Occurred();
}

PyObject* not_plain() {
    PyErr_Clear();
    return PyLong_FromLong(kNotPlain);
}

// No exception of torch's may leave an entry point of C: a tensor without storage (inside torch.func.vmap, say)
// throws where its sizes, its data pointer or its stream are asked for.  The Python path then raises its own.
template <PyObject* (*F)(PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    try {
        return F(args, nargs);
    } catch (const std::exception&) {
        return not_plain();
    }
}

// attn_fwd(q, k, v, out, lse, causal, scale, stream)
PyObject* attn_fwd(PyObject* const* args, Py_ssize_t nargs) {
    if (nargs != 8 || !g_attn) return not_plain();
    const at::Tensor *q = plain_tensor(args[0], 4), *k = plain_tensor(args[1], 4), *v = plain_tensor(args[2], 4),
                     *out = plain_tensor(args[3], 4), *lse = plain_tensor(args[4], 3);
    if (!q || !k || !v || !out || !lse) return not_plain();
    const int dt = dtype_code(*q);
    if (dt < 0 || k->scalar_type() != q->scalar_type() || v->scalar_type() != q->scalar_type() ||
        out->scalar_type() != q->scalar_type() || lse->scalar_type() != at::kFloat || k->sizes() != q->sizes() ||
        v->sizes() != q->sizes() || out->sizes() != q->sizes() || lse->sizes() != q->sizes().slice(0, 3))
        return not_plain();
    const int causal = PyObject_IsTrue(args[5]);
    const double scale = PyFloat_AsDouble(args[6]);
    void* stream;
    if (causal < 0 || (scale == -1.0 && PyErr_Occurred()) || !stream_of(args[7], *q, &stream)) return not_plain();
    void *const pq = q->data_ptr(), *const pk = k->data_ptr(), *const pv = v->data_ptr(), *const po = out->data_ptr(),
               *const pl = lse->data_ptr();
    const int B = (int)q->size(0), H = (int)q->size(1), N = (int)q->size(2), d = (int)q->size(3);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = g_attn(pq, pk, pv, po, (float*)pl, B, H, N, d, causal, (float)scale, dt, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

// gemm_lrelu(a, b, c, slope, stream)
PyObject* gemm_lrelu(PyObject* const* args, Py_ssize_t nargs) {
    if (nargs != 5 || !g_gemm) return not_plain();
    const at::Tensor *a = plain_tensor(args[0], 2), *b = plain_tensor(args[1], 2), *c = plain_tensor(args[2], 2);
    if (!a || !b || !c) return not_plain();
    const int dt = dtype_code(*a);
    if (dt < 0 || b->scalar_type() != a->scalar_type() || c->scalar_type() != a->scalar_type() || b->size(0) != a->size(1) ||
        c->size(0) != a->size(0) || c->size(1) != b->size(1))
        return not_plain();
    const double slope = PyFloat_AsDouble(args[3]);
    void* stream;
    if ((slope == -1.0 && PyErr_Occurred()) || !stream_of(args[4], *a, &stream)) return not_plain();
    void *const pa = a->data_ptr(), *const pb = b->data_ptr(), *const pc = c->data_ptr();
    const int M = (int)a->size(0), N = (int)b->size(1), K = (int)a->size(1);
    Workspace ws(stream, a->device().index());
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = g_gemm(pa, pb, pc, M, N, K, (float)slope, dt, stream, &Workspace::take, &ws);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

// Arguments of the calls below.  Each reader clears `ok` where what it finds is not plain.

struct Reader {
    int device;
    bool ok = true;

    explicit Reader(PyObject* first) : device(-1) {
        if (THPVariable_Check(first)) {
            const at::Tensor& t = THPVariable_Unpack(first);
            if (t.defined() && t.is_cuda()) device = t.device().index();
        }
        if (device < 0 || c10::hip::current_device() != device) ok = false;
    }
    // A strided tensor of this device with `dim` sizes below 2^31 and channels on end.
    const at::Tensor* strided(PyObject* o, int dim) {
        if (ok && THPVariable_Check(o)) {
            const at::Tensor& t = THPVariable_Unpack(o);
            if (t.defined() && t.layout() == at::kStrided && t.is_cuda() && t.device().index() == device && t.dim() == dim && t.numel() > 0 &&
                t.stride(dim - 1) == 1) {
                bool small = true;
                for (int i = 0; i < dim; ++i) small = small && t.size(i) <= INT_MAX;
                if (small) return &t;
            }
        }
        ok = false;
        return nullptr;
    }
    const at::Tensor* whole(PyObject* o, int dim, at::ScalarType type) {
        const at::Tensor* t = strided(o, dim);
        if (t && t->is_contiguous() && t->scalar_type() == type) return t;
        ok = false;
        return nullptr;
    }
    const at::Tensor* whole_or_none(PyObject* o, int dim, at::ScalarType type) { return o == Py_None ? nullptr : whole(o, dim, type); }
    const at::Tensor* cache(PyObject* o) {
        const at::Tensor* t = whole(o, 4, at::kByte);
        if (t && t->size(3) % 17) ok = false;
        return ok ? t : nullptr;
    }
    bool truth(PyObject* o) {
        const int x = PyObject_IsTrue(o);
        if (x < 0) ok = false;
        return x > 0;
    }
    double number(PyObject* o) {
        const double x = PyFloat_AsDouble(o);
        if (x == -1.0 && PyErr_Occurred()) ok = false;
        return x;
    }
    int integer(PyObject* o) {
        const long long x = PyLong_CheckExact(o) ? PyLong_AsLongLong(o) : -1;
        if (x < 0 || x > INT_MAX) ok = false;
        return ok ? (int)x : 0;
    }
};

void* data(const at::Tensor* t) { return t ? t->data_ptr() : nullptr; }
long long stride(const at::Tensor* t, int i) { return t->size(i) > 1 ? t->stride(i) : 0; }

// cos and sin, [rows, d/2]: the same sizes
bool tables(Reader& r, PyObject* c, PyObject* s, int d, const at::Tensor** cos, const at::Tensor** sin) {
    *cos = r.whole(c, 2, at::kFloat), *sin = r.whole(s, 2, at::kFloat);
    return r.ok && (*cos)->size(1) == d / 2 && (*sin)->sizes() == (*cos)->sizes();
}

// kv4_append(k, v, cache, slots, cos, sin, positions, interleaved, stream)
PyObject* append(PyObject* const* args, Py_ssize_t nargs) {
    if (nargs != 9 || !g_kv4_append) return not_plain();
    Reader r(args[2]);
    const at::Tensor *k = r.strided(args[0], 3), *v = r.strided(args[1], 3), *cache = r.cache(args[2]), *slots = r.whole(args[3], 1, at::kInt);
    if (!r.ok) return not_plain();
    const int dt = dtype_code(*k), T = (int)k->size(0), heads = (int)cache->size(1), d = (int)(cache->size(3) / 17 * 16);
    if (dt < 0 || v->scalar_type() != k->scalar_type() || v->sizes() != k->sizes() || k->size(1) != heads || k->size(2) != d || slots->size(0) != T)
        return not_plain();
    const at::Tensor *cos = nullptr, *sin = nullptr, *positions = nullptr;
    if (args[4] != Py_None) {
        positions = r.whole(args[6], 1, at::kInt);
        if (!tables(r, args[4], args[5], d, &cos, &sin) || positions->size(0) != T) return not_plain();
    } else if (args[5] != Py_None) {
        return not_plain();
    }
    const bool pairs = r.truth(args[7]);
    void* stream;
    if (!r.ok || !stream_of(args[8], *cache, &stream)) return not_plain();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = g_kv4_append(data(k), stride(k, 0), stride(k, 1), data(v), stride(v, 0), stride(v, 1), data(cache), (const int*)data(slots),
                                (const float*)data(cos), (const float*)data(sin), (const int*)data(positions), cos ? (int)cos->size(0) : 0, pairs,
                                T, heads, d, (int)cache->size(0), (int)cache->size(2), dt, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

// kv4_read(cache, slots, k, v, stream)
PyObject* read(PyObject* const* args, Py_ssize_t nargs) {
    if (nargs != 5 || !g_kv4_read) return not_plain();
    Reader r(args[0]);
    const at::Tensor *cache = r.cache(args[0]), *slots = r.whole(args[1], 1, at::kInt);
    const at::Tensor *k = args[2] == Py_None ? nullptr : r.strided(args[2], 3), *v = args[3] == Py_None ? nullptr : r.strided(args[3], 3);
    if (!r.ok || (!k && !v)) return not_plain();
    const int T = (int)slots->size(0), heads = (int)cache->size(1), d = (int)(cache->size(3) / 17 * 16), dt = dtype_code(k ? *k : *v);
    for (const at::Tensor* t : {k, v})
        if (t && (!t->is_contiguous() || dtype_code(*t) != dt || dt < 0 || t->size(0) != T || t->size(1) != heads || t->size(2) != d)) return not_plain();
    void* stream;
    if (!stream_of(args[4], *cache, &stream)) return not_plain();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = g_kv4_read(data(cache), (const int*)data(slots), data(k), data(v), T, heads, d, (int)cache->size(0), (int)cache->size(2), dt, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

// kv4_attn(q, cache, tables, lens, out, lse, causal, scale, cu_q, max_q, workspace, stream)
PyObject* cached_attn(PyObject* const* args, Py_ssize_t nargs) {
    if (nargs != 12 || !g_kv4_attn) return not_plain();
    Reader r(args[1]);
    const at::Tensor *q = r.strided(args[0], 3), *cache = r.cache(args[1]), *table = r.whole(args[2], 2, at::kInt), *lens = r.whole(args[3], 1, at::kInt),
                     *out = r.strided(args[4], 3), *lse = r.whole(args[5], 2, at::kFloat), *cu = r.whole_or_none(args[8], 1, at::kInt);
    if (!r.ok) return not_plain();
    const int dt = dtype_code(*q), T = (int)q->size(0), H = (int)q->size(1), heads = (int)cache->size(1), d = (int)(cache->size(3) / 17 * 16),
              B = (int)table->size(0), width = (int)table->size(1), page = (int)cache->size(2);
    if (dt < 0 || !q->is_contiguous() || !out->is_contiguous() || out->sizes() != q->sizes() || out->scalar_type() != q->scalar_type() || q->size(2) != d ||
        lse->size(0) != T || lse->size(1) != H || lens->size(0) != B || (cu ? cu->size(0) != B + 1 || args[9] == Py_None : T % B != 0))
        return not_plain();
    const int max_q = args[9] == Py_None ? T / B : r.integer(args[9]);
    const bool causal = r.truth(args[6]);
    const double scale = r.number(args[7]);
    void* stream;
    if (!r.ok || (!cu && max_q != T / B) || !stream_of(args[11], *q, &stream)) return not_plain();
    const long long need = g_kv4_attn_workspace(T, B, H, heads, d, page, width, max_q);
    if (need < 0) return PyLong_FromLong(need);
    void* given = nullptr;
    if (args[10] != Py_None) {
        if (!THPVariable_Check(args[10])) return not_plain();
        const at::Tensor& t = THPVariable_Unpack(args[10]);
        if (!t.defined() || !t.is_cuda() || t.device().index() != r.device || !t.is_contiguous() || (long long)t.nbytes() < need) return not_plain();
        given = t.data_ptr();
    }
    void *const pq = data(q), *const pc = data(cache), *const pt = data(table), *const pn = data(lens), *const pu = data(cu), *const po = data(out),
               *const pl = data(lse);
    const int pages = (int)cache->size(0);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    {
        Workspace own(stream, r.device, true);
        void* ws = given ? given : need ? own.take(need) : nullptr;
        rc = g_kv4_attn(pq, pc, (const int*)pt, (const int*)pn, (const int*)pu, po, (float*)pl, T, B, H, heads, d, pages, page, width, max_q, causal,
                        (float)scale, dt, ws, ws ? need : 0, stream);
    }
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

struct RopeArgs {
    const at::Tensor* like = nullptr;
    int heads[2] = {0, 0}, dt = -1, B = 0, N = 0, d = 0, f32 = 0;
    const at::Tensor *cos = nullptr, *sin = nullptr, *positions = nullptr, *w[2] = {nullptr, nullptr};

    // A tensor of heads (z: of queries or keys) of one type and the sizes of those before it; None where `heads` has none.
    bool heads_of(Reader& r, PyObject* o, int z, qk_heads* h) {
        *h = {nullptr, 0, 0, 0};
        if (o == Py_None) return heads[z] == 0;
        const at::Tensor* t = r.strided(o, 4);
        if (!t) return false;
        if (!like) like = t, dt = dtype_code(*t), B = (int)t->size(0), N = (int)t->size(1), d = (int)t->size(3);
        if (!heads[z]) heads[z] = (int)t->size(2);
        if (dt < 0 || t->scalar_type() != like->scalar_type() || t->size(0) != B || t->size(1) != N || t->size(2) != heads[z] || t->size(3) != d) return false;
        *h = {t->data_ptr(), stride(t, 0), stride(t, 1), stride(t, 2)};
        return true;
    }
    bool others(Reader& r, PyObject* const* a) {  // cos, sin, positions, q_weight, k_weight
        if (!tables(r, a[0], a[1], d, &cos, &sin)) return false;
        positions = r.whole(a[2], 2, at::kInt);
        if (!r.ok || positions->size(0) != B || positions->size(1) != N) return false;
        for (int z = 0; z < 2; ++z) {
            if (a[3 + z] == Py_None) continue;
            w[z] = r.strided(a[3 + z], 1);
            if (!r.ok || w[z]->size(0) != d) return false;
            const at::ScalarType type = w[z]->scalar_type();
            if ((type != at::kFloat && type != like->scalar_type()) || (z && w[0] && w[0]->scalar_type() != type)) return false;
            f32 = type == at::kFloat;
        }
        return true;
    }
};

// qk_norm_rope(q, k, q_out, k_out, cos, sin, positions, q_weight, k_weight, eps, interleaved, stream)
PyObject* norm_rope(PyObject* const* args, Py_ssize_t nargs) {
    if (nargs != 12 || !g_rope) return not_plain();
    Reader r(args[4]);
    RopeArgs a;
    qk_heads h[4];
    for (int i = 0; i < 4; ++i)
        if (!a.heads_of(r, args[i], i % 2, &h[i])) return not_plain();
    for (int z = 0; z < 2; ++z)
        if (!h[z].data != !h[2 + z].data) return not_plain();
    if (!a.like || !a.others(r, args + 4)) return not_plain();
    const double eps = r.number(args[9]);
    const bool pairs = r.truth(args[10]);
    void* stream;
    if (!r.ok || !stream_of(args[11], *a.like, &stream)) return not_plain();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = g_rope(&h[0], &h[1], &h[2], &h[3], data(a.w[0]), data(a.w[1]), a.f32, (const float*)data(a.cos), (const float*)data(a.sin),
                (const int*)data(a.positions), (int)a.cos->size(0), (float)eps, pairs, a.B, a.N, a.heads[0], a.heads[1], a.d, a.dt, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

// qk_norm_rope_bwd(dq_out, dk_out, q, k, dq, dk, cos, sin, positions, q_weight, k_weight, dq_weight, dk_weight, eps, interleaved, workspace, stream),
// without a workspace of the caller's: one is left to Python.
PyObject* norm_rope_bwd(PyObject* const* args, Py_ssize_t nargs) {
    if (nargs != 17 || !g_rope_bwd || args[15] != Py_None) return not_plain();
    Reader r(args[6]);
    RopeArgs a;
    qk_heads h[6];
    for (int i : {0, 1, 4, 5})
        if (!a.heads_of(r, args[i], i % 2, &h[i])) return not_plain();
    for (int z = 0; z < 2; ++z) {
        if (!h[z].data != !h[4 + z].data || (args[9 + z] != Py_None && !h[z].data) || (args[9 + z] == Py_None) != (args[11 + z] == Py_None)) return not_plain();
        h[2 + z] = {nullptr, 0, 0, 0};
        if (args[9 + z] != Py_None && (args[2 + z] == Py_None || !a.heads_of(r, args[2 + z], z, &h[2 + z]))) return not_plain();
    }
    if (!a.like || !a.others(r, args + 6)) return not_plain();
    const at::Tensor* dw[2] = {r.whole_or_none(args[11], 1, at::kFloat), r.whole_or_none(args[12], 1, at::kFloat)};
    for (int z = 0; z < 2; ++z)
        if (r.ok && dw[z] && dw[z]->size(0) != a.d) return not_plain();
    const double eps = r.number(args[13]);
    const bool pairs = r.truth(args[14]);
    void* stream;
    if (!r.ok || !stream_of(args[16], *a.like, &stream)) return not_plain();
    const long long need = a.w[0] || a.w[1] ? g_rope_bwd_workspace(a.B, a.N, a.heads[0], a.heads[1], a.d) : 0;
    if (need < 0) return PyLong_FromLong(need);
    long rc = kNotPlain;
    Py_BEGIN_ALLOW_THREADS
    {
        Workspace own(stream, r.device, true);
        void* ws = need ? own.take(need) : nullptr;
        if (ws || !need)
            rc = g_rope_bwd(&h[0], &h[1], &h[2], &h[3], &h[4], &h[5], data(a.w[0]), data(a.w[1]), a.f32, (float*)data(dw[0]), (float*)data(dw[1]),
                            (const float*)data(a.cos), (const float*)data(a.sin), (const int*)data(a.positions), (int)a.cos->size(0), (float)eps, pairs,
                            a.B, a.N, a.heads[0], a.heads[1], a.d, a.dt, ws, need, stream);
    }
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

// memory_of_a_pool(address): whether torch's allocator has it in a pool other than the common one
PyObject* memory_of_a_pool(PyObject* const* args, Py_ssize_t nargs) {
    if (nargs != 1) return not_plain();
    return PyBool_FromLong(in_private_pool(PyLong_AsVoidPtr(args[0])));
}

// bind_cached(addresses of kv4_append, kv4_read, kv4_attn, kv4_attn_workspace, qk_norm_rope, qk_norm_rope_bwd and qk_norm_rope_bwd_workspace)
PyObject* bind_cached(PyObject*, PyObject* args) {
    unsigned long long f[7];
    if (!PyArg_ParseTuple(args, "KKKKKKK", &f[0], &f[1], &f[2], &f[3], &f[4], &f[5], &f[6])) return nullptr;
    g_kv4_append = (decltype(g_kv4_append))f[0], g_kv4_read = (decltype(g_kv4_read))f[1], g_kv4_attn = (decltype(g_kv4_attn))f[2];
    g_kv4_attn_workspace = (decltype(g_kv4_attn_workspace))f[3], g_rope = (decltype(g_rope))f[4], g_rope_bwd = (decltype(g_rope_bwd))f[5];
    g_rope_bwd_workspace = (decltype(g_rope_bwd_workspace))f[6];
    Py_RETURN_NONE;
}

// bind(addresses of the library's attn_fwd, gemm_lrelu_with and gemm_lrelu_capturing)
PyObject* bind(PyObject*, PyObject* args) {
    unsigned long long attn = 0, gemm = 0, capturing = 0;
    if (!PyArg_ParseTuple(args, "KKK", &attn, &gemm, &capturing)) return nullptr;
    g_attn = (AttnFn)attn;
    g_capturing = (CapturingFn)capturing;
    g_gemm = (GemmFn)gemm;
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {{"attn_fwd", (PyCFunction)(void (*)(void))guarded<attn_fwd>, METH_FASTCALL, "0, a library error, or NOT_PLAIN"},
                         {"gemm_lrelu", (PyCFunction)(void (*)(void))guarded<gemm_lrelu>, METH_FASTCALL, "0, a library error, or NOT_PLAIN"},
                         {"kv4_append", (PyCFunction)(void (*)(void))guarded<append>, METH_FASTCALL, "0, a library error, or NOT_PLAIN"},
                         {"kv4_read", (PyCFunction)(void (*)(void))guarded<read>, METH_FASTCALL, "0, a library error, or NOT_PLAIN"},
                         {"kv4_attn", (PyCFunction)(void (*)(void))guarded<cached_attn>, METH_FASTCALL, "0, a library error, or NOT_PLAIN"},
                         {"qk_norm_rope", (PyCFunction)(void (*)(void))guarded<norm_rope>, METH_FASTCALL, "0, a library error, or NOT_PLAIN"},
                         {"qk_norm_rope_bwd", (PyCFunction)(void (*)(void))guarded<norm_rope_bwd>, METH_FASTCALL, "0, a library error, or NOT_PLAIN"},
                         {"memory_of_a_pool", (PyCFunction)(void (*)(void))guarded<memory_of_a_pool>, METH_FASTCALL, "whether an address is a private pool's"},
                         {"bind_cached", bind_cached, METH_VARARGS, "addresses of the library's entry points"},
                         {"bind", bind, METH_VARARGS, "addresses of the library's entry points"},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native() {
    PyObject* m = PyModule_Create(&module);
    if (m && PyModule_AddIntConstant(m, "NOT_PLAIN", kNotPlain) < 0) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
