// The Python entry points' fast path (module _pqnative): checks and marshals tensors and enqueues through the C ABI.
//
// A scoring step over a small catalogue takes the GPU some 10 us; marshalled in Python (ctypes, torch.cuda.current_stream(),
// torch.empty(): about 2 us apiece) the same step took 28 us, most of it the interpreter.  Here a call costs well under a
// microsecond beside its kernel launches (about 3 us each in the HIP runtime).  No computation and no policy: whatever
// does not fit a function's plain case (a tensor that is not on the current device, of another type, not contiguous, a
// shape that disagrees) is answered with None, and binding.py's own code reports it.
#include <Python.h>

#include <limits.h>

#include <ATen/core/Tensor.h>
#include <ATen/hip/EmptyTensor.h>
#include <c10/core/Allocator.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "pqtopk.h"
#include "pqtopk_train.h"
#include "pqtopk_probs.h"

namespace {

PyObject* none() { Py_RETURN_NONE; }

// A contiguous tensor of that type on the current device, else nullptr.
const at::Tensor* plain(PyObject* o, at::ScalarType type, int device) {
    if (!THPVariable_Check(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.get_device() != device || t.scalar_type() != type || !t.is_contiguous()) return nullptr;
    return &t;
}

at::Tensor empty(at::IntArrayRef size, at::ScalarType type, int device) {
    return at::detail::empty_cuda(size, type, c10::Device(c10::DeviceType::CUDA, (c10::DeviceIndex)device), c10::nullopt);
}

void* current_stream() { return static_cast<void*>(c10::hip::getCurrentHIPStream().stream()); }

// The interpreter is free for other threads while the HIP runtime enqueues (it blocks when its queue is full).
template <typename F>
int without_gil(F&& f) {
    PyThreadState* t = PyEval_SaveThread();
    const int rc = f();
    PyEval_RestoreThread(t);
    return rc;
}

template <typename F>
PyObject* guarded(F&& f) {
    try {
        return f();
    } catch (const std::exception& e) {                       // (out of memory, mostly: torch's own words)
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// subitem_scores(queries, centroids, out | None) -> S, an error code (int), or None
PyObject* subitem_scores(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (n != 3) return none();
        const int device = c10::hip::current_device();
        const at::Tensor *q = plain(args[0], at::kFloat, device), *c = plain(args[1], at::kFloat, device);
        if (!q || !c || q->dim() != 2 || c->dim() != 3) return none();
        const int64_t B = q->size(0), d = q->size(1), m = c->size(0), b = c->size(1);
        if (m * c->size(2) != d) return none();
        PyObject* result = args[2];
        at::Tensor made;
        const at::Tensor* S;
        if (result == Py_None) {
            made = empty({B, m, b}, at::kFloat, device);
            S = &made;
            result = nullptr;
        } else {
            S = plain(result, at::kFloat, device);
            if (!S) return none();
        }
        const float *phi = q->const_data_ptr<float>(), *psi = c->const_data_ptr<float>();
        float* out = S->mutable_data_ptr<float>();
        void* st = current_stream();
        const int rc = without_gil([&]() { return pq_subitem_scores(phi, psi, out, (int)B, (int)d, (int)m, (int)b, st); });
        if (rc != PQ_OK) return PyLong_FromLong(rc);
        if (result) { Py_INCREF(result); return result; }
        return THPVariable_Wrap(std::move(made));
    });
}

// Outputs and workspace of a TopK call: the caller's, or made here.  The workspace made here is given back to torch's
// allocator when the call has been enqueued: memory freed on a stream is only handed out again behind the work enqueued there.
struct TopKBuffers {
    at::Tensor made_ids, made_scores;
    c10::DataPtr made_ws;
    const at::Tensor *ids = nullptr, *scores = nullptr;
    void* ws = nullptr;
    size_t ws_bytes = 0;

    template <typename Need>
    bool set(PyObject* ws_o, PyObject* ids_o, PyObject* scores_o, int64_t B, int64_t K, int device, Need&& need) {
        if (ids_o != Py_None && !(ids = plain(ids_o, at::kInt, device))) return false;
        if (scores_o != Py_None && !(scores = plain(scores_o, at::kFloat, device))) return false;
        if (ws_o != Py_None) {
            if (!THPVariable_Check(ws_o)) return false;
            const at::Tensor& t = THPVariable_Unpack(ws_o);
            ws = t.mutable_data_ptr();
            ws_bytes = (size_t)t.numel();
        } else {
            ws_bytes = need();
            if (ws_bytes < 16) ws_bytes = 16;
            made_ws = c10::GetAllocator(c10::DeviceType::CUDA)->allocate(ws_bytes);
            ws = made_ws.get();
        }
        if (!ids) { made_ids = empty({B, K}, at::kInt, device); ids = &made_ids; }
        if (!scores) { made_scores = empty({B, K}, at::kFloat, device); scores = &made_scores; }
        return true;
    }
    PyObject* result(PyObject* ids_o, PyObject* scores_o) {
        PyObject* i = ids_o != Py_None ? (Py_INCREF(ids_o), ids_o) : THPVariable_Wrap(std::move(made_ids));
        PyObject* s = scores_o != Py_None ? (Py_INCREF(scores_o), scores_o) : THPVariable_Wrap(std::move(made_scores));
        PyObject* r = PyTuple_New(2);
        PyTuple_SET_ITEM(r, 0, i);
        PyTuple_SET_ITEM(r, 1, s);
        return r;
    }
};

bool as_int(PyObject* o, int64_t* out) {
    if (!PyLong_Check(o)) return false;
    *out = PyLong_AsLongLong(o);
    if (*out == -1 && PyErr_Occurred()) { PyErr_Clear(); return false; }
    return *out >= 1 && *out <= PQ_MAX_K;                     // (anything else: the Python code's business)
}

// score_topk(codes, S, K, workspace | None, out_ids | None, out_scores | None) -> (ids, scores), an error code, or None
template <bool WIDE>
PyObject* score_topk(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        int64_t K;
        if (n != 6 || !as_int(args[2], &K)) return none();
        const int device = c10::hip::current_device();
        const at::Tensor *g = plain(args[0], WIDE ? at::kUInt16 : at::kByte, device), *S = plain(args[1], at::kFloat, device);
        if (!g || !S || g->dim() != 2 || S->dim() != 3) return none();
        const int64_t N = g->size(0), m = g->size(1), B = S->size(0), b = S->size(2);
        if (S->size(1) != m) return none();
        TopKBuffers io;
        auto need = [&]() { return WIDE ? pq_score_topk_u16_workspace_bytes(N, (int)B, (int)m, (int)b, (int)K)
                                        : pq_score_topk_workspace_bytes(N, (int)B, (int)m, (int)b, (int)K); };
        if (!io.set(args[3], args[4], args[5], B, K, device, need)) return none();
        int* ids = io.ids->mutable_data_ptr<int>();
        float *scores = io.scores->mutable_data_ptr<float>();
        const float* s = S->const_data_ptr<float>();
        const void* codes = g->const_data_ptr();
        void* st = current_stream();
        const int rc = without_gil([&]() {
            return WIDE ? pq_score_topk_u16(static_cast<const uint16_t*>(codes), s, N, (int)B, (int)m, (int)b, (int)K, ids, scores, io.ws,
                                            io.ws_bytes, st)
                        : pq_score_topk(static_cast<const uint8_t*>(codes), s, N, (int)B, (int)m, (int)b, (int)K, ids, scores, io.ws,
                                        io.ws_bytes, st);
        });
        if (rc != PQ_OK) return PyLong_FromLong(rc);
        return io.result(args[4], args[5]);
    });
}

// score_topk_subset(codes, S, subset, K, workspace | None, out_ids | None, out_scores | None) -> as score_topk
PyObject* score_topk_subset(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        int64_t K;
        if (n != 7 || !as_int(args[3], &K)) return none();
        const int device = c10::hip::current_device();
        const at::Tensor *g = plain(args[0], at::kByte, device), *S = plain(args[1], at::kFloat, device), *v = plain(args[2], at::kInt, device);
        if (!g || !S || !v || g->dim() != 2 || S->dim() != 3 || v->dim() != 1) return none();
        const int64_t N = g->size(0), m = g->size(1), B = S->size(0), b = S->size(2), nv = v->size(0);
        if (S->size(1) != m) return none();
        TopKBuffers io;
        if (!io.set(args[4], args[5], args[6], B, K, device,
                    [&]() { return pq_score_topk_subset_workspace_bytes(nv, (int)B, (int)m, (int)b, (int)K); }))
            return none();
        const uint8_t* codes = g->const_data_ptr<uint8_t>();
        const float* s = S->const_data_ptr<float>();
        const int* list = v->const_data_ptr<int>();
        int* ids = io.ids->mutable_data_ptr<int>();
        float* scores = io.scores->mutable_data_ptr<float>();
        void* st = current_stream();
        const int rc = without_gil([&]() {
            return pq_score_topk_subset(codes, s, list, nv, N, (int)B, (int)m, (int)b, (int)K, ids, scores, io.ws, io.ws_bytes, st);
        });
        if (rc != PQ_OK) return PyLong_FromLong(rc);
        return io.result(args[5], args[6]);
    });
}

// ---- the scoring head's training and its four-bit form

// A size as the C ABI takes it.  One that no int holds becomes the largest, which every call rejects: cut off it might be a valid one.
int narrow(int64_t n) { return n > INT_MAX ? INT_MAX : (int)n; }

// An output of a call: the caller's tensor, checked, or one made here; bad: there is one and it does not fit.
struct Output {
    PyObject* given = nullptr;
    at::Tensor made;
    const at::Tensor* t = nullptr;
    bool bad = false;

    Output(PyObject* o, at::IntArrayRef size, at::ScalarType type, int device) {
        if (o == Py_None) {
            made = empty(size, type, device);
            t = &made;
        } else {
            t = plain(o, type, device);
            given = o;
            bad = !t || t->sizes() != size;
        }
    }
    float* floats() { return t->mutable_data_ptr<float>(); }
    PyObject* object() {
        if (!given) return THPVariable_Wrap(std::move(made));
        Py_INCREF(given);
        return given;
    }
};

PyObject* pair(Output& a, Output& b) {
    PyObject* r = PyTuple_New(2);
    if (!r) return nullptr;
    PyTuple_SET_ITEM(r, 0, a.object());
    PyTuple_SET_ITEM(r, 1, b.object());
    return r;
}

// A call's scratch: the caller's uint8 tensor, or memory given back to torch's allocator when the call has been enqueued.
struct Scratch {
    c10::DataPtr made;
    void* p = nullptr;
    size_t bytes = 0;
    bool bad = false;

    Scratch(PyObject* o, size_t need, int device) {
        if (o == Py_None) {
            bytes = need < 16 ? 16 : need;
            made = c10::GetAllocator(c10::DeviceType::CUDA)->allocate(bytes);
            p = made.get();
        } else {
            const at::Tensor* t = plain(o, at::kByte, device);
            bad = !t;
            if (t) { p = t->mutable_data_ptr(); bytes = (size_t)t->numel(); }
        }
    }
};

bool vector_of(const at::Tensor* t, int64_t n) { return t && t->dim() == 1 && t->size(0) == n; }

// cross_entropy(codes, S, targets, workspace | None, loss | None, lse | None) -> (loss, lse), an error code, or None
template <bool WIDE>
PyObject* cross_entropy(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (n != 6) return none();
        const int device = c10::hip::current_device();
        const at::Tensor *g = plain(args[0], WIDE ? at::kUInt16 : at::kByte, device), *S = plain(args[1], at::kFloat, device), *t = plain(args[2], at::kInt, device);
        if (!g || !S || g->dim() != 2 || S->dim() != 3 || S->size(1) != g->size(1) || !vector_of(t, S->size(0))) return none();
        const int64_t N = g->size(0), m = g->size(1), B = S->size(0), b = S->size(2);
        Output loss(args[4], {B}, at::kFloat, device), lse(args[5], {B}, at::kFloat, device);
        Scratch ws(args[3], WIDE ? pq_cross_entropy_u16_workspace_bytes(N, narrow(B), narrow(m), narrow(b)) : pq_cross_entropy_workspace_bytes(N, narrow(B), narrow(m), narrow(b)), device);
        if (loss.bad || lse.bad || ws.bad) return none();
        const void* codes = g->const_data_ptr();
        const float* s = S->const_data_ptr<float>();
        const int* targets = t->const_data_ptr<int>();
        float *l = loss.floats(), *e = lse.floats();
        void* st = current_stream();
        const int rc = without_gil([&]() {
            return WIDE ? pq_cross_entropy_u16(static_cast<const uint16_t*>(codes), s, targets, N, narrow(B), narrow(m), narrow(b), l, e, ws.p, ws.bytes, st)
                        : pq_cross_entropy(static_cast<const uint8_t*>(codes), s, targets, N, narrow(B), narrow(m), narrow(b), l, e, ws.p, ws.bytes, st);
        });
        return rc != PQ_OK ? PyLong_FromLong(rc) : pair(loss, lse);
    });
}

// cross_entropy_backward(codes, S, targets, lse, grad_loss, workspace | None, out | None) -> dS, an error code, or None
template <bool WIDE>
PyObject* cross_entropy_backward(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (n != 7) return none();
        const int device = c10::hip::current_device();
        const at::Tensor *g = plain(args[0], WIDE ? at::kUInt16 : at::kByte, device), *S = plain(args[1], at::kFloat, device), *t = plain(args[2], at::kInt, device);
        const at::Tensor *e = plain(args[3], at::kFloat, device), *w = plain(args[4], at::kFloat, device);
        if (!g || !S || g->dim() != 2 || S->dim() != 3 || S->size(1) != g->size(1)) return none();
        const int64_t N = g->size(0), m = g->size(1), B = S->size(0), b = S->size(2);
        if (!vector_of(t, B) || !vector_of(e, B) || !vector_of(w, B)) return none();
        Output dS(args[6], S->sizes(), at::kFloat, device);
        Scratch ws(args[5], WIDE ? pq_cross_entropy_u16_backward_workspace_bytes(N, narrow(B), narrow(m), narrow(b)) : pq_cross_entropy_backward_workspace_bytes(N, narrow(B), narrow(m), narrow(b)), device);
        if (dS.bad || ws.bad) return none();
        const void* codes = g->const_data_ptr();
        const float *s = S->const_data_ptr<float>(), *lse = e->const_data_ptr<float>(), *grad = w->const_data_ptr<float>();
        const int* targets = t->const_data_ptr<int>();
        float* out = dS.floats();
        void* st = current_stream();
        const int rc = without_gil([&]() {
            return WIDE ? pq_cross_entropy_u16_backward(static_cast<const uint16_t*>(codes), s, targets, lse, grad, N, narrow(B), narrow(m), narrow(b), out, ws.p, ws.bytes, st)
                        : pq_cross_entropy_backward(static_cast<const uint8_t*>(codes), s, targets, lse, grad, N, narrow(B), narrow(m), narrow(b), out, ws.p, ws.bytes, st);
        });
        return rc != PQ_OK ? PyLong_FromLong(rc) : dS.object();
    });
}

// subitem_scores_backward(dS, queries, centroids, workspace | None, dqueries | None, dcentroids | None) -> (dqueries, dcentroids), an error code, or None
PyObject* subitem_scores_backward(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (n != 6) return none();
        const int device = c10::hip::current_device();
        const at::Tensor *g = plain(args[0], at::kFloat, device), *q = plain(args[1], at::kFloat, device), *c = plain(args[2], at::kFloat, device);
        if (!g || !q || !c || g->dim() != 3 || q->dim() != 2 || c->dim() != 3) return none();
        const int64_t B = q->size(0), d = q->size(1), m = c->size(0), b = c->size(1);
        if (m * c->size(2) != d || g->size(0) != B || g->size(1) != m || g->size(2) != b) return none();
        Output dq(args[4], q->sizes(), at::kFloat, device), dc(args[5], c->sizes(), at::kFloat, device);
        Scratch ws(args[3], pq_subitem_scores_backward_workspace_bytes(narrow(B), narrow(d), narrow(m), narrow(b)), device);
        if (dq.bad || dc.bad || ws.bad) return none();
        const float *dS = g->const_data_ptr<float>(), *phi = q->const_data_ptr<float>(), *psi = c->const_data_ptr<float>();
        float *dphi = dq.floats(), *dpsi = dc.floats();
        void* st = current_stream();
        const int rc = without_gil([&]() { return pq_subitem_scores_backward(dS, phi, psi, dphi, dpsi, narrow(B), narrow(d), narrow(m), narrow(b), ws.p, ws.bytes, st); });
        return rc != PQ_OK ? PyLong_FromLong(rc) : pair(dq, dc);
    });
}

// W and queries of one type; its number in the C ABI, or -1
int dense_type(const at::Tensor& W) {
    return W.scalar_type() == at::kFloat ? PQ_FLOAT32 : W.scalar_type() == at::kBFloat16 ? PQ_BFLOAT16 : W.scalar_type() == at::kHalf ? PQ_FLOAT16 : -1;
}

// default_cross_entropy(W, queries, targets, workspace | None, loss | None, lse | None) -> (loss, lse), an error code, or None
PyObject* default_cross_entropy(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (n != 6 || !THPVariable_Check(args[0])) return none();
        const int device = c10::hip::current_device();
        const int type = dense_type(THPVariable_Unpack(args[0]));
        if (type < 0) return none();
        const at::ScalarType scalar = THPVariable_Unpack(args[0]).scalar_type();
        const at::Tensor *W = plain(args[0], scalar, device), *q = plain(args[1], scalar, device), *t = plain(args[2], at::kInt, device);
        if (!W || !q || W->dim() != 2 || q->dim() != 2 || W->size(1) != q->size(1) || !vector_of(t, q->size(0))) return none();
        const int64_t N = W->size(0), d = W->size(1), B = q->size(0);
        Output loss(args[4], {B}, at::kFloat, device), lse(args[5], {B}, at::kFloat, device);
        Scratch ws(args[3], pq_default_cross_entropy_workspace_bytes(N, narrow(B), narrow(d), type), device);
        if (loss.bad || lse.bad || ws.bad) return none();
        const void *w = W->const_data_ptr(), *h = q->const_data_ptr();
        const int* targets = t->const_data_ptr<int>();
        float *l = loss.floats(), *e = lse.floats();
        void* st = current_stream();
        const int rc = without_gil([&]() { return pq_default_cross_entropy(w, h, targets, N, narrow(B), narrow(d), type, l, e, ws.p, ws.bytes, st); });
        return rc != PQ_OK ? PyLong_FromLong(rc) : pair(loss, lse);
    });
}

// default_cross_entropy_backward(W, queries, targets, lse, grad_loss, workspace | None, dqueries | None, dW | None)
// -> (dqueries, dW), an error code, or None
PyObject* default_cross_entropy_backward(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (n != 8 || !THPVariable_Check(args[0])) return none();
        const int device = c10::hip::current_device();
        const int type = dense_type(THPVariable_Unpack(args[0]));
        if (type < 0) return none();
        const at::ScalarType scalar = THPVariable_Unpack(args[0]).scalar_type();
        const at::Tensor *W = plain(args[0], scalar, device), *q = plain(args[1], scalar, device), *t = plain(args[2], at::kInt, device);
        const at::Tensor *e = plain(args[3], at::kFloat, device), *g = plain(args[4], at::kFloat, device);
        if (!W || !q || W->dim() != 2 || q->dim() != 2 || W->size(1) != q->size(1)) return none();
        const int64_t N = W->size(0), d = W->size(1), B = q->size(0);
        if (!vector_of(t, B) || !vector_of(e, B) || !vector_of(g, B)) return none();
        Output dq(args[6], q->sizes(), scalar, device), dW(args[7], W->sizes(), scalar, device);
        Scratch ws(args[5], pq_default_cross_entropy_backward_workspace_bytes(N, narrow(B), narrow(d), type), device);
        if (dq.bad || dW.bad || ws.bad) return none();
        const void *w = W->const_data_ptr(), *h = q->const_data_ptr();
        const int* targets = t->const_data_ptr<int>();
        const float *lse = e->const_data_ptr<float>(), *grad = g->const_data_ptr<float>();
        void *out_h = dq.t->mutable_data_ptr(), *out_w = dW.t->mutable_data_ptr();
        void* st = current_stream();
        const int rc = without_gil([&]() {
            return pq_default_cross_entropy_backward(w, h, targets, lse, grad, N, narrow(B), narrow(d), type, out_h, out_w, ws.p, ws.bytes, st);
        });
        return rc != PQ_OK ? PyLong_FromLong(rc) : pair(dq, dW);
    });
}

// default_scores_q4(packed, scales, queries, out | None) -> scores, an error code, or None
PyObject* default_scores_q4(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (n != 4) return none();
        const int device = c10::hip::current_device();
        const at::Tensor *p = plain(args[0], at::kByte, device), *s = plain(args[1], at::kBFloat16, device), *q = plain(args[2], at::kFloat, device);
        if (!p || !s || !q || p->dim() != 2 || s->dim() != 2 || q->dim() != 2) return none();
        const int64_t N = p->size(0), B = q->size(0), d = q->size(1), groups = s->size(1);
        if (s->size(0) != N || p->size(1) * 2 != d || groups < 1 || d % groups != 0) return none();
        int64_t ld = (N + 3) / 4 * 4;
        if (args[3] != Py_None) {
            const at::Tensor* given = plain(args[3], at::kFloat, device);
            if (!given || given->dim() != 2) return none();
            ld = given->size(1);
        }
        Output out(args[3], {B, ld}, at::kFloat, device);
        if (out.bad) return none();
        const uint8_t* packed = p->const_data_ptr<uint8_t>();
        const uint16_t* scales = static_cast<const uint16_t*>(s->const_data_ptr());
        const float* phi = q->const_data_ptr<float>();
        float* scores = out.floats();
        void* st = current_stream();
        const int rc = without_gil([&]() { return pq_default_scores_q4(packed, scales, phi, N, narrow(B), narrow(d), narrow(d / groups), scores, ld, st); });
        return rc != PQ_OK ? PyLong_FromLong(rc) : out.object();
    });
}

// ---- Enqueue: an entry point with its arguments fixed; calling the object enqueues and returns `result`.  Base class of
// binding.py's Prepared classes, which keep the tensors alive and say what an error code means (`failed`).
enum Entry { kUnset, kSubitem, kTopK, kTopKU16, kTopKSubset };

struct Enqueue {
    PyObject_HEAD
    int entry;
    void *in0, *in1, *in2, *out0, *out1, *ws, *stream;
    long long N, n;
    size_t ws_bytes;
    int B, d, m, b, K;
    PyObject *result, *failed;
};

PyObject* enqueue_call(PyObject* self, PyObject*, PyObject*) {
    const Enqueue* e = reinterpret_cast<Enqueue*>(self);
    const int rc = without_gil([e]() -> int {
        const float* in1 = static_cast<const float*>(e->in1);
        int* ids = static_cast<int*>(e->out0);
        float* scores = static_cast<float*>(e->out1);
        switch (e->entry) {
            case kSubitem:
                return pq_subitem_scores(static_cast<const float*>(e->in0), in1, static_cast<float*>(e->out0), e->B, e->d, e->m, e->b, e->stream);
            case kTopK:
                return pq_score_topk(static_cast<const uint8_t*>(e->in0), in1, e->N, e->B, e->m, e->b, e->K, ids, scores, e->ws, e->ws_bytes,
                                     e->stream);
            case kTopKU16:
                return pq_score_topk_u16(static_cast<const uint16_t*>(e->in0), in1, e->N, e->B, e->m, e->b, e->K, ids, scores, e->ws,
                                         e->ws_bytes, e->stream);
            case kTopKSubset:
                return pq_score_topk_subset(static_cast<const uint8_t*>(e->in0), in1, static_cast<const int*>(e->in2), e->n, e->N, e->B, e->m,
                                            e->b, e->K, ids, scores, e->ws, e->ws_bytes, e->stream);
            default: return PQ_ERR_NULL;
        }
    });
    if (rc != PQ_OK) {
        if (e->failed) return PyObject_CallFunction(e->failed, "i", rc);
        PyErr_SetString(PyExc_RuntimeError, "called before it was prepared");
        return nullptr;
    }
    Py_INCREF(e->result);
    return e->result;
}

// _bind(entry, in0, in1, in2, n, N, B, d, m, b, K, out0, out1, ws, ws_bytes, stream, result, failed)
PyObject* enqueue_bind(PyObject* self, PyObject* args) {
    Enqueue* e = reinterpret_cast<Enqueue*>(self);
    int entry, B, d, m, b, K;
    unsigned long long in0, in1, in2, out0, out1, ws, ws_bytes, stream;
    long long n, N;
    PyObject *result, *failed;
    if (!PyArg_ParseTuple(args, "iKKKLLiiiiiKKKKKOO", &entry, &in0, &in1, &in2, &n, &N, &B, &d, &m, &b, &K, &out0, &out1, &ws, &ws_bytes,
                          &stream, &result, &failed))
        return nullptr;
    e->in0 = (void*)in0; e->in1 = (void*)in1; e->in2 = (void*)in2; e->out0 = (void*)out0; e->out1 = (void*)out1;
    e->ws = (void*)ws; e->ws_bytes = (size_t)ws_bytes; e->stream = (void*)stream;
    e->n = n; e->N = N; e->B = B; e->d = d; e->m = m; e->b = b; e->K = K;
    Py_INCREF(result);
    Py_INCREF(failed);
    Py_XSETREF(e->result, result);
    Py_XSETREF(e->failed, failed);
    e->entry = entry;
    Py_RETURN_NONE;
}

int enqueue_traverse(PyObject* self, visitproc visit, void* arg) {
    Enqueue* e = reinterpret_cast<Enqueue*>(self);
    Py_VISIT(e->result);
    Py_VISIT(e->failed);
    return 0;
}
int enqueue_clear(PyObject* self) {
    Enqueue* e = reinterpret_cast<Enqueue*>(self);
    e->entry = kUnset;
    Py_CLEAR(e->result);
    Py_CLEAR(e->failed);
    return 0;
}
void enqueue_dealloc(PyObject* self) {
    PyObject_GC_UnTrack(self);
    enqueue_clear(self);
    Py_TYPE(self)->tp_free(self);
}

// A call by sub-ids of one or two bytes (first: codes, second: S) or by the default scorer (W, queries): its sizes as the C ABI takes them.
enum Head { SUB_IDS, WIDE_SUB_IDS, DENSE };
struct HeadArgs {
    const at::Tensor *first = nullptr, *second = nullptr;
    int64_t N = 0, B = 0;
    int x = 0, y = 0;                                            // m, b or d, type
    const void *p = nullptr, *q = nullptr;

    template <Head H>
    bool set(PyObject* a, PyObject* b, int device) {
        if (H == DENSE) {
            if (!THPVariable_Check(a)) return false;
            const at::Tensor& W = THPVariable_Unpack(a);
            y = dense_type(W);
            if (y < 0 || !(first = plain(a, W.scalar_type(), device)) || !(second = plain(b, W.scalar_type(), device))) return false;
            if (first->dim() != 2 || second->dim() != 2 || first->size(1) != second->size(1)) return false;
            x = narrow(first->size(1));
        } else {
            first = plain(a, H == WIDE_SUB_IDS ? at::kUInt16 : at::kByte, device);
            second = plain(b, at::kFloat, device);
            if (!first || !second || first->dim() != 2 || second->dim() != 3 || second->size(1) != first->size(1)) return false;
            x = narrow(first->size(1));
            y = narrow(second->size(2));
        }
        N = first->size(0);
        B = second->size(0);
        p = first->const_data_ptr();
        q = second->const_data_ptr();
        return true;
    }
    const uint8_t* codes() const { return static_cast<const uint8_t*>(p); }
    const uint16_t* wide_codes() const { return static_cast<const uint16_t*>(p); }
    const float* S() const { return static_cast<const float*>(q); }
};

bool rows_of(const at::Tensor* t, int64_t B) { return t && t->dim() == 2 && t->size(0) == B; }

// A number argument; false (and no error set) if it is none.
bool number(PyObject* o, float& x) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) { PyErr_Clear(); return false; }
    x = (float)v;
    return true;
}

// log_probs(first, second, items | None, K, temperature, workspace | None, log_probs | None, entropy | None, lse | None, top_items | None,
//           top_log_probs | None) -> (log_probs, entropy, lse, top_items, top_log_probs), an error code, or None
template <Head H>
PyObject* log_probs(PyObject*, PyObject* const* args, Py_ssize_t count) {
    return guarded([&]() -> PyObject* {
        if (count != 11) return none();
        const int device = c10::hip::current_device();
        HeadArgs a;
        if (!a.set<H>(args[0], args[1], device) || !PyLong_Check(args[3])) return none();
        const long long K = PyLong_AsLongLong(args[3]);
        if (K == -1 && PyErr_Occurred()) { PyErr_Clear(); return none(); }
        float T;
        if (K < 0 || K > INT_MAX || !number(args[4], T)) return none();
        const at::Tensor* items = nullptr;
        if (args[2] != Py_None && !rows_of(items = plain(args[2], at::kInt, device), a.B)) return none();
        const int64_t n = items ? items->size(1) : 0;
        const int B = narrow(a.B);
        Scratch ws(args[5], H == DENSE ? pq_default_log_probs_workspace_bytes(a.N, B, a.x, a.y, (int)K) : H == WIDE_SUB_IDS
                   ? pq_log_probs_u16_workspace_bytes(a.N, B, a.x, a.y, (int)K) : pq_log_probs_workspace_bytes(a.N, B, a.x, a.y, (int)K), device);
        Output lp(args[6], {a.B, n}, at::kFloat, device), entropy(args[7], {a.B}, at::kFloat, device), lse(args[8], {a.B}, at::kFloat, device);
        Output top(args[9], {a.B, (int64_t)K}, at::kInt, device), top_lp(args[10], {a.B, (int64_t)K}, at::kFloat, device);
        if (ws.bad || lp.bad || entropy.bad || lse.bad || top.bad || top_lp.bad) return none();
        const int* ids = items ? items->const_data_ptr<int>() : nullptr;
        float *l = lp.floats(), *h = entropy.floats(), *e = lse.floats(), *tl = top_lp.floats();
        int* ti = top.t->mutable_data_ptr<int>();
        void* st = current_stream();
        const int rc = without_gil([&]() {
            if (H == DENSE) return pq_default_log_probs(a.p, a.q, ids, a.N, B, a.x, a.y, narrow(n), (int)K, T, l, h, e, ti, tl, ws.p, ws.bytes, st);
            if (H == WIDE_SUB_IDS) return pq_log_probs_u16(a.wide_codes(), a.S(), ids, a.N, B, a.x, a.y, narrow(n), (int)K, T, l, h, e, ti, tl, ws.p, ws.bytes, st);
            return pq_log_probs(a.codes(), a.S(), ids, a.N, B, a.x, a.y, narrow(n), (int)K, T, l, h, e, ti, tl, ws.p, ws.bytes, st);
        });
        if (rc != PQ_OK) return PyLong_FromLong(rc);
        PyObject* r = PyTuple_New(5);
        if (!r) return nullptr;
        Output* outputs[5] = {&lp, &entropy, &lse, &top, &top_lp};
        for (int i = 0; i < 5; ++i) PyTuple_SET_ITEM(r, i, outputs[i]->object());
        return r;
    });
}

// distillation(first, second, teacher_items, teacher_scores, temperature, workspace | None, loss | None, lse | None) -> (loss, lse), an error code, or None
template <Head H>
PyObject* distillation(PyObject*, PyObject* const* args, Py_ssize_t count) {
    return guarded([&]() -> PyObject* {
        if (count != 8) return none();
        const int device = c10::hip::current_device();
        HeadArgs a;
        float T;
        if (!a.set<H>(args[0], args[1], device) || !number(args[4], T)) return none();
        const at::Tensor *items = plain(args[2], at::kInt, device), *scores = plain(args[3], at::kFloat, device);
        if (!rows_of(items, a.B) || !rows_of(scores, a.B) || items->size(1) != scores->size(1)) return none();
        const int B = narrow(a.B), K = narrow(items->size(1));
        Scratch ws(args[5], H == DENSE ? pq_default_distillation_workspace_bytes(a.N, B, a.x, a.y, K) : H == WIDE_SUB_IDS
                   ? pq_distillation_u16_workspace_bytes(a.N, B, a.x, a.y, K) : pq_distillation_workspace_bytes(a.N, B, a.x, a.y, K), device);
        Output loss(args[6], {a.B}, at::kFloat, device), lse(args[7], {a.B}, at::kFloat, device);
        if (ws.bad || loss.bad || lse.bad) return none();
        const int* ids = items->const_data_ptr<int>();
        const float* u = scores->const_data_ptr<float>();
        float *l = loss.floats(), *e = lse.floats();
        void* st = current_stream();
        const int rc = without_gil([&]() {
            if (H == DENSE) return pq_default_distillation(a.p, a.q, ids, u, a.N, B, a.x, a.y, K, T, l, e, ws.p, ws.bytes, st);
            if (H == WIDE_SUB_IDS) return pq_distillation_u16(a.wide_codes(), a.S(), ids, u, a.N, B, a.x, a.y, K, T, l, e, ws.p, ws.bytes, st);
            return pq_distillation(a.codes(), a.S(), ids, u, a.N, B, a.x, a.y, K, T, l, e, ws.p, ws.bytes, st);
        });
        return rc != PQ_OK ? PyLong_FromLong(rc) : pair(loss, lse);
    });
}

// distillation_backward(first, second, teacher_items, teacher_scores, lse, grad_loss, temperature, workspace | None, dS | None) -> dS, or with
// dqueries | None, dW | None at the end -> (dqueries, dW); an error code, or None
template <Head H>
PyObject* distillation_backward(PyObject*, PyObject* const* args, Py_ssize_t count) {
    return guarded([&]() -> PyObject* {
        if (count != (H == DENSE ? 10 : 9)) return none();
        const int device = c10::hip::current_device();
        HeadArgs a;
        float T;
        if (!a.set<H>(args[0], args[1], device) || !number(args[6], T)) return none();
        const at::Tensor *items = plain(args[2], at::kInt, device), *scores = plain(args[3], at::kFloat, device);
        const at::Tensor *e = plain(args[4], at::kFloat, device), *g = plain(args[5], at::kFloat, device);
        if (!rows_of(items, a.B) || !rows_of(scores, a.B) || items->size(1) != scores->size(1) || !vector_of(e, a.B) || !vector_of(g, a.B)) return none();
        const int B = narrow(a.B), K = narrow(items->size(1));
        Scratch ws(args[7], H == DENSE ? pq_default_distillation_backward_workspace_bytes(a.N, B, a.x, a.y, K) : H == WIDE_SUB_IDS
                   ? pq_distillation_u16_backward_workspace_bytes(a.N, B, a.x, a.y, K) : pq_distillation_backward_workspace_bytes(a.N, B, a.x, a.y, K), device);
        const int* ids = items->const_data_ptr<int>();
        const float *u = scores->const_data_ptr<float>(), *lse = e->const_data_ptr<float>(), *grad = g->const_data_ptr<float>();
        void* st = current_stream();
        Output one(args[8], a.second->sizes(), a.second->scalar_type(), device);                       // dS, or dqueries
        if (ws.bad || one.bad) return none();
        void* first_out = one.t->mutable_data_ptr();
        if (H == DENSE) {
            Output dW(args[9], a.first->sizes(), a.first->scalar_type(), device);
            if (dW.bad) return none();
            void* second_out = dW.t->mutable_data_ptr();
            const int rc = without_gil([&]() {
                return pq_default_distillation_backward(a.p, a.q, ids, u, lse, grad, a.N, B, a.x, a.y, K, T, first_out, second_out, ws.p, ws.bytes, st);
            });
            return rc != PQ_OK ? PyLong_FromLong(rc) : pair(one, dW);
        }
        float* dS = static_cast<float*>(first_out);
        const int rc = without_gil([&]() {
            if (H == WIDE_SUB_IDS) return pq_distillation_u16_backward(a.wide_codes(), a.S(), ids, u, lse, grad, a.N, B, a.x, a.y, K, T, dS, ws.p, ws.bytes, st);
            return pq_distillation_backward(a.codes(), a.S(), ids, u, lse, grad, a.N, B, a.x, a.y, K, T, dS, ws.p, ws.bytes, st);
        });
        return rc != PQ_OK ? PyLong_FromLong(rc) : one.object();
    });
}

PyMethodDef enqueue_methods[] = {{"_bind", enqueue_bind, METH_VARARGS, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyTypeObject enqueue_type = {PyVarObject_HEAD_INIT(nullptr, 0) "_pqnative.Enqueue"};

PyMethodDef functions[] = {
    {"subitem_scores", (PyCFunction)(void (*)(void))subitem_scores, METH_FASTCALL, nullptr},
    {"score_topk", (PyCFunction)(void (*)(void))score_topk<false>, METH_FASTCALL, nullptr},
    {"score_topk_u16", (PyCFunction)(void (*)(void))score_topk<true>, METH_FASTCALL, nullptr},
    {"score_topk_subset", (PyCFunction)(void (*)(void))score_topk_subset, METH_FASTCALL, nullptr},
    {"log_probs", (PyCFunction)(void (*)(void))log_probs<SUB_IDS>, METH_FASTCALL, nullptr},
    {"log_probs_u16", (PyCFunction)(void (*)(void))log_probs<WIDE_SUB_IDS>, METH_FASTCALL, nullptr},
    {"default_log_probs", (PyCFunction)(void (*)(void))log_probs<DENSE>, METH_FASTCALL, nullptr},
    {"distillation", (PyCFunction)(void (*)(void))distillation<SUB_IDS>, METH_FASTCALL, nullptr},
    {"distillation_u16", (PyCFunction)(void (*)(void))distillation<WIDE_SUB_IDS>, METH_FASTCALL, nullptr},
    {"default_distillation", (PyCFunction)(void (*)(void))distillation<DENSE>, METH_FASTCALL, nullptr},
    {"distillation_backward", (PyCFunction)(void (*)(void))distillation_backward<SUB_IDS>, METH_FASTCALL, nullptr},
    {"distillation_u16_backward", (PyCFunction)(void (*)(void))distillation_backward<WIDE_SUB_IDS>, METH_FASTCALL, nullptr},
    {"default_distillation_backward", (PyCFunction)(void (*)(void))distillation_backward<DENSE>, METH_FASTCALL, nullptr},
    {"cross_entropy", (PyCFunction)(void (*)(void))cross_entropy<false>, METH_FASTCALL, nullptr},
    {"cross_entropy_u16", (PyCFunction)(void (*)(void))cross_entropy<true>, METH_FASTCALL, nullptr},
    {"cross_entropy_backward", (PyCFunction)(void (*)(void))cross_entropy_backward<false>, METH_FASTCALL, nullptr},
    {"cross_entropy_u16_backward", (PyCFunction)(void (*)(void))cross_entropy_backward<true>, METH_FASTCALL, nullptr},
    {"subitem_scores_backward", (PyCFunction)(void (*)(void))subitem_scores_backward, METH_FASTCALL, nullptr},
    {"default_cross_entropy", (PyCFunction)(void (*)(void))default_cross_entropy, METH_FASTCALL, nullptr},
    {"default_cross_entropy_backward", (PyCFunction)(void (*)(void))default_cross_entropy_backward, METH_FASTCALL, nullptr},
    {"default_scores_q4", (PyCFunction)(void (*)(void))default_scores_q4, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_pqnative", nullptr, -1, functions, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__pqnative() {
    enqueue_type.tp_basicsize = sizeof(Enqueue);
    enqueue_type.tp_flags = Py_TPFLAGS_DEFAULT | Py_TPFLAGS_BASETYPE | Py_TPFLAGS_HAVE_GC;
    enqueue_type.tp_new = PyType_GenericNew;
    enqueue_type.tp_call = enqueue_call;
    enqueue_type.tp_methods = enqueue_methods;
    enqueue_type.tp_traverse = enqueue_traverse;
    enqueue_type.tp_clear = enqueue_clear;
    enqueue_type.tp_dealloc = enqueue_dealloc;
    if (PyType_Ready(&enqueue_type) < 0) return nullptr;
    PyObject* mod = PyModule_Create(&module);
    if (!mod) return nullptr;
    Py_INCREF(&enqueue_type);
    PyModule_AddObject(mod, "Enqueue", reinterpret_cast<PyObject*>(&enqueue_type));
    PyModule_AddIntConstant(mod, "SUBITEM", kSubitem);
    PyModule_AddIntConstant(mod, "TOPK", kTopK);
    PyModule_AddIntConstant(mod, "TOPK_U16", kTopKU16);
    PyModule_AddIntConstant(mod, "TOPK_SUBSET", kTopKSubset);
    return mod;
}
