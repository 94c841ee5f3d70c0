// The per-call path of the Python binding for the calls that a decoder makes
// once per frame (advance, fused_greedy_step, fused_topk, beam_step) or round
// (draft, verify, kv_append, attend, kv_fork, kv_copy, kv_compact): argument checks,
// output allocation and the C ABI call without interpreter work in between.
// Each function answers the ordinary call (plain contiguous device tensors,
// the current stream) and returns None for anything else, which the Python
// method then handles, and reports, by itself; a failing C call returns its
// code.  Everything that can fail otherwise, the results' Python objects among
// it, comes before the C call: after it the step has been enqueued, and None
// would make the Python method enqueue it a second time.
//
// An enqueued call cost the host 4.4 us (advance) to 9.9 us (top-k, three
// outputs allocated), more than the kernels of small batches take, and 2.4 us
// of it are the launch: 3.1 us and 6.0 us here.
#include <Python.h>

#include <ATen/ops/empty.h>
#include <c10/core/GradMode.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <cstdint>

#include "ngpu_lm.h"

namespace {

// The library's entry points, bound from the handle that the binding loaded.
decltype(&ngpu_lm_advance) g_advance;
decltype(&ngpu_lm_fused_greedy_step) g_step;
decltype(&ngpu_lm_fused_topk) g_topk;
decltype(&ngpu_lm_draft) g_draft;
decltype(&ngpu_lm_verify_workspace) g_verify_workspace;
decltype(&ngpu_lm_verify) g_verify;
decltype(&ngpu_lm_kv_append) g_kv_append;
decltype(&ngpu_lm_attend_workspace) g_attend_workspace;
decltype(&ngpu_lm_attend) g_attend;
decltype(&ngpu_lm_kv_append8) g_kv_append8;
decltype(&ngpu_lm_attend8_workspace) g_attend8_workspace;
decltype(&ngpu_lm_attend8) g_attend8;
decltype(&ngpu_lm_kv_copy) g_kv_copy;
decltype(&ngpu_lm_kv_copy8) g_kv_copy8;
decltype(&ngpu_lm_kv_fork_workspace) g_kv_fork_workspace;
decltype(&ngpu_lm_kv_fork) g_kv_fork;
decltype(&ngpu_lm_kv_compact_workspace) g_kv_compact_workspace;
decltype(&ngpu_lm_kv_compact) g_kv_compact;
decltype(&ngpu_lm_kv_move) g_kv_move;
decltype(&ngpu_lm_beam_step_workspace) g_beam_step_workspace;
decltype(&ngpu_lm_beam_step) g_beam_step;

PyObject *none() {
    PyErr_Clear();   // the Python method meets the error again, or does not
    Py_RETURN_NONE;
}

struct Ref {   // an owned reference
    PyObject *p = nullptr;
    Ref() = default;
    explicit Ref(PyObject *o) : p(o) {}
    Ref(const Ref &) = delete;
    ~Ref() { Py_XDECREF(p); }
    PyObject *release() {
        PyObject *o = p;
        p = nullptr;
        return o;
    }
};

const at::Tensor *tensor_of(PyObject *o, at::ScalarType type) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    return t.scalar_type() == type && t.layout() == at::kStrided && t.is_cuda() ? &t : nullptr;
}
const at::Tensor *dense(PyObject *o, at::ScalarType type) {
    const at::Tensor *t = tensor_of(o, type);
    return t && t->is_contiguous() ? t : nullptr;
}

// An output: the caller's contiguous tensor of at least n entries, or a new one.
struct Output {
    Ref object;
    at::Tensor t;
    bool set(PyObject *o, at::ScalarType type, int64_t n, at::IntArrayRef shape, const at::Tensor &like) {
        if (o == Py_None) {
            t = at::empty(shape, like.options().dtype(type));
            object.p = THPVariable_Wrap(t);
            return object.p && t.is_contiguous();
        }
        const at::Tensor *x = dense(o, type);
        if (!x || x->numel() < n) return false;
        Py_INCREF(o);
        object.p = o;
        t = *x;
        return true;
    }
};

bool whole(PyObject *o, int64_t &v) {   // an int (no conversion that could run user code)
    if (!PyLong_CheckExact(o)) return false;
    int overflow = 0;
    v = PyLong_AsLongLongAndOverflow(o, &overflow);
    return overflow == 0;
}
bool real(PyObject *o, float &v) {
    if (!PyFloat_CheckExact(o)) return false;
    v = static_cast<float>(PyFloat_AS_DOUBLE(o));
    return true;
}

template <class F>
int without_gil(F f) {
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f();
    Py_END_ALLOW_THREADS
    return rc;
}

void *current_stream() { return c10::hip::getCurrentHIPStream().stream(); }

// advance(handle, V, states, scores or None, next or None)
PyObject *advance(PyObject *, PyObject *const *a, Py_ssize_t n) try {
    int64_t h, V;
    if (n != 5 || !whole(a[0], h) || !whole(a[1], V)) return none();
    const at::Tensor *states = dense(a[2], at::kInt);
    if (!states) return none();
    const int64_t B = states->numel();
    Output scores, next;
    if (!scores.set(a[3], at::kFloat, B * V, {B, V}, *states) || !next.set(a[4], at::kInt, B * V, {B, V}, *states))
        return none();
    const auto *st = static_cast<const int32_t *>(states->data_ptr());
    auto *sc = static_cast<float *>(scores.t.data_ptr());
    auto *nx = static_cast<int32_t *>(next.t.data_ptr());
    Ref result(PyTuple_Pack(2, scores.object.p, next.object.p));
    if (!result.p) return none();
    void *stream = current_stream();
    const int rc = without_gil([&] { return g_advance(reinterpret_cast<const ngpu_lm *>(h), st, B, sc, nx, stream); });
    return rc != NGPU_OK ? PyLong_FromLong(rc) : result.release();
} catch (const std::exception &) {
    return none();   // nothing was enqueued: the C call, and what follows it, throws nothing
}

// step(handle, V, asr, lam, states, prev or None, mode, tokens or None)
PyObject *step(PyObject *, PyObject *const *a, Py_ssize_t n) try {
    int64_t h, V, mode;
    float lam;
    if (n != 8 || !whole(a[0], h) || !whole(a[1], V) || !real(a[3], lam) || !whole(a[6], mode) || mode < 0 || mode > 3)
        return none();
    const at::Tensor *asr = tensor_of(a[2], at::kFloat), *states = dense(a[4], at::kInt);
    const at::Tensor *prev = a[5] == Py_None ? nullptr : dense(a[5], at::kInt);
    if (!asr || !states || (a[5] != Py_None && !prev) || asr->dim() != 2 || asr->stride(1) != 1) return none();
    const int64_t B = asr->size(0);
    if (asr->size(1) < V + (mode != NGPU_FUSION_PLAIN) || states->numel() != B || (prev && prev->numel() != B))
        return none();
    Output tokens;
    if (!tokens.set(a[7], at::kInt, B, {B}, *asr)) return none();
    const auto *row = static_cast<const float *>(asr->data_ptr());
    auto *st = static_cast<int32_t *>(states->data_ptr());
    auto *pv = prev ? static_cast<int32_t *>(prev->data_ptr()) : nullptr;
    auto *tk = static_cast<int32_t *>(tokens.t.data_ptr());
    const int64_t ld = asr->stride(0);
    void *stream = current_stream();
    const int rc = without_gil([&] {
        return g_step(reinterpret_cast<const ngpu_lm *>(h), row, B, ld, static_cast<int32_t>(mode), lam, st, pv, tk,
                      stream);
    });
    return rc != NGPU_OK ? PyLong_FromLong(rc) : tokens.object.release();
} catch (const std::exception &) {
    return none();
}

// topk(handle, V, asr, lam, k, states, tokens or None, scores or None, next or None)
PyObject *topk(PyObject *, PyObject *const *a, Py_ssize_t n) try {
    int64_t h, V, k;
    float lam;
    if (n != 9 || !whole(a[0], h) || !whole(a[1], V) || !real(a[3], lam) || !whole(a[4], k) || k < 1 ||
        k > NGPU_LM_MAX_TOPK)
        return none();
    const at::Tensor *asr = tensor_of(a[2], at::kFloat), *states = dense(a[5], at::kInt);
    if (!asr || !states || asr->dim() != 2 || asr->stride(1) != 1) return none();
    const int64_t B = asr->size(0);
    if (asr->size(1) < V || states->numel() != B) return none();
    Output tokens, scores, next;
    if (!tokens.set(a[6], at::kInt, B * k, {B, k}, *asr) || !scores.set(a[7], at::kFloat, B * k, {B, k}, *asr) ||
        !next.set(a[8], at::kInt, B * k, {B, k}, *asr))
        return none();
    const auto *row = static_cast<const float *>(asr->data_ptr());
    const auto *st = static_cast<const int32_t *>(states->data_ptr());
    auto *tk = static_cast<int32_t *>(tokens.t.data_ptr());
    auto *sc = static_cast<float *>(scores.t.data_ptr());
    auto *nx = static_cast<int32_t *>(next.t.data_ptr());
    const int64_t ld = asr->stride(0);
    Ref result(PyTuple_Pack(3, tokens.object.p, scores.object.p, next.object.p));
    if (!result.p) return none();
    void *stream = current_stream();
    const int rc = without_gil([&] {
        return g_topk(reinterpret_cast<const ngpu_lm *>(h), row, B, ld, lam, static_cast<int32_t>(k), st, tk, sc, nx,
                      stream);
    });
    return rc != NGPU_OK ? PyLong_FromLong(rc) : result.release();
} catch (const std::exception &) {
    return none();
}

// bind(addresses of ngpu_lm_advance, ngpu_lm_fused_greedy_step, ngpu_lm_fused_topk)
PyObject *bind(PyObject *, PyObject *const *a, Py_ssize_t n) {
    int64_t p[3];
    if (n != 3 || !whole(a[0], p[0]) || !whole(a[1], p[1]) || !whole(a[2], p[2])) {
        PyErr_SetString(PyExc_TypeError, "bind takes three addresses");
        return nullptr;
    }
    g_advance = reinterpret_cast<decltype(g_advance)>(p[0]);
    g_step = reinterpret_cast<decltype(g_step)>(p[1]);
    g_topk = reinterpret_cast<decltype(g_topk)>(p[2]);
    return none();
}

// ---- drafting, verification, cache append and attention

bool on_current_device(const at::Tensor &t) { return t.device().index() == c10::hip::current_device(); }

// Whether a call without a backward pass would lose a gradient (the Python function refuses it).
bool tracked(const at::Tensor *t) { return t && t->requires_grad() && c10::GradMode::is_enabled(); }

// A device tensor of this type and shape on `like`'s device, or None where it may
// be: with unit stride in its last dimension (rows) or contiguous.
struct Input {
    const at::Tensor *t = nullptr;
    bool set(PyObject *o, at::ScalarType type, at::IntArrayRef shape, const at::Tensor &like, bool rows,
             bool optional = false) {
        if (o == Py_None) return optional;
        const at::Tensor *x = tensor_of(o, type);
        if (!x || x->device() != like.device() || x->sizes() != shape) return false;
        if (!(rows ? shape.back() <= 1 || x->stride(-1) == 1 : x->is_contiguous())) return false;
        t = x;
        return true;
    }
    template <class T = void>
    T *ptr() const {
        return t ? static_cast<T *>(t->data_ptr()) : nullptr;
    }
    int64_t stride(int64_t i) const { return t ? t->stride(i) : 0; }
};

// A temperature; one that only rounds to 0, which is greedy, is left to the Python function, which refuses it.
bool temperature_of(PyObject *o, float &t) { return real(o, t) && (t != 0.0f || PyFloat_AS_DOUBLE(o) == 0.0); }

int32_t type_code(at::ScalarType t) {
    return t == at::kFloat ? NGPU_F32 : (t == at::kHalf ? NGPU_F16 : (t == at::kBFloat16 ? NGPU_BF16 : -1));
}
const at::Tensor *any_tensor(PyObject *o, int64_t dims) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    return t.layout() == at::kStrided && t.is_cuda() && t.dim() == dims && type_code(t.scalar_type()) >= 0 ? &t : nullptr;
}
at::Tensor scratch(size_t bytes, const at::Tensor &like) {
    return at::empty({int64_t(bytes)}, like.options().dtype(at::kByte));
}
PyObject *held(const at::Tensor &t) {   // a new reference, None for an undefined tensor
    if (!t.defined()) Py_RETURN_NONE;
    return THPVariable_Wrap(t);
}
PyObject *answer(int rc, Ref &result) { return rc != NGPU_OK ? PyLong_FromLong(rc) : result.release(); }

// draft(handle, V, states, k, noise or None, temperature, last or None)
PyObject *draft(PyObject *, PyObject *const *a, Py_ssize_t n) try {
    int64_t h, V, k;
    float temperature;
    if (n != 7 || !whole(a[0], h) || !whole(a[1], V) || !whole(a[3], k) || !temperature_of(a[5], temperature) || k < 1 ||
        k > NGPU_LM_MAX_DRAFT)
        return none();
    const at::Tensor *states = dense(a[2], at::kInt);
    if (!states || !on_current_device(*states)) return none();
    const int64_t B = states->numel();
    const bool sample = temperature != 0.0f;
    Input noise, last;
    if (sample && !noise.set(a[4], at::kFloat, {B, k, V}, *states, true)) return none();
    if (!last.set(a[6], at::kInt, {B}, *states, false, true)) return none();
    const auto ints = states->options();
    const at::Tensor tokens = at::empty({B, k}, ints), after = at::empty({B, k + 1}, ints);
    const at::Tensor rows = sample ? at::empty({B, k, V}, ints.dtype(at::kFloat)) : at::Tensor();
    Ref t(held(tokens)), s(held(after)), r(held(rows));
    if (!t.p || !s.p || !r.p) return none();
    Ref result(PyTuple_Pack(3, t.p, s.p, r.p));
    if (!result.p) return none();
    void *stream = current_stream();
    const int rc = without_gil([&] {
        return g_draft(reinterpret_cast<const ngpu_lm *>(h), states->const_data_ptr<int32_t>(), last.ptr<int32_t>(), B,
                       int32_t(k), temperature, noise.ptr<float>(), noise.stride(0), noise.stride(1),
                       tokens.data_ptr<int32_t>(), after.data_ptr<int32_t>(),
                       sample ? rows.data_ptr<float>() : nullptr, stream);
    });
    return answer(rc, result);
} catch (const std::exception &) {
    return none();
}

// verify(logits, tokens, logprobs, uniforms, noise, temperature, lengths, draft_states), tensors from
// logprobs on or None
PyObject *verify(PyObject *, PyObject *const *a, Py_ssize_t n) try {
    float temperature;
    if (n != 8 || !temperature_of(a[5], temperature)) return none();
    const at::Tensor *logits = any_tensor(a[0], 3);
    if (!logits || logits->size(1) < 1 || !on_current_device(*logits)) return none();
    const int64_t B = logits->size(0), K = logits->size(1) - 1, V = logits->size(2);
    if (V > 1 && logits->stride(2) != 1) return none();
    const bool sample = temperature != 0.0f;
    Input tokens, logprobs, uniforms, noise, lengths, states;
    if (!tokens.set(a[1], at::kInt, {B, K}, *logits, false) ||
        (sample && (!logprobs.set(a[2], at::kFloat, {B, K, V}, *logits, true, true) ||
                    !uniforms.set(a[3], at::kFloat, {B, K}, *logits, false, K == 0) ||
                    !noise.set(a[4], at::kFloat, {B, V}, *logits, true))) ||
        !lengths.set(a[6], at::kInt, {B}, *logits, false, true) ||
        !states.set(a[7], at::kInt, {B, K + 1}, *logits, false, true))
        return none();
    const auto ints = logits->options().dtype(at::kInt);
    const at::Tensor out = at::empty({B, K + 1}, ints), kept = at::empty({B}, ints);
    const at::Tensor after = states.t ? at::empty({B}, ints) : at::Tensor();
    const size_t bytes = K <= NGPU_LM_MAX_DRAFT ? g_verify_workspace(B, int32_t(K), V) : 0;
    const at::Tensor workspace = scratch(bytes, *logits);
    Ref o(held(out)), c(held(kept)), s(held(after));
    if (!o.p || !c.p || !s.p) return none();
    Ref result(PyTuple_Pack(3, o.p, c.p, s.p));
    if (!result.p) return none();
    const ngpu_verify_t args{B, int32_t(K), V, type_code(logits->scalar_type()), logits->data_ptr(), logits->stride(0),
                             logits->stride(1), tokens.ptr<int32_t>(), lengths.ptr<int32_t>(), logprobs.ptr<float>(),
                             logprobs.stride(0), logprobs.stride(1), uniforms.ptr<float>(), noise.ptr<float>(),
                             noise.stride(0), temperature, states.ptr<int32_t>(), out.data_ptr<int32_t>(),
                             kept.data_ptr<int32_t>(), states.t ? after.data_ptr<int32_t>() : nullptr};
    void *stream = current_stream();
    const int rc = without_gil([&] { return g_verify(&args, workspace.data_ptr(), bytes, stream); });
    return answer(rc, result);
} catch (const std::exception &) {
    return none();
}

// The cache of two [pages, page size, heads, dim] tensors.
bool layout_of(PyObject *v, int32_t code, ngpu_kv_cache_t &c, const at::Tensor &keys) {
    if (!on_current_device(keys)) return false;
    Input values;
    if (!values.set(v, keys.scalar_type(), keys.sizes(), keys, true)) return false;
    if (keys.size(3) > 1 && keys.stride(3) != 1) return false;
    if (tracked(&keys) || tracked(values.t)) return false;
    for (int i = 1; i < 4; ++i)
        if (keys.size(i) > INT32_MAX) return false;
    c = {code, int32_t(keys.size(2)), int32_t(keys.size(3)), int32_t(keys.size(1)),
         keys.size(0), keys.data_ptr(), values.ptr(), keys.stride(0), keys.stride(1), keys.stride(2),
         values.stride(0), values.stride(1), values.stride(2)};
    return true;
}
bool cache_of(PyObject *k, PyObject *v, ngpu_kv_cache_t &c, const at::Tensor *&keys) {
    keys = any_tensor(k, 4);
    return keys && keys->scalar_type() != at::kFloat && layout_of(v, type_code(keys->scalar_type()), c, *keys);
}
// The same of 8 bits with its scales, for queries, keys and values of `type`.
bool scales_of(PyObject *o, const at::Tensor &keys, int64_t blocks, const at::Tensor *&t) {
    t = tensor_of(o, at::kFloat);
    return t && t->dim() == 3 && t->device() == keys.device() && t->size(0) == keys.size(0) && t->size(1) == blocks &&
           t->size(2) == keys.size(2) && !tracked(t);
}
bool cache8_of(PyObject *k, PyObject *v, PyObject *ks, PyObject *vs, at::ScalarType type, ngpu_kv_cache8_t &c,
               const at::Tensor *&keys) {
    keys = tensor_of(k, at::kFloat8_e4m3fn);
    if (!keys || keys->dim() != 4 || (type != at::kHalf && type != at::kBFloat16) ||
        !layout_of(v, type_code(type), c.cache, *keys))
        return false;
    const at::Tensor *a = tensor_of(ks, at::kFloat), *b;
    if (!a || a->dim() != 3 || a->size(1) < 1 || keys->size(1) % a->size(1) != 0 || !scales_of(ks, *keys, a->size(1), a) ||
        !scales_of(vs, *keys, a->size(1), b))
        return false;
    c.block = int32_t(keys->size(1) / a->size(1));
    c.k_scale = static_cast<float *>(a->data_ptr());
    c.v_scale = static_cast<float *>(b->data_ptr());
    c.k_scale_stride_page = a->stride(0), c.k_scale_stride_block = a->stride(1), c.k_scale_stride_head = a->stride(2);
    c.v_scale_stride_page = b->stride(0), c.v_scale_stride_block = b->stride(1), c.v_scale_stride_head = b->stride(2);
    return true;
}
// A page table: [rows, any width].
bool table_of(PyObject *o, int64_t rows, const at::Tensor &like, Input &t) {
    const at::Tensor *x = tensor_of(o, at::kInt);
    return x && x->dim() == 2 && t.set(o, at::kInt, {rows, x->size(1)}, like, true);
}

// kv_append(k, v, k_cache, v_cache, pages, start, positions, cos, sin, layout, q, lengths[, k_scale, v_scale]);
// positions, cos with sin, q and lengths may be None
PyObject *kv_append(PyObject *, PyObject *const *a, Py_ssize_t n) try {
    int64_t layout;
    ngpu_kv_cache8_t cache8;
    ngpu_kv_cache_t &cache = cache8.cache;
    const bool eight = n == 14;
    const at::Tensor *keys, *k = n == 12 || eight ? any_tensor(a[0], 4) : nullptr;
    if (!k || !(eight ? cache8_of(a[2], a[3], a[12], a[13], k->scalar_type(), cache8, keys) : cache_of(a[2], a[3], cache, keys)) ||
        !whole(a[9], layout) || layout < 0 || layout > 1)
        return none();
    const int64_t S = k->size(0), T = k->size(1);
    const at::ScalarType type = eight ? k->scalar_type() : keys->scalar_type();
    Input kx, v, q, pages, start, lengths, positions, cos, sin;
    if (!kx.set(a[0], type, {S, T, cache.heads, cache.dim}, *keys, true) ||
        !v.set(a[1], type, k->sizes(), *keys, true) || !table_of(a[4], S, *keys, pages) ||
        !start.set(a[5], at::kInt, {S}, *keys, false) || !lengths.set(a[11], at::kInt, {S}, *keys, false, true))
        return none();
    if (a[7] != Py_None) {
        const at::Tensor *table = dense(a[7], at::kFloat);
        if (!table || table->dim() != 2 || table->size(1) > NGPU_LM_MAX_HEAD_DIM ||
            !cos.set(a[7], at::kFloat, table->sizes(), *keys, false) ||
            !sin.set(a[8], at::kFloat, table->sizes(), *keys, false) ||
            !positions.set(a[6], at::kInt, {S, T}, *keys, false, true))
            return none();
    } else if (a[8] != Py_None) {
        return none();
    }
    at::Tensor out;
    if (a[10] != Py_None) {
        const at::Tensor *x = any_tensor(a[10], 4);
        if (!x || x->size(2) > INT32_MAX || !q.set(a[10], type, {S, T, x->size(2), cache.dim}, *keys, true))
            return none();
        out = at::empty(x->sizes(), k->options());
    }
    if (tracked(kx.t) || tracked(v.t) || tracked(q.t) || tracked(cos.t) || tracked(sin.t)) return none();
    Ref result(q.t ? held(out) : Py_NewRef(Py_True));   // (None would say that the call was not made)
    if (!result.p) return none();
    const ngpu_kv_append_t args{S, T, kx.ptr(), v.ptr(), kx.stride(0), kx.stride(1), kx.stride(2), v.stride(0),
                                v.stride(1), v.stride(2), q.ptr(), q.t ? int32_t(q.t->size(2)) : 0, q.stride(0),
                                q.stride(1), q.stride(2), q.t ? out.data_ptr() : nullptr, pages.ptr<int32_t>(),
                                pages.t->size(1), pages.stride(0), start.ptr<int32_t>(), lengths.ptr<int32_t>(),
                                cos.t ? int32_t(2 * cos.t->size(1)) : 0, int32_t(layout), positions.ptr<int32_t>(),
                                cos.ptr<float>(), sin.ptr<float>(), cos.t ? cos.t->size(0) : 0};
    void *stream = current_stream();
    const int rc = without_gil([&] { return eight ? g_kv_append8(&cache8, &args, stream) : g_kv_append(&cache, &args, stream); });
    return answer(rc, result);
} catch (const std::exception &) {
    return none();
}

// attend(q, k_cache, v_cache, pages, lengths, prefix_pages, prefix_lengths, q_lengths, scale[, k_scale, v_scale]), pages
// with lengths, prefix_pages with prefix_lengths, q_lengths and scale may be None: the output alone
PyObject *attend(PyObject *, PyObject *const *a, Py_ssize_t n) try {
    float scale;
    ngpu_kv_cache8_t cache8;
    ngpu_kv_cache_t &cache = cache8.cache;
    const bool eight = n == 11;
    const at::Tensor *keys, *x = n == 9 || eight ? any_tensor(a[0], 4) : nullptr;
    if (!x || !(eight ? cache8_of(a[1], a[2], a[9], a[10], x->scalar_type(), cache8, keys) : cache_of(a[1], a[2], cache, keys)) ||
        x->size(2) > INT32_MAX)
        return none();
    if (a[8] == Py_None)
        scale = float(1.0 / std::sqrt(double(cache.dim)));
    else if (!real(a[8], scale))
        return none();
    const int64_t S = x->size(0), T = x->size(1);
    Input q, pages, lengths, prefix, prefix_lengths, q_lengths;
    if (!q.set(a[0], eight ? x->scalar_type() : keys->scalar_type(), {S, T, x->size(2), cache.dim}, *keys, true) ||
        !q_lengths.set(a[7], at::kInt, {S}, *keys, false, true) || (a[3] == Py_None) != (a[4] == Py_None) ||
        (a[5] == Py_None) != (a[6] == Py_None) || tracked(q.t))
        return none();
    if (a[3] != Py_None && (!table_of(a[3], S, *keys, pages) || pages.t->size(1) == 0 ||
                            !lengths.set(a[4], at::kInt, {S}, *keys, false)))
        return none();
    int64_t G = 0;
    if (a[5] != Py_None) {
        const at::Tensor *t = tensor_of(a[5], at::kInt);
        if (!t || t->dim() != 2 || t->size(0) < 1) return none();
        G = t->size(0);
        if (!table_of(a[5], G, *keys, prefix) || !prefix_lengths.set(a[6], at::kInt, {G}, *keys, false)) return none();
    }
    const at::Tensor out = at::empty(x->sizes(), x->options());
    ngpu_attend_t args{S, T, int32_t(x->size(2)), q.ptr(), q.stride(0), q.stride(1), q.stride(2),
                       q_lengths.ptr<int32_t>(), G, prefix.ptr<int32_t>(), prefix.t ? prefix.t->size(1) : 0,
                       prefix.stride(0), prefix_lengths.ptr<int32_t>(), pages.ptr<int32_t>(),
                       pages.t ? pages.t->size(1) : 0, pages.stride(0), lengths.ptr<int32_t>(), scale, out.data_ptr(),
                       nullptr};
    const size_t bytes = eight ? g_attend8_workspace(&cache8, &args) : g_attend_workspace(&cache, &args);
    const at::Tensor workspace = scratch(bytes, *keys);
    Ref result(held(out));
    if (!result.p) return none();
    void *stream = current_stream();
    const int rc = without_gil([&] {
        return eight ? g_attend8(&cache8, &args, workspace.data_ptr(), bytes, stream)
                     : g_attend(&cache, &args, workspace.data_ptr(), bytes, stream);
    });
    return answer(rc, result);
} catch (const std::exception &) {
    return none();
}

// ---- the beam search's calls

// beam_step(handle, V, asr, lam, states, scores, k or None, last or None, mode)
PyObject *beam_step(PyObject *, PyObject *const *a, Py_ssize_t n) try {
    int64_t h, V, k, mode;
    float lam;
    if (n != 9 || !whole(a[0], h) || !whole(a[1], V) || !real(a[3], lam) || !whole(a[8], mode) || mode < 0 || mode > 3)
        return none();
    const at::Tensor *asr = tensor_of(a[2], at::kFloat);
    if (!asr || asr->dim() != 3 || !on_current_device(*asr) || asr->stride(2) != 1) return none();
    const int64_t B = asr->size(0), W = asr->size(1);
    if (asr->size(2) < V + (mode != NGPU_FUSION_PLAIN) || W < 1 || W > NGPU_LM_MAX_BEAMS) return none();
    k = W;
    if (a[6] != Py_None && (!whole(a[6], k) || k < 1 || k > NGPU_LM_MAX_BEAMS)) return none();
    Input states, scores, last;
    if (!states.set(a[4], at::kInt, {B, W}, *asr, false) || !scores.set(a[5], at::kFloat, {B, W}, *asr, false) ||
        !last.set(a[7], at::kInt, {B, W}, *asr, false, true) || tracked(asr) || tracked(scores.t))
        return none();
    const auto ints = states.t->options();
    const at::Tensor tokens = at::empty({B, k}, ints), parents = at::empty({B, k}, ints), after = at::empty({B, k}, ints),
                     best = at::empty({B, k}, asr->options());
    const size_t bytes = g_beam_step_workspace(B, int32_t(W), int32_t(k));
    const at::Tensor workspace = scratch(bytes, *asr);
    Ref t(held(tokens)), p(held(parents)), b(held(best)), s(held(after));
    if (!t.p || !p.p || !b.p || !s.p) return none();
    Ref result(PyTuple_Pack(4, t.p, p.p, b.p, s.p));
    if (!result.p) return none();
    const ngpu_beam_step_t args{B, int32_t(W), int32_t(k), int32_t(mode), lam, static_cast<const float *>(asr->data_ptr()),
                                asr->stride(0), asr->stride(1), states.ptr<int32_t>(), scores.ptr<float>(),
                                last.ptr<int32_t>(), tokens.data_ptr<int32_t>(), parents.data_ptr<int32_t>(),
                                best.data_ptr<float>(), after.data_ptr<int32_t>()};
    void *stream = current_stream();
    const int rc = without_gil(
        [&] { return g_beam_step(reinterpret_cast<const ngpu_lm *>(h), &args, workspace.data_ptr(), bytes, stream); });
    return answer(rc, result);
} catch (const std::exception &) {
    return none();
}

// kv_fork(pages, lengths, parents, refs, page size, tokens: an int or a tensor)
PyObject *kv_fork(PyObject *, PyObject *const *a, Py_ssize_t n) try {
    int64_t page_size, T = 0;
    if (n != 6 || !whole(a[4], page_size) || page_size < INT32_MIN || page_size > INT32_MAX) return none();
    const at::Tensor *refs = dense(a[3], at::kInt), *parents = dense(a[2], at::kInt), *table = tensor_of(a[0], at::kInt);
    if (!refs || refs->dim() != 1 || !on_current_device(*refs) || !parents || parents->dim() != 2 ||
        parents->device() != refs->device() || !table || table->dim() != 2)
        return none();
    const int64_t G = parents->size(0), K = parents->size(1), rows = table->size(0), width = table->size(1);
    if (G < 1 || rows % G != 0) return none();
    Input pages, lengths, tokens;
    if (!pages.set(a[0], at::kInt, {rows, width}, *refs, true) || !lengths.set(a[1], at::kInt, {rows}, *refs, false) ||
        (!whole(a[5], T) && (a[5] == Py_None || !tokens.set(a[5], at::kInt, {G, K}, *refs, false))))
        return none();
    const auto ints = refs->options();
    const at::Tensor made = at::empty({G * K, width}, ints), after = at::empty({G * K}, ints),
                     copies = at::empty({G * K, 3}, ints);
    const size_t bytes = g_kv_fork_workspace(G, K, refs->numel());
    const at::Tensor workspace = scratch(bytes, *refs);
    Ref m(held(made)), l(held(after)), c(held(copies));
    if (!m.p || !l.p || !c.p) return none();
    Ref result(PyTuple_Pack(3, m.p, l.p, c.p));
    if (!result.p) return none();
    const ngpu_kv_fork_t args{G, rows / G, K, pages.ptr<int32_t>(), width, pages.stride(0), lengths.ptr<int32_t>(),
                              static_cast<const int32_t *>(parents->data_ptr()), tokens.ptr<int32_t>(), T,
                              int32_t(page_size), refs->numel(), static_cast<int32_t *>(refs->data_ptr()),
                              made.data_ptr<int32_t>(), after.data_ptr<int32_t>(), copies.data_ptr<int32_t>()};
    void *stream = current_stream();
    const int rc = without_gil([&] { return g_kv_fork(&args, workspace.data_ptr(), bytes, stream); });
    return answer(rc, result);
} catch (const std::exception &) {
    return none();
}

// kv_copy(k_cache, v_cache, copies[, k_scale, v_scale]): True
PyObject *kv_copy(PyObject *, PyObject *const *a, Py_ssize_t n) try {
    ngpu_kv_cache8_t cache;
    const at::Tensor *keys, *copies = n == 3 || n == 5 ? dense(a[2], at::kInt) : nullptr;
    if (!copies || copies->dim() != 2 || copies->size(1) != 3 ||
        !(n == 5 ? cache8_of(a[0], a[1], a[3], a[4], at::kHalf, cache, keys) : cache_of(a[0], a[1], cache.cache, keys)) ||
        copies->device() != keys->device())
        return none();
    const auto *rows = static_cast<const int32_t *>(copies->data_ptr());
    const int64_t count = copies->size(0);
    void *stream = current_stream();
    const int rc = without_gil([&] {
        return n == 5 ? g_kv_copy8(&cache, rows, count, stream) : g_kv_copy(&cache.cache, rows, count, stream);
    });
    return rc != NGPU_OK ? PyLong_FromLong(rc) : Py_NewRef(Py_True);
} catch (const std::exception &) {
    return none();
}

// kv_compact(refs, page size, tables: a tuple)
PyObject *kv_compact(PyObject *, PyObject *const *a, Py_ssize_t n) try {
    constexpr Py_ssize_t kMost = 8;
    int64_t page_size;
    if (n != 3 || !whole(a[1], page_size) || page_size < INT32_MIN || page_size > INT32_MAX || !PyTuple_CheckExact(a[2]))
        return none();
    const at::Tensor *refs = dense(a[0], at::kInt), *tables[kMost];
    const Py_ssize_t count = PyTuple_GET_SIZE(a[2]);
    if (!refs || refs->dim() != 1 || !on_current_device(*refs) || count > kMost) return none();
    for (Py_ssize_t i = 0; i < count; ++i) {
        const at::Tensor *t = tables[i] = tensor_of(PyTuple_GET_ITEM(a[2], i), at::kInt);
        if (!t || t->dim() != 2 || t->device() != refs->device() || (t->size(1) > 1 && t->stride(1) != 1) ||
            (t->size(0) > 1 && t->stride(0) < t->size(1)))
            return none();
        for (Py_ssize_t j = 0; j < i; ++j)
            if (t->numel() > 0 && tables[j]->numel() > 0 && t->data_ptr() == tables[j]->data_ptr()) return none();
    }
    const int64_t P = refs->numel();
    const at::Tensor copies = at::empty({P / 2, 3}, refs->options()), moved = at::empty({P}, refs->options());
    const size_t bytes = g_kv_compact_workspace(P);
    const at::Tensor workspace = scratch(bytes, *refs);
    Ref c(held(copies)), m(held(moved));
    if (!c.p || !m.p) return none();
    Ref result(PyTuple_Pack(2, c.p, m.p));
    if (!result.p) return none();
    void *stream = current_stream();
    const int rc = without_gil([&] {
        int r = g_kv_compact(static_cast<int32_t *>(refs->data_ptr()), P, int32_t(page_size), copies.data_ptr<int32_t>(),
                             moved.data_ptr<int32_t>(), workspace.data_ptr(), bytes, stream);
        for (Py_ssize_t i = 0; i < count && r == NGPU_OK; ++i)
            r = g_kv_move(static_cast<int32_t *>(tables[i]->data_ptr()), tables[i]->size(0), tables[i]->size(1),
                          tables[i]->stride(0), moved.data_ptr<int32_t>(), P, stream);
        return r;
    });
    return answer(rc, result);
} catch (const std::exception &) {
    return none();
}

// The entry points of a call, in this order.
template <class... F>
PyObject *bind_all(PyObject *const *a, Py_ssize_t n, const char *error, F &...f) {
    int64_t p[sizeof...(F)];
    for (size_t i = 0; i < sizeof...(F); ++i)
        if (size_t(n) != sizeof...(F) || !whole(a[i], p[i])) {
            PyErr_SetString(PyExc_TypeError, error);
            return nullptr;
        }
    size_t at = 0;
    ((f = reinterpret_cast<F>(p[at++])), ...);
    return none();
}
// bind_serving(addresses of ngpu_lm_draft, ngpu_lm_verify_workspace, ngpu_lm_verify, ngpu_lm_kv_append,
// ngpu_lm_attend_workspace, ngpu_lm_attend)
PyObject *bind_serving(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return bind_all(a, n, "bind_serving takes six addresses", g_draft, g_verify_workspace, g_verify, g_kv_append,
                    g_attend_workspace, g_attend);
}
// bind_beam(addresses of the entry points below)
PyObject *bind_beam(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return bind_all(a, n, "bind_beam takes twelve addresses", g_kv_append8, g_attend8_workspace, g_attend8, g_kv_copy,
                    g_kv_copy8, g_kv_fork_workspace, g_kv_fork, g_kv_compact_workspace, g_kv_compact, g_kv_move,
                    g_beam_step_workspace, g_beam_step);
}

// The torch.__version__ of the headers this was compiled with.
PyObject *torch_version(PyObject *, PyObject *const *, Py_ssize_t) { return PyUnicode_FromString(NGPU_TORCH_VERSION); }

template <PyObject *(*F)(PyObject *, PyObject *const *, Py_ssize_t)>
PyMethodDef method(const char *name) {
    return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(F)), METH_FASTCALL, nullptr};
}
PyMethodDef g_methods[] = {method<advance>("advance"), method<step>("step"), method<topk>("topk"),
                           method<bind>("bind"), method<draft>("draft"), method<verify>("verify"),
                           method<kv_append>("kv_append"), method<attend>("attend"),
                           method<beam_step>("beam_step"), method<kv_fork>("kv_fork"), method<kv_copy>("kv_copy"),
                           method<kv_compact>("kv_compact"), method<bind_beam>("bind_beam"),
                           method<bind_serving>("bind_serving"), method<torch_version>("torch_version"),
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_fastcall", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fastcall() { return PyModule_Create(&g_module); }
