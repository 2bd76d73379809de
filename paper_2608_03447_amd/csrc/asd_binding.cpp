// The binding's fast path: argument checks, output allocation and the C call of
// the per-round entry points in native code.
//
// Each function takes the address of the library's entry point and the call's
// arguments, checks them as the Python functions do, and makes the call on the
// current stream.  It returns (accept_len, next_token) or True, or the library's
// status when that is not ASD_OK, or None, with nothing done, for any argument
// that is not the ordinary one (a scalar gate, a tensor on another device, a
// layout to copy, a subclass, a wrong shape, an active dispatch mode): the
// Python function then takes the call, converts or copies what it accepts and
// raises what it refuses.
//
// A call's checks, pointers and outputs in Python took more host time than the
// GPU needs for a small round.  Host time per call of the public functions, before
// and after: one request with 8 drafts of 32,000 logits 15.5 and 5.8 us (3.8 of it
// in this module and the launch; the call itself 15.5 and 7.3 us, now the
// kernel's time); verify with commit 20.0 and 8.2 us; the opportunity statistic
// 12.2 and 3.5 us; the fused output layer 21.9 and 10.5; calls of the decoding
// operators, GPU time included, an append of one block 23.7 and 7.7.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>

#include "../../include/asd.h"

#ifndef ASD_BINDING_HASH
#define ASD_BINDING_HASH "unhashed"
#endif

namespace {

using at::ScalarType;

// A dense GPU tensor of this type on the current device, or nullptr.
const at::Tensor* dense(PyObject* o, ScalarType type, int device) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.defined() || t.layout() != at::kStrided || !t.is_cuda() || !t.has_storage() ||
        t.get_device() != device || t.scalar_type() != type || !t.is_contiguous())
        return nullptr;
    return &t;
}

// Pointer of a vector of `n` elements (any length for n < 0); false if it is
// not one.  None gives nullptr where `optional`.
bool vec(PyObject* o, ScalarType type, int64_t n, int device, void** out, bool optional = false) {
    *out = nullptr;
    if (o == Py_None) return optional;
    const at::Tensor* t = dense(o, type, device);
    if (!t || t->dim() != 1 || (n >= 0 && t->size(0) != n)) return false;
    *out = t->data_ptr();
    return true;
}

int current_device(PyObject* o) {
    if (c10::impl::TorchDispatchModeTLS::any_modes_set() || !THPVariable_CheckExact(o)) return -1;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.defined() || !t.is_cuda()) return -1;
    const int device = t.get_device();
    return device == c10::hip::current_device() ? device : -1;
}

void* current_stream(int device) {
    return (void*)c10::hip::getCurrentHIPStream((c10::DeviceIndex)device).stream();
}

// The arguments that every verifying call shares, from args[0]: draft tokens,
// block lengths, gates, caps, ledgers, row offsets, accepted lengths, next
// tokens, argmax, regret.
constexpr int kShared = 10;
struct Shared {
    int32_t n = 0;
    int64_t rows = 0;
    void *draft, *lens, *tau, *cap, *budget, *offsets, *accept, *next, *argmax, *regret;
    void* stream = nullptr;
    PyObject* outputs[2] = {nullptr, nullptr};       // owned references
    at::Tensor fresh[2];

    bool take(PyObject* const* a, int64_t total_rows, int device) {
        rows = total_rows;
        const at::Tensor* l = dense(a[1], ScalarType::Int, device);
        if (!l || l->dim() != 1 || l->size(0) > INT32_MAX) return false;
        n = (int32_t)l->size(0);
        lens = l->data_ptr();
        const at::Tensor* b = dense(a[4], ScalarType::Float, device);
        if (!b || b->dim() != 2 || b->size(0) != n || b->size(1) != 2) return false;
        budget = b->data_ptr();
        if (!vec(a[0], ScalarType::Int, rows, device, &draft) ||
            !vec(a[2], ScalarType::Float, n, device, &tau) ||
            !vec(a[3], ScalarType::Int, n, device, &cap) ||
            !vec(a[5], ScalarType::Long, n, device, &offsets, true) ||
            !vec(a[6], ScalarType::Int, n, device, &accept, true) ||
            !vec(a[7], ScalarType::Int, n, device, &next, true) ||
            !vec(a[8], ScalarType::Int, rows, device, &argmax, true) ||
            !vec(a[9], ScalarType::Float, rows, device, &regret, true))
            return false;
        void** const ptr[2] = {&accept, &next};
        for (int k = 0; k < 2; ++k) {
            if (a[6 + k] != Py_None) {        // also an empty one, whose pointer is null
                Py_INCREF(a[6 + k]);
                outputs[k] = a[6 + k];
            } else {
                fresh[k] = at::empty({n}, l->options().requires_grad(false));
                *ptr[k] = fresh[k].data_ptr();
            }
        }
        stream = current_stream(device);
        return true;
    }
    // (accept_len, next_token), or the status of a call that failed.
    PyObject* result(asd_status st) {
        if (st != ASD_OK) return PyLong_FromLong(st);
        for (int k = 0; k < 2; ++k)
            if (!outputs[k] && !(outputs[k] = THPVariable_Wrap(std::move(fresh[k])))) return nullptr;
        return PyTuple_Pack(2, outputs[0], outputs[1]);
    }
    ~Shared() {
        Py_XDECREF(outputs[0]);
        Py_XDECREF(outputs[1]);
    }
};

PyObject* done(asd_status st) {
    if (st != ASD_OK) return PyLong_FromLong(st);
    Py_RETURN_TRUE;
}

template <typename F>
F entry(PyObject* address) {
    return reinterpret_cast<F>(PyLong_AsVoidPtr(address));
}

// Runs a library call without the interpreter lock.
template <typename Call>
asd_status unlocked(Call&& call) {
    asd_status st;
    Py_BEGIN_ALLOW_THREADS;
    st = call();
    Py_END_ALLOW_THREADS;
    return st;
}

// Logits [rows, V] in f32 or bf16: type code, sizes and pointer.
struct Logits {
    asd_dtype dtype;
    int64_t rows, vocab;
    void* ptr;
    bool take(PyObject* o, int device) {
        const at::Tensor* t = dense(o, ScalarType::BFloat16, device);
        dtype = ASD_BF16;
        if (!t) {
            t = dense(o, ScalarType::Float, device);
            dtype = ASD_F32;
        }
        if (!t || t->dim() != 2) return false;
        rows = t->size(0);
        vocab = t->size(1);
        ptr = t->data_ptr();
        return true;
    }
};

// verify(entry, logits, shared...): asd_verify and asd_verify_static
PyObject* verify(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    if (nargs != 2 + kShared) Py_RETURN_NONE;
    const int device = current_device(a[1]);
    Logits z;
    Shared s;
    if (device < 0 || !z.take(a[1], device) || !s.take(a + 2, z.rows, device)) Py_RETURN_NONE;
    const auto f = entry<decltype(&asd_verify)>(a[0]);
    return s.result(unlocked([&] {
        return f(z.ptr, z.dtype, z.vocab, s.n, s.rows, (const int32_t*)s.draft,
                 (const int32_t*)s.lens, (const int64_t*)s.offsets, (const float*)s.tau,
                 (const int32_t*)s.cap, (asd_budget*)s.budget, (int32_t*)s.accept,
                 (int32_t*)s.next, (int32_t*)s.argmax, (float*)s.regret, s.stream);
    }));
    END_HANDLE_TH_ERRORS
}

// verify_ex(entry, logits, flags, shared...): the library's workspace
PyObject* verify_ex(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    if (nargs != 3 + kShared || !PyLong_CheckExact(a[2])) Py_RETURN_NONE;
    const long flags = PyLong_AsLong(a[2]);
    if (flags < 0 || flags > (long)INT32_MAX) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    const int device = current_device(a[1]);
    Logits z;
    Shared s;
    if (device < 0 || !z.take(a[1], device) || !s.take(a + 3, z.rows, device)) Py_RETURN_NONE;
    const auto f = entry<decltype(&asd_verify_ex)>(a[0]);
    return s.result(unlocked([&] {
        return f(z.ptr, z.dtype, z.vocab, s.n, s.rows, (const int32_t*)s.draft,
                 (const int32_t*)s.lens, (const int64_t*)s.offsets, (const float*)s.tau,
                 (const int32_t*)s.cap, (asd_budget*)s.budget, (int32_t*)s.accept,
                 (int32_t*)s.next, (int32_t*)s.argmax, (float*)s.regret, (uint32_t)flags, s.stream,
                 nullptr, 0);
    }));
    END_HANDLE_TH_ERRORS
}

// verify_commit(entry, logits, tokens, seq_len, committed, shared...)
PyObject* verify_commit(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    if (nargs != 5 + kShared) Py_RETURN_NONE;
    const int device = current_device(a[1]);
    Logits z;
    Shared s;
    if (device < 0 || !z.take(a[1], device)) Py_RETURN_NONE;
    const at::Tensor* tokens = dense(a[2], ScalarType::Int, device);
    const at::Tensor* lens = dense(a[6], ScalarType::Int, device);
    void *seq_len, *committed;
    if (!tokens || tokens->dim() != 2 || !lens || lens->dim() != 1 ||
        tokens->size(0) != lens->size(0) ||
        !vec(a[3], ScalarType::Long, lens->size(0), device, &seq_len) ||
        !vec(a[4], ScalarType::Int, lens->size(0), device, &committed, true) ||
        !s.take(a + 5, z.rows, device))
        Py_RETURN_NONE;
    void* const t = tokens->data_ptr();
    const int64_t capacity = tokens->size(1);
    const auto f = entry<decltype(&asd_verify_commit)>(a[0]);
    return s.result(unlocked([&] {
        return f(z.ptr, z.dtype, z.vocab, s.n, s.rows, (const int32_t*)s.draft,
                 (const int32_t*)s.lens, (const int64_t*)s.offsets, (const float*)s.tau,
                 (const int32_t*)s.cap, (asd_budget*)s.budget, (int32_t*)s.accept,
                 (int32_t*)s.next, (int32_t*)s.argmax, (float*)s.regret, (int32_t*)t, capacity,
                 (int64_t*)seq_len, (int32_t*)committed, s.stream, nullptr, 0);
    }));
    END_HANDLE_TH_ERRORS
}

bool integer(PyObject* o, int64_t* out) {
    if (!PyLong_CheckExact(o)) return false;
    *out = PyLong_AsLongLong(o);
    if (*out == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        return false;
    }
    return true;
}

// verify_partials(entry, partials, shard_vocab, vocab, shared...)
PyObject* verify_partials(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    if (nargs != 4 + kShared) Py_RETURN_NONE;
    const int device = current_device(a[1]);
    int64_t width, vocab;
    const at::Tensor* p = device < 0 ? nullptr : dense(a[1], ScalarType::Int, device);
    Shared s;
    if (!p || p->dim() != 3 || p->size(2) != 4 || p->size(0) > INT32_MAX || !integer(a[2], &width) ||
        !integer(a[3], &vocab) || !s.take(a + 4, p->size(1), device))
        Py_RETURN_NONE;
    const void* const ptr = p->data_ptr();
    const int32_t shards = (int32_t)p->size(0);
    const auto f = entry<decltype(&asd_verify_partials)>(a[0]);
    return s.result(unlocked([&] {
        return f((const asd_row_partial*)ptr, shards, width, vocab, s.n, s.rows,
                 (const int32_t*)s.draft, (const int32_t*)s.lens, (const int64_t*)s.offsets,
                 (const float*)s.tau, (const int32_t*)s.cap, (asd_budget*)s.budget,
                 (int32_t*)s.accept, (int32_t*)s.next, (int32_t*)s.argmax, (float*)s.regret,
                 s.stream);
    }));
    END_HANDLE_TH_ERRORS
}

// lmhead_verify(entry, hidden, weight, shared...)
PyObject* lmhead_verify(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    if (nargs != 3 + kShared) Py_RETURN_NONE;
    const int device = current_device(a[1]);
    if (device < 0) Py_RETURN_NONE;
    const at::Tensor* h = dense(a[1], ScalarType::BFloat16, device);
    const at::Tensor* w = dense(a[2], ScalarType::BFloat16, device);
    Shared s;
    if (!h || !w || h->dim() != 2 || w->dim() != 2 || h->size(1) != w->size(1) ||
        !s.take(a + 3, h->size(0), device))
        Py_RETURN_NONE;
    const void *hp = h->data_ptr(), *wp = w->data_ptr();
    const int64_t d = h->size(1), vocab = w->size(0);
    const auto f = entry<decltype(&asd_lmhead_verify)>(a[0]);
    return s.result(unlocked([&] {
        return f(hp, wp, d, vocab, s.n, s.rows, (const int32_t*)s.draft, (const int32_t*)s.lens,
                 (const int64_t*)s.offsets, (const float*)s.tau, (const int32_t*)s.cap,
                 (asd_budget*)s.budget, (int32_t*)s.accept, (int32_t*)s.next, (int32_t*)s.argmax,
                 (float*)s.regret, s.stream);
    }));
    END_HANDLE_TH_ERRORS
}

// shard_argmax(entry, shard_logits, vocab_offset, vocab, draft, partials)
PyObject* shard_argmax(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    if (nargs != 6) Py_RETURN_NONE;
    const int device = current_device(a[1]);
    Logits z;
    int64_t offset, vocab;
    void* draft;
    if (device < 0 || !z.take(a[1], device) || !integer(a[2], &offset) || !integer(a[3], &vocab) ||
        !vec(a[4], ScalarType::Int, z.rows, device, &draft))
        Py_RETURN_NONE;
    const at::Tensor* p = dense(a[5], ScalarType::Int, device);
    if (!p || p->dim() != 2 || p->size(0) != z.rows || p->size(1) != 4) Py_RETURN_NONE;
    void *out = p->data_ptr(), *stream = current_stream(device);
    const auto f = entry<decltype(&asd_shard_argmax)>(a[0]);
    return done(unlocked([&] {
        return f(z.ptr, z.dtype, z.vocab, offset, vocab, z.rows, (const int32_t*)draft,
                 (asd_row_partial*)out, stream);
    }));
    END_HANDLE_TH_ERRORS
}

// opportunity(entry, draft, argmax, regret, vocab, lens, taus, ps, counts,
// mismatches, offsets)
PyObject* opportunity(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    if (nargs != 11) Py_RETURN_NONE;
    const int device = current_device(a[1]);
    if (device < 0) Py_RETURN_NONE;
    const at::Tensor* x = dense(a[1], ScalarType::Int, device);
    const at::Tensor* lens = dense(a[5], ScalarType::Int, device);
    const at::Tensor* taus = dense(a[6], ScalarType::Float, device);
    const at::Tensor* ps = dense(a[7], ScalarType::Int, device);
    const at::Tensor* counts = dense(a[8], ScalarType::Long, device);
    int64_t vocab;
    void *argmax, *regret, *mismatches, *offsets;
    if (!x || x->dim() != 1 || !lens || lens->dim() != 1 || lens->size(0) > INT32_MAX || !taus ||
        taus->dim() != 1 || taus->size(0) > INT32_MAX || !ps || ps->dim() != 1 ||
        ps->size(0) > INT32_MAX || !counts || counts->dim() != 2 ||
        counts->size(0) != taus->size(0) || counts->size(1) != ps->size(0) ||
        !integer(a[4], &vocab) || !vec(a[2], ScalarType::Int, x->size(0), device, &argmax) ||
        !vec(a[3], ScalarType::Float, x->size(0), device, &regret) ||
        !vec(a[9], ScalarType::Long, 1, device, &mismatches) ||
        !vec(a[10], ScalarType::Long, lens->size(0), device, &offsets, true))
        Py_RETURN_NONE;
    const int64_t rows = x->size(0);
    const int32_t n = (int32_t)lens->size(0), nt = (int32_t)taus->size(0), np = (int32_t)ps->size(0);
    void *xp = x->data_ptr(), *lp = lens->data_ptr(), *tp = taus->data_ptr(), *pp = ps->data_ptr();
    void *cp = counts->data_ptr(), *stream = current_stream(device);
    const auto f = entry<decltype(&asd_opportunity)>(a[0]);
    return done(unlocked([&] {
        return f((const int32_t*)xp, (const int32_t*)argmax, (const float*)regret, vocab, n, rows,
                 (const int32_t*)lp, (const int64_t*)offsets, (const float*)tp, nt,
                 (const int32_t*)pp, np, (uint64_t*)cp, (uint64_t*)mismatches, stream);
    }));
    END_HANDLE_TH_ERRORS
}

// A strided GPU tensor on the current device with elements, or nullptr.
const at::Tensor* strided(PyObject* o, int device) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.defined() || t.layout() != at::kStrided || !t.is_cuda() || !t.has_storage() ||
        t.get_device() != device || t.numel() == 0)
        return nullptr;
    return &t;
}

bool half_type(const at::Tensor& t, asd_dtype* out) {
    *out = t.scalar_type() == ScalarType::BFloat16 ? ASD_BF16 : ASD_F16;
    return t.scalar_type() == ScalarType::BFloat16 || t.scalar_type() == ScalarType::Half;
}

// [rows, heads, D] in bf16 or f16 with the heads of a row dense; a type, rows or dim that are set already
// are those it has to have.
struct Heads {
    const at::Tensor* t = nullptr;
    void* ptr = nullptr;
    int64_t stride = 0, heads = 0;
    bool take(PyObject* o, int device, const at::Tensor* like) {
        t = strided(o, device);
        if (!t || t->dim() != 3) return false;
        if (like && (t->scalar_type() != like->scalar_type() || t->size(0) != like->size(0) ||
                     t->size(2) != like->size(2)))
            return false;
        heads = t->size(1);
        const int64_t d = t->size(2);
        if ((d > 1 && t->stride(2) != 1) || (heads > 1 && t->stride(1) != d) || heads > INT32_MAX ||
            d > INT32_MAX)
            return false;
        stride = t->size(0) > 1 ? t->stride(0) : heads * d;
        ptr = t->data_ptr();
        return true;
    }
};

// The batch and the cache of the decoding operators, from args[0]: key cache, value cache, page table,
// cache lengths, block lengths, row offsets.
constexpr int kPaged = 6;
struct Paged {
    asd_paged_cache cache;
    int32_t n = 0;
    void *cached, *lens, *offsets;
    bool take(PyObject* const* a, int device, const at::Tensor& like) {
        const at::Tensor *k = strided(a[0], device), *v = strided(a[1], device);
        if (!k || !v || k->dim() != 4 || v->dim() != 4 || k->scalar_type() != like.scalar_type() ||
            v->scalar_type() != like.scalar_type() || k->size(3) != like.size(2) ||
            k->sizes() != v->sizes() || k->strides() != v->strides() ||
            (k->size(3) > 1 && k->stride(3) != 1))
            return false;
        const at::Tensor* l = dense(a[4], ScalarType::Int, device);
        const at::Tensor* table = dense(a[2], ScalarType::Int, device);
        if (!l || l->dim() != 1 || l->size(0) > INT32_MAX || !table || table->dim() != 2 ||
            table->size(0) != l->size(0) || table->size(1) > INT32_MAX || k->size(1) > INT32_MAX ||
            k->size(2) > INT32_MAX || !vec(a[3], ScalarType::Long, l->size(0), device, &cached) ||
            !vec(a[5], ScalarType::Long, l->size(0), device, &offsets, true))
            return false;
        n = (int32_t)l->size(0);
        lens = l->data_ptr();
        // a stride over one entry is never used; torch leaves it with any value
        const auto step = [k](int i) { return k->size(i) > 1 ? k->stride(i) : 0; };
        cache = {k->data_ptr(), v->data_ptr(), k->size(0), step(0), step(1), step(2),
                 (const int32_t*)table->data_ptr(), (int32_t)table->size(1), (int32_t)k->size(1),
                 (int32_t)k->size(2), (int32_t)k->size(3)};
        return true;
    }
};

// A caller's workspace, or None.
bool space(PyObject* o, int device, void** ptr, size_t* bytes) {
    *ptr = nullptr;
    *bytes = 0;
    if (o == Py_None) return true;
    const at::Tensor* t = dense(o, ScalarType::Byte, device);
    if (!t || t->numel() == 0) return false;
    *ptr = t->data_ptr();
    *bytes = (size_t)t->numel();
    return true;
}

// An output that the caller gave (owned reference) or a fresh one.
struct Output {
    PyObject* given = nullptr;
    at::Tensor fresh;
    void* ptr = nullptr;
    void keep(PyObject* o, void* p) {
        Py_INCREF(o);
        given = o;
        ptr = p;
    }
    void make(at::IntArrayRef sizes, const at::TensorOptions& options) {
        fresh = at::empty(sizes, options.requires_grad(false));
        ptr = fresh.data_ptr();
    }
    PyObject* result(asd_status st) {
        if (st != ASD_OK) return PyLong_FromLong(st);
        if (!given) return THPVariable_Wrap(std::move(fresh));
        Py_INCREF(given);
        return given;
    }
    ~Output() { Py_XDECREF(given); }
};

// rope_append(entry, k, q, v, paged..., inv_freq, q_norm, k_norm, eps, positions, interleaved, out_q):
// out_q, or True without q
PyObject* rope_append(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    constexpr int kRest = 4 + kPaged;
    if (nargs != kRest + 7 || !PyFloat_CheckExact(a[kRest + 3]) || !PyBool_Check(a[kRest + 5]))
        Py_RETURN_NONE;
    const int device = current_device(a[1]);
    Heads k, v, q, out;
    Paged p;
    asd_dtype dtype;
    if (device < 0 || !k.take(a[1], device, nullptr) || !half_type(*k.t, &dtype) ||
        !v.take(a[3], device, k.t) || v.heads != k.heads || !p.take(a + 4, device, *k.t) ||
        p.cache.num_heads != k.heads)
        Py_RETURN_NONE;
    const int64_t rows = k.t->size(0), dim = k.t->size(2);
    PyObject* const* r = a + kRest;
    void *freq, *q_norm, *k_norm, *positions;
    const ScalarType type = k.t->scalar_type();
    if (!vec(r[0], ScalarType::Float, -1, device, &freq, true) ||
        !vec(r[1], type, dim, device, &q_norm, true) || !vec(r[2], type, dim, device, &k_norm, true) ||
        !vec(r[4], ScalarType::Long, rows, device, &positions, true))
        Py_RETURN_NONE;
    const int64_t rot = r[0] == Py_None ? 0 : 2 * THPVariable_Unpack(r[0]).numel();
    if (rot > dim) Py_RETURN_NONE;
    Output o;
    if (a[2] == Py_None) {
        if (r[6] != Py_None) Py_RETURN_NONE;
    } else {
        if (!q.take(a[2], device, k.t)) Py_RETURN_NONE;
        if (r[6] == Py_None) {
            o.make(q.t->sizes(), q.t->options());
            out.stride = q.heads * dim;
        } else {
            if (!out.take(r[6], device, k.t) || out.heads != q.heads) Py_RETURN_NONE;
            o.keep(r[6], out.ptr);
        }
    }
    const float eps = (float)PyFloat_AS_DOUBLE(r[3]);
    const uint32_t flags = r[5] == Py_True ? (uint32_t)ASD_ROPE_INTERLEAVED : 0u;
    void* const stream = current_stream(device);
    const auto f = entry<decltype(&asd_rope_append)>(a[0]);
    const asd_status st = unlocked([&] {
        return f(q.ptr, k.ptr, v.ptr, dtype, q.stride, k.stride, v.stride, (int32_t)q.heads, q_norm,
                 k_norm, eps, (const float*)freq, (int32_t)rot, flags, (const int64_t*)positions,
                 &p.cache, p.n, rows, (const int32_t*)p.lens, (const int64_t*)p.offsets,
                 (const int64_t*)p.cached, o.ptr, out.stride, stream);
    });
    return a[2] == Py_None ? done(st) : o.result(st);
    END_HANDLE_TH_ERRORS
}

// block_attention(entry, q, paged..., scale, mask, out, workspace)
PyObject* block_attention(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    constexpr int kRest = 2 + kPaged;
    if (nargs != kRest + 4) Py_RETURN_NONE;
    const int device = current_device(a[1]);
    Heads q;
    Paged p;
    asd_dtype dtype;
    if (device < 0 || !q.take(a[1], device, nullptr) || !half_type(*q.t, &dtype) ||
        !p.take(a + 2, device, *q.t))
        Py_RETURN_NONE;
    const int64_t rows = q.t->size(0), dim = q.t->size(2);
    PyObject* const* r = a + kRest;
    void *mask = nullptr, *ws;
    int32_t words = 0;
    size_t ws_bytes;
    if (r[0] != Py_None && !PyFloat_CheckExact(r[0])) Py_RETURN_NONE;
    const float scale =
        (float)(r[0] == Py_None ? 1.0 / std::sqrt((double)dim) : PyFloat_AS_DOUBLE(r[0]));
    if (r[1] != Py_None) {
        const at::Tensor* m = dense(r[1], ScalarType::Long, device);
        if (!m || m->dim() != 2 || m->size(0) != rows || m->size(1) < 1 || m->size(1) > INT32_MAX)
            Py_RETURN_NONE;
        mask = m->data_ptr();
        words = (int32_t)m->size(1);
    }
    Output o;
    if (r[2] == Py_None) {
        o.make(q.t->sizes(), q.t->options());
    } else {
        const at::Tensor* t = dense(r[2], q.t->scalar_type(), device);
        if (!t || t->sizes() != q.t->sizes()) Py_RETURN_NONE;
        o.keep(r[2], t->data_ptr());
    }
    if (!space(r[3], device, &ws, &ws_bytes)) Py_RETURN_NONE;
    void* const stream = current_stream(device);
    const auto f = entry<decltype(&asd_block_attention)>(a[0]);
    return o.result(unlocked([&] {
        return f(q.ptr, dtype, q.stride, (int32_t)q.heads, scale, &p.cache, p.n, rows,
                 (const int32_t*)p.lens, (const int64_t*)p.offsets, (const int64_t*)p.cached,
                 (const uint64_t*)mask, words, o.ptr, stream, ws, ws_bytes);
    }));
    END_HANDLE_TH_ERRORS
}

// sample(entry, logits, uniform, temperature, top_k, top_p, min_p, out_token, out_prob, workspace)
PyObject* sample(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    if (nargs != 10) Py_RETURN_NONE;
    const int device = current_device(a[1]);
    const at::Tensor* z = device < 0 ? nullptr : strided(a[1], device);
    if (!z || z->dim() != 2) Py_RETURN_NONE;
    asd_dtype dtype = ASD_F32;
    if (z->scalar_type() != ScalarType::Float && !half_type(*z, &dtype)) Py_RETURN_NONE;
    const int64_t rows = z->size(0), vocab = z->size(1), stride = rows > 1 ? z->stride(0) : vocab;
    void *uniform, *temperature, *top_k, *top_p, *min_p, *prob, *token, *ws;
    size_t ws_bytes;
    if ((vocab > 1 && z->stride(1) != 1) || stride < vocab ||
        !vec(a[2], ScalarType::Float, rows, device, &uniform) ||
        !vec(a[3], ScalarType::Float, rows, device, &temperature, true) ||
        !vec(a[4], ScalarType::Int, rows, device, &top_k, true) ||
        !vec(a[5], ScalarType::Float, rows, device, &top_p, true) ||
        !vec(a[6], ScalarType::Float, rows, device, &min_p, true) ||
        !vec(a[7], ScalarType::Int, rows, device, &token, true) ||
        !vec(a[8], ScalarType::Float, rows, device, &prob, true) ||
        !space(a[9], device, &ws, &ws_bytes))
        Py_RETURN_NONE;
    Output o;
    if (a[7] != Py_None)
        o.keep(a[7], token);
    else
        o.make({rows}, z->options().dtype(ScalarType::Int));
    const void* const ptr = z->data_ptr();
    void* const stream = current_stream(device);
    const auto f = entry<decltype(&asd_sample)>(a[0]);
    return o.result(unlocked([&] {
        return f(ptr, dtype, vocab, rows, stride, (const float*)temperature, (const int32_t*)top_k,
                 (const float*)top_p, (const float*)min_p, (const float*)uniform, (int32_t*)o.ptr,
                 (float*)prob, stream, ws, ws_bytes);
    }));
    END_HANDLE_TH_ERRORS
}

PyObject* source_hash(PyObject*, PyObject*) { return PyUnicode_FromString(ASD_BINDING_HASH); }

#define ASD_FAST(name) \
    {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ASD_FAST(verify),        ASD_FAST(verify_ex),
                         ASD_FAST(verify_commit), ASD_FAST(verify_partials),
                         ASD_FAST(lmhead_verify), ASD_FAST(shard_argmax),
                         ASD_FAST(opportunity),   ASD_FAST(rope_append),
                         ASD_FAST(block_attention), ASD_FAST(sample),
                         {"source_hash", source_hash, METH_NOARGS, nullptr},
                         {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_asd_binding", nullptr, -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__asd_binding(void) { return PyModule_Create(&module); }
