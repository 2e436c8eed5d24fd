// Argument marshalling of the hot calls in native code: the CPython face of the C ABI that binding.py's methods use.
//
// What bounds it: a decoding cycle makes one to three calls per layer, each a few microseconds of device work, so the
// host time per call decides whether the stream ever runs dry.  Through ctypes a call cost 8.5 - 10 us (conversion of
// 8 to 17 arguments, a c_void_p object for each pointer, the stream looked up through three Python layers) of which
// the launch itself is 2 - 3; here the tensors' device pointers and torch's current stream are read directly.
//
// Every function takes the context handle as an integer first and returns the vispec_status; tensors must be
// contiguous CUDA tensors (AssertionError otherwise), None stands for NULL.  The interpreter lock is released around
// the C call.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <c10/util/Exception.h>
#include <torch/csrc/autograd/python_variable.h>

#include <climits>
#include <initializer_list>
#include <string>

#include "vispec.h"

namespace {

// One call's arguments, read from left to right.  After a failed conversion `ok` is false and an exception is set.
struct Args {
    PyObject* const* a;
    Py_ssize_t n;
    Py_ssize_t i = 0;
    bool ok = true;

    Args(PyObject* const* args, Py_ssize_t nargs, Py_ssize_t want) : a(args), n(nargs) {
        if (nargs != want) {
            PyErr_Format(PyExc_TypeError, "%zd arguments expected, %zd given", want, nargs);
            ok = false;
        }
    }
    vispec_ctx* ctx() {
        if (!ok) return nullptr;
        void* p = PyLong_AsVoidPtr(a[i++]);
        if (!p && PyErr_Occurred()) ok = false;
        return static_cast<vispec_ctx*>(p);
    }
    int num() {
        if (!ok) return 0;
        const long v = PyLong_AsLong(a[i++]);
        if (v == -1 && PyErr_Occurred()) {
            ok = false;
        } else if (v < INT_MIN || v > INT_MAX) {
            PyErr_SetString(PyExc_OverflowError, "an integer of 32 bits is expected");
            ok = false;
        }
        return static_cast<int>(v);
    }
    float real() {
        if (!ok) return 0.f;
        const double v = PyFloat_AsDouble(a[i++]);
        if (v == -1.0 && PyErr_Occurred()) ok = false;
        return static_cast<float>(v);
    }
    // The tensor whose sizes the call needs (at least / exactly `dims` of them); nullptr with an exception otherwise.
    const at::Tensor* tensor(int dims, bool exact = true) {
        if (!ok) return nullptr;
        PyObject* o = a[i];
        if (!THPVariable_Check(o)) {
            PyErr_SetString(PyExc_TypeError, "a CUDA tensor is expected");
            ok = false;
            return nullptr;
        }
        const at::Tensor& t = THPVariable_Unpack(o);
        if (exact ? t.dim() != dims : t.dim() < dims) {
            PyErr_Format(PyExc_ValueError, "a tensor of %d dimensions is expected, got %d", dims, (int)t.dim());
            ok = false;
            return nullptr;
        }
        return &t;
    }
    template <typename T = void>
    T* ptr() {
        if (!ok) return nullptr;
        PyObject* o = a[i++];
        if (o == Py_None) return nullptr;
        if (!THPVariable_Check(o)) {
            PyErr_SetString(PyExc_TypeError, "a CUDA tensor or None is expected");
            ok = false;
            return nullptr;
        }
        const at::Tensor& t = THPVariable_Unpack(o);
        if (!t.is_cuda() || !t.is_contiguous()) {
            PyErr_SetString(PyExc_AssertionError, "device pointers must come from contiguous CUDA tensors");
            ok = false;
            return nullptr;
        }
        return static_cast<T*>(t.data_ptr());
    }
    // A tensor's memory, which has to be on the current device.  Looked at in this order: a fake tensor has neither memory nor,
    // maybe, a device, and its address of zero would pass for an argument that is not given.
    void* memory(const at::Tensor& t) {
        void* const p = t.data_ptr();
        if (!p && t.numel() > 0) {
            PyErr_SetString(PyExc_RuntimeError, "a tensor has no storage");
            ok = false;
        } else if (t.get_device() != c10::cuda::current_device()) {
            PyErr_SetString(PyExc_ValueError, "tensors must be on the current CUDA device");
            ok = false;
        }
        return p;
    }
    // [T, heads, D] bf16 on the current device, a token's heads contiguous, tokens any number of elements apart.  T < 0: the
    // tensor's own count is taken over, otherwise it has to be T.  None: nullptr.
    struct Rows { void* p = nullptr; int64_t stride = 0; };
    Rows rows(int64_t& T, int heads, int D) {
        Rows r;
        if (!ok) return r;
        if (a[i] == Py_None) { ++i; return r; }
        const at::Tensor* t = tensor(3);
        if (!t) return r;
        ++i;
        if (!t->is_cuda() || t->scalar_type() != at::kBFloat16) {
            PyErr_SetString(PyExc_ValueError, "rows must be bfloat16 CUDA tensors");
            ok = false;
        } else if ((T >= 0 && t->size(0) != T) || t->size(1) != heads || t->size(2) != D) {
            PyErr_Format(PyExc_ValueError, "rows of %lld tokens, %d heads and head size %d are expected", (long long)(T < 0 ? t->size(0) : T), heads, D);
            ok = false;
        } else if (t->size(0) > 0 && (t->stride(2) != 1 || (heads > 1 && t->stride(1) != D))) {
            PyErr_SetString(PyExc_ValueError, "a token's heads must be contiguous");
            ok = false;
        }
        if (!ok) return r;
        if (t->size(0) > INT_MAX) { PyErr_SetString(PyExc_ValueError, "too many tokens"); ok = false; return r; }
        T = t->size(0);
        r.p = memory(*t);
        r.stride = T > 1 ? t->stride(0) : (int64_t)heads * D;      // (one token: whatever its stride says is not used)
        return r;
    }
    // Are the sizes of t those of `want`, or those with neighbours joined or split?  (As many elements in another order of dimensions
    // are not: every size up to some point has to multiply to the same as some sizes of the other.)
    static bool fits(const at::Tensor& t, std::initializer_list<int64_t> want) {
        auto ends_in = [](const int64_t* x, size_t nx, const int64_t* y, size_t ny) {
            int64_t px = 1, py = 1;
            for (size_t i = 0, j = 0; i < nx; ++i) {
                px *= x[i];
                while (py < px && j < ny) py *= y[j++];
                if (py != px) return false;
            }
            return true;
        };
        int64_t n = 1;
        for (int64_t w : want) n *= w;
        const auto have = t.sizes();
        return t.numel() == n && (n == 0 || ends_in(have.data(), have.size(), want.begin(), want.size()) ||
                                  ends_in(want.begin(), want.size(), have.data(), have.size()));
    }
    // A contiguous tensor of `type` and the given sizes on the current device ({}: any).  None: nullptr, where it may be.
    void* dense(at::ScalarType type, std::initializer_list<int64_t> want, bool optional = false) {
        if (!ok) return nullptr;
        PyObject* o = a[i];
        if (o == Py_None && optional) { ++i; return nullptr; }
        if (!THPVariable_Check(o)) {
            PyErr_SetString(PyExc_TypeError, "a CUDA tensor is expected");
            ok = false;
            return nullptr;
        }
        const at::Tensor& t = THPVariable_Unpack(o);
        if (!t.is_cuda() || t.scalar_type() != type || !t.is_contiguous() ||
            (want.size() > 0 && !fits(t, want))) {
            std::string shape;
            for (int64_t w : want) shape += (shape.empty() ? "" : ", ") + std::to_string(w);
            PyErr_Format(PyExc_ValueError, "a contiguous %s CUDA tensor of shape [%s] is expected",
                         c10::toString(type), want.size() > 0 ? shape.c_str() : "any");
            ok = false;
            return nullptr;
        }
        ++i;
        return memory(t);
    }
    int32_t* ints(std::initializer_list<int64_t> want, bool optional = false) { return static_cast<int32_t*>(dense(at::kInt, want, optional)); }
    const vispec_rope_axes* axes() {                                // address of the struct (RopeAxes keeps it), 0: none
        if (!ok) return nullptr;
        void* p = PyLong_AsVoidPtr(a[i++]);
        if (!p && PyErr_Occurred()) ok = false;
        return static_cast<const vispec_rope_axes*>(p);
    }
};

void* stream() { return c10::cuda::getCurrentCUDAStream().stream(); }

// The interpreter lock is given up for as long as this lives.
struct Unlocked {
    PyThreadState* state = PyEval_SaveThread();
    ~Unlocked() { PyEval_RestoreThread(state); }
};

// The call itself, without the interpreter lock.
template <typename F>
PyObject* finish(const Args& g, F&& call) {
    if (!g.ok) return nullptr;
    void* const st = stream();
    int rc;
    {
        Unlocked unlocked;
        rc = call(st);
    }
    return PyLong_FromLong(rc);
}

// What the interpreter calls: an exception that torch throws on the way - a tensor without storage (a fake or wrapped one) has
// no data pointer, a process without a usable device has no current stream - becomes a RuntimeError; past this frame it would
// end the process.
template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject* self, PyObject* const* args, Py_ssize_t nargs) {
    try {
        return F(self, args, nargs);
    } catch (const c10::Error& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what_without_backtrace());
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
    }
    return nullptr;
}

int size(const at::Tensor* t, int d) { return t ? static_cast<int>(t->size(d)) : 0; }

#define NATIVE(name) PyObject* name(PyObject*, PyObject* const* args, Py_ssize_t nargs)

NATIVE(tree_mask_build) {   // handle, parents, tree_mask, depth
    Args g(args, nargs, 4);
    vispec_ctx* c = g.ctx();
    const at::Tensor* t = g.tensor(2);
    const int B = size(t, 0), N = size(t, 1);
    auto* parents = g.ptr<int32_t>(); auto* mask = g.ptr<uint64_t>(); auto* depth = g.ptr<int32_t>();
    return finish(g, [&](void* st) { return vispec_tree_mask_build(c, parents, B, N, mask, depth, st); });
}

NATIVE(tree_verify_attn) {  // handle, layer, q, k_cache, v_cache, kv_len, tree_mask, positions, scale, out, lse
    Args g(args, nargs, 11);
    vispec_ctx* c = g.ctx();
    const int layer = g.num();
    const at::Tensor* t = g.tensor(2, false);
    const int B = size(t, 0), N = size(t, 1);
    auto* q = g.ptr(); auto* k = g.ptr(); auto* v = g.ptr();
    auto* kv_len = g.ptr<int32_t>(); auto* mask = g.ptr<uint64_t>(); auto* pos = g.ptr<int32_t>();
    const float scale = g.real();
    auto* out = g.ptr(); auto* lse = g.ptr<float>();
    return finish(g, [&](void* st) { return vispec_tree_verify_attn(c, layer, q, k, v, kv_len, mask, pos, B, N, scale, out, lse, st); });
}

NATIVE(tree_verify_attn_rope) {  // handle, layer, q, k_new, v_new, rope_table, kv_len, tree_mask, scale, out, lse
    Args g(args, nargs, 11);
    vispec_ctx* c = g.ctx();
    const int layer = g.num();
    const at::Tensor* t = g.tensor(2, false);
    const int B = size(t, 0), N = size(t, 1);
    auto* q = g.ptr(); auto* k = g.ptr(); auto* v = g.ptr(); auto* table = g.ptr();
    auto* kv_len = g.ptr<int32_t>(); auto* mask = g.ptr<uint64_t>();
    const float scale = g.real();
    auto* out = g.ptr(); auto* lse = g.ptr<float>();
    return finish(g, [&](void* st) { return vispec_tree_verify_attn_rope(c, layer, q, k, v, table, kv_len, mask, B, N, scale, out, lse, st); });
}

NATIVE(tree_verify_attn_paged) {  // handle, layer, q, kv_len, block_table, tree_mask, scale, out, lse
    Args g(args, nargs, 9);
    vispec_ctx* c = g.ctx();
    const int layer = g.num();
    const at::Tensor* t = g.tensor(2, false);
    const int B = size(t, 0), N = size(t, 1);
    auto* q = g.ptr(); auto* kv_len = g.ptr<int32_t>();
    const int stride = size(g.tensor(2), 1);
    auto* table = g.ptr<int32_t>(); auto* mask = g.ptr<uint64_t>();
    const float scale = g.real();
    auto* out = g.ptr(); auto* lse = g.ptr<float>();
    return finish(g, [&](void* st) { return vispec_tree_verify_attn_paged(c, layer, q, kv_len, table, stride, mask, B, N, scale, out, lse, st); });
}

NATIVE(tree_verify_attn_static) {  // q, k_cache, v_cache, kv_len, tree_mask, scale, out, lse, status_word
    Args g(args, nargs, 9);
    const at::Tensor* t = g.tensor(4);
    const int B = size(t, 0), N = size(t, 1), Hq = size(t, 2), D = size(t, 3);
    auto* q = g.ptr();
    const at::Tensor* tk = g.tensor(4);
    const int Hkv = size(tk, 1), S_max = size(tk, 2);
    auto* k = g.ptr(); auto* v = g.ptr(); auto* kv_len = g.ptr<int32_t>(); auto* mask = g.ptr<uint64_t>();
    const float scale = g.real();
    auto* out = g.ptr(); auto* lse = g.ptr<float>(); auto* status = g.ptr<int>();
    return finish(g, [&](void* st) { return vispec_tree_verify_attn_static(q, k, v, kv_len, mask, B, N, Hq, Hkv, D, S_max, scale, out, lse, status, st); });
}

NATIVE(rope_table_build) {  // handle, positions, theta, table
    Args g(args, nargs, 4);
    vispec_ctx* c = g.ctx();
    const at::Tensor* t = g.tensor(2);
    const int B = size(t, 0), N = size(t, 1);
    auto* pos = g.ptr<int32_t>();
    const float theta = g.real();
    auto* table = g.ptr();
    return finish(g, [&](void* st) { return vispec_rope_table_build(c, pos, B, N, theta, table, st); });
}

NATIVE(rope_tree_rows) {  // handle, layer, q, k_new, v_new, positions, kv_len, theta
    Args g(args, nargs, 8);
    vispec_ctx* c = g.ctx();
    const int layer = g.num();
    auto* q = g.ptr(); auto* k = g.ptr(); auto* v = g.ptr();
    const at::Tensor* t = g.tensor(2);
    const int B = size(t, 0), N = size(t, 1);
    auto* pos = g.ptr<int32_t>(); auto* kv_len = g.ptr<int32_t>();
    const float theta = g.real();
    return finish(g, [&](void* st) { return vispec_rope_tree_rows(c, layer, q, k, v, pos, kv_len, B, N, theta, st); });
}

NATIVE(rope_tree_rows_paged) {  // handle, layer, q, k_new, v_new, positions, kv_len, block_table, theta
    Args g(args, nargs, 9);
    vispec_ctx* c = g.ctx();
    const int layer = g.num();
    auto* q = g.ptr(); auto* k = g.ptr(); auto* v = g.ptr();
    const at::Tensor* t = g.tensor(2);
    const int B = size(t, 0), N = size(t, 1);
    auto* pos = g.ptr<int32_t>(); auto* kv_len = g.ptr<int32_t>();
    const int stride = size(g.tensor(2), 1);
    auto* table = g.ptr<int32_t>();
    const float theta = g.real();
    return finish(g, [&](void* st) { return vispec_rope_tree_rows_paged(c, layer, q, k, v, pos, kv_len, table, stride, B, N, theta, st); });
}

NATIVE(accept) {  // handle, draft_ids, target_ids, parents, path, accept_len, bonus
    Args g(args, nargs, 7);
    vispec_ctx* c = g.ctx();
    auto* draft = g.ptr<int32_t>(); auto* target = g.ptr<int32_t>();
    const at::Tensor* t = g.tensor(2);
    const int B = size(t, 0), N = size(t, 1);
    auto* parents = g.ptr<int32_t>(); auto* path = g.ptr<int32_t>(); auto* alen = g.ptr<int32_t>(); auto* bonus = g.ptr<int32_t>();
    return finish(g, [&](void* st) { return vispec_accept(c, draft, target, parents, B, N, path, alen, bonus, st); });
}

NATIVE(accept_commit) {  // handle, layer_begin, layer_end, draft_ids, target_ids, parents, kv_len, path, accept_len, bonus, kv_len_out
    Args g(args, nargs, 11);
    vispec_ctx* c = g.ctx();
    const int lb = g.num(), le = g.num();
    auto* draft = g.ptr<int32_t>(); auto* target = g.ptr<int32_t>();
    const at::Tensor* t = g.tensor(2);
    const int B = size(t, 0), N = size(t, 1);
    auto* parents = g.ptr<int32_t>(); auto* kv_len = g.ptr<int32_t>(); auto* path = g.ptr<int32_t>();
    auto* alen = g.ptr<int32_t>(); auto* bonus = g.ptr<int32_t>(); auto* out = g.ptr<int32_t>();
    return finish(g, [&](void* st) { return vispec_accept_commit(c, lb, le, draft, target, parents, kv_len, B, N, path, alen, bonus, out, st); });
}

NATIVE(accept_commit_paged) {  // ... kv_len, block_table, path, accept_len, bonus, kv_len_out
    Args g(args, nargs, 12);
    vispec_ctx* c = g.ctx();
    const int lb = g.num(), le = g.num();
    auto* draft = g.ptr<int32_t>(); auto* target = g.ptr<int32_t>();
    const at::Tensor* t = g.tensor(2);
    const int B = size(t, 0), N = size(t, 1);
    auto* parents = g.ptr<int32_t>(); auto* kv_len = g.ptr<int32_t>();
    const int stride = size(g.tensor(2), 1);
    auto* table = g.ptr<int32_t>(); auto* path = g.ptr<int32_t>();
    auto* alen = g.ptr<int32_t>(); auto* bonus = g.ptr<int32_t>(); auto* out = g.ptr<int32_t>();
    return finish(g, [&](void* st) { return vispec_accept_commit_paged(c, lb, le, draft, target, parents, kv_len, table, stride, B, N, path, alen, bonus, out, st); });
}

NATIVE(kv_compact) {  // handle, layer_begin, layer_end, path, accept_len, kv_len, kv_len_out
    Args g(args, nargs, 7);
    vispec_ctx* c = g.ctx();
    const int lb = g.num(), le = g.num();
    const at::Tensor* t = g.tensor(2);
    const int B = size(t, 0), N = size(t, 1);
    auto* path = g.ptr<int32_t>(); auto* alen = g.ptr<int32_t>(); auto* kv_len = g.ptr<int32_t>(); auto* out = g.ptr<int32_t>();
    return finish(g, [&](void* st) { return vispec_kv_compact(c, lb, le, path, alen, kv_len, out, B, N, st); });
}

NATIVE(kv_compact_paged) {  // handle, layer_begin, layer_end, path, accept_len, kv_len, block_table, kv_len_out
    Args g(args, nargs, 8);
    vispec_ctx* c = g.ctx();
    const int lb = g.num(), le = g.num();
    const at::Tensor* t = g.tensor(2);
    const int B = size(t, 0), N = size(t, 1);
    auto* path = g.ptr<int32_t>(); auto* alen = g.ptr<int32_t>(); auto* kv_len = g.ptr<int32_t>();
    const int stride = size(g.tensor(2), 1);
    auto* table = g.ptr<int32_t>(); auto* out = g.ptr<int32_t>();
    return finish(g, [&](void* st) { return vispec_kv_compact_paged(c, lb, le, path, alen, kv_len, table, stride, out, B, N, st); });
}

NATIVE(accept_sampled) {  // handle, draft_ids, parents, p_target, p_draft, u_accept, u_bonus, path, accept_len, bonus
    Args g(args, nargs, 10);
    vispec_ctx* c = g.ctx();
    auto* draft = g.ptr<int32_t>(); auto* parents = g.ptr<int32_t>();
    const at::Tensor* t = g.tensor(3);
    const int B = size(t, 0), N = size(t, 1), V = size(t, 2);
    auto* p = g.ptr<float>(); auto* ph = g.ptr<float>(); auto* ua = g.ptr<float>(); auto* ub = g.ptr<float>();
    auto* path = g.ptr<int32_t>(); auto* alen = g.ptr<int32_t>(); auto* bonus = g.ptr<int32_t>();
    return finish(g, [&](void* st) { return vispec_accept_sampled(c, draft, parents, p, ph, ua, ub, B, N, V, path, alen, bonus, st); });
}

NATIVE(tree_rerank) {  // handle, cand_parent, cand_token, cand_score, K, parents, draft_ids, selected
    Args g(args, nargs, 8);
    vispec_ctx* c = g.ctx();
    const at::Tensor* t = g.tensor(2);
    const int B = size(t, 0), M = size(t, 1);
    auto* cp = g.ptr<int32_t>(); auto* ct = g.ptr<int32_t>(); auto* cs = g.ptr<float>();
    const int K = g.num();
    auto* parents = g.ptr<int32_t>(); auto* ids = g.ptr<int32_t>(); auto* sel = g.ptr<int32_t>();
    return finish(g, [&](void* st) { return vispec_tree_rerank(c, cp, ct, cs, B, M, K, parents, ids, sel, st); });
}

// handle, Hq, Hkv, D, q, k, positions, axes, q_out, k_out
NATIVE(rope_axes_rows) {
    Args g(args, nargs, 10);
    vispec_ctx* c = g.ctx();
    const int Hq = g.num(), Hkv = g.num(), D = g.num();
    int64_t T = -1;
    const auto q = g.rows(T, Hq, D), k = g.rows(T, Hkv, D);
    if (g.ok && T < 0) { PyErr_SetString(PyExc_TypeError, "q, k or both are tensors"); g.ok = false; }
    if (g.ok) g.i = 7;                     // the axes say how many positions there are
    const vispec_rope_axes* axes = g.axes();
    const auto qo = g.rows(T, Hq, D), ko = g.rows(T, Hkv, D);
    if (g.ok) g.i = 6;
    auto* pos = axes ? g.ints({axes->n_axes, T}) : g.ints({});
    return finish(g, [&](void* st) { return vispec_rope_axes_rows(c, q.p, q.stride, k.p, k.stride, pos, (int)T, axes, qo.p, qo.stride, ko.p, ko.stride, st); });
}

// handle, Hq, Hkv, D, layer, q, k_new, v_new, positions, axes, cu_len, kv_len, [block_table,] q_out, kv_len_out
template <bool PAGED>
PyObject* kv_append_call(PyObject* const* args, Py_ssize_t nargs) {
    Args g(args, nargs, PAGED ? 15 : 14);
    vispec_ctx* c = g.ctx();
    const int Hq = g.num(), Hkv = g.num(), D = g.num(), layer = g.num();
    int64_t T = -1;
    if (g.ok) g.i = 6;
    const auto k = g.rows(T, Hkv, D), v = g.rows(T, Hkv, D);
    if (g.ok && (T < 0)) { PyErr_SetString(PyExc_TypeError, "k_new and v_new are tensors"); g.ok = false; }
    if (g.ok) g.i = 5;
    const auto q = g.rows(T, Hq, D);
    if (g.ok) g.i = 9;
    const vispec_rope_axes* axes = g.axes();
    if (g.ok) g.i = 8;
    auto* pos = axes ? g.ints({axes->n_axes, T}, true) : g.ints({}, true);
    if (g.ok) g.i = 11;
    const at::Tensor* tl = g.tensor(1);
    const int B = tl ? (int)tl->size(0) : 0;
    if (g.ok) g.i = 10;
    auto* cu = g.ints({B + 1});
    auto* kv_len = g.ints({B});
    int stride = 0;
    int32_t* table = nullptr;
    if (PAGED) {
        const at::Tensor* tt = g.tensor(2);
        stride = tt ? (int)tt->size(1) : 0;
        table = g.ints({B, stride});
    }
    const auto qo = g.rows(T, Hq, D);
    auto* len_out = g.ints({B}, true);
    return finish(g, [&](void* st) {
        return PAGED ? vispec_kv_append_paged(c, layer, q.p, q.stride, k.p, k.stride, v.p, v.stride, pos, axes, cu, kv_len, table, stride, B, (int)T, qo.p, qo.stride, len_out, st)
                     : vispec_kv_append(c, layer, q.p, q.stride, k.p, k.stride, v.p, v.stride, pos, axes, cu, kv_len, B, (int)T, qo.p, qo.stride, len_out, st);
    });
}
NATIVE(kv_append) { return kv_append_call<false>(args, nargs); }
NATIVE(kv_append_paged) { return kv_append_call<true>(args, nargs); }

// handle, Hq, Hkv, D, layer, q, kv_len, block_table, prefix_len, tree_mask, scale, scratch, out, lse
NATIVE(tree_verify_attn_prefix_paged) {
    Args g(args, nargs, 14);
    vispec_ctx* c = g.ctx();
    const int Hq = g.num(), Hkv = g.num(), D = g.num(), layer = g.num();
    (void)Hkv;
    const at::Tensor* t = g.tensor(4);
    const int64_t B = size(t, 0), N = size(t, 1);
    auto* q = g.dense(at::kBFloat16, {B, N, Hq, D});
    auto* kv_len = g.ints({B});
    const int stride = size(g.tensor(2), 1);
    auto* table = g.ints({B, stride});
    const int prefix = g.num();
    auto* mask = static_cast<uint64_t*>(g.dense(at::kLong, {B, N, (N + 63) / 64}));
    const float scale = g.real();
    const at::Tensor* ts = g.tensor(1);
    auto* scratch = g.dense(at::kByte, {});
    const size_t bytes = ts ? (size_t)ts->numel() : 0;
    auto* out = g.dense(at::kBFloat16, {B, N, Hq, D});
    auto* lse = static_cast<float*>(g.dense(at::kFloat, {B, Hq, N}, true));
    return finish(g, [&](void* st) { return vispec_tree_verify_attn_prefix_paged(c, layer, q, kv_len, table, stride, prefix, mask, (int)B, (int)N, scale, scratch, bytes, out, lse, st); });
}

#define ENTRY(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(guarded<name>)), METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {
    ENTRY(tree_mask_build), ENTRY(tree_verify_attn), ENTRY(tree_verify_attn_rope), ENTRY(tree_verify_attn_paged),
    ENTRY(tree_verify_attn_static), ENTRY(rope_table_build), ENTRY(rope_tree_rows), ENTRY(rope_tree_rows_paged),
    ENTRY(accept), ENTRY(accept_commit), ENTRY(accept_commit_paged), ENTRY(kv_compact), ENTRY(kv_compact_paged),
    ENTRY(accept_sampled), ENTRY(tree_rerank), ENTRY(rope_axes_rows), ENTRY(kv_append), ENTRY(kv_append_paged),
    ENTRY(tree_verify_attn_prefix_paged), {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_native", "Hot calls of libvispec without ctypes", -1, kMethods,
                       nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native() { return PyModule_Create(&kModule); }
