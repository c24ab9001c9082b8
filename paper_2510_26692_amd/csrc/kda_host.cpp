// The decode calls of the Python binding (kda.py), those of the softmax-attention layers (attn.py) and those of draft trees and shared pages (tree.py), marshalled natively: a decode step of one sequence takes the device 4 us, and the
// checks, descriptors and ctypes of the general path 10 us of the host (measured in a loop of kda_recurrent_step, 1 sequence x 32
// heads: 9.9 us a call through kda.py alone, 4.2 to 5.0 here; kda_cache_append of one token 17 and 5.2).
//
// Only calls that are regular in every respect are taken: plain contiguous device tensors of the expected types and shapes on
// one device.  For anything else, and for whatever cannot be told here, the functions return None, and kda.py's own path decides
// and words the error.  A status other than KDA_OK comes back as a number, which kda.py raises.  Nothing is kept between calls
// but the addresses of the library's entry points, and the entry points are handed over by kda.py, so that both ways call the
// same library.
#include <Python.h>

#include <cmath>

#include <ATen/ATen.h>
#include <c10/core/DeviceGuard.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include "kda.h"

namespace {

decltype(&kda_recurrent_step) step_entry;
decltype(&kda_recurrent_steps) steps_entry;
decltype(&kda_cache_append) append_entry;
decltype(&kda_cache_attn) attend_entry;
decltype(&kda_cache_attn_workspace_size) attend_size_entry;
decltype(&kda_window_attn_fwd) fwd_entry;
decltype(&kda_window_attn_bwd) bwd_entry;
decltype(&kda_window_attn_bwd_workspace_size) bwd_size_entry;
decltype(&kda_rotate) rotate_entry;
decltype(&kda_cache_tree_attn) tree_attend_entry;
decltype(&kda_cache_tree_attn_workspace_size) tree_attend_size_entry;
decltype(&kda_cache_keep) keep_entry;
decltype(&kda_cache_copy_pages) copy_entry;
decltype(&kda_tree_steps) tree_steps_entry;
decltype(&kda_tree_commit) tree_commit_entry;
decltype(&kda_pages_fork) fork_entry;
decltype(&kda_pages_reserve) reserve_entry;
decltype(&kda_pages_reserve_workspace_size) reserve_size_entry;
PyObject *raw_stream;                                        // device index -> current stream, as a number

struct Irregular {};

// A tensor argument: exactly torch's own class, with memory of its own and nothing (vmap, a tracer) wrapped around it.
const at::Tensor &plain(PyObject *x)
{
    if (!THPVariable_CheckExact(x)) throw Irregular{};
    const at::Tensor &t = THPVariable_Unpack(x);
    using K = c10::DispatchKey;
    static const c10::DispatchKeySet wrapped({K::Python, K::PythonTLSSnapshot, K::Fake, K::Functionalize, K::FuncTorchBatched,
                                              K::FuncTorchGradWrapper, K::Conjugate, K::Negative, K::ZeroTensor});
    if (t.key_set().has_any(wrapped) || !t.has_storage()) throw Irregular{};
    return t;
}

struct Checked {
    c10::DeviceIndex device;
    explicit Checked(const at::Tensor &t) : device(t.device().index()) {}
    const at::Tensor &operator()(const at::Tensor &t, at::ScalarType type, at::IntArrayRef shape) const
    {
        if (!t.is_cuda() || t.device().index() != device || t.scalar_type() != type || t.sizes() != shape || !t.is_contiguous())
            throw Irregular{};
        return t;
    }
    const at::Tensor &operator()(PyObject *x, at::ScalarType type, at::IntArrayRef shape) const { return (*this)(plain(x), type, shape); }
};

// The device that launches go to, for as long as this lives.  (A guard that sets a device which is current already costs 0.1 us.)
class Current {
    c10::OptionalDeviceGuard guard;
public:
    explicit Current(c10::Device device)
    {
        if (c10::impl::VirtualGuardImpl(device.type()).getDevice() != device) guard.reset_device(device);
    }
};

float number(PyObject *x)
{
    if (PyFloat_CheckExact(x)) return (float)PyFloat_AS_DOUBLE(x);
    if (PyLong_CheckExact(x)) return (float)PyLong_AsDouble(x);
    throw Irregular{};
}

int code(at::ScalarType t)
{
    if (t == at::kFloat) return KDA_F32;
    if (t == at::kBFloat16) return KDA_BF16;
    throw Irregular{};
}

// o as the caller passed it, or a fresh one
at::Tensor output(PyObject *o, PyObject *out_dtype, const at::Tensor &v, const Checked &check)
{
    at::ScalarType type = at::kFloat;
    if (o != Py_None) type = plain(o).scalar_type();
    if (out_dtype != Py_None) {
        if (!THPDtype_Check(out_dtype)) throw Irregular{};
        const at::ScalarType asked = reinterpret_cast<THPDtype *>(out_dtype)->scalar_type;
        if (o != Py_None && asked != type) throw Irregular{};
        type = asked;
    }
    (void)code(type);
    if (o != Py_None) return check(o, type, v.sizes());
    return at::empty(v.sizes(), v.options().dtype(type));
}

void *stream_of(c10::DeviceIndex device)
{
    PyObject *index = PyLong_FromLong(device), *s = index ? PyObject_CallOneArg(raw_stream, index) : nullptr;
    Py_XDECREF(index);
    void *p = s ? PyLong_AsVoidPtr(s) : nullptr;
    Py_XDECREF(s);
    if (PyErr_Occurred()) { PyErr_Clear(); throw Irregular{}; }
    return p;
}

PyObject *finish(kda_status st, PyObject *o, const at::Tensor &out)
{
    if (st != KDA_OK) return PyLong_FromLong((long)st);
    if (o != Py_None) { Py_INCREF(o); return o; }
    return THPVariable_Wrap(out);
}

template <typename F> PyObject *guarded(F &&f)
{
    try {
        return f();
    } catch (...) {                                          // (whatever it was: kda.py meets it again, and says so)
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

kda_dims decode_dims(int64_t N, int64_t tokens, int64_t H, int64_t dk, int64_t dv, int in, int out, float scale)
{
    if (N > 0x7fffffff || H > 0x7fffffff || dk > 0x7fffffff || dv > 0x7fffffff) throw Irregular{};
    kda_dims d{};
    d.batch = (int32_t)N; d.seqlen = tokens; d.heads = (int32_t)H; d.dk = (int32_t)dk; d.dv = (int32_t)dv; d.chunk = 64;
    d.num_seqs = (int32_t)N; d.in_dtype = (kda_dtype)in; d.out_dtype = (kda_dtype)out; d.scale = scale;
    return d;
}

// step(q, k, v, log_alpha, beta, S, scale, o, out_dtype)
PyObject *step(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        if (n != 9 || !step_entry) throw Irregular{};
        const at::Tensor &q = plain(a[0]);
        if (q.dim() != 3) throw Irregular{};
        const at::Tensor &v = plain(a[2]);
        if (v.dim() != 3) throw Irregular{};
        const int64_t N = q.size(0), H = q.size(1), dk = q.size(2), dv = v.size(2);
        const at::ScalarType type = q.scalar_type();
        const Checked check(q);
        check(q, type, {N, H, dk});
        const at::Tensor &k = check(a[1], type, {N, H, dk});
        check(v, type, {N, H, dv});
        const at::Tensor &la = check(a[3], type, {N, H, dk}), &beta = check(a[4], type, {N, H});
        const at::Tensor &S = check(a[5], at::kFloat, {N, H, dk, dv});
        const int in = code(type);
        const float scale = number(a[6]);
        const at::Tensor o = output(a[7], a[8], v, check);
        const kda_dims d = decode_dims(N, 1, H, dk, dv, in, code(o.scalar_type()), scale);
        const Current on(q.device());
        void *stream = stream_of(check.device);
        kda_status st;
        Py_BEGIN_ALLOW_THREADS
        st = step_entry(&d, q.data_ptr(), k.data_ptr(), v.data_ptr(), la.data_ptr(), beta.data_ptr(), static_cast<float *>(S.data_ptr()),
                        o.data_ptr(), stream);
        Py_END_ALLOW_THREADS
        return finish(st, a[7], o);
    });
}

// steps(q, k, v, log_alpha, beta, S_pool, state_indices, scale, o, out_dtype, form, l2norm_eps, a_scale, dt_bias, out_gate, norm_weight, rms_eps)
// form: 0 plain, 1 scalar gate, 2 fused stages with the prologue, 3 without
PyObject *steps(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        if (n != 17 || !steps_entry) throw Irregular{};
        const long form = PyLong_CheckExact(a[10]) ? PyLong_AsLong(a[10]) : -1;
        if (form < 0 || form > 3) throw Irregular{};
        const at::Tensor &q = plain(a[0]);
        if (q.dim() != 4) throw Irregular{};
        const at::Tensor &v = plain(a[2]);
        if (v.dim() != 4) throw Irregular{};
        const int64_t N = q.size(0), T = q.size(1), H = q.size(2), dk = q.size(3), dv = v.size(3);
        const at::ScalarType type = q.scalar_type();
        const Checked check(q);
        check(q, type, {N, T, H, dk});
        const at::Tensor &k = check(a[1], type, {N, T, H, dk});
        check(v, type, {N, T, H, dv});
        const at::Tensor &la = form == 1 ? check(a[3], type, {N, T, H}) : check(a[3], type, {N, T, H, dk});
        const at::Tensor &beta = check(a[4], type, {N, T, H}), &S = plain(a[5]);
        if (S.dim() != 4) throw Irregular{};
        check(S, at::kFloat, {S.size(0), H, dk, dv});
        const int32_t *indices = nullptr;
        if (a[6] != Py_None) indices = static_cast<const int32_t *>(check(a[6], at::kInt, {N}).data_ptr());
        else if (S.size(0) < N) throw Irregular{};
        const int in = code(type);
        const float scale = number(a[7]);
        kda_prologue pro{};
        kda_epilogue epi{};
        const bool gated = form >= 2 && a[14] != Py_None;
        if (form == 2) {
            pro.l2norm_eps = number(a[11]);
            if (a[12] != Py_None) pro.a_scale = static_cast<const float *>(check(a[12], at::kFloat, {H}).data_ptr());
            if (a[13] != Py_None) pro.dt_bias = static_cast<const float *>(check(a[13], at::kFloat, {H, dk}).data_ptr());
        }
        if (gated) {
            epi.rms_eps = number(a[16]);
            epi.gate = check(a[14], type, v.sizes()).data_ptr();
            if (a[15] != Py_None) epi.norm_weight = static_cast<const float *>(check(a[15], at::kFloat, {dv}).data_ptr());
        }
        const at::Tensor o = output(a[8], a[9], v, check);
        const kda_dims d = decode_dims(N, T, H, dk, dv, in, code(o.scalar_type()), scale);
        const uint32_t flags = (form == 1 ? KDA_STEPS_SCALAR_GATE : 0) | (a[8] == Py_None ? KDA_STEPS_ZERO_SKIPPED : 0);
        const Current on(q.device());
        void *stream = stream_of(check.device);
        kda_status st;
        Py_BEGIN_ALLOW_THREADS
        st = steps_entry(&d, form == 2 ? &pro : nullptr, gated ? &epi : nullptr, q.data_ptr(), k.data_ptr(), v.data_ptr(), la.data_ptr(),
                         beta.data_ptr(), static_cast<float *>(S.data_ptr()), indices, o.data_ptr(), flags, stream);
        Py_END_ALLOW_THREADS
        return finish(st, a[8], o);
    });
}

int64_t whole(PyObject *x)
{
    if (!PyLong_CheckExact(x)) throw Irregular{};
    const int64_t v = PyLong_AsLongLong(x);
    if (v == -1 && PyErr_Occurred()) throw Irregular{};
    return v;
}
bool truth(PyObject *x)
{
    if (x != Py_True && x != Py_False) throw Irregular{};
    return x == Py_True;
}
int32_t narrow(int64_t n)
{
    if (n < 0 || n > 0x7fffffff) throw Irregular{};
    return (int32_t)n;
}
float attn_scale(PyObject *x, int64_t dim) { return x == Py_None ? (float)(1.0 / std::sqrt((double)dim)) : number(x); }
at::Tensor bytes(size_t n, const at::Tensor &like) { return at::empty({(int64_t)n}, like.options().dtype(at::kByte)); }

// The cache's arguments a[0..5]: k_cache, v_cache, k_scale, v_scale, block_table, kv_lens.
kda_cache cache_of(PyObject *const *a, const Checked &check, int64_t N, int64_t Hq, int64_t Hk, int64_t d)
{
    const at::Tensor &k = plain(a[0]), &table = plain(a[4]);
    if (k.dim() != 4 || table.dim() != 2) throw Irregular{};
    const int64_t P = k.size(0), page = k.size(2);
    check(k, at::kFloat8_e4m3fn, {P, Hk, page, d});
    check(table, at::kInt, {N, table.size(1)});
    kda_cache c{};
    c.num_seqs = narrow(N); c.heads_q = narrow(Hq); c.heads_kv = narrow(Hk); c.dim = narrow(d); c.page_size = narrow(page);
    c.num_pages = P; c.max_pages = narrow(table.size(1));
    c.k = k.data_ptr(); c.v = check(a[1], at::kFloat8_e4m3fn, k.sizes()).data_ptr();
    c.k_scale = static_cast<float *>(check(a[2], at::kFloat, {P, Hk}).data_ptr());
    c.v_scale = static_cast<float *>(check(a[3], at::kFloat, {P, Hk}).data_ptr());
    c.block_table = static_cast<const int32_t *>(table.data_ptr());
    c.kv_lens = static_cast<const int32_t *>(check(a[5], at::kInt, {N}).data_ptr());
    return c;
}

// (the first of two results and the second, None where there is none)
PyObject *pair(kda_status st, PyObject *given0, const at::Tensor &t0, PyObject *given1, const at::Tensor &t1)
{
    if (st != KDA_OK) return PyLong_FromLong((long)st);
    auto object = [](PyObject *given, const at::Tensor &t) -> PyObject * {
        if (given == Py_None && t.defined()) return THPVariable_Wrap(t);
        Py_INCREF(given);
        return given;
    };
    PyObject *a = object(given0, t0), *b = a ? object(given1, t1) : nullptr, *r = b ? PyTuple_Pack(2, a, b) : nullptr;
    Py_XDECREF(a);
    Py_XDECREF(b);
    if (!r) throw Irregular{};
    return r;
}

// append(k, v, k_cache, v_cache, k_scale, v_scale, block_table, kv_lens, cu_seqlens, inv_freq, interleaved, q, q_out, k_out, want_k)
PyObject *append(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        if (n != 15 || !append_entry) throw Irregular{};
        const at::Tensor &k = plain(a[0]);
        if (k.dim() != 4) throw Irregular{};
        const int64_t B = k.size(0), T = k.size(1), Hk = k.size(2), d = k.size(3);
        const Checked check(k);
        check(k, at::kBFloat16, {B, T, Hk, d});
        const at::Tensor &v = check(a[1], at::kBFloat16, k.sizes());
        int64_t N = B, Hq = Hk;
        const int32_t *cu = nullptr;
        if (a[8] != Py_None) {
            const at::Tensor &t = plain(a[8]);
            if (t.dim() != 1 || t.size(0) < 1 || B != 1) throw Irregular{};
            cu = static_cast<const int32_t *>(check(t, at::kInt, t.sizes()).data_ptr());
            N = t.size(0) - 1;
        }
        at::Tensor q, q_out, k_out;
        uint32_t flags = 0;
        if (a[11] != Py_None) {
            q = plain(a[11]);
            if (q.dim() != 4) throw Irregular{};
            Hq = q.size(2);
            check(q, at::kBFloat16, {B, T, Hq, d});
            if (a[12] != Py_None) q_out = check(a[12], at::kBFloat16, q.sizes());
            else { q_out = at::empty(q.sizes(), q.options()); flags |= KDA_APPEND_ZERO_Q; }
        } else if (a[12] != Py_None) {
            throw Irregular{};
        }
        if (a[13] != Py_None) k_out = check(a[13], at::kBFloat16, k.sizes());
        else if (truth(a[14])) { k_out = at::empty(k.sizes(), k.options()); flags |= KDA_APPEND_ZERO_K; }
        const kda_cache c = cache_of(a + 2, check, N, Hq, Hk, d);
        kda_rope rope{};
        if (a[9] != Py_None) {
            const at::Tensor &f = plain(a[9]);
            if (f.dim() != 1) throw Irregular{};
            rope.inv_freq = static_cast<const float *>(check(f, at::kFloat, f.sizes()).data_ptr());
            rope.num_freqs = narrow(f.size(0));
            rope.interleaved = truth(a[10]);
        }
        const Current on(k.device());
        void *stream = stream_of(check.device);
        kda_status st;
        Py_BEGIN_ALLOW_THREADS
        st = append_entry(&c, T, k.data_ptr(), v.data_ptr(), 0, 0, cu, a[9] != Py_None ? &rope : nullptr, k_out.defined() ? k_out.data_ptr() : nullptr,
                          q.defined() ? q.data_ptr() : nullptr, 0, q_out.defined() ? q_out.data_ptr() : nullptr, flags, stream);
        Py_END_ALLOW_THREADS
        return pair(st, a[12], q_out, a[13], k_out);
    });
}

// attend(q, k_cache, v_cache, k_scale, v_scale, block_table, kv_lens, window, sinks, scale, max_kv_len, o, out_dtype)
PyObject *attend(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        if (n != 13 || !attend_entry) throw Irregular{};
        const at::Tensor &q = plain(a[0]), &kc = plain(a[1]);
        if (q.dim() != 4 || kc.dim() != 4) throw Irregular{};
        const int64_t N = q.size(0), T = q.size(1), Hq = q.size(2), d = q.size(3);
        const Checked check(q);
        check(q, at::kBFloat16, {N, T, Hq, d});
        const kda_cache c = cache_of(a + 1, check, N, Hq, kc.size(1), d);
        const at::Tensor o = output(a[11], a[12], q, check);
        kda_cache_query query{};
        query.tokens = narrow(T); query.window = whole(a[7]); query.sinks = narrow(whole(a[8])); query.scale = attn_scale(a[9], d);
        query.max_kv_len = whole(a[10]); query.out_dtype = (kda_dtype)code(o.scalar_type());
        const size_t need = attend_size_entry(&c, &query);
        const at::Tensor ws = need ? bytes(need, q) : at::Tensor();
        const Current on(q.device());
        void *stream = stream_of(check.device);
        kda_status st;
        Py_BEGIN_ALLOW_THREADS
        st = attend_entry(&c, &query, q.data_ptr(), o.data_ptr(), need ? ws.data_ptr() : nullptr, need, stream);
        Py_END_ALLOW_THREADS
        return finish(st, a[11], o);
    });
}

// The dims of a fixed batch.
kda_attn_dims attn_dims(const at::Tensor &q, const at::Tensor &k, const Checked &check, PyObject *window, PyObject *sinks, PyObject *scale, int out)
{
    kda_attn_dims d{};
    check(q, at::kBFloat16, q.sizes());
    check(k, at::kBFloat16, {q.size(0), q.size(1), k.size(2), q.size(3)});
    d.batch = d.num_seqs = narrow(q.size(0)); d.seqlen = q.size(1); d.heads_q = narrow(q.size(2)); d.heads_kv = narrow(k.size(2)); d.dim = narrow(q.size(3));
    d.in_dtype = KDA_BF16; d.out_dtype = (kda_dtype)out; d.scale = attn_scale(scale, q.size(3)); d.window = whole(window); d.sinks = narrow(whole(sinks));
    return d;
}

// window_fwd(q, k, v, window, sinks, scale, o, lse, want_lse, out_dtype): a fixed batch
PyObject *window_fwd(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        if (n != 10 || !fwd_entry) throw Irregular{};
        const at::Tensor &q = plain(a[0]), &k = plain(a[1]);
        if (q.dim() != 4 || k.dim() != 4) throw Irregular{};
        const Checked check(q);
        const at::Tensor o = output(a[6], a[9], q, check);
        const kda_attn_dims d = attn_dims(q, k, check, a[3], a[4], a[5], code(o.scalar_type()));
        const at::Tensor &v = check(a[2], at::kBFloat16, k.sizes());
        at::Tensor lse;
        if (a[7] != Py_None) lse = check(a[7], at::kFloat, {q.size(0), q.size(2), q.size(1)});
        else if (truth(a[8])) lse = at::empty({q.size(0), q.size(2), q.size(1)}, q.options().dtype(at::kFloat));
        const Current on(q.device());
        void *stream = stream_of(check.device);
        kda_status st;
        Py_BEGIN_ALLOW_THREADS
        st = fwd_entry(&d, q.data_ptr(), k.data_ptr(), v.data_ptr(), nullptr, o.data_ptr(), lse.defined() ? static_cast<float *>(lse.data_ptr()) : nullptr, stream);
        Py_END_ALLOW_THREADS
        return pair(st, a[6], o, a[7], lse);
    });
}

// window_bwd(q, k, v, o, lse, do, window, sinks, scale): a fixed batch; (dq, dk, dv)
PyObject *window_bwd(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        if (n != 9 || !bwd_entry) throw Irregular{};
        const at::Tensor &q = plain(a[0]), &k = plain(a[1]);
        if (q.dim() != 4 || k.dim() != 4) throw Irregular{};
        const Checked check(q);
        const kda_attn_dims d = attn_dims(q, k, check, a[6], a[7], a[8], KDA_BF16);
        const at::Tensor &v = check(a[2], at::kBFloat16, k.sizes()), &o = check(a[3], at::kBFloat16, q.sizes());
        const at::Tensor &lse = check(a[4], at::kFloat, {q.size(0), q.size(2), q.size(1)}), &d_o = check(a[5], at::kBFloat16, q.sizes());
        const at::Tensor dq = at::empty(q.sizes(), q.options()), dk = at::empty(k.sizes(), k.options()), dv = at::empty(k.sizes(), k.options());
        const size_t need = bwd_size_entry(&d);
        const at::Tensor ws = bytes(need ? need : 256, q);
        const Current on(q.device());
        void *stream = stream_of(check.device);
        kda_status st;
        Py_BEGIN_ALLOW_THREADS
        st = bwd_entry(&d, q.data_ptr(), k.data_ptr(), v.data_ptr(), nullptr, o.data_ptr(), static_cast<const float *>(lse.data_ptr()), d_o.data_ptr(),
                       dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), ws.data_ptr(), need ? need : 256, stream);
        Py_END_ALLOW_THREADS
        if (st != KDA_OK) return PyLong_FromLong((long)st);
        PyObject *r = PyTuple_New(3);
        if (!r) throw Irregular{};
        int i = 0;
        for (const at::Tensor &t : {dq, dk, dv}) {
            PyObject *w = THPVariable_Wrap(t);
            if (!w) { Py_DECREF(r); throw Irregular{}; }
            PyTuple_SET_ITEM(r, i++, w);
        }
        return r;
    });
}

const int32_t *int32s(PyObject *x, const Checked &check, at::IntArrayRef shape) { return static_cast<const int32_t *>(check(x, at::kInt, shape).data_ptr()); }
PyObject *nothing(kda_status st)
{
    if (st != KDA_OK) return PyLong_FromLong((long)st);
    Py_RETURN_TRUE;                                          // (None is a call that this way leaves to the other)
}

// rotate(q, k, positions, inv_freq, axes, interleaved, inverse, q_out, k_out); axes: None or bytes
PyObject *rotate(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        if (n != 9 || !rotate_entry) throw Irregular{};
        const at::Tensor &q = plain(a[0]), &pos = plain(a[2]), &f = plain(a[3]);
        if (q.dim() != 4 || f.dim() != 1 || (pos.dim() != 2 && pos.dim() != 3)) throw Irregular{};
        const Checked check(q);
        const at::ScalarType type = q.scalar_type();
        check(q, type, q.sizes());
        const int64_t B = q.size(0), T = q.size(1);
        kda_rotation r{};
        r.batch = narrow(B); r.seqlen = T; r.heads_q = narrow(q.size(2)); r.dim = narrow(q.size(3)); r.dtype = (kda_dtype)code(type);
        at::Tensor k, q_out, k_out;
        if (a[1] != Py_None) {
            k = plain(a[1]);
            if (k.dim() != 4) throw Irregular{};
            check(k, type, {B, T, k.size(2), q.size(3)});
            r.heads_k = narrow(k.size(2));
            k_out = a[8] != Py_None ? check(a[8], type, k.sizes()) : at::empty(k.sizes(), k.options());
        } else if (a[8] != Py_None) {
            throw Irregular{};
        }
        q_out = a[7] != Py_None ? check(a[7], type, q.sizes()) : at::empty(q.sizes(), q.options());
        r.axes = pos.dim() == 3 ? narrow(pos.size(0)) : 1;
        if (pos.dim() == 3) check(pos, at::kInt, {r.axes, B, T});
        else check(pos, at::kInt, {B, T});
        r.num_freqs = narrow(f.size(0));
        r.inv_freq = static_cast<const float *>(check(f, at::kFloat, f.sizes()).data_ptr());
        if (a[4] != Py_None) {
            if (!PyBytes_CheckExact(a[4]) || PyBytes_GET_SIZE(a[4]) != r.num_freqs) throw Irregular{};
            r.axis_of_freq = reinterpret_cast<const uint8_t *>(PyBytes_AS_STRING(a[4]));
        }
        r.interleaved = truth(a[5]);
        r.inverse = truth(a[6]);
        const Current on(q.device());
        void *stream = stream_of(check.device);
        kda_status st;
        Py_BEGIN_ALLOW_THREADS
        st = rotate_entry(&r, q.data_ptr(), k.defined() ? k.data_ptr() : nullptr, static_cast<const int32_t *>(pos.data_ptr()), q_out.data_ptr(),
                          k_out.defined() ? k_out.data_ptr() : nullptr, stream);
        Py_END_ALLOW_THREADS
        return pair(st, a[7], q_out, a[8], k_out);
    });
}

// tree_attend(q, k_cache, v_cache, k_scale, v_scale, block_table, kv_lens, parents, window, sinks, scale, max_kv_len, o, out_dtype)
PyObject *tree_attend(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        if (n != 14 || !tree_attend_entry) throw Irregular{};
        const at::Tensor &q = plain(a[0]), &kc = plain(a[1]);
        if (q.dim() != 4 || kc.dim() != 4) throw Irregular{};
        const int64_t N = q.size(0), T = q.size(1), Hq = q.size(2), d = q.size(3);
        const Checked check(q);
        check(q, at::kBFloat16, {N, T, Hq, d});
        const kda_cache c = cache_of(a + 1, check, N, Hq, kc.size(1), d);
        const int32_t *parents = int32s(a[7], check, {N, T});
        const at::Tensor o = output(a[12], a[13], q, check);
        kda_cache_query query{};
        query.tokens = narrow(T); query.window = whole(a[8]); query.sinks = narrow(whole(a[9])); query.scale = attn_scale(a[10], d);
        query.max_kv_len = whole(a[11]); query.out_dtype = (kda_dtype)code(o.scalar_type());
        const size_t need = tree_attend_size_entry(&c, &query);
        const at::Tensor ws = need ? bytes(need, q) : at::Tensor();
        const Current on(q.device());
        void *stream = stream_of(check.device);
        kda_status st;
        Py_BEGIN_ALLOW_THREADS
        st = tree_attend_entry(&c, &query, q.data_ptr(), parents, o.data_ptr(), need ? ws.data_ptr() : nullptr, need, stream);
        Py_END_ALLOW_THREADS
        return finish(st, a[12], o);
    });
}

// A layer's or a stack's cache a[0..3], and its layers.
kda_cache stack_of(PyObject *const *a, const at::Tensor &k, const Checked &check, int32_t &layers)
{
    if (k.dim() != 4 && k.dim() != 5) throw Irregular{};
    const int at = k.dim() - 4;
    layers = at ? narrow(k.size(0)) : 1;
    check(k, at::kFloat8_e4m3fn, k.sizes());
    kda_cache c{};
    c.num_pages = k.size(at); c.heads_q = c.heads_kv = narrow(k.size(at + 1)); c.page_size = narrow(k.size(at + 2)); c.dim = narrow(k.size(at + 3));
    c.k = k.data_ptr(); c.v = check(a[1], at::kFloat8_e4m3fn, k.sizes()).data_ptr();
    c.k_scale = static_cast<float *>(check(a[2], at::kFloat, k.sizes().slice(0, at + 2)).data_ptr());
    c.v_scale = static_cast<float *>(check(a[3], at::kFloat, k.sizes().slice(0, at + 2)).data_ptr());
    return c;
}

// keep(k_cache, v_cache, k_scale, v_scale, block_table, kv_lens, kept)
PyObject *keep(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        if (n != 7 || !keep_entry) throw Irregular{};
        const at::Tensor &k = plain(a[0]), &table = plain(a[4]), &kept = plain(a[6]);
        if (table.dim() != 2 || kept.dim() != 2) throw Irregular{};
        const Checked check(k);
        int32_t layers;
        kda_cache c = stack_of(a, k, check, layers);
        const int64_t N = table.size(0);
        c.num_seqs = narrow(N); c.max_pages = narrow(table.size(1));
        c.block_table = int32s(a[4], check, {N, table.size(1)});
        c.kv_lens = int32s(a[5], check, {N});
        const int32_t *path = int32s(a[6], check, {N, kept.size(1)});
        const Current on(k.device());
        void *stream = stream_of(check.device);
        kda_status st;
        Py_BEGIN_ALLOW_THREADS
        st = keep_entry(&c, layers, path, narrow(kept.size(1)), stream);
        Py_END_ALLOW_THREADS
        return nothing(st);
    });
}

// copy_pages(k_cache, v_cache, k_scale, v_scale, pairs)
PyObject *copy_pages(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        if (n != 5 || !copy_entry) throw Irregular{};
        const at::Tensor &k = plain(a[0]), &pairs = plain(a[4]);
        if (pairs.dim() != 2) throw Irregular{};
        const Checked check(k);
        int32_t layers;
        const kda_cache c = stack_of(a, k, check, layers);
        const int32_t *list = int32s(a[4], check, {pairs.size(0), 2});
        const Current on(k.device());
        void *stream = stream_of(check.device);
        kda_status st;
        Py_BEGIN_ALLOW_THREADS
        st = copy_entry(&c, layers, list, pairs.size(0), stream);
        Py_END_ALLOW_THREADS
        return nothing(st);
    });
}

// fork(block_table, page_refs, source)
PyObject *fork_rows(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        if (n != 3 || !fork_entry) throw Irregular{};
        const at::Tensor &table = plain(a[0]), &refs = plain(a[1]);
        if (table.dim() != 2 || refs.dim() != 1) throw Irregular{};
        const Checked check(table);
        check(table, at::kInt, table.sizes());
        check(refs, at::kInt, refs.sizes());
        const int32_t *source = int32s(a[2], check, {table.size(0)});
        const Current on(table.device());
        void *stream = stream_of(check.device);
        kda_status st;
        Py_BEGIN_ALLOW_THREADS
        st = fork_entry(static_cast<int32_t *>(table.data_ptr()), narrow(table.size(0)), narrow(table.size(1)), static_cast<int32_t *>(refs.data_ptr()),
                        refs.size(0), source, stream);
        Py_END_ALLOW_THREADS
        return nothing(st);
    });
}

// reserve(block_table, kv_lens, new_lens, page_refs, page_size, copies, missing)
PyObject *reserve(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        if (n != 7 || !reserve_entry) throw Irregular{};
        const at::Tensor &table = plain(a[0]), &refs = plain(a[3]);
        if (table.dim() != 2 || refs.dim() != 1) throw Irregular{};
        const Checked check(table);
        check(table, at::kInt, table.sizes());
        check(refs, at::kInt, refs.sizes());
        const int64_t N = table.size(0);
        const int32_t *lens = int32s(a[1], check, {N}), *after = int32s(a[2], check, {N});
        const at::Tensor copies = a[5] != Py_None ? check(a[5], at::kInt, {N, 2}) : at::empty({N, 2}, table.options());
        const at::Tensor missing = a[6] != Py_None ? check(a[6], at::kInt, {1}) : at::empty({1}, table.options());
        const int32_t rows = narrow(N), columns = narrow(table.size(1)), page = narrow(whole(a[4]));
        const size_t need = reserve_size_entry(rows, columns, refs.size(0));
        const at::Tensor ws = need ? bytes(need, table) : at::Tensor();
        const Current on(table.device());
        void *stream = stream_of(check.device);
        kda_status st;
        Py_BEGIN_ALLOW_THREADS
        st = reserve_entry(static_cast<int32_t *>(table.data_ptr()), rows, columns, page, static_cast<int32_t *>(refs.data_ptr()), refs.size(0), lens, after,
                           static_cast<int32_t *>(copies.data_ptr()), static_cast<int32_t *>(missing.data_ptr()), need ? ws.data_ptr() : nullptr, need, stream);
        Py_END_ALLOW_THREADS
        return pair(st, a[5], copies, a[6], missing);
    });
}

// What kda_tree_steps and kda_tree_commit share: a[0..5] are k, v, log_alpha, beta, S_pool, state_indices.
struct Delta {
    kda_dims d;
    const void *k, *v, *la, *beta;
    float *S;
    const int32_t *indices = nullptr;
    Delta(PyObject *const *a, const at::Tensor &kt, const Checked &check, bool scalar_gate, int out, float scale)
    {
        const at::Tensor &vt = plain(a[1]), &St = plain(a[4]);
        if (kt.dim() != 4 || vt.dim() != 4 || St.dim() != 4) throw Irregular{};
        const int64_t N = kt.size(0), T = kt.size(1), H = kt.size(2), dk = kt.size(3), dv = vt.size(3);
        const at::ScalarType type = kt.scalar_type();
        k = check(kt, type, {N, T, H, dk}).data_ptr();
        v = check(vt, type, {N, T, H, dv}).data_ptr();
        la = scalar_gate ? check(a[2], type, {N, T, H}).data_ptr() : check(a[2], type, {N, T, H, dk}).data_ptr();
        beta = check(a[3], type, {N, T, H}).data_ptr();
        S = static_cast<float *>(check(St, at::kFloat, {St.size(0), H, dk, dv}).data_ptr());
        if (a[5] != Py_None) indices = int32s(a[5], check, {N});
        else if (St.size(0) < N) throw Irregular{};
        d = decode_dims(N, T, H, dk, dv, code(type), out, scale);
    }
};

// tree_steps(k, v, log_alpha, beta, S_pool, state_indices, q, parents, scale, o, out_dtype, scalar_gate)
PyObject *tree_steps(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        if (n != 12 || !tree_steps_entry) throw Irregular{};
        const at::Tensor &k = plain(a[0]), &v = plain(a[1]);
        const Checked check(k);
        const bool scalar = truth(a[11]);
        const at::Tensor o = output(a[9], a[10], v, check);
        const Delta x(a, k, check, scalar, code(o.scalar_type()), number(a[8]));
        const at::Tensor &q = check(a[6], k.scalar_type(), k.sizes());
        const int32_t *parents = int32s(a[7], check, {k.size(0), k.size(1)});
        const Current on(k.device());
        void *stream = stream_of(check.device);
        kda_status st;
        Py_BEGIN_ALLOW_THREADS
        st = tree_steps_entry(&x.d, q.data_ptr(), x.k, x.v, x.la, x.beta, x.S, x.indices, parents, o.data_ptr(), scalar ? KDA_STEPS_SCALAR_GATE : 0, stream);
        Py_END_ALLOW_THREADS
        return finish(st, a[9], o);
    });
}

// tree_commit(k, v, log_alpha, beta, S_pool, state_indices, kept, scalar_gate)
PyObject *tree_commit(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        if (n != 8 || !tree_commit_entry) throw Irregular{};
        const at::Tensor &k = plain(a[0]), &kept = plain(a[6]);
        if (kept.dim() != 2) throw Irregular{};
        const Checked check(k);
        const bool scalar = truth(a[7]);
        const Delta x(a, k, check, scalar, KDA_F32, 1.f);
        const int32_t *path = int32s(a[6], check, {k.size(0), kept.size(1)});
        const Current on(k.device());
        void *stream = stream_of(check.device);
        kda_status st;
        Py_BEGIN_ALLOW_THREADS
        st = tree_commit_entry(&x.d, x.k, x.v, x.la, x.beta, x.S, x.indices, path, narrow(kept.size(1)), scalar ? KDA_STEPS_SCALAR_GATE : 0, stream);
        Py_END_ALLOW_THREADS
        return nothing(st);
    });
}

// bind_tree(addresses of kda_rotate, kda_cache_tree_attn, kda_cache_tree_attn_workspace_size, kda_cache_keep, kda_cache_copy_pages, kda_tree_steps,
// kda_tree_commit, kda_pages_fork, kda_pages_reserve, kda_pages_reserve_workspace_size), after bind
PyObject *bind_tree(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 10) { PyErr_SetString(PyExc_TypeError, "bind_tree takes ten arguments"); return nullptr; }
    void *p[10];
    for (int i = 0; i < 10; ++i) p[i] = PyLong_AsVoidPtr(a[i]);
    if (PyErr_Occurred()) return nullptr;
    rotate_entry = reinterpret_cast<decltype(rotate_entry)>(p[0]);
    tree_attend_entry = reinterpret_cast<decltype(tree_attend_entry)>(p[1]);
    tree_attend_size_entry = reinterpret_cast<decltype(tree_attend_size_entry)>(p[2]);
    keep_entry = reinterpret_cast<decltype(keep_entry)>(p[3]);
    copy_entry = reinterpret_cast<decltype(copy_entry)>(p[4]);
    tree_steps_entry = reinterpret_cast<decltype(tree_steps_entry)>(p[5]);
    tree_commit_entry = reinterpret_cast<decltype(tree_commit_entry)>(p[6]);
    fork_entry = reinterpret_cast<decltype(fork_entry)>(p[7]);
    reserve_entry = reinterpret_cast<decltype(reserve_entry)>(p[8]);
    reserve_size_entry = reinterpret_cast<decltype(reserve_size_entry)>(p[9]);
    Py_RETURN_NONE;
}

// bind_attn(addresses of kda_cache_append, kda_cache_attn, kda_cache_attn_workspace_size, kda_window_attn_fwd, kda_window_attn_bwd,
// kda_window_attn_bwd_workspace_size), after bind
PyObject *bind_attn(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 6) { PyErr_SetString(PyExc_TypeError, "bind_attn takes six arguments"); return nullptr; }
    void *p[6];
    for (int i = 0; i < 6; ++i) p[i] = PyLong_AsVoidPtr(a[i]);
    if (PyErr_Occurred()) return nullptr;
    append_entry = reinterpret_cast<decltype(append_entry)>(p[0]);
    attend_entry = reinterpret_cast<decltype(attend_entry)>(p[1]);
    attend_size_entry = reinterpret_cast<decltype(attend_size_entry)>(p[2]);
    fwd_entry = reinterpret_cast<decltype(fwd_entry)>(p[3]);
    bwd_entry = reinterpret_cast<decltype(bwd_entry)>(p[4]);
    bwd_size_entry = reinterpret_cast<decltype(bwd_size_entry)>(p[5]);
    Py_RETURN_NONE;
}

// bind(address of kda_recurrent_step, address of kda_recurrent_steps, function from a device index to its current stream)
PyObject *bind(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 3) { PyErr_SetString(PyExc_TypeError, "bind takes three arguments"); return nullptr; }
    void *one = PyLong_AsVoidPtr(a[0]), *many = PyLong_AsVoidPtr(a[1]);
    if (PyErr_Occurred()) return nullptr;
    step_entry = reinterpret_cast<decltype(step_entry)>(one);
    steps_entry = reinterpret_cast<decltype(steps_entry)>(many);
    Py_INCREF(a[2]);
    Py_XDECREF(raw_stream);
    raw_stream = a[2];
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"bind", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(bind)), METH_FASTCALL, nullptr},
    {"step", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(step)), METH_FASTCALL, nullptr},
    {"steps", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(steps)), METH_FASTCALL, nullptr},
    {"bind_attn", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(bind_attn)), METH_FASTCALL, nullptr},
    {"append", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(append)), METH_FASTCALL, nullptr},
    {"attend", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(attend)), METH_FASTCALL, nullptr},
    {"window_fwd", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(window_fwd)), METH_FASTCALL, nullptr},
    {"window_bwd", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(window_bwd)), METH_FASTCALL, nullptr},
    {"bind_tree", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(bind_tree)), METH_FASTCALL, nullptr},
    {"rotate", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(rotate)), METH_FASTCALL, nullptr},
    {"tree_attend", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(tree_attend)), METH_FASTCALL, nullptr},
    {"keep", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(keep)), METH_FASTCALL, nullptr},
    {"copy_pages", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(copy_pages)), METH_FASTCALL, nullptr},
    {"fork", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(fork_rows)), METH_FASTCALL, nullptr},
    {"reserve", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(reserve)), METH_FASTCALL, nullptr},
    {"tree_steps", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(tree_steps)), METH_FASTCALL, nullptr},
    {"tree_commit", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(tree_commit)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_kda_host", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__kda_host(void) { return PyModule_Create(&module); }
