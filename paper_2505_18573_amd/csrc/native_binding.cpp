// The binding's hot calls without Python between the tensors and libe3.so.  A call of a few microseconds on the GPU took as
// long in Python: about 0.7 us per checked tensor, 0.8 to 1.4 us per foreign call, 1.1 us per allocated output.
// One pass among others, in Python / here: 64 x 8 advantages 5.7 / 3.6 us (the kernel 2.9), the objective of 512
// rollouts 11.6 / 9.4 us (its kernels 8.9), a step of 512 rows, whose host work lies between two launches, 72.9 / 69.8 us,
// log-probs with the measured gap of 1 row x 1000 16.5 / 10.9.
//
// Every function takes the arguments of the Python function it serves, and does what that does when they are ordinary: plain
// torch tensors of the right type, size and device, Python ints and floats.  It returns the outputs; or the
// library's status if that is not E3_OK; or None, with nothing done, for arguments that are not ordinary, which
// binding.py then treats itself: errors are found and worded in one place.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/util/Exception.h>
#include <torch/csrc/autograd/python_variable.h>

#include <array>

#include "../../include/e3.h"

namespace {

// Entry points of the library that binding.py has loaded, and torch's handle of the current stream.
decltype(&e3_grpo_advantages) p_advantages;
decltype(&e3_grpo_objective) p_objective;
decltype(&e3_workspace_bytes) p_workspace_bytes;
decltype(&e3_sample_entropy) p_sample;
decltype(&e3_restricted_workspace_bytes) p_restricted_bytes;
decltype(&e3_sample_restricted_ws) p_restricted;
decltype(&e3_logprob_entropy_advantages) p_logprob;
decltype(&e3_logprob_entropy_gap) p_gap;
decltype(&e3_temperature_update) p_temperature;
decltype(&e3_cache_append) p_cache_append;
decltype(&e3_cache_read) p_cache_read;
decltype(&e3_prefix_attention_workspace_bytes) p_attention_bytes;
decltype(&e3_prefix_attention) p_attention;
decltype(&e3_verify_workspace_bytes) p_verify_bytes;
decltype(&e3_verify_drafts) p_verify;
decltype(&e3_rotate) p_rotate;
decltype(&e3_beam_workspace_bytes) p_beam_bytes;
decltype(&e3_beam_select) p_beam_select;
decltype(&e3_beam_reorder) p_beam_reorder;
decltype(&e3_cache_copy) p_cache_copy;
decltype(&e3_window_attention) p_window;
decltype(&e3_window_attention_workspace_bytes) p_window_bytes;
decltype(&e3_cache_append_rotated) p_append_rotated;
PyObject* raw_stream = nullptr;

// A call's arguments as they are read: `ok` falls at the first one that is not ordinary.
struct Reader {
    bool ok = true;
    at::Device dev = at::Device(at::kCPU);

    const at::Tensor* plain(PyObject* o)
    {
        if (!ok || !THPVariable_CheckExact(o)) { ok = false; return nullptr; }
        const at::Tensor& t = THPVariable_Unpack(o);
        if (!t.defined() || t.layout() != at::kStrided || !t.has_storage() || t.is_neg()
            || t.key_set().has(c10::DispatchKey::Python)) { ok = false; return nullptr; }
        return &t;
    }
    // the vector that names the device
    const at::Tensor* first(PyObject* o)
    {
        const at::Tensor* t = plain(o);
        if (t == nullptr || !t->is_cuda()) { ok = false; return nullptr; }
        dev = t->device();
        return t;
    }
    // a vector of n elements, or None
    void* vector(PyObject* o, at::ScalarType type, int64_t n)
    {
        if (o == Py_None) return nullptr;
        const at::Tensor* t = plain(o);
        if (t == nullptr || t->scalar_type() != type || t->dim() != 1 || t->size(0) != n || !t->is_contiguous()
            || t->device() != dev) { ok = false; return nullptr; }
        return t->data_ptr();
    }
    // one element, also in pinned host memory
    void* scalar(PyObject* o, at::ScalarType type)
    {
        if (o == Py_None) return nullptr;
        const at::Tensor* t = plain(o);
        if (t == nullptr || t->scalar_type() != type || t->dim() != 1 || t->size(0) != 1
            || (t->device() != dev && !(t->is_cpu() && t->is_pinned()))) { ok = false; return nullptr; }
        return t->data_ptr();
    }
    int64_t integer(PyObject* o)
    {
        if (!PyLong_CheckExact(o)) { ok = false; return 0; }
        int overflow = 0;
        const long long v = PyLong_AsLongLongAndOverflow(o, &overflow);
        if (overflow != 0) ok = false;
        return v;
    }
    int32_t integer32(PyObject* o)
    {
        const int64_t v = integer(o);
        if (v != (int32_t)v) ok = false;
        return (int32_t)v;
    }
    uint64_t word(PyObject* o)                                    // modulo 2^64
    {
        if (!PyLong_CheckExact(o)) { ok = false; return 0; }
        return PyLong_AsUnsignedLongLongMask(o);
    }
    double number(PyObject* o)
    {
        if (PyFloat_CheckExact(o)) return PyFloat_AS_DOUBLE(o);
        return (double)integer(o);
    }
    void* stream()
    {
        PyObject* index = PyLong_FromLong(dev.index());
        PyObject* s = index ? PyObject_CallOneArg(raw_stream, index) : nullptr;
        Py_XDECREF(index);
        void* p = s ? PyLong_AsVoidPtr(s) : nullptr;
        Py_XDECREF(s);
        if (PyErr_Occurred()) { PyErr_Clear(); ok = false; }
        return p;
    }
};

struct Logits {
    const void* p = nullptr;
    int dtype = 0;
    int64_t rows = 0, V = 0, pitch = 0;
    Logits(Reader& r, PyObject* o)
    {
        const at::Tensor* t = r.first(o);
        if (t == nullptr || t->dim() != 2) { r.ok = false; return; }
        if (t->scalar_type() == at::kBFloat16) dtype = E3_BF16;
        else if (t->scalar_type() == at::kFloat) dtype = E3_F32;
        else { r.ok = false; return; }
        rows = t->size(0); V = t->size(1);
        if (V > 1 && t->stride(1) != 1) { r.ok = false; return; }
        pitch = rows > 1 ? t->stride(0) : std::max(V, t->stride(0));
        p = t->data_ptr();
    }
};

// An output: the caller's tensor, or one of n elements.
struct Output {
    PyObject* object = nullptr;
    void* p = nullptr;
    Output() = default;
    Output(const Output&) = delete;
    ~Output() { Py_XDECREF(object); }
    void make(Reader& r, at::ScalarType type, int64_t n)
    {
        if (!r.ok) return;
        const at::Tensor t = at::empty({n}, at::TensorOptions().dtype(type).device(r.dev));
        p = t.data_ptr();
        object = THPVariable_Wrap(t);
        if (object == nullptr) { PyErr_Clear(); r.ok = false; }
    }
    // n elements of a vector, from `from` on: several small outputs are one allocation (0.9 us of the calling thread each)
    void part(Reader& r, const at::Tensor& of, int64_t from, int64_t n)
    {
        const at::Tensor t = at::detail::make_tensor<at::TensorImpl>(at::TensorImpl::VIEW, at::Storage(of.storage()), of.key_set(), of.dtype());
        t.unsafeGetTensorImpl()->set_storage_offset(from);
        t.unsafeGetTensorImpl()->set_sizes_contiguous({n});
        p = t.data_ptr();
        object = THPVariable_Wrap(t);
        if (object == nullptr) { PyErr_Clear(); r.ok = false; }
    }
    void take(PyObject* given) { Py_INCREF(given); object = given; }
    void take_or_make(Reader& r, PyObject* given, at::ScalarType type, int64_t n)
    {
        if (given == Py_None) return make(r, type, n);
        p = r.vector(given, type, n);
        take(given);
    }
    // the same for a tensor of any shape
    template <size_t N>
    void shaped(Reader& r, PyObject* given, at::ScalarType type, const std::array<int64_t, N>& shape)
    {
        if (given != Py_None) {
            const at::Tensor* t = r.plain(given);
            if (t == nullptr || t->scalar_type() != type || t->sizes() != at::IntArrayRef(shape.data(), N) || t->device() != r.dev
                || !t->is_contiguous()) { r.ok = false; return; }
            p = t->data_ptr();
            return take(given);
        }
        if (!r.ok) return;
        const at::Tensor t = at::empty(at::IntArrayRef(shape.data(), N), at::TensorOptions().dtype(type).device(r.dev));
        p = t.data_ptr();
        object = THPVariable_Wrap(t);
        if (object == nullptr) { PyErr_Clear(); r.ok = false; }
    }
    PyObject* release() { PyObject* o = object; object = nullptr; return o; }
};

// The vocabulary pass's workspace argument: a tensor, None (allocate what is needed) or False (none).
struct Workspace {
    at::Tensor own;
    void* p = nullptr;
    size_t bytes = 0;
    void make(Reader& r, size_t need)
    {
        if (!r.ok || need == 0) return;
        own = at::empty({(int64_t)need}, at::TensorOptions().dtype(at::kByte).device(r.dev));
        p = own.data_ptr();
        bytes = need;
    }
    Workspace(Reader& r, PyObject* o, int64_t rows, int64_t V)
    {
        if (o == Py_False) return;
        if (o == Py_None) { make(r, p_workspace_bytes(rows, V)); return; }
        const at::Tensor* t = r.plain(o);
        if (t == nullptr) return;
        p = t->data_ptr();
        bytes = (size_t)t->numel() * t->element_size();
    }
    // The restricted sampler's: None allocates what is needed where `may_allocate`, and goes without where the memory is not there.
    Workspace(Reader& r, PyObject* o, size_t need, bool may_allocate)
    {
        if (o == Py_False) return;
        if (o == Py_None) {
            if (!may_allocate) return;
            try { make(r, need); } catch (const c10::OutOfMemoryError&) { own = at::Tensor(); p = nullptr; bytes = 0; }
            return;
        }
        const at::Tensor* t = r.plain(o);
        if (t == nullptr || t->device() != r.dev || !t->is_contiguous()) { r.ok = false; return; }
        p = t->data_ptr();
        bytes = (size_t)t->numel() * t->element_size();
    }
};

PyObject* unusual() { Py_RETURN_NONE; }

template <typename Call, typename Done>
PyObject* run(Reader& r, Call&& call, Done&& done)
{
    void* const stream = r.ok ? r.stream() : nullptr;
    if (!r.ok) return unusual();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = call(stream);
    Py_END_ALLOW_THREADS
    return rc == E3_OK ? done() : PyLong_FromLong(rc);
}

// C++ errors (an allocation that fails) leave the call to binding.py, which meets them again and reports them.
template <typename F>
PyObject* guarded(F&& f)
{
    try { return f(); } catch (...) { PyErr_Clear(); return unusual(); }
}

// rewards, group_offsets, ddof, eps, adv_out
PyObject* advantages(PyObject*, PyObject* const* a, Py_ssize_t n_args)
{
    if (n_args != 5) return unusual();
    return guarded([&]() -> PyObject* {
        Reader r;
        const at::Tensor* rewards = r.first(a[0]);
        const at::Tensor* offsets = r.ok ? r.plain(a[1]) : nullptr;
        if (!r.ok || rewards->dim() != 1 || offsets->dim() != 1) return unusual();
        const int64_t n = rewards->size(0), groups = offsets->size(0) - 1;
        const void* pr = r.vector(a[0], at::kFloat, n);
        const void* po = r.vector(a[1], at::kInt, groups + 1);
        const int32_t ddof = r.integer32(a[2]);
        const double eps = r.number(a[3]);
        if (groups != (int32_t)groups) return unusual();
        Output adv;
        adv.take_or_make(r, a[4], at::kFloat, n);
        return run(r, [&](void* s) { return p_advantages((const float*)pr, (const int32_t*)po, (int32_t)groups, ddof, (float)eps, (float*)adv.p, s); },
                   [&] { return adv.release(); });
    });
}

// logp_new, logp_old, seq_offsets, adv, group_offsets, clip_eps, want_token_terms
PyObject* objective(PyObject*, PyObject* const* a, Py_ssize_t n_args)
{
    if (n_args != 7 || !PyBool_Check(a[6])) return unusual();
    return guarded([&]() -> PyObject* {
        Reader r;
        const at::Tensor* logp = r.first(a[0]);
        const at::Tensor* adv = r.ok ? r.plain(a[3]) : nullptr;
        const at::Tensor* groups = r.ok ? r.plain(a[4]) : nullptr;
        if (!r.ok || logp->dim() != 1 || adv->dim() != 1 || groups->dim() != 1) return unusual();
        const int64_t T = logp->size(0), N = adv->size(0), B = groups->size(0) - 1;
        if (N != (int32_t)N || B != (int32_t)B) return unusual();
        const void* p_new = r.vector(a[0], at::kFloat, T);
        const void* p_old = a[1] == Py_None ? (r.ok = false, nullptr) : r.vector(a[1], at::kFloat, T);
        const void* p_seq = a[2] == Py_None ? (r.ok = false, nullptr) : r.vector(a[2], at::kInt, N + 1);
        const void* p_adv = r.vector(a[3], at::kFloat, N);
        const void* p_grp = r.vector(a[4], at::kInt, B + 1);
        const double clip = r.number(a[5]);
        Output J, mean, terms;
        if (a[6] == Py_True) terms.make(r, at::kFloat, T);
        else terms.take(Py_None);
        mean.make(r, at::kDouble, N);
        J.make(r, at::kDouble, 1);
        return run(r, [&](void* s) {
                       return p_objective((const float*)p_new, (const float*)p_old, (const int32_t*)p_seq, (const float*)p_adv, (int32_t)N,
                                          (const int32_t*)p_grp, (int32_t)B, (float)clip, (float*)terms.p, (double*)mean.p, (double*)J.p, s);
                   },
                   [&] { return PyTuple_Pack(3, J.object, mean.object, terms.object); });
    });
}

// logits, tau_rows, tau_scalar, seed, row_base, token_out, logp_out, entropy_out, workspace
PyObject* sample(PyObject*, PyObject* const* a, Py_ssize_t n_args)
{
    if (n_args != 9) return unusual();
    return guarded([&]() -> PyObject* {
        Reader r;
        const Logits l(r, a[0]);
        const void* tau = r.vector(a[1], at::kFloat, l.rows);
        const double tau_scalar = r.number(a[2]);
        const uint64_t seed = r.word(a[3]), row_base = r.word(a[4]);
        if (!r.ok) return unusual();
        Output token, logp, entropy;
        token.take_or_make(r, a[5], at::kInt, l.rows);
        logp.take_or_make(r, a[6], at::kFloat, l.rows);
        entropy.take_or_make(r, a[7], at::kFloat, l.rows);
        const Workspace ws(r, a[8], l.rows, l.V);
        return run(r, [&](void* s) {
                       return p_sample(l.p, l.dtype, l.rows, l.V, l.pitch, (const float*)tau, (float)tau_scalar, seed, row_base,
                                       (int32_t*)token.p, (float*)logp.p, (float*)entropy.p, ws.p, ws.bytes, s);
                   },
                   [&] { return PyTuple_Pack(3, token.object, logp.object, entropy.object); });
    });
}

// logits, tau_rows, tau_scalar, top_k, top_p, seed, row_base, token_out, logp_out, kept_out, workspace
PyObject* restricted(PyObject*, PyObject* const* a, Py_ssize_t n_args)
{
    if (n_args != 11) return unusual();
    return guarded([&]() -> PyObject* {
        Reader r;
        const Logits l(r, a[0]);
        const void* tau = r.vector(a[1], at::kFloat, l.rows);
        const double tau_scalar = r.number(a[2]);
        const int32_t top_k = r.integer32(a[3]);
        const double top_p = r.number(a[4]);
        const uint64_t seed = r.word(a[5]), row_base = r.word(a[6]);
        if (!r.ok) return unusual();
        Output token, logp, kept;
        token.take_or_make(r, a[7], at::kInt, l.rows);
        logp.take_or_make(r, a[8], at::kFloat, l.rows);
        kept.take_or_make(r, a[9], at::kInt, l.rows);
        const bool may_allocate = a[7] == Py_None || a[8] == Py_None || a[9] == Py_None;
        const Workspace ws(r, a[10], p_restricted_bytes(l.dtype, l.rows, l.V, top_k), may_allocate);
        return run(r, [&](void* s) {
                       return p_restricted(l.p, l.dtype, l.rows, l.V, l.pitch, (const float*)tau, (float)tau_scalar, top_k, (float)top_p, seed,
                                           row_base, (int32_t*)token.p, (float*)logp.p, (int32_t*)kept.p, ws.p, ws.bytes, s);
                   },
                   [&] { return PyTuple_Pack(3, token.object, logp.object, kept.object); });
    });
}

// logits, target_ids, row_mask, tau_rows, tau_scalar, rewards, group_offsets, ddof, eps, logp_out, entropy_out,
// entropy_sum_out, entropy_count_out, adv_out, workspace, want_sum; rewards None: no advantages
PyObject* logprob(PyObject*, PyObject* const* a, Py_ssize_t n_args)
{
    if (n_args != 16 || !PyBool_Check(a[15])) return unusual();
    return guarded([&]() -> PyObject* {
        Reader r;
        const Logits l(r, a[0]);
        const void* target = r.vector(a[1], at::kInt, l.rows);
        const void* mask = r.vector(a[2], at::kByte, l.rows);
        const void* tau = r.vector(a[3], at::kFloat, l.rows);
        const double tau_scalar = r.number(a[4]);
        if (!r.ok) return unusual();
        int64_t n = 0, groups = 0;
        const bool with_groups = a[5] != Py_None;
        const void *rewards = nullptr, *offsets = nullptr;
        if (with_groups) {
            const at::Tensor *tr = r.plain(a[5]), *to = r.ok ? r.plain(a[6]) : nullptr;
            if (!r.ok || tr->dim() != 1 || to->dim() != 1) return unusual();
            n = tr->size(0); groups = to->size(0) - 1;
            rewards = r.vector(a[5], at::kFloat, n);
            offsets = r.vector(a[6], at::kInt, groups + 1);
            if (groups != (int32_t)groups) return unusual();
        }
        const int32_t ddof = r.integer32(a[7]);
        const double eps = r.number(a[8]);
        Output logp, entropy, sum, count, adv;
        if (a[9] == Py_None && a[1] == Py_None) logp.take(Py_None);
        else logp.take_or_make(r, a[9], at::kFloat, l.rows);
        entropy.take_or_make(r, a[10], at::kFloat, l.rows);
        const bool want_sum = a[15] == Py_True;
        auto sum_out = [&](Output& o, PyObject* given, at::ScalarType type) {
            if (given == Py_None && want_sum) return o.make(r, type, 1);
            o.p = r.scalar(given, type);
            o.take(given);
        };
        sum_out(sum, a[11], at::kDouble);
        sum_out(count, a[12], at::kLong);
        if (with_groups) adv.take_or_make(r, a[13], at::kFloat, n);
        const Workspace ws(r, a[14], l.rows, l.V);
        return run(r, [&](void* s) {
                       return p_logprob(l.p, l.dtype, l.rows, l.V, l.pitch, (const int32_t*)target, (const uint8_t*)mask, (const float*)tau,
                                        (float)tau_scalar, (float*)logp.p, (float*)entropy.p, (double*)sum.p, (int64_t*)count.p,
                                        (const float*)rewards, (const int32_t*)offsets, (int32_t)groups, ddof, (float)eps, (float*)adv.p,
                                        ws.p, ws.bytes, s);
                   },
                   [&] {
                       return with_groups ? PyTuple_Pack(5, logp.object, entropy.object, sum.object, count.object, adv.object)
                                          : PyTuple_Pack(4, logp.object, entropy.object, sum.object, count.object);
                   });
    });
}

// logits, target_ids, row_mask, tau_rows, tau_scalar, workspace
PyObject* logprob_gap(PyObject*, PyObject* const* a, Py_ssize_t n_args)
{
    if (n_args != 6) return unusual();
    return guarded([&]() -> PyObject* {
        Reader r;
        const Logits l(r, a[0]);
        const void* target = r.vector(a[1], at::kInt, l.rows);
        const void* mask = r.vector(a[2], at::kByte, l.rows);
        const void* tau = r.vector(a[3], at::kFloat, l.rows);
        const double tau_scalar = r.number(a[4]);
        if (!r.ok) return unusual();
        Output logp, entropy, gap, sum, gap_sum, count;
        if (a[1] == Py_None) logp.take(Py_None);
        else logp.make(r, at::kFloat, l.rows);
        entropy.make(r, at::kFloat, l.rows);
        gap.make(r, at::kFloat, l.rows);
        sum.make(r, at::kDouble, 1);
        gap_sum.make(r, at::kDouble, 1);
        count.make(r, at::kLong, 1);
        const Workspace ws(r, a[5], l.rows, l.V);
        return run(r, [&](void* s) {
                       return p_gap(l.p, l.dtype, l.rows, l.V, l.pitch, (const int32_t*)target, (const uint8_t*)mask, (const float*)tau,
                                    (float)tau_scalar, (float*)logp.p, (float*)entropy.p, (float*)gap.p, (double*)sum.p, (double*)gap_sum.p,
                                    (int64_t*)count.p, ws.p, ws.bytes, s);
                   },
                   [&] { return PyTuple_Pack(6, logp.object, entropy.object, gap.object, sum.object, gap_sum.object, count.object); });
    });
}

// A cache as binding.py's E3Cache holds it: a tuple of k, v, k_scale, v_scale.
struct Cache {
    e3_cache c{};
    Cache(Reader& r, PyObject* o)
    {
        if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 4) { r.ok = false; return; }
        const at::Tensor* k = r.first(PyTuple_GET_ITEM(o, 0));
        const at::Tensor* v = r.ok ? r.plain(PyTuple_GET_ITEM(o, 1)) : nullptr;
        if (!r.ok || k->dim() != 4 || v->dim() != 5 || !k->is_contiguous() || !v->is_contiguous() || v->device() != r.dev
            || v->scalar_type() != k->scalar_type()) { r.ok = false; return; }
        const auto ks = k->sizes(), vs = v->sizes();
        if (vs[0] != ks[0] || vs[1] != ks[1] || vs[2] != ks[2] / 8 || vs[3] != ks[3] || vs[4] != 8) { r.ok = false; return; }
        const bool fp8 = k->scalar_type() == at::kFloat8_e4m3fn;
        if (!fp8 && k->scalar_type() != at::kBFloat16) { r.ok = false; return; }
        for (int i = 1; i < 4; ++i)
            if (ks[i] != (int32_t)ks[i]) { r.ok = false; return; }
        c.k = k->data_ptr();
        c.v = v->data_ptr();
        for (int i = 0; i < 2; ++i) {
            PyObject* const scale = PyTuple_GET_ITEM(o, 2 + i);
            if ((scale == Py_None) == fp8) { r.ok = false; return; }
            if (!fp8) continue;
            const at::Tensor* t = r.plain(scale);
            if (t == nullptr || t->scalar_type() != at::kByte || t->dim() != 3 || t->size(0) != ks[0] || t->size(1) != ks[1] || t->size(2) != ks[2]
                || t->device() != r.dev || !t->is_contiguous()) { r.ok = false; return; }
            (i == 0 ? c.k_scale : c.v_scale) = (uint8_t*)t->data_ptr();
        }
        c.num_pages = ks[0]; c.kv_heads = (int32_t)ks[1]; c.page_size = (int32_t)ks[2]; c.head_dim = (int32_t)ks[3];
        c.dtype = fp8 ? E3_E4M3 : E3_BF16;
    }
};

int float_type(Reader& r, at::ScalarType t)
{
    if (t != at::kBFloat16 && t != at::kFloat) r.ok = false;
    return t == at::kFloat ? E3_F32 : E3_BF16;
}

// a dimension's stride; one of a single element has none of its own
int64_t step_of(const at::Tensor* t, int64_t dim) { return t->size(dim) > 1 ? t->stride(dim) : 0; }

// cache, k, v, slots; True where it was done
PyObject* cache_append(PyObject*, PyObject* const* a, Py_ssize_t n_args)
{
    if (n_args != 4) return unusual();
    return guarded([&]() -> PyObject* {
        Reader r;
        const Cache cache(r, a[0]);
        const at::Tensor* k = r.ok ? r.plain(a[1]) : nullptr;
        const at::Tensor* v = r.ok ? r.plain(a[2]) : nullptr;
        const at::Tensor* slots = r.ok ? r.plain(a[3]) : nullptr;
        if (!r.ok || slots->dim() != 1) return unusual();
        const int64_t n = slots->size(0);
        const void* ps = r.vector(a[3], at::kLong, n);
        for (const at::Tensor* t : {k, v})
            if (t->scalar_type() != k->scalar_type() || t->dim() != 3 || t->size(0) != n || t->size(1) != cache.c.kv_heads
                || t->size(2) != cache.c.head_dim || t->device() != r.dev || (n > 0 && t->stride(2) != 1)) return unusual();
        const int type = float_type(r, k->scalar_type());
        return run(r, [&](void* s) {
                       return p_cache_append(&cache.c, k->data_ptr(), v->data_ptr(), type, n, step_of(k, 0), step_of(k, 1), step_of(v, 0),
                                             step_of(v, 1), (const int64_t*)ps, s);
                   },
                   [&]() -> PyObject* { Py_RETURN_TRUE; });
    });
}

// rotary positions as binding.py's E3Rotary holds them (freqs, axis, neighbours), and the tokens' positions
struct Turns {
    e3_rotary c{};
    const int64_t* positions = nullptr;
    int64_t stride = 0;
    Turns(Reader& r, PyObject* o, PyObject* of, int64_t tokens)
    {
        if (!r.ok || !PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 3 || !PyBool_Check(PyTuple_GET_ITEM(o, 2))) { r.ok = false; return; }
        const at::Tensor* f = r.plain(PyTuple_GET_ITEM(o, 0));
        const at::Tensor* p = r.ok ? r.plain(of) : nullptr;
        if (!r.ok || f->dim() != 1 || f->size(0) != (int32_t)f->size(0) || f->size(0) > 1 << 20) { r.ok = false; return; }
        const int64_t pairs = f->size(0), dims = p->dim();
        c.freqs = (const double*)r.vector(PyTuple_GET_ITEM(o, 0), at::kDouble, pairs);
        c.axis = (const uint8_t*)r.vector(PyTuple_GET_ITEM(o, 1), at::kByte, pairs);
        if (!r.ok || (dims != 1 && dims != 2) || p->scalar_type() != at::kLong || p->size(dims - 1) != tokens || p->device() != r.dev
            || (tokens > 1 && p->stride(dims - 1) != 1)) { r.ok = false; return; }
        const int64_t axes = dims == 2 ? p->size(0) : 1;
        if (axes > 1 << 20 || (c.axis == nullptr && axes != 1)) { r.ok = false; return; }
        c.rot_dim = (int32_t)(2 * pairs); c.axes = (int32_t)axes; c.neighbours = PyTuple_GET_ITEM(o, 2) == Py_True;
        positions = (const int64_t*)p->data_ptr();
        stride = axes > 1 ? p->stride(0) : 0;
    }
};

bool unit_columns(const at::Tensor* t) { return t->numel() == 0 || t->size(2) < 2 || t->stride(2) == 1; }

// an output [tokens][heads][D] of any strides with columns next to each other
const at::Tensor* rows_of_heads(Reader& r, Output& out, PyObject* given, at::ScalarType type, const std::array<int64_t, 3>& shape)
{
    if (given == Py_None) {
        out.shaped(r, given, type, shape);
        return r.ok ? &THPVariable_Unpack(out.object) : nullptr;
    }
    const at::Tensor* t = r.plain(given);
    if (t == nullptr || t->scalar_type() != type || t->sizes() != at::IntArrayRef(shape.data(), 3) || t->device() != r.dev || !unit_columns(t)) {
        r.ok = false;
        return nullptr;
    }
    out.p = t->data_ptr();
    out.take(given);
    return t;
}

// x, rotary, positions, out, inverse
PyObject* rotate(PyObject*, PyObject* const* a, Py_ssize_t n_args)
{
    if (n_args != 5 || !PyBool_Check(a[4])) return unusual();
    return guarded([&]() -> PyObject* {
        Reader r;
        const at::Tensor* x = r.first(a[0]);
        if (!r.ok || x->dim() != 3 || !unit_columns(x)) return unusual();
        const int type = float_type(r, x->scalar_type());
        const int64_t n = x->size(0), heads = x->size(1), D = x->size(2);
        const Turns turns(r, a[1], a[2], n);
        if (!r.ok) return unusual();
        Output out;
        const at::Tensor* o = rows_of_heads(r, out, a[3], x->scalar_type(), {n, heads, D});
        return run(r, [&](void* s) {
                       return p_rotate(&turns.c, turns.positions, turns.stride, x->data_ptr(), type, n, heads, D, step_of(x, 0), step_of(x, 1), out.p,
                                       step_of(o, 0), step_of(o, 1), a[4] == Py_True, s);
                   },
                   [&] { return out.release(); });
    });
}

// cache, q, k, v, rotary, positions, slots, q_out; the turned queries, True where there are none
PyObject* append_rotated(PyObject*, PyObject* const* a, Py_ssize_t n_args)
{
    if (n_args != 8) return unusual();
    return guarded([&]() -> PyObject* {
        Reader r;
        const Cache cache(r, a[0]);
        const at::Tensor* k = r.ok ? r.plain(a[2]) : nullptr;
        const at::Tensor* v = r.ok ? r.plain(a[3]) : nullptr;
        const at::Tensor* slots = r.ok ? r.plain(a[6]) : nullptr;
        const at::Tensor* q = r.ok && a[1] != Py_None ? r.plain(a[1]) : nullptr;
        if (!r.ok || slots->dim() != 1 || (q == nullptr && a[7] != Py_None)) return unusual();
        const int64_t n = slots->size(0);
        const void* ps = r.vector(a[6], at::kLong, n);
        for (const at::Tensor* t : {k, v})
            if (t->scalar_type() != k->scalar_type() || t->dim() != 3 || t->size(0) != n || t->size(1) != cache.c.kv_heads
                || t->size(2) != cache.c.head_dim || t->device() != r.dev || !unit_columns(t)) return unusual();
        const int type = float_type(r, k->scalar_type());
        const Turns turns(r, a[4], a[5], n);
        if (!r.ok) return unusual();
        Output out;
        const at::Tensor* o = nullptr;
        if (q != nullptr) {
            if (q->scalar_type() != k->scalar_type() || q->dim() != 3 || q->size(0) != n || q->size(2) != cache.c.head_dim || q->device() != r.dev
                || !unit_columns(q)) return unusual();
            o = rows_of_heads(r, out, a[7], k->scalar_type(), {n, q->size(1), q->size(2)});
            if (!r.ok) return unusual();
        }
        return run(r, [&](void* s) {
                       return p_append_rotated(&cache.c, &turns.c, turns.positions, turns.stride, q ? q->data_ptr() : nullptr, k->data_ptr(),
                                               v->data_ptr(), type, n, q ? q->size(1) : 0, q ? step_of(q, 0) : 0, q ? step_of(q, 1) : 0,
                                               step_of(k, 0), step_of(k, 1), step_of(v, 0), step_of(v, 1), (const int64_t*)ps, out.p,
                                               o ? step_of(o, 0) : 0, o ? step_of(o, 1) : 0, s);
                   },
                   [&]() -> PyObject* { if (q == nullptr) Py_RETURN_TRUE; return out.release(); });
    });
}

// cache, slots, whether bf16 (or fp32), k_out, v_out
PyObject* cache_read(PyObject*, PyObject* const* a, Py_ssize_t n_args)
{
    if (n_args != 5 || !PyBool_Check(a[2])) return unusual();
    return guarded([&]() -> PyObject* {
        Reader r;
        const Cache cache(r, a[0]);
        const at::Tensor* slots = r.ok ? r.plain(a[1]) : nullptr;
        if (!r.ok || slots->dim() != 1) return unusual();
        const int64_t n = slots->size(0);
        const void* ps = r.vector(a[1], at::kLong, n);
        const at::ScalarType type = a[2] == Py_True ? at::kBFloat16 : at::kFloat;
        const std::array<int64_t, 3> shape = {n, cache.c.kv_heads, cache.c.head_dim};
        Output k, v;
        k.shaped(r, a[3], type, shape);
        v.shaped(r, a[4], type, shape);
        return run(r, [&](void* s) { return p_cache_read(&cache.c, (const int64_t*)ps, n, k.p, v.p, type == at::kFloat ? E3_F32 : E3_BF16, s); },
                   [&] { return PyTuple_Pack(2, k.object, v.object); });
    });
}

// q, cache, group_offsets, prefix_pages, prefix_lens, row_pages, row_lens, scale, out, lse_out, workspace, want_lse
PyObject* attention(PyObject*, PyObject* const* a, Py_ssize_t n_args)
{
    if (n_args != 12 || !PyBool_Check(a[11])) return unusual();
    return guarded([&]() -> PyObject* {
        Reader r;
        const Cache cache(r, a[1]);
        const at::Tensor* q = r.ok ? r.plain(a[0]) : nullptr;
        if (!r.ok || q->dim() != 4 || q->scalar_type() != at::kBFloat16 || q->device() != r.dev || q->size(3) != cache.c.head_dim
            || (q->numel() > 0 && q->stride(3) != 1)) return unusual();
        const int64_t rows = q->size(0), T = q->size(1), heads = q->size(2), D = q->size(3);
        auto table = [&](PyObject* o, int64_t n, int64_t* width) -> const int32_t* {
            const at::Tensor* t = r.plain(o);
            if (t == nullptr || t->scalar_type() != at::kInt || t->dim() != 2 || t->size(0) != n || !t->is_contiguous()
                || t->device() != r.dev) { r.ok = false; return nullptr; }
            *width = t->size(1);
            return (const int32_t*)t->data_ptr();
        };
        int64_t groups = 0, prefix_width = 0, row_width = 0;
        const void *offsets = nullptr, *prefix_lens = nullptr;
        const int32_t* prefix_pages = nullptr;
        if (a[2] != Py_None) {
            const at::Tensor* off = r.plain(a[2]);
            if (off == nullptr || off->dim() != 1 || a[3] == Py_None || a[4] == Py_None) return unusual();
            groups = off->size(0) - 1;
            offsets = r.vector(a[2], at::kInt, groups + 1);
            prefix_pages = table(a[3], groups, &prefix_width);
            prefix_lens = r.vector(a[4], at::kInt, groups);
        }
        const int32_t* row_pages = table(a[5], rows, &row_width);
        if (a[6] == Py_None) return unusual();
        const void* row_lens = r.vector(a[6], at::kInt, rows);
        const double scale = r.number(a[7]);
        if (!r.ok) return unusual();
        Output out, lse;
        out.shaped(r, a[8], at::kBFloat16, std::array<int64_t, 4>{rows, T, heads, D});
        if (a[9] == Py_None && a[11] == Py_False) lse.take(Py_None);
        else lse.shaped(r, a[9], at::kFloat, std::array<int64_t, 3>{rows, T, heads});
        const size_t need = a[10] == Py_None ? p_attention_bytes(rows, T, heads, cache.c.kv_heads, D, groups) : 0;
        const Workspace ws(r, a[10] == Py_False ? Py_True : a[10], need, true);       // False is no workspace here: left to binding.py
        if (a[10] == Py_None && need > 0 && ws.p == nullptr) return unusual();         // no memory: reported there
        return run(r, [&](void* s) {
                       return p_attention(&cache.c, q->data_ptr(), rows, T, heads, step_of(q, 0), step_of(q, 1), step_of(q, 2),
                                          groups > 0 ? (const int32_t*)offsets : nullptr, groups, prefix_pages, prefix_width, (const int32_t*)prefix_lens,
                                          row_pages, row_width, (const int32_t*)row_lens, (float)scale, out.p, (float*)lse.p, ws.p, ws.bytes, s);
                   },
                   [&] { return PyTuple_Pack(2, out.object, lse.object); });
    });
}

// q, cache, query_offsets, row_pages, row_lens, window, sinks, scale, out, lse_out, workspace, want_lse
PyObject* window(PyObject*, PyObject* const* a, Py_ssize_t n_args)
{
    if (n_args != 12 || !PyBool_Check(a[11])) return unusual();
    return guarded([&]() -> PyObject* {
        Reader r;
        const Cache cache(r, a[1]);
        const at::Tensor* q = r.ok ? r.plain(a[0]) : nullptr;
        const at::Tensor* offsets = r.ok ? r.plain(a[2]) : nullptr;
        const at::Tensor* pages = r.ok ? r.plain(a[3]) : nullptr;
        if (!r.ok || q->dim() != 3 || q->scalar_type() != at::kBFloat16 || q->device() != r.dev || q->size(2) != cache.c.head_dim || !unit_columns(q)
            || offsets->dim() != 1 || offsets->size(0) < 1 || a[4] == Py_None) return unusual();
        const int64_t tokens = q->size(0), heads = q->size(1), D = q->size(2), rows = offsets->size(0) - 1;
        const void* of = r.vector(a[2], at::kInt, rows + 1);
        if (pages->scalar_type() != at::kInt || pages->dim() != 2 || pages->size(0) != rows || !pages->is_contiguous() || pages->device() != r.dev)
            return unusual();
        const void* lens = r.vector(a[4], at::kInt, rows);
        const int64_t width = r.integer(a[5]), sinks = r.integer(a[6]);
        const double scale = r.number(a[7]);
        if (!r.ok) return unusual();
        Output out, lse;
        out.shaped(r, a[8], at::kBFloat16, std::array<int64_t, 3>{tokens, heads, D});
        if (a[9] == Py_None && a[11] == Py_False) lse.take(Py_None);
        else lse.shaped(r, a[9], at::kFloat, std::array<int64_t, 2>{tokens, heads});
        const size_t need = a[10] == Py_None ? p_window_bytes(rows, tokens, heads, cache.c.kv_heads, D) : 0;
        const Workspace ws(r, a[10] == Py_False ? Py_True : a[10], need, true);
        if (a[10] == Py_None && need > 0 && ws.p == nullptr) return unusual();
        return run(r, [&](void* s) {
                       return p_window(&cache.c, q->data_ptr(), tokens, heads, step_of(q, 0), step_of(q, 1), (const int32_t*)of, rows,
                                       (const int32_t*)pages->data_ptr(), pages->size(1), (const int32_t*)lens, width, sinks, (float)scale, out.p,
                                       (float*)lse.p, ws.p, ws.bytes, s);
                   },
                   [&] { return PyTuple_Pack(2, out.object, lse.object); });
    });
}

// logits, draft_tokens, draft_logits, draft_lens, tau_rows, tau_scalar, seed, row_base, draft_tau_rows, accepted_out, token_out,
// logp_out, entropy_out, workspace
PyObject* verify(PyObject*, PyObject* const* a, Py_ssize_t n_args)
{
    if (n_args != 14) return unusual();
    return guarded([&]() -> PyObject* {
        Reader r;
        const at::Tensor* z = r.first(a[0]);
        if (!r.ok || z->dim() != 3 || z->size(1) < 1) return unusual();
        const int type = float_type(r, z->scalar_type());
        const int64_t rows = z->size(0), positions = z->size(1), V = z->size(2), drafts = positions - 1;
        if (drafts != (int32_t)drafts) return unusual();
        // row and position strides, of a dimension of one what binding.py gives
        auto strides = [&](const at::Tensor* t, int64_t* of_row, int64_t* of_position) {
            if (V > 1 && t->stride(2) != 1) { r.ok = false; return; }
            *of_position = t->size(1) > 1 ? t->stride(1) : (V + 7) / 8 * 8;
            *of_row = rows > 1 ? t->stride(0) : *of_position * t->size(1);
        };
        int64_t row_stride = 0, position_stride = 0, draft_row = 0, draft_position = 0;
        strides(z, &row_stride, &position_stride);
        const void* d = nullptr;
        if (a[2] != Py_None) {
            const at::Tensor* t = r.plain(a[2]);
            if (t == nullptr || t->scalar_type() != z->scalar_type() || t->dim() != 3 || t->size(0) != rows || t->size(1) != drafts
                || t->size(2) != V || t->device() != r.dev) return unusual();
            if (drafts > 0) strides(t, &draft_row, &draft_position);
            d = t->data_ptr();
        }
        const void* tokens = nullptr;
        if (a[1] != Py_None) {
            const at::Tensor* t = r.plain(a[1]);
            if (t == nullptr || t->scalar_type() != at::kInt || t->dim() != 2 || t->size(0) != rows || t->size(1) != drafts || !t->is_contiguous()
                || t->device() != r.dev) return unusual();
            tokens = t->data_ptr();
        } else if (drafts > 0) return unusual();
        const void* lens = r.vector(a[3], at::kInt, rows);
        const void* tau = r.vector(a[4], at::kFloat, rows);
        const double tau_scalar = r.number(a[5]);
        const uint64_t seed = r.word(a[6]), row_base = r.word(a[7]);
        const void* draft_tau = r.vector(a[8], at::kFloat, rows);
        if (!r.ok) return unusual();
        const std::array<int64_t, 2> shape = {rows, positions};
        Output accepted, token, logp, entropy;
        accepted.take_or_make(r, a[9], at::kInt, rows);
        token.shaped(r, a[10], at::kInt, shape);
        logp.shaped(r, a[11], at::kFloat, shape);
        entropy.shaped(r, a[12], at::kFloat, shape);
        const size_t need = a[13] == Py_None ? p_verify_bytes(rows, (int32_t)drafts, V) : 0;
        const Workspace ws(r, a[13] == Py_False ? Py_True : a[13], need, true);
        if (a[13] == Py_None && need > 0 && ws.p == nullptr) return unusual();
        return run(r, [&](void* s) {
                       return p_verify(z->data_ptr(), type, rows, (int32_t)drafts, V, row_stride, position_stride, (const int32_t*)tokens,
                                       (const int32_t*)lens, d, draft_row, draft_position, (const float*)tau, (float)tau_scalar, (const float*)draft_tau,
                                       seed, row_base, (int32_t*)accepted.p, (int32_t*)token.p, (float*)logp.p, (float*)entropy.p, ws.p, ws.bytes, s);
                   },
                   [&] { return PyTuple_Pack(4, accepted.object, token.object, logp.object, entropy.object); });
    });
}

// logits, scores, keep, tau, finished, eos_token, parent_out, token_out, score_out, workspace
PyObject* beam_select(PyObject*, PyObject* const* a, Py_ssize_t n_args)
{
    if (n_args != 10) return unusual();
    return guarded([&]() -> PyObject* {
        Reader r;
        const at::Tensor* z = r.first(a[0]);
        if (!r.ok || z->dim() != 3) return unusual();
        const int type = float_type(r, z->scalar_type());
        const int64_t seqs = z->size(0), beams = z->size(1), V = z->size(2);
        if ((V > 1 && z->stride(2) != 1) || beams != (int32_t)beams || a[1] == Py_None) return unusual();
        // of a dimension of one what binding.py gives
        const int64_t beam_stride = beams > 1 ? z->stride(1) : (V + 7) / 8 * 8;
        const int64_t seq_stride = seqs > 1 ? z->stride(0) : beam_stride * beams;
        auto table = [&](PyObject* o, at::ScalarType kind) -> const void* {
            if (o == Py_None) return nullptr;
            const at::Tensor* t = r.plain(o);
            if (t == nullptr || t->scalar_type() != kind || t->dim() != 2 || t->size(0) != seqs || t->size(1) != beams || !t->is_contiguous()
                || t->device() != r.dev) { r.ok = false; return nullptr; }
            return t->data_ptr();
        };
        const void* scores = table(a[1], at::kFloat);
        const void* finished = table(a[4], at::kByte);
        const int32_t keep = r.integer32(a[2]), eos = r.integer32(a[5]);
        const double tau = r.number(a[3]);
        if (!r.ok || keep < 1 || keep > E3_MAX_KEEP) return unusual();
        const std::array<int64_t, 2> shape = {seqs, keep};
        Output parent, token, score;
        parent.shaped(r, a[6], at::kInt, shape);
        token.shaped(r, a[7], at::kInt, shape);
        score.shaped(r, a[8], at::kFloat, shape);
        const size_t need = a[9] == Py_None ? p_beam_bytes(seqs, (int32_t)beams, V) : 0;
        const Workspace ws(r, a[9] == Py_False ? Py_True : a[9], need, true);
        if (a[9] == Py_None && need > 0 && ws.p == nullptr) return unusual();
        return run(r, [&](void* s) {
                       return p_beam_select(z->data_ptr(), type, seqs, (int32_t)beams, V, seq_stride, beam_stride, (const float*)scores, keep, (float)tau,
                                            (const uint8_t*)finished, eos, (int32_t*)parent.p, (int32_t*)token.p, (float*)score.p, ws.p, ws.bytes, s);
                   },
                   [&] { return PyTuple_Pack(3, parent.object, token.object, score.object); });
    });
}

// parent, row_pages, row_lens, page_size, pages_out, lens_out, src_out, dst_out, counts_out
PyObject* beam_reorder(PyObject*, PyObject* const* a, Py_ssize_t n_args)
{
    if (n_args != 9) return unusual();
    return guarded([&]() -> PyObject* {
        Reader r;
        const at::Tensor* parent = r.first(a[0]);
        const at::Tensor* pages = r.ok ? r.plain(a[1]) : nullptr;
        if (!r.ok || parent->dim() != 2 || parent->scalar_type() != at::kInt || !parent->is_contiguous() || parent->size(1) != (int32_t)parent->size(1)
            || pages->dim() != 2 || pages->scalar_type() != at::kInt || pages->size(0) != parent->numel() || !pages->is_contiguous()
            || pages->device() != r.dev || a[2] == Py_None) return unusual();
        const int64_t seqs = parent->size(0), beams = parent->size(1), rows = seqs * beams, width = pages->size(1);
        const void* lens = r.vector(a[2], at::kInt, rows);
        const int32_t page = r.integer32(a[3]);
        if (!r.ok) return unusual();
        Output out_pages, out[4];
        out_pages.shaped(r, a[4], at::kInt, std::array<int64_t, 2>{rows, width});
        if (r.ok && a[5] == Py_None && a[6] == Py_None && a[7] == Py_None && a[8] == Py_None) {
            const int64_t apart = (rows + 15) / 16 * 16;                       // aligned like allocations for any vector load
            const at::Tensor all = at::empty({4 * apart}, at::TensorOptions().dtype(at::kInt).device(r.dev));
            for (int i = 0; i < 4; ++i) out[i].part(r, all, i * apart, rows);
        }
        else
            for (int i = 0; i < 4; ++i) out[i].take_or_make(r, a[5 + i], at::kInt, rows);
        return run(r, [&](void* s) {
                       return p_beam_reorder((const int32_t*)parent->data_ptr(), seqs, (int32_t)beams, (const int32_t*)pages->data_ptr(), width,
                                             (const int32_t*)lens, page, (int32_t*)out_pages.p, (int32_t*)out[0].p, (int32_t*)out[1].p,
                                             (int32_t*)out[2].p, (int32_t*)out[3].p, s);
                   },
                   [&] { return PyTuple_Pack(5, out_pages.object, out[0].object, out[1].object, out[2].object, out[3].object); });
    });
}

// cache, src_pages, dst_pages, counts; True where it was done
PyObject* cache_copy(PyObject*, PyObject* const* a, Py_ssize_t n_args)
{
    if (n_args != 4) return unusual();
    return guarded([&]() -> PyObject* {
        Reader r;
        const Cache cache(r, a[0]);
        const at::Tensor* src = r.ok ? r.plain(a[1]) : nullptr;
        if (!r.ok || src->dim() != 1 || a[2] == Py_None || a[3] == Py_None) return unusual();
        const int64_t n = src->size(0);
        const void* from = r.vector(a[1], at::kInt, n);
        const void* to = r.vector(a[2], at::kInt, n);
        const void* counts = r.vector(a[3], at::kInt, n);
        return run(r, [&](void* s) { return p_cache_copy(&cache.c, (const int32_t*)from, (const int32_t*)to, (const int32_t*)counts, n, s); },
                   [&]() -> PyObject* { Py_RETURN_TRUE; });
    });
}

// tau_t, H_t, H_init, vocab, t, t_anneal, t_max, eta, tau_min, tau_max
PyObject* temperature(PyObject*, PyObject* const* a, Py_ssize_t n_args)
{
    if (n_args != 10) return unusual();
    Reader r;
    const double tau = r.number(a[0]), H = r.number(a[1]), H0 = r.number(a[2]);
    const int64_t vocab = r.integer(a[3]), t = r.integer(a[4]), t_anneal = r.integer(a[5]), t_max = r.integer(a[6]);
    const double eta = r.number(a[7]), lo = r.number(a[8]), hi = r.number(a[9]);
    if (!r.ok) return unusual();
    double next = 0.0, target = 0.0;
    const int rc = p_temperature(tau, H, H0, vocab, t, t_anneal, t_max, eta, lo, hi, &next, &target);
    return rc == E3_OK ? Py_BuildValue("dd", next, target) : PyLong_FromLong(rc);
}

// The library's entry points by name (a dict of addresses), and torch's handle of the current stream.
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n_args)
{
    if (n_args != 2 || !PyDict_Check(a[0]) || !PyCallable_Check(a[1])) {
        PyErr_SetString(PyExc_TypeError, "bind(addresses, current_raw_stream)");
        return nullptr;
    }
    bool all = true;
    auto get = [&](const char* name, auto& to) {
        PyObject* v = PyDict_GetItemString(a[0], name);
        void* p = v && PyLong_Check(v) ? PyLong_AsVoidPtr(v) : nullptr;
        if (p == nullptr) all = false;
        to = reinterpret_cast<std::remove_reference_t<decltype(to)>>(p);
    };
    get("e3_grpo_advantages", p_advantages);
    get("e3_grpo_objective", p_objective);
    get("e3_workspace_bytes", p_workspace_bytes);
    get("e3_sample_entropy", p_sample);
    get("e3_restricted_workspace_bytes", p_restricted_bytes);
    get("e3_sample_restricted_ws", p_restricted);
    get("e3_logprob_entropy_advantages", p_logprob);
    get("e3_logprob_entropy_gap", p_gap);
    get("e3_temperature_update", p_temperature);
    get("e3_cache_append", p_cache_append);
    get("e3_cache_read", p_cache_read);
    get("e3_prefix_attention_workspace_bytes", p_attention_bytes);
    get("e3_prefix_attention", p_attention);
    get("e3_verify_workspace_bytes", p_verify_bytes);
    get("e3_verify_drafts", p_verify);
    get("e3_rotate", p_rotate);
    get("e3_beam_workspace_bytes", p_beam_bytes);
    get("e3_beam_select", p_beam_select);
    get("e3_beam_reorder", p_beam_reorder);
    get("e3_cache_copy", p_cache_copy);
    get("e3_window_attention", p_window);
    get("e3_window_attention_workspace_bytes", p_window_bytes);
    get("e3_cache_append_rotated", p_append_rotated);
    if (!all) { PyErr_SetString(PyExc_ValueError, "an entry point is missing"); return nullptr; }
    Py_INCREF(a[1]);
    Py_XSETREF(raw_stream, a[1]);
    Py_RETURN_NONE;
}

template <typename F>
constexpr PyCFunction fast(F* f) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)); }

PyMethodDef methods[] = {
    {"bind", fast(bind), METH_FASTCALL, nullptr},
    {"advantages", fast(advantages), METH_FASTCALL, nullptr},
    {"objective", fast(objective), METH_FASTCALL, nullptr},
    {"sample", fast(sample), METH_FASTCALL, nullptr},
    {"restricted", fast(restricted), METH_FASTCALL, nullptr},
    {"logprob", fast(logprob), METH_FASTCALL, nullptr},
    {"logprob_advantages", fast(logprob), METH_FASTCALL, nullptr},
    {"logprob_gap", fast(logprob_gap), METH_FASTCALL, nullptr},
    {"temperature", fast(temperature), METH_FASTCALL, nullptr},
    {"cache_append", fast(cache_append), METH_FASTCALL, nullptr},
    {"cache_read", fast(cache_read), METH_FASTCALL, nullptr},
    {"attention", fast(attention), METH_FASTCALL, nullptr},
    {"verify", fast(verify), METH_FASTCALL, nullptr},
    {"rotate", fast(rotate), METH_FASTCALL, nullptr},
    {"beam_select", fast(beam_select), METH_FASTCALL, nullptr},
    {"beam_reorder", fast(beam_reorder), METH_FASTCALL, nullptr},
    {"cache_copy", fast(cache_copy), METH_FASTCALL, nullptr},
    {"window", fast(window), METH_FASTCALL, nullptr},
    {"append_rotated", fast(append_rotated), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native() { return PyModule_Create(&module); }
