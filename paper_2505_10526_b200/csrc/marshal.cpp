// Argument marshalling of the calls a decoding loop makes every step: tensors are checked and their addresses taken here
// instead of by half a dozen attribute reads per tensor in Python (25 tensors a step: about 8 us of 26 on a step whose kernels
// take 20).  The functions called are those of the C ABI library the binding has loaded; bind() hands their addresses in.
#include <Python.h>

#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <memory>

#include "massv.h"

namespace {

decltype(&massv_verify_attn) g_verify_attn = nullptr;
decltype(&massv_accept) g_accept = nullptr;
decltype(&massv_kv_commit) g_kv_commit = nullptr;
decltype(&massv_sample_top_p) g_sample_top_p = nullptr;
decltype(&massv_tvd) g_tvd = nullptr;
decltype(&massv_rotary) g_rotary = nullptr;
decltype(&massv_verify_attn_shared) g_verify_attn_shared = nullptr;
decltype(&massv_logits_apply) g_logits_apply = nullptr;
decltype(&massv_accept_logits) g_accept_logits = nullptr;
decltype(&massv_history_add) g_history_add = nullptr;
PyObject *g_attn_desc = nullptr, *g_accept_desc = nullptr, *g_rope_desc = nullptr, *g_logit_rules = nullptr, *g_sized_rules = nullptr;       // the ctypes structures of the descriptors

const char* dtype_name(c10::ScalarType t) {
    switch (t) {
        case c10::ScalarType::BFloat16: return "torch.bfloat16";
        case c10::ScalarType::Float: return "torch.float32";
        case c10::ScalarType::Int: return "torch.int32";
        default: return c10::toString(t);
    }
}

// Sets a Python error and leaves by exception, so that one catch per call cleans up.
struct PythonError {};
[[noreturn]] void fail(PyObject* type, const char* text) { PyErr_SetString(type, text); throw PythonError(); }

// Address of a tensor's data; None is a null pointer.  dtype Undefined: any.
void* pointer(PyObject* obj, c10::ScalarType dtype) {
    if (obj == Py_None) return nullptr;
    if (!THPVariable_Check(obj)) fail(PyExc_AttributeError, "massv: tensors expected");
    const at::Tensor& t = THPVariable_Unpack(obj);
    if (!t.is_cuda()) fail(PyExc_ValueError, "massv: tensors must live on a CUDA device");
    if (!t.is_contiguous()) fail(PyExc_ValueError, "massv: tensors must be contiguous");
    if (dtype != c10::ScalarType::Undefined && t.scalar_type() != dtype) {
        PyErr_Format(PyExc_ValueError, "massv: expected %s, got %s", dtype_name(dtype), dtype_name(t.scalar_type()));
        throw PythonError();
    }
    return t.mutable_data_ptr();
}
void* bf16(PyObject* o) { return pointer(o, c10::ScalarType::BFloat16); }
float* f32(PyObject* o) { return static_cast<float*>(pointer(o, c10::ScalarType::Float)); }
int32_t* i32(PyObject* o) { return static_cast<int32_t*>(pointer(o, c10::ScalarType::Int)); }
void* any(PyObject* o) { return pointer(o, c10::ScalarType::Undefined); }
size_t elements(PyObject* o) { return o == Py_None ? 0 : (size_t)THPVariable_Unpack(o).numel(); }      // (behind any(): a tensor)

// The same for a tensor that has to live on the device whose stream the call goes to.
const at::Tensor& on_device(PyObject* obj) {
    if (!THPVariable_Check(obj)) fail(PyExc_AttributeError, "massv: tensors expected");
    const at::Tensor& t = THPVariable_Unpack(obj);
    if (!t.is_cuda()) fail(PyExc_ValueError, "massv: tensors must live on a CUDA device");
    if (t.get_device() != c10::cuda::current_device()) fail(PyExc_ValueError, "massv: tensors must live on the current device");
    return t;
}
void* here(PyObject* obj, c10::ScalarType dtype) {
    if (obj != Py_None) on_device(obj);
    return pointer(obj, dtype);
}
// The same with at least n elements.  (n as a double: no product of a descriptor's fields overflows it; a descriptor whose product is
// nonsense is the library's to refuse.)
void* at_least(PyObject* obj, c10::ScalarType dtype, double n, const char* name) {
    void* data = here(obj, dtype);
    if ((double)elements(obj) < n && obj != Py_None) {
        PyErr_Format(PyExc_ValueError, "massv: %s has fewer elements than the call takes", name);
        throw PythonError();
    }
    return data;
}

// Tokens of heads * d consecutive bf16 elements, evenly spaced: a dense tensor [..., heads, d] or a slice of a fused projection's output.
struct Tokens { void* data = nullptr; int64_t stride = 0; };
Tokens tokens_of(PyObject* obj, int64_t n, int64_t heads, int64_t d) {
    Tokens r;
    if (obj == Py_None) return r;
    const at::Tensor& t = on_device(obj);
    if (t.scalar_type() != c10::ScalarType::BFloat16) {
        PyErr_Format(PyExc_ValueError, "massv: expected torch.bfloat16, got %s", dtype_name(t.scalar_type()));
        throw PythonError();
    }
    const int64_t dims = t.dim();
    if (dims < 3 || t.size(dims - 1) != d || t.size(dims - 2) != heads || t.numel() != n * heads * d) fail(PyExc_ValueError, "massv: tokens must be [..., heads, head_dim], as many as the descriptor says");
    if (t.stride(dims - 1) != 1 || (heads > 1 && t.stride(dims - 2) != d)) fail(PyExc_ValueError, "massv: a token's heads must be contiguous");
    int64_t count = 1;
    r.stride = heads * d;
    for (int64_t i = dims - 3; i >= 0; --i) {
        if (t.size(i) == 1) continue;
        if (count == 1) r.stride = t.stride(i);
        else if (t.stride(i) != r.stride * count) fail(PyExc_ValueError, "massv: tokens must be evenly spaced");
        count *= t.size(i);
    }
    r.data = t.mutable_data_ptr();
    return r;
}

// A descriptor: the bytes of its ctypes structure (or of one derived from it, which begins with the same fields).
template <typename Desc>
struct DescOf {
    Py_buffer view;
    DescOf(PyObject* o, PyObject* type) {
        const int is = PyObject_IsInstance(o, type);
        if (is < 0) throw PythonError();
        if (is == 0) fail(PyExc_TypeError, "massv: wrong descriptor");
        if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) throw PythonError();
        if (view.len < (Py_ssize_t)sizeof(Desc)) { PyBuffer_Release(&view); fail(PyExc_TypeError, "massv: wrong descriptor"); }
    }
    DescOf(const DescOf&) = delete;
    DescOf& operator=(const DescOf&) = delete;
    ~DescOf() { PyBuffer_Release(&view); }
    const Desc* get() const { return static_cast<const Desc*>(view.buf); }
};

// Rules as logit_rules makes them: with the tensors' lengths (-1: no tensor) and their device (-1: no tensors).
struct SizedRules { massv_logit_rules rules; int64_t sizes[10]; int32_t device; };
// Whether the rules' tensors are long enough for the call and live where it runs (rules filled in by hand hold bare addresses, as in C).
void check_rules(PyObject* obj, const massv_logit_rules* rules, int64_t batch, int64_t rows, int64_t vocab) {
    const int is = PyObject_IsInstance(obj, g_sized_rules);
    if (is < 0) throw PythonError();
    if (is == 0 || batch < 1 || rows < 1 || vocab < 1) return;
    const SizedRules& r = *reinterpret_cast<const SizedRules*>(rules);
    static const char* const kNames[10] = {"allowed", "bias_start", "bias_tokens", "bias_values", "prompt_bits", "output_bits", "counts", "repetition", "frequency", "presence"};
    const double words = (double)((vocab + 31) / 32), b = (double)batch;
    const double need[10] = {b * rows * words, b + 1, 0, 0, b * words, b * words, b * vocab, b, b, b};
    for (int i = 0; i < 10; ++i)
        if (r.sizes[i] >= 0 && (double)r.sizes[i] < need[i]) {
            PyErr_Format(PyExc_ValueError, "massv: the rules' %s has fewer elements than the call's batch and vocabulary take", kNames[i]);
            throw PythonError();
        }
    if (r.device >= 0 && r.device != c10::cuda::current_device()) fail(PyExc_ValueError, "massv: the rules' tensors must live on the current device");
}

massv_stream_t stream() { return reinterpret_cast<massv_stream_t>(c10::cuda::getCurrentCUDAStream().stream()); }

long integer(PyObject* o) { const long v = PyLong_AsLong(o); if (v == -1 && PyErr_Occurred()) throw PythonError(); return v; }
int32_t int_of(PyObject* o) {                                    // an int32, whole
    const long v = integer(o);
    if (v != (int32_t)v) fail(PyExc_OverflowError, "massv: a size does not fit in 32 bits");
    return (int32_t)v;
}
double number(PyObject* o) {                                     // whatever float() takes
    PyObject* f = PyNumber_Float(o);
    if (!f) throw PythonError();
    const double v = PyFloat_AS_DOUBLE(f);
    Py_DECREF(f);
    return v;
}

// Runs `call` (arguments in, status out) with the argument count checked and C++ exceptions turned into Python's; the
// library call itself runs without the interpreter lock.
template <typename Call>
PyObject* guarded(Py_ssize_t given, Py_ssize_t wanted, Call&& call) {
    try {
        if (given != wanted) fail(PyExc_TypeError, "massv: wrong number of arguments");
        return PyLong_FromLong(call());
    } catch (const PythonError&) {
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}
template <typename F>
int unlocked(F&& f) {
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f();
    Py_END_ALLOW_THREADS
    return rc;
}

PyObject* py_verify_attn(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 13, [&] {
        const DescOf<massv_attn_desc> d(a[0], g_attn_desc);
        void *q = bf16(a[1]), *kn = bf16(a[2]), *vn = bf16(a[3]), *kp = bf16(a[4]), *vp = bf16(a[5]);
        int32_t *table = i32(a[6]), *lens = i32(a[7]);
        void* out = bf16(a[8]);
        float *out32 = f32(a[9]), *lse = f32(a[10]);
        void* ws = any(a[11]);
        const size_t ws_bytes = elements(a[11]);
        int32_t* status = i32(a[12]);
        const massv_stream_t s = stream();
        return unlocked([&] { return g_verify_attn(d.get(), q, kn, vn, kp, vp, table, lens, out, out32, lse, ws, ws_bytes, status, s); });
    });
}
PyObject* py_accept(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 13, [&] {
        const DescOf<massv_accept_desc> d(a[0], g_accept_desc);
        void *h = bf16(a[1]), *w = bf16(a[2]);
        int32_t* drafts = i32(a[3]);
        float *q = f32(a[4]), *ua = f32(a[5]), *us = f32(a[6]);
        int32_t *tokens = i32(a[7]), *lens = i32(a[8]);
        float *logits = f32(a[9]), *probs = f32(a[10]);
        void* ws = any(a[11]);
        const size_t ws_bytes = elements(a[11]);
        int32_t* status = i32(a[12]);
        const massv_stream_t s = stream();
        return unlocked([&] { return g_accept(d.get(), h, w, drafts, q, ua, us, tokens, lens, logits, probs, ws, ws_bytes, status, s); });
    });
}
PyObject* py_kv_commit(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 5, [&] {
        const int32_t batch = (int32_t)integer(a[0]), gamma = (int32_t)integer(a[1]);
        int32_t *lens = i32(a[2]), *seq = i32(a[3]), *status = i32(a[4]);
        const massv_stream_t s = stream();
        return unlocked([&] { return g_kv_commit(batch, gamma, lens, seq, status, s); });
    });
}
PyObject* py_sample_top_p(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 9, [&] {
        const int32_t rows = (int32_t)integer(a[0]), vocab = (int32_t)integer(a[1]);
        const float T = (float)number(a[2]), top_p = (float)number(a[3]);
        float *z = f32(a[4]), *u = f32(a[5]);
        int32_t* tokens = i32(a[6]);
        float* probs = f32(a[7]);
        int32_t* status = i32(a[8]);
        const massv_stream_t s = stream();
        return unlocked([&] { return g_sample_top_p(rows, vocab, T, top_p, z, u, tokens, probs, status, s); });
    });
}
PyObject* py_tvd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 7, [&] {
        const DescOf<massv_accept_desc> d(a[0], g_accept_desc);
        float *z = f32(a[1]), *q = f32(a[2]), *tvd = f32(a[3]), *acc = f32(a[4]);
        void* ws = any(a[5]);
        const size_t ws_bytes = elements(a[5]);
        int32_t* status = i32(a[6]);
        const massv_stream_t s = stream();
        return unlocked([&] { return g_tvd(d.get(), z, q, tvd, acc, ws, ws_bytes, status, s); });
    });
}

PyObject* py_rotary(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 9, [&] {
        const DescOf<massv_rope_desc> d(a[0], g_rope_desc);
        const massv_rope_desc& g = *d.get();
        const int64_t count = (int64_t)g.batch * g.rows;
        const uint64_t* turns = static_cast<const uint64_t*>(here(a[1], c10::ScalarType::Long));
        if (a[1] != Py_None && (int64_t)elements(a[1]) != g.rot_dim / 2) fail(PyExc_ValueError, "massv: turns must have rot_dim / 2 values");
        const Tokens q = tokens_of(a[2], count, g.n_q_heads, g.head_dim), k = tokens_of(a[3], count, g.n_kv_heads, g.head_dim);
        const Tokens qo = tokens_of(a[4], count, g.n_q_heads, g.head_dim), ko = tokens_of(a[5], count, g.n_kv_heads, g.head_dim);
        const double tokens = (double)g.batch * g.rows;
        const auto ints = [&](int i, double least, const char* name) { return static_cast<int32_t*>(at_least(a[i], c10::ScalarType::Int, least, name)); };
        int32_t *const pos[3] = {ints(6, tokens * g.n_axes, "positions"), ints(7, g.batch, "seq_lens"), ints(8, g.batch, "pos_delta")};
        const massv_stream_t s = stream();
        return unlocked([&] { return g_rotary(d.get(), turns, q.data, q.stride, k.data, k.stride, pos[0], pos[1], pos[2], qo.data, qo.stride, ko.data, ko.stride, s); });
    });
}
PyObject* py_verify_attn_shared(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 15, [&] {
        const DescOf<massv_attn_desc> d(a[0], g_attn_desc);
        const massv_attn_desc& g = *d.get();
        const double rows = (double)g.batch * (g.gamma + 1.0), q_size = rows * g.n_q_heads * g.head_dim, new_size = rows * g.n_kv_heads * g.head_dim;
        const double pool = (double)g.num_pages * g.n_kv_heads * g.page_size * g.head_dim;
        const auto in = [&](int i, c10::ScalarType t, double least, const char* name) { return at_least(a[i], t, least, name); };
        constexpr auto BF = c10::ScalarType::BFloat16, I = c10::ScalarType::Int, F = c10::ScalarType::Float;
        if (a[1] == Py_None || a[2] == Py_None) fail(PyExc_ValueError, "massv: groups expected");
        int32_t *start = static_cast<int32_t*>(here(a[1], I)), *shared = static_cast<int32_t*>(here(a[2], I));
        const int64_t groups = THPVariable_Unpack(a[2]).numel();
        if (THPVariable_Unpack(a[1]).numel() != groups + 1) fail(PyExc_ValueError, "massv: group_start has one entry more than shared_lens");
        void *q = in(3, BF, q_size, "q"), *kn = in(4, BF, new_size, "k_new"), *vn = in(5, BF, new_size, "v_new"), *kp = in(6, BF, pool, "k_pages"), *vp = in(7, BF, pool, "v_pages");
        int32_t *table = static_cast<int32_t*>(in(8, I, (double)g.batch * g.max_pages_per_seq, "page_table")), *lens = static_cast<int32_t*>(in(9, I, g.batch, "seq_lens"));
        void* out = in(10, BF, q_size, "out");
        float *out32 = static_cast<float*>(in(11, F, q_size, "out_f32")), *lse = static_cast<float*>(in(12, F, rows * g.n_q_heads, "lse"));
        void* ws = here(a[13], c10::ScalarType::Undefined);
        const size_t ws_bytes = elements(a[13]);
        int32_t* status = static_cast<int32_t*>(in(14, I, 1, "dev_status"));
        const massv_stream_t s = stream();
        return unlocked([&] { return g_verify_attn_shared(d.get(), (int32_t)groups, start, shared, q, kn, vn, kp, vp, table, lens, out, out32, lse, ws, ws_bytes, status, s); });
    });
}
PyObject* py_logits_apply(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 8, [&] {
        const int32_t batch = int_of(a[0]), gamma = int_of(a[1]), vocab = int_of(a[2]);
        const DescOf<massv_logit_rules> rules(a[3], g_logit_rules);
        check_rules(a[3], rules.get(), batch, (int64_t)gamma + 1, vocab);
        constexpr auto I = c10::ScalarType::Int, F = c10::ScalarType::Float;
        const double size = (double)batch * (gamma + 1.0) * vocab;
        float *z = static_cast<float*>(at_least(a[4], F, size, "logits")), *out = static_cast<float*>(at_least(a[5], F, size, "logits_out"));
        int32_t *drafts = static_cast<int32_t*>(at_least(a[6], I, (double)batch * gamma, "draft_tokens")), *status = static_cast<int32_t*>(at_least(a[7], I, 1, "dev_status"));
        const massv_stream_t s = stream();
        return unlocked([&] { return g_logits_apply(batch, gamma, vocab, rules.get(), z, out, drafts, status, s); });
    });
}
PyObject* py_accept_logits(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 13, [&] {
        const DescOf<massv_accept_desc> d(a[0], g_accept_desc);
        const std::unique_ptr<DescOf<massv_logit_rules>> rules(a[1] == Py_None ? nullptr : new DescOf<massv_logit_rules>(a[1], g_logit_rules));
        if (rules) check_rules(a[1], rules->get(), d.get()->batch, (int64_t)d.get()->gamma + 1, d.get()->vocab);
        const double batch = d.get()->batch, drafted = batch * d.get()->gamma, rows = drafted + batch, vocab = d.get()->vocab;
        const auto f = [&](int i, double least, const char* name) { return static_cast<float*>(at_least(a[i], c10::ScalarType::Float, least, name)); };
        const auto w = [&](int i, double least, const char* name) { return static_cast<int32_t*>(at_least(a[i], c10::ScalarType::Int, least, name)); };
        float *z = f(2, rows * vocab, "logits"), *out = f(3, rules ? rows * vocab : 0, "logits_out");
        int32_t* drafts = w(4, drafted, "draft_tokens");
        const double sampling = d.get()->temperature > 0.f ? 1 : 0;          // (not read at T = 0)
        float *q = f(5, sampling * drafted * vocab, "draft_probs"), *ua = f(6, sampling * drafted, "u_accept"), *us = f(7, sampling * rows, "u_sample");
        int32_t *tokens = w(8, rows, "out_tokens"), *lens = w(9, batch, "accept_len");
        float* probs = f(10, rows * vocab, "probs_out");
        void* ws = here(a[11], c10::ScalarType::Undefined);
        const size_t ws_bytes = elements(a[11]);
        int32_t* status = w(12, 1, "dev_status");
        const massv_stream_t s = stream();
        return unlocked([&] { return g_accept_logits(d.get(), rules ? rules->get() : nullptr, z, out, drafts, q, ua, us, tokens, lens, probs, ws, ws_bytes, status, s); });
    });
}
PyObject* py_history_add(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 8, [&] {
        const int32_t batch = int_of(a[0]), vocab = int_of(a[1]), n_max = int_of(a[3]);
        const auto w = [&](int i, double least, const char* name) { return static_cast<int32_t*>(at_least(a[i], c10::ScalarType::Int, least, name)); };
        int32_t *tokens = w(2, (double)batch * n_max, "tokens"), *lens = w(4, batch, "lens"), *bits = w(5, (double)batch * ((vocab + 31LL) / 32), "bits"),
                *counts = w(6, (double)batch * vocab, "counts"), *status = w(7, 1, "dev_status");
        const massv_stream_t s = stream();
        return unlocked([&] { return g_history_add(batch, vocab, tokens, n_max, lens, reinterpret_cast<uint32_t*>(bits), counts, status, s); });
    });
}

PyObject* py_bind(PyObject*, PyObject* args) {
    unsigned long long attn, accept, commit, top_p, tvd, rotary, shared, apply, accept_logits, history;
    PyObject *attn_desc, *accept_desc, *rope_desc, *logit_rules, *sized_rules;
    if (!PyArg_ParseTuple(args, "KKKKKKKKKKO!O!O!O!O!", &attn, &accept, &commit, &top_p, &tvd, &rotary, &shared, &apply, &accept_logits, &history, &PyType_Type, &attn_desc,
                          &PyType_Type, &accept_desc, &PyType_Type, &rope_desc, &PyType_Type, &logit_rules, &PyType_Type, &sized_rules))
        return nullptr;
    const auto keep = [](PyObject*& slot, PyObject* type) { Py_INCREF(type); Py_XSETREF(slot, type); };
    keep(g_attn_desc, attn_desc); keep(g_accept_desc, accept_desc); keep(g_rope_desc, rope_desc); keep(g_logit_rules, logit_rules); keep(g_sized_rules, sized_rules);
    g_rotary = reinterpret_cast<decltype(g_rotary)>(rotary);
    g_verify_attn_shared = reinterpret_cast<decltype(g_verify_attn_shared)>(shared);
    g_logits_apply = reinterpret_cast<decltype(g_logits_apply)>(apply);
    g_accept_logits = reinterpret_cast<decltype(g_accept_logits)>(accept_logits);
    g_history_add = reinterpret_cast<decltype(g_history_add)>(history);
    g_verify_attn = reinterpret_cast<decltype(g_verify_attn)>(attn);
    g_accept = reinterpret_cast<decltype(g_accept)>(accept);
    g_kv_commit = reinterpret_cast<decltype(g_kv_commit)>(commit);
    g_sample_top_p = reinterpret_cast<decltype(g_sample_top_p)>(top_p);
    g_tvd = reinterpret_cast<decltype(g_tvd)>(tvd);
    Py_RETURN_NONE;
}

#define MASSV_FAST(f) reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(f)), METH_FASTCALL
PyMethodDef g_methods[] = {
    {"bind", py_bind, METH_VARARGS, "addresses of the C ABI functions, types of the descriptors"},
    {"verify_attn", MASSV_FAST(py_verify_attn), nullptr},
    {"accept", MASSV_FAST(py_accept), nullptr},
    {"kv_commit", MASSV_FAST(py_kv_commit), nullptr},
    {"sample_top_p", MASSV_FAST(py_sample_top_p), nullptr},
    {"tvd", MASSV_FAST(py_tvd), nullptr},
    {"rotary", MASSV_FAST(py_rotary), nullptr},
    {"verify_attn_shared", MASSV_FAST(py_verify_attn_shared), nullptr},
    {"logits_apply", MASSV_FAST(py_logits_apply), nullptr},
    {"accept_logits", MASSV_FAST(py_accept_logits), nullptr},
    {"history_add", MASSV_FAST(py_history_add), nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&g_module); }
