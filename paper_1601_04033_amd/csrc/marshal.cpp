// Native argument marshalling of the binding's calls (module _marshal): plain
// arguments (contiguous device tensors of the right type and length, integers,
// floats, sequences of them) become the C ABI's arguments without a Python
// bytecode per tensor.  An argument that is not plain in this sense (another
// tensor type or subclass, a wrong length, a number that Python converts by
// its own rules) makes a call return None with nothing done; the binding then
// takes its general way in Python, which converts or rejects it.  The two ways
// make the same library call with the same arguments.
//
// Host time per call, back to back, with the library call in it (3.5 us with
// one kernel launch): a pass of K = 1 / 16 / 32 gradients 8.4 / 20.5 / 33.2 us
// marshalled in Python, 3.7 / 4.0 / 4.2 us here; a selection (two launches)
// 12.3 and 6.3 us, a sparse apply 8.0 and 4.0 us.
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include <stdint.h>
#include <string.h>

#include "../../include/fasgd_client.h"

namespace {

// the library's entry points, by the order of kNames
constexpr const char* kNames[] = {
    "fasgd_apply_updates", "sasgd_apply_updates", "bfasgd_select_compact", "bfasgd_select_compact_batch",
    "bfasgd_apply_sparse", "fasgd_apply_with_push", "fasgd_apply_with_push_and_select", "fasgd_apply_pushes",
    "bfasgd_apply_cached", "bfasgd_apply_fetch", "bfasgd_decide_segments", "bfasgd_apply_segments"};
constexpr int kCount = sizeof kNames / sizeof kNames[0];
struct Entry {
    decltype(&::fasgd_apply_updates) fasgd_apply_updates;
    decltype(&::sasgd_apply_updates) sasgd_apply_updates;
    decltype(&::bfasgd_select_compact) bfasgd_select_compact;
    decltype(&::bfasgd_select_compact_batch) bfasgd_select_compact_batch;
    decltype(&::bfasgd_apply_sparse) bfasgd_apply_sparse;
    decltype(&::fasgd_apply_with_push) fasgd_apply_with_push;
    decltype(&::fasgd_apply_with_push_and_select) fasgd_apply_with_push_and_select;
    decltype(&::fasgd_apply_pushes) fasgd_apply_pushes;
    decltype(&::bfasgd_apply_cached) bfasgd_apply_cached;
    decltype(&::bfasgd_apply_fetch) bfasgd_apply_fetch;
    decltype(&::bfasgd_decide_segments) bfasgd_decide_segments;
    decltype(&::bfasgd_apply_segments) bfasgd_apply_segments;
};
static_assert(sizeof(Entry) == kCount * sizeof(void*), "one pointer per name");
// and the client's, by the order of kClientNames
constexpr const char* kClientNames[] = {"client_dropout", "client_residual_norm_forward",
                                        "client_residual_norm_backward", "client_fp8_quantize", "client_fp8_matmul",
                                        "client_fp8_linear", "client_vocab_loss_forward",
                                        "client_vocab_loss_backward", "client_vocab_distill_forward",
                                        "client_vocab_distill_backward"};
constexpr int kClientCount = sizeof kClientNames / sizeof kClientNames[0];
struct ClientEntry {
    decltype(&::client_dropout) client_dropout;
    decltype(&::client_residual_norm_forward) client_residual_norm_forward;
    decltype(&::client_residual_norm_backward) client_residual_norm_backward;
    decltype(&::client_fp8_quantize) client_fp8_quantize;
    decltype(&::client_fp8_matmul) client_fp8_matmul;
    decltype(&::client_fp8_linear) client_fp8_linear;
    decltype(&::client_vocab_loss_forward) client_vocab_loss_forward;
    decltype(&::client_vocab_loss_backward) client_vocab_loss_backward;
    decltype(&::client_vocab_distill_forward) client_vocab_distill_forward;
    decltype(&::client_vocab_distill_backward) client_vocab_distill_backward;
};
static_assert(sizeof(ClientEntry) == kClientCount * sizeof(void*), "one pointer per name");
ClientEntry g_client;                 // set by bind_client()
Entry g_lib;                          // set by bind(), once, before any other call
PyObject* g_current_stream = nullptr; // callable: the current stream's handle as an int

// One call's arguments.  Every getter returns a usable value while `plain`
// holds; afterwards nothing that they return is used.
struct Args {
    PyObject* const* v;
    bool plain = true;
    Py_buffer state_view{};
    Py_buffer seg_view{};
    PyObject* held[3] = {nullptr, nullptr, nullptr};   // fast sequences of this call
    int n_held = 0;

    explicit Args(PyObject* const* args) : v(args) {}
    ~Args()
    {
        if (state_view.obj) PyBuffer_Release(&state_view);
        if (seg_view.obj) PyBuffer_Release(&seg_view);
        for (int i = 0; i < n_held; ++i) Py_DECREF(held[i]);
    }
    Args(const Args&) = delete;
    Args& operator=(const Args&) = delete;

    // The argument is not plain.  Of the exceptions that its conversion may
    // have raised, those that say so are dropped, as the general way raises
    // them again; any other (an interrupt, a signal handler's, no memory)
    // stays set, and finish() lets it out.
    bool refuse()
    {
        if (PyErr_Occurred() &&
            (PyErr_ExceptionMatches(PyExc_TypeError) || PyErr_ExceptionMatches(PyExc_ValueError) ||
             PyErr_ExceptionMatches(PyExc_OverflowError) || PyErr_ExceptionMatches(PyExc_AttributeError) ||
             PyErr_ExceptionMatches(PyExc_BufferError)))
            PyErr_Clear();
        plain = false;
        return false;
    }

    // the fasgd_state struct (a ctypes Structure, by its buffer)
    fasgd_state* state(int i)
    {
        if (!plain) return nullptr;
        if (PyObject_GetBuffer(v[i], &state_view, PyBUF_WRITABLE) != 0 ||
            state_view.len != static_cast<Py_ssize_t>(sizeof(fasgd_state))) {
            refuse();
            return nullptr;
        }
        return static_cast<fasgd_state*>(state_view.buf);
    }

    // a contiguous device tensor of `type` with at least `least` elements and,
    // when `exactly` >= 0, that many; the element count goes to *n
    void* tensor_of(PyObject* o, c10::ScalarType type, int64_t exactly, int64_t least = 0, int64_t* n = nullptr)
    {
        if (!plain) return nullptr;
        if (!THPVariable_CheckExact(o)) {
            refuse();
            return nullptr;
        }
        try {
            const at::Tensor& t = THPVariable_Unpack(o);
            const int64_t count = t.numel();
            if (!t.is_cuda() || t.scalar_type() != type || !t.is_contiguous() || (exactly >= 0 && count != exactly) ||
                count < least) {
                refuse();
                return nullptr;
            }
            if (n) *n = count;
            return t.data_ptr();
        } catch (...) {   // a tensor without storage: the general way says so
            refuse();
            return nullptr;
        }
    }
    void* tensor(int i, c10::ScalarType type, int64_t exactly, int64_t least = 0, int64_t* n = nullptr)
    {
        return tensor_of(v[i], type, exactly, least, n);
    }
    float* floats(int i, int64_t exactly, int64_t* n = nullptr)
    {
        return static_cast<float*>(tensor(i, c10::ScalarType::Float, exactly, 0, n));
    }
    int32_t* ints(int i, int64_t exactly, int64_t* n = nullptr)
    {
        return static_cast<int32_t*>(tensor(i, c10::ScalarType::Int, exactly, 0, n));
    }
    int64_t* counts(int i, int64_t exactly)
    {
        return static_cast<int64_t*>(tensor(i, c10::ScalarType::Long, exactly));
    }
    // a [B, columns] tensor's columns
    int64_t columns(int i, int64_t B)
    {
        if (!plain) return 0;
        try {
            if (THPVariable_CheckExact(v[i])) {
                const at::Tensor& t = THPVariable_Unpack(v[i]);
                if (t.dim() == 2 && t.size(0) == B) return t.size(1);
            }
        } catch (...) {
        }
        refuse();
        return 0;
    }
    // the list index (None where it may be absent)
    uint32_t* seg_start(int i, int64_t length, bool required, bool whole = false)
    {
        if (!plain || (v[i] == Py_None && !required)) return nullptr;
        return static_cast<uint32_t*>(tensor(i, c10::ScalarType::Int, whole ? length : -1, length));
    }

    int64_t integer_of(PyObject* o)
    {
        if (!plain) return 0;
        PyObject* x = PyNumber_Index(o);   // an int, or what says it is one (numpy's)
        if (!x) {
            refuse();
            return 0;
        }
        int over = 0;
        const long long r = PyLong_AsLongLongAndOverflow(x, &over);
        Py_DECREF(x);
        if (over || (r == -1 && PyErr_Occurred())) {
            refuse();
            return 0;
        }
        return r;
    }
    int64_t int64(int i) { return integer_of(v[i]); }
    int32_t narrow(int64_t r)
    {
        if (r < INT32_MIN || r > INT32_MAX) refuse();
        return static_cast<int32_t>(r);
    }
    int32_t int32(int i) { return narrow(integer_of(v[i])); }
    // any integer, by its low 64 bits
    uint64_t seed(int i)
    {
        if (!plain) return 0;
        PyObject* x = PyNumber_Index(v[i]);
        if (!x) {
            refuse();
            return 0;
        }
        const uint64_t r = PyLong_AsUnsignedLongLongMask(x);
        Py_DECREF(x);
        if (PyErr_Occurred()) refuse();
        return r;
    }
    // what ctypes takes for a float: any number (numpy's too)
    float real(int i)
    {
        if (!plain) return 0.0f;
        const double d = PyFloat_AsDouble(v[i]);
        if (d == -1.0 && PyErr_Occurred()) refuse();
        return static_cast<float>(d);
    }

    // a sequence of n (n < 0: any number, 1 .. most); lists and tuples are taken as they are, so a list's items are
    // read through integer_at() wherever Python code may have run since
    PyObject* sequence(int i, int64_t n, int64_t most, int64_t* count)
    {
        if (!plain) return nullptr;
        if (!PyList_CheckExact(v[i]) && !PyTuple_CheckExact(v[i]) && !PySequence_Check(v[i])) {
            refuse();
            return nullptr;
        }
        PyObject* f = PySequence_Fast(v[i], "");
        if (!f) {
            refuse();
            return nullptr;
        }
        held[n_held++] = f;
        const int64_t k = PySequence_Fast_GET_SIZE(f);
        if ((n >= 0 && k != n) || k < 1 || k > most) {
            refuse();
            return nullptr;
        }
        if (count) *count = k;
        return f;
    }
    // the integer at place k of a sequence: its conversion may run Python code, which may change the sequence
    int64_t integer_at(PyObject* f, int64_t k)
    {
        if (!plain) return 0;
        if (k >= PySequence_Fast_GET_SIZE(f)) {
            refuse();
            return 0;
        }
        PyObject* o = PySequence_Fast_GET_ITEM(f, k);
        Py_INCREF(o);
        const int64_t r = integer_of(o);
        Py_DECREF(o);
        return r;
    }
    int64_t gradients(int i, int64_t P, const float** out, int64_t most)
    {
        int64_t K = 0;
        PyObject* f = sequence(i, -1, most, &K);
        for (int64_t k = 0; plain && k < K; ++k)   // no Python code runs in between
            out[k] = static_cast<const float*>(tensor_of(PySequence_Fast_GET_ITEM(f, k), c10::ScalarType::Float, P));
        return K;
    }
    void clients(int i, int64_t K, int32_t* out)
    {
        PyObject* f = sequence(i, K, K, nullptr);
        for (int64_t k = 0; plain && k < K; ++k) out[k] = narrow(integer_at(f, k));
    }
    void timestamps(int i, int64_t K, int64_t* out)
    {
        PyObject* f = sequence(i, K, K, nullptr);
        for (int64_t k = 0; plain && k < K; ++k) out[k] = integer_at(f, k);
    }
    // host offsets of S + 1 segments: a C-contiguous one-dimensional int64 array
    const int64_t* segments(int i, int32_t* S)
    {
        if (!plain) return nullptr;
        if (PyObject_GetBuffer(v[i], &seg_view, PyBUF_FORMAT | PyBUF_C_CONTIGUOUS) != 0) {
            seg_view.obj = nullptr;
            refuse();
            return nullptr;
        }
        const char* f = seg_view.format;
        if (seg_view.ndim != 1 || seg_view.itemsize != 8 || !f || (f[0] != 'l' && f[0] != 'q') || f[1] ||
            seg_view.len / 8 - 1 < 0 || seg_view.len / 8 - 1 > INT32_MAX) {
            refuse();
            return nullptr;
        }
        *S = static_cast<int32_t>(seg_view.len / 8 - 1);
        return static_cast<const int64_t*>(seg_view.buf);
    }
    // the stream's handle, or it itself; None: the current stream (looked up last, after every tensor was found to be a device one)
    hipStream_t stream(int i)
    {
        if (!plain) return nullptr;
        PyObject* h;
        if (v[i] == Py_None) {
            h = PyObject_CallNoArgs(g_current_stream);
            if (!h) {   // whatever it raises is the call's
                plain = false;
                return nullptr;
            }
        } else if (PyLong_CheckExact(v[i])) {   // a raw handle
            h = v[i];
            Py_INCREF(h);
        } else {
            h = PyObject_GetAttrString(v[i], "cuda_stream");
        }
        if (!h || !PyLong_Check(h)) {
            Py_XDECREF(h);
            refuse();
            return nullptr;
        }
        void* p = PyLong_AsVoidPtr(h);
        Py_DECREF(h);
        if (PyErr_Occurred()) refuse();
        return static_cast<hipStream_t>(p);
    }
};

int64_t index_length(int64_t P) { return P < 1 ? 0 : (P + 255) / 256 + 1; }

// The library call itself, without the interpreter's lock; None unless the arguments were plain, or the exception
// that a getter left set.
template <typename Call>
PyObject* finish(Args& a, Call call)
{
    if (!a.plain) {
        if (PyErr_Occurred()) return nullptr;
        Py_RETURN_NONE;
    }
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = static_cast<int>(call());
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

bool arity(Py_ssize_t n, Py_ssize_t want)
{
    if (n == want && g_current_stream) return true;
    PyErr_SetString(PyExc_TypeError, "_marshal: wrong number of arguments, or bind() not called");
    return false;
}

// (state, grads, clients, grad_ts, stream)
template <bool FASGD>
PyObject* dense(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    if (!arity(n, 5)) return nullptr;
    Args a(args);
    fasgd_state* st = a.state(0);
    const float* g[FASGD_MAX_K];
    int32_t cl[FASGD_MAX_K];
    int64_t ts[FASGD_MAX_K];
    const int64_t K = a.gradients(1, st ? st->P : 0, g, FASGD_MAX_K);
    a.clients(2, K, cl);
    a.timestamps(3, K, ts);
    hipStream_t s = a.stream(4);
    return finish(a, [&] {
        return (FASGD ? g_lib.fasgd_apply_updates : g_lib.sasgd_apply_updates)(st, g, cl, ts, static_cast<int32_t>(K), s);
    });
}

// (state, grad, c, eps_c, seed, T, client, out_idx, out_val, d_count, workspace, seg_start, stream)
PyObject* select_compact(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    if (!arity(n, 13)) return nullptr;
    Args a(args);
    fasgd_state* st = a.state(0);
    const int64_t P = st ? st->P : 0;
    int64_t cap = 0, ws = 0;
    const float* g = a.floats(1, P);
    const float c = a.real(2), eps_c = a.real(3);
    const uint64_t seed = a.seed(4);
    const int64_t T = a.int64(5);
    const int32_t client = a.int32(6);
    int32_t* idx = a.ints(7, -1, &cap);
    float* val = a.floats(8, cap);
    int64_t* cnt = a.counts(9, -1);
    void* w = a.tensor(10, c10::ScalarType::Byte, -1, 0, &ws);
    uint32_t* seg = a.seg_start(11, index_length(P), false);
    hipStream_t s = a.stream(12);
    return finish(a, [&] {
        return g_lib.bfasgd_select_compact(st, g, c, eps_c, seed, T, client, idx, val, cap, cnt, seg, w,
                                           static_cast<size_t>(ws), s);
    });
}

// (state, grads, c, eps_c, seed, T, clients, out_idx, out_val, d_count, workspace, seg_start, stream)
PyObject* select_compact_batch(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    if (!arity(n, 13)) return nullptr;
    Args a(args);
    fasgd_state* st = a.state(0);
    const int64_t P = st ? st->P : 0;
    const float* g[FASGD_MAX_BATCH];
    int64_t T[FASGD_MAX_BATCH], ws = 0;
    int32_t cl[FASGD_MAX_BATCH];
    const int64_t B = a.gradients(1, P, g, FASGD_MAX_BATCH);
    const float c = a.real(2), eps_c = a.real(3);
    const uint64_t seed = a.seed(4);
    a.timestamps(5, B, T);
    a.clients(6, B, cl);
    const int64_t cap = a.columns(7, B);
    a.columns(8, B);
    int32_t* idx = a.ints(7, B * cap);
    float* val = a.floats(8, B * cap);
    int64_t* cnt = a.counts(9, B);
    void* w = a.tensor(10, c10::ScalarType::Byte, -1, 0, &ws);
    if (a.plain && a.v[11] != Py_None && a.columns(11, B) != index_length(P)) a.refuse();
    uint32_t* seg = a.seg_start(11, B * index_length(P), false, true);
    hipStream_t s = a.stream(12);
    return finish(a, [&] {
        return g_lib.bfasgd_select_compact_batch(st, static_cast<int32_t>(B), g, c, eps_c, seed, T, cl, idx, val, cap, cnt,
                                                 seg, w, static_cast<size_t>(ws), s);
    });
}

// (state, idx, val, d_count, client, grad_ts, stream)
PyObject* apply_sparse(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    if (!arity(n, 7)) return nullptr;
    Args a(args);
    fasgd_state* st = a.state(0);
    int64_t cap = 0;
    const int32_t* idx = a.ints(1, -1, &cap);
    const float* val = a.floats(2, cap);
    const int64_t* cnt = a.counts(3, -1);
    const int32_t client = a.int32(4);
    const int64_t ts = a.int64(5);
    hipStream_t s = a.stream(6);
    return finish(a, [&] { return g_lib.bfasgd_apply_sparse(st, idx, val, cnt, cap, client, ts, s); });
}

// (state, push_idx, push_val, push_count, push_seg_start, push_client, push_grad_ts, grads, clients, grad_ts, stream)
PyObject* with_push(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    if (!arity(n, 11)) return nullptr;
    Args a(args);
    fasgd_state* st = a.state(0);
    const int64_t P = st ? st->P : 0;
    int64_t cap = 0;
    const float* g[FASGD_MAX_K];
    int32_t cl[FASGD_MAX_K];
    int64_t ts[FASGD_MAX_K];
    const int32_t* idx = a.ints(1, -1, &cap);
    const float* val = a.floats(2, cap);
    const int64_t* cnt = a.counts(3, -1);
    const uint32_t* seg = a.seg_start(4, index_length(P), true);
    const int32_t client = a.int32(5);
    const int64_t push_ts = a.int64(6);
    const int64_t K = a.gradients(7, P, g, FASGD_MAX_K);
    a.clients(8, K, cl);
    a.timestamps(9, K, ts);
    hipStream_t s = a.stream(10);
    return finish(a, [&] {
        return g_lib.fasgd_apply_with_push(st, idx, val, cnt, seg, cap, client, push_ts, g, cl, ts,
                                           static_cast<int32_t>(K), s);
    });
}

// (state, push_idx, push_val, push_count, push_seg_start, push_client, push_grad_ts, grads, clients, grad_ts,
//  next_grad, next_client, c, eps_c, seed, out_idx, out_val, out_count, out_seg_start, workspace, stream)
PyObject* with_push_and_select(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    if (!arity(n, 21)) return nullptr;
    Args a(args);
    fasgd_state* st = a.state(0);
    const int64_t P = st ? st->P : 0;
    int64_t cap = 0, out_cap = 0, ws = 0;
    const float* g[FASGD_MAX_K];
    int32_t cl[FASGD_MAX_K];
    int64_t ts[FASGD_MAX_K];
    const int32_t* idx = a.ints(1, -1, &cap);
    const float* val = a.floats(2, cap);
    const int64_t* cnt = a.counts(3, -1);
    const uint32_t* seg = a.seg_start(4, index_length(P), true);
    const int32_t client = a.int32(5);
    const int64_t push_ts = a.int64(6);
    const int64_t K = a.gradients(7, P, g, FASGD_MAX_K);
    a.clients(8, K, cl);
    a.timestamps(9, K, ts);
    const float* next = a.floats(10, P);
    const int32_t next_client = a.int32(11);
    const float c = a.real(12), eps_c = a.real(13);
    const uint64_t seed = a.seed(14);
    int32_t* out_idx = a.ints(15, -1, &out_cap);
    float* out_val = a.floats(16, out_cap);
    int64_t* out_cnt = a.counts(17, -1);
    uint32_t* out_seg = a.seg_start(18, index_length(P), false);
    void* w = a.tensor(19, c10::ScalarType::Byte, -1, 0, &ws);
    hipStream_t s = a.stream(20);
    return finish(a, [&] {
        return g_lib.fasgd_apply_with_push_and_select(st, idx, val, cnt, seg, cap, client, push_ts, g, cl, ts,
                                                      static_cast<int32_t>(K), next, next_client, c, eps_c, seed, out_idx,
                                                      out_val, out_cap, out_cnt, out_seg, w, static_cast<size_t>(ws), s);
    });
}

// (state, idx, val, d_count, seg_start, clients, grad_ts, stream)
PyObject* apply_pushes(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    if (!arity(n, 8)) return nullptr;
    Args a(args);
    fasgd_state* st = a.state(0);
    const int64_t P = st ? st->P : 0;
    int32_t cl[FASGD_MAX_BATCH];
    int64_t ts[FASGD_MAX_BATCH], B = 0;
    PyObject* f = a.sequence(5, -1, FASGD_MAX_BATCH, &B);
    for (int64_t b = 0; a.plain && b < B; ++b) cl[b] = a.narrow(a.integer_at(f, b));
    a.timestamps(6, B, ts);
    const int64_t cap = a.columns(1, B);
    a.columns(2, B);
    const int32_t* idx = a.ints(1, B * cap);
    const float* val = a.floats(2, B * cap);
    const int64_t* cnt = a.counts(3, B);
    if (a.columns(4, B) != index_length(P)) a.refuse();
    const uint32_t* seg = a.seg_start(4, B * index_length(P), true, true);
    hipStream_t s = a.stream(7);
    return finish(a, [&] {
        return g_lib.fasgd_apply_pushes(st, static_cast<int32_t>(B), idx, val, cnt, seg, cap, cl, ts, s);
    });
}

// (state, idx, val, d_count, cache, client, grad_ts, seg_start, stream)
PyObject* apply_cached(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    if (!arity(n, 9)) return nullptr;
    Args a(args);
    fasgd_state* st = a.state(0);
    const int64_t P = st ? st->P : 0;
    int64_t cap = 0;
    const int32_t* idx = a.ints(1, -1, &cap);
    const float* val = a.floats(2, cap);
    const int64_t* cnt = a.counts(3, -1);
    float* cache = a.floats(4, P);
    const int32_t client = a.int32(5);
    const int64_t ts = a.int64(6);
    const uint32_t* seg = a.seg_start(7, index_length(P), false);
    hipStream_t s = a.stream(8);
    return finish(a, [&] { return g_lib.bfasgd_apply_cached(st, idx, val, cnt, seg, cap, cache, client, ts, s); });
}

// (theta_client, idx, val, d_count, seg_start, stream)
PyObject* apply_fetch(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    if (!arity(n, 6)) return nullptr;
    Args a(args);
    int64_t P = 0, cap = 0;
    float* copy = a.floats(0, -1, &P);
    const int32_t* idx = a.ints(1, -1, &cap);
    const float* val = a.floats(2, cap);
    const int64_t* cnt = a.counts(3, -1);
    const uint32_t* seg = a.seg_start(4, index_length(P), false);
    hipStream_t s = a.stream(5);
    return finish(a, [&] { return g_lib.bfasgd_apply_fetch(copy, P, idx, val, cnt, seg, cap, s); });
}

// (state, seg, c, eps_c, seed, T, client, d_transmit, workspace, stream)
PyObject* decide_segments(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    if (!arity(n, 10)) return nullptr;
    Args a(args);
    fasgd_state* st = a.state(0);
    int32_t S = 0;
    int64_t ws = 0;
    const int64_t* seg = a.segments(1, &S);
    const float c = a.real(2), eps_c = a.real(3);
    const uint64_t seed = a.seed(4);
    const int64_t T = a.int64(5);
    const int32_t client = a.int32(6);
    uint8_t* send = static_cast<uint8_t*>(a.tensor(7, c10::ScalarType::Byte, S));
    void* w = a.tensor(8, c10::ScalarType::Byte, -1, 0, &ws);
    hipStream_t s = a.stream(9);
    return finish(a, [&] {
        return g_lib.bfasgd_decide_segments(st, seg, S, c, eps_c, seed, T, client, send, w, static_cast<size_t>(ws), s);
    });
}

// (state, grad, seg, d_transmit, client, grad_ts, stream)
PyObject* apply_segments(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    if (!arity(n, 7)) return nullptr;
    Args a(args);
    fasgd_state* st = a.state(0);
    int32_t S = 0;
    const float* g = a.floats(1, st ? st->P : 0);
    const int64_t* seg = a.segments(2, &S);
    const uint8_t* send = static_cast<const uint8_t*>(a.tensor(3, c10::ScalarType::Byte, -1, S));   // one byte per segment
    const int32_t client = a.int32(4);
    const int64_t ts = a.int64(5);
    hipStream_t s = a.stream(6);
    return finish(a, [&] { return g_lib.bfasgd_apply_segments(st, g, seg, S, send, client, ts, s); });
}

// ---- the client's operators

// A matrix of activations: one or two dimensions, last stride 1.
struct Matrix {
    void* p = nullptr;
    int64_t rows = 0, cols = 0, ld = 0;
    int32_t dtype = -1;
    int dim = 0;
};

struct ClientArgs : Args {
    Py_buffer operand_view[2] = {};
    explicit ClientArgs(PyObject* const* args) : Args(args) {}
    ~ClientArgs()
    {
        for (Py_buffer& b : operand_view)
            if (b.obj) PyBuffer_Release(&b);
    }

    Matrix matrix(int i)
    {
        Matrix m;
        if (!plain) return m;
        if (!THPVariable_CheckExact(v[i])) {
            refuse();
            return m;
        }
        try {
            const at::Tensor& t = THPVariable_Unpack(v[i]);
            switch (t.scalar_type()) {
            case c10::ScalarType::Float: m.dtype = CLIENT_F32; break;
            case c10::ScalarType::BFloat16: m.dtype = CLIENT_BF16; break;
            case c10::ScalarType::Half: m.dtype = CLIENT_F16; break;
            default: break;
            }
            m.dim = static_cast<int>(t.dim());
            if (!t.is_cuda() || m.dtype < 0 || m.dim < 1 || m.dim > 2) {
                refuse();
                return m;
            }
            m.rows = m.dim == 2 ? t.size(0) : 1;
            m.cols = t.size(m.dim - 1);
            if (m.cols > 1 && t.stride(m.dim - 1) != 1) {
                refuse();
                return m;
            }
            m.ld = m.rows > 1 ? t.stride(0) : m.cols;
            m.p = t.data_ptr();
        } catch (...) {
            refuse();
        }
        return m;
    }
    // one of the shape and type of `like`; None where it may be absent
    Matrix matrix_like(int i, const Matrix& like, bool optional = false)
    {
        if (!plain || (optional && v[i] == Py_None)) return Matrix{};
        const Matrix m = matrix(i);
        if (plain && (m.dtype != like.dtype || m.dim != like.dim || m.rows != like.rows || m.cols != like.cols)) refuse();
        return m;
    }
    // an optional parameter vector
    float* parameters(int i, int64_t n) { return plain && v[i] != Py_None ? floats(i, n) : nullptr; }
    double wide_real(PyObject* o)
    {
        if (!plain) return 0.0;
        const double d = PyFloat_AsDouble(o);
        if (d == -1.0 && PyErr_Occurred()) refuse();
        return d;
    }
    uint64_t seed_of(PyObject* o)
    {
        if (!plain) return 0;
        PyObject* x = PyNumber_Index(o);
        if (!x) {
            refuse();
            return 0;
        }
        const uint64_t r = PyLong_AsUnsignedLongLongMask(x);
        Py_DECREF(x);
        if (PyErr_Occurred()) refuse();
        return r;
    }
    // an 8-bit operand's struct (a ctypes Structure, by its buffer); None: NULL
    client_fp8_operand* operand(int i, int which)
    {
        if (!plain || v[i] == Py_None) return nullptr;
        if (PyObject_GetBuffer(v[i], &operand_view[which], PyBUF_WRITABLE) != 0 ||
            operand_view[which].len != static_cast<Py_ssize_t>(sizeof(client_fp8_operand))) {
            refuse();
            return nullptr;
        }
        return static_cast<client_fp8_operand*>(operand_view[which].buf);
    }
    void* workspace(int i, int64_t* n)
    {
        *n = 0;
        return plain && v[i] != Py_None ? tensor(i, c10::ScalarType::Byte, -1, 0, n) : nullptr;
    }
    // a contiguous int64 tensor [rows] (columns NULL) or [rows][*columns]
    const int64_t* indices(int i, int64_t rows, int64_t* columns)
    {
        if (!plain) return nullptr;
        try {
            if (THPVariable_CheckExact(v[i])) {
                const at::Tensor& t = THPVariable_Unpack(v[i]);
                if (t.dim() == (columns ? 2 : 1) && t.size(0) == rows) {
                    if (columns) *columns = t.size(1);
                    return static_cast<const int64_t*>(tensor(i, c10::ScalarType::Long, -1));
                }
            }
        } catch (...) {
        }
        refuse();
        return nullptr;
    }
    // x, w and the scale of their logits
    client_vocab_head head(int x, int w, int scale)
    {
        client_vocab_head op;
        memset(&op, 0, sizeof op);
        const Matrix a = matrix(x), b = matrix(w);
        if (plain && (a.dim != 2 || b.dim != 2 || a.dtype != b.dtype || a.cols != b.cols)) refuse();
        op.rows = a.rows;
        op.cols = a.cols;
        op.vocab = b.rows;
        op.dtype = a.dtype;
        op.logit_scale = real(scale);
        op.x = a.p;
        op.ld_x = a.ld;
        op.w = b.p;
        op.ld_w = b.ld;
        return op;
    }
    // a teacher's logits, contiguous and of x's type, at `columns` classes a row
    const void* teacher(int i, const client_vocab_head& op, int64_t columns)
    {
        const Matrix m = matrix(i);
        if (plain && (m.dim != 2 || m.dtype != op.dtype || m.rows != op.rows || m.cols != columns || columns > INT32_MAX ||
                      (m.rows > 1 && m.ld != m.cols)))
            refuse();
        return m.p;
    }
    // dx, dw, dloss, grad_scale, accumulate
    struct Gradients {
        Matrix dx, dw;
        const float* dloss;
        float scale;
        bool add;
    };
    Gradients gradients_of(int at, const client_vocab_head& op)
    {
        Gradients g;
        if (plain && v[at] != Py_None) {
            g.dx = matrix(at);
            if (plain && (g.dx.dim != 2 || g.dx.dtype != op.dtype || g.dx.rows != op.rows || g.dx.cols != op.cols)) refuse();
        }
        g.dw.dtype = CLIENT_F32;
        if (plain && v[at + 1] != Py_None) {
            g.dw = matrix(at + 1);
            if (plain && (g.dw.dim != 2 || (g.dw.dtype != CLIENT_F32 && g.dw.dtype != op.dtype) || g.dw.rows != op.vocab ||
                          g.dw.cols != op.cols))
                refuse();
        }
        g.dloss = parameters(at + 2, op.rows);
        g.scale = real(at + 3);
        g.add = truth(at + 4);
        return g;
    }
    // a truth value
    bool truth(int i)
    {
        if (v[i] != Py_True && v[i] != Py_False) refuse();
        return v[i] == Py_True;
    }
    // the type of a product's output, with the choice of short sums
    int32_t output_type(const Matrix& m, int i) { return truth(i) ? m.dtype | CLIENT_FP8_SHORT_SUMS : m.dtype; }
    // gate forms as the binding's general way tells them apart
    bool gate(int i, const Matrix& like, int32_t* form, void** p, int64_t* ld)
    {
        *form = CLIENT_GATE_NONE;
        *p = nullptr;
        *ld = 0;
        if (!plain || v[i] == Py_None) return plain;
        const Matrix g = matrix(i);
        if (!plain) return false;
        const bool same = g.dtype == like.dtype && g.dim == like.dim && g.rows == like.rows && g.cols == like.cols;
        if (same && (g.dim == 2 || g.dtype != CLIENT_F32)) {
            *form = CLIENT_GATE_FULL;
            *ld = g.ld;
        } else if (g.dtype != CLIENT_F32) {
            return refuse();
        } else if (g.dim == 1 && g.cols == like.cols) {
            *form = CLIENT_GATE_CHANNEL;
        } else if (g.dim == 2 && g.cols == 1 && g.rows == like.rows && (g.ld == 1 || g.rows == 1)) {
            *form = CLIENT_GATE_ROW;
        } else {
            return refuse();
        }
        *p = g.p;
        return true;
    }
    // from `at` on: kind, w_post, b_post, gate, gate_act, w_pre, b_pre, residual_scale, eps, dropout, index_base
    client_residual_norm norm(int at, const Matrix& x)
    {
        client_residual_norm op;
        memset(&op, 0, sizeof op);
        op.rows = x.rows;
        op.cols = x.cols;
        op.dtype = x.dtype;
        op.kind = int32(at);
        op.w_post = parameters(at + 1, x.cols);
        op.b_post = parameters(at + 2, x.cols);
        void* g = nullptr;
        gate(at + 3, x, &op.gate_form, &g, &op.ld_gate);
        op.gate = g;
        op.gate_act = int32(at + 4);
        op.w_pre = parameters(at + 5, x.cols);
        op.b_pre = parameters(at + 6, x.cols);
        op.residual_scale = real(at + 7);
        op.eps = real(at + 8);
        if (plain && v[at + 9] != Py_None) {
            PyObject* d = v[at + 9];
            if (!PyTuple_CheckExact(d) || PyTuple_GET_SIZE(d) != 5) {
                refuse();
                return op;
            }
            op.p = wide_real(PyTuple_GET_ITEM(d, 0));
            op.seed = seed_of(PyTuple_GET_ITEM(d, 1));
            op.T = integer_of(PyTuple_GET_ITEM(d, 2));
            op.client = narrow(integer_of(PyTuple_GET_ITEM(d, 3)));
            op.site = narrow(integer_of(PyTuple_GET_ITEM(d, 4)));
        }
        op.index_base = int64(at + 10);
        return op;
    }
};

// (x, out, p, seed, T, client, site, residual, index_base, stream)
PyObject* client_dropout_call(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    if (!arity(n, 10)) return nullptr;
    ClientArgs a(args);
    const Matrix x = a.matrix(0), y = a.matrix_like(1, x), r = a.matrix_like(7, x, true);
    const double p = a.wide_real(args[2]);
    const uint64_t seed = a.seed(3);
    const int64_t T = a.int64(4);
    const int32_t client = a.int32(5), site = a.int32(6);
    const int64_t base = a.int64(8);
    hipStream_t s = a.stream(9);
    return finish(a, [&] {
        return g_client.client_dropout(x.p, x.ld, r.p, r.ld, y.p, y.ld, x.rows, x.cols, x.dtype, p, seed, T, client,
                                       site, base, s);
    });
}

// (branch, residual, sum, normed, stats, the operator's 11, stream)
PyObject* norm_forward_call(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    if (!arity(n, 17)) return nullptr;
    ClientArgs a(args);
    const Matrix x = a.matrix(0), r = a.matrix_like(1, x, true), sum = a.matrix_like(2, x), h = a.matrix_like(3, x, true);
    float* stats = a.floats(4, 4 * x.rows);
    const client_residual_norm op = a.norm(5, x);
    hipStream_t s = a.stream(16);
    return finish(a, [&] {
        return g_client.client_residual_norm_forward(&op, x.p, x.ld, r.p, r.ld, sum.p, sum.ld, h.p, h.ld, stats, s);
    });
}

// (branch, sum, stats, dsum, dnormed, dbranch, dresidual, dw_post, db_post, dgate, dw_pre, db_pre, workspace, the
// operator's 11, stream)
PyObject* norm_backward_call(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    if (!arity(n, 25)) return nullptr;
    ClientArgs a(args);
    const Matrix x = a.matrix(0), sum = a.matrix_like(1, x, true);
    const float* stats = a.floats(2, 4 * x.rows);
    const Matrix ds = a.matrix_like(3, x, true), dh = a.matrix_like(4, x, true), dx = a.matrix_like(5, x),
                 dr = a.matrix_like(6, x, true);
    float* dwp = a.parameters(7, x.cols);
    float* dbp = a.parameters(8, x.cols);
    int32_t form = 0;
    void* dg = nullptr;
    int64_t ld_dg = 0;
    a.gate(9, x, &form, &dg, &ld_dg);
    float* dwn = a.parameters(10, x.cols);
    float* dbn = a.parameters(11, x.cols);
    int64_t ws = 0;
    void* w = a.workspace(12, &ws);
    const client_residual_norm op = a.norm(13, x);
    if (a.plain && dg && form != op.gate_form) a.refuse();
    hipStream_t s = a.stream(24);
    return finish(a, [&] {
        return g_client.client_residual_norm_backward(&op, x.p, x.ld, sum.p, sum.ld, stats, ds.p, ds.ld, dh.p, dh.ld, dx.p,
                                                      dx.ld, dr.p, dr.ld, dwp, dbp, dg, ld_dg, dwn, dbn, w,
                                                      static_cast<size_t>(ws), s);
    });
}

// (x, by_rows, by_cols, block_rows, stream)
PyObject* quantize_call(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    if (!arity(n, 5)) return nullptr;
    ClientArgs a(args);
    const Matrix x = a.matrix(0);
    const client_fp8_operand *r = a.operand(1, 0), *c = a.operand(2, 1);
    const int32_t block = a.int32(3);
    hipStream_t s = a.stream(4);
    return finish(a, [&] { return g_client.client_fp8_quantize(x.p, x.ld, x.rows, x.cols, x.dtype, block, r, c, s); });
}

// (a, b, out, accumulate, workspace, stream, short sums)
PyObject* matmul_call(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    if (!arity(n, 7)) return nullptr;
    ClientArgs a(args);
    const client_fp8_operand *x = a.operand(0, 0), *y = a.operand(1, 1);
    const Matrix c = a.matrix(2);
    if (a.plain && (!x || !y || c.rows != x->rows || c.cols != y->rows)) a.refuse();
    const bool add = a.truth(3);
    const int32_t type = a.output_type(c, 6);
    int64_t ws = 0;
    void* w = a.workspace(4, &ws);
    hipStream_t s = a.stream(5);
    return finish(a, [&] {
        return g_client.client_fp8_matmul(x, y, c.p, c.ld, type, add, w, static_cast<size_t>(ws), s);
    });
}

// (x, w, out, workspace, stream, short sums)
PyObject* linear_call(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    if (!arity(n, 6)) return nullptr;
    ClientArgs a(args);
    const Matrix x = a.matrix(0);
    const client_fp8_operand* w = a.operand(1, 0);
    const Matrix y = a.matrix(2);
    if (a.plain && (!w || x.dtype != y.dtype || x.cols != w->k || y.rows != x.rows || y.cols != w->rows)) a.refuse();
    const int32_t type = a.output_type(y, 5);
    int64_t ws = 0;
    void* p = a.workspace(3, &ws);
    hipStream_t s = a.stream(4);
    return finish(a, [&] {
        return g_client.client_fp8_linear(x.p, x.ld, x.rows, w, y.p, y.ld, type, p, static_cast<size_t>(ws), s);
    });
}

// (x, w, targets, loss, lse, picked, smoothing, z_loss, logit_scale, workspace, stream)
PyObject* vocab_loss_forward_call(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    if (!arity(n, 11)) return nullptr;
    ClientArgs a(args);
    const client_vocab_head op = a.head(0, 1, 8);
    const int64_t* targets = a.indices(2, op.rows, nullptr);
    float *loss = a.floats(3, op.rows), *lse = a.floats(4, op.rows), *picked = a.floats(5, op.rows);
    const float smoothing = a.real(6), z_loss = a.real(7);
    int64_t ws = 0;
    void* w = a.workspace(9, &ws);
    hipStream_t s = a.stream(10);
    return finish(a, [&] {
        return g_client.client_vocab_loss_forward(&op, targets, smoothing, z_loss, loss, lse, picked, w,
                                                  static_cast<size_t>(ws), s);
    });
}

// (x, w, targets, lse, picked, dx, dw, dloss, grad_scale, accumulate, smoothing, z_loss, logit_scale, workspace, stream)
PyObject* vocab_loss_backward_call(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    if (!arity(n, 15)) return nullptr;
    ClientArgs a(args);
    const client_vocab_head op = a.head(0, 1, 12);
    const int64_t* targets = a.indices(2, op.rows, nullptr);
    const float *lse = a.floats(3, op.rows), *picked = a.floats(4, op.rows);
    const ClientArgs::Gradients g = a.gradients_of(5, op);
    const float smoothing = a.real(10), z_loss = a.real(11);
    int64_t ws = 0;
    void* w = a.workspace(13, &ws);
    hipStream_t s = a.stream(14);
    return finish(a, [&] {
        return g_client.client_vocab_loss_backward(&op, targets, smoothing, z_loss, lse, picked, g.dloss, g.scale, g.dx.p,
                                                   g.dx.ld, g.dw.p, g.dw.ld, g.dw.dtype, g.add, w,
                                                   static_cast<size_t>(ws), s);
    });
}

// (x, w, index, teacher, loss, lse, picked, teacher_scale, teacher_lse, logit_scale, workspace, stream)
PyObject* vocab_distill_forward_call(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    if (!arity(n, 12)) return nullptr;
    ClientArgs a(args);
    const client_vocab_head op = a.head(0, 1, 9);
    int64_t k = 0;
    const int64_t* index = a.indices(2, op.rows, &k);
    const void* teacher = a.teacher(3, op, k);
    float *loss = a.floats(4, op.rows), *lse = a.floats(5, op.rows), *picked = a.floats(6, op.rows * k);
    const float scale = a.real(7);
    const float* teacher_lse = a.parameters(8, op.rows);
    int64_t ws = 0;
    void* w = a.workspace(10, &ws);
    hipStream_t s = a.stream(11);
    return finish(a, [&] {
        return g_client.client_vocab_distill_forward(&op, index, teacher, static_cast<int32_t>(k), scale, teacher_lse, loss,
                                                     lse, picked, w, static_cast<size_t>(ws), s);
    });
}

// (x, w, index, teacher, lse, picked, dx, dw, dloss, grad_scale, accumulate, teacher_scale, teacher_lse, logit_scale,
// workspace, stream)
PyObject* vocab_distill_backward_call(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    if (!arity(n, 16)) return nullptr;
    ClientArgs a(args);
    const client_vocab_head op = a.head(0, 1, 13);
    int64_t k = 0;
    const int64_t* index = a.indices(2, op.rows, &k);
    const void* teacher = a.teacher(3, op, k);
    const float *lse = a.floats(4, op.rows), *picked = a.floats(5, op.rows * k);
    const ClientArgs::Gradients g = a.gradients_of(6, op);
    const float scale = a.real(11);
    const float* teacher_lse = a.parameters(12, op.rows);
    int64_t ws = 0;
    void* w = a.workspace(14, &ws);
    hipStream_t s = a.stream(15);
    return finish(a, [&] {
        return g_client.client_vocab_distill_backward(&op, index, teacher, static_cast<int32_t>(k), scale, teacher_lse, lse,
                                                      picked, g.dloss, g.scale, g.dx.p, g.dx.ld, g.dw.p, g.dw.ld,
                                                      g.dw.dtype, g.add, w, static_cast<size_t>(ws), s);
    });
}

// bind_client(addresses of the entry points in kClientNames' order), after bind()
PyObject* bind_client(PyObject*, PyObject* list)
{
    if (!PyList_Check(list) || PyList_GET_SIZE(list) != kClientCount) {
        PyErr_SetString(PyExc_ValueError, "_marshal.bind_client: one address per entry point");
        return nullptr;
    }
    void* p[kClientCount];
    for (int i = 0; i < kClientCount; ++i) {
        p[i] = PyLong_AsVoidPtr(PyList_GET_ITEM(list, i));
        if (PyErr_Occurred()) return nullptr;
        if (!p[i]) {
            PyErr_SetString(PyExc_ValueError, "_marshal.bind_client: NULL address");
            return nullptr;
        }
    }
    memcpy(&g_client, p, sizeof g_client);
    Py_RETURN_NONE;
}

// bind(addresses of the entry points in kNames' order, current-stream callable)
PyObject* bind(PyObject*, PyObject* args)
{
    PyObject *list, *stream;
    if (!PyArg_ParseTuple(args, "O!O", &PyList_Type, &list, &stream)) return nullptr;
    if (PyList_GET_SIZE(list) != kCount || !PyCallable_Check(stream)) {
        PyErr_SetString(PyExc_ValueError, "_marshal.bind: one address per entry point and a callable");
        return nullptr;
    }
    void* p[kCount];
    for (int i = 0; i < kCount; ++i) {
        p[i] = PyLong_AsVoidPtr(PyList_GET_ITEM(list, i));
        if (PyErr_Occurred()) return nullptr;
        if (!p[i]) {
            PyErr_SetString(PyExc_ValueError, "_marshal.bind: NULL address");
            return nullptr;
        }
    }
    memcpy(&g_lib, p, sizeof g_lib);
    Py_INCREF(stream);
    Py_XSETREF(g_current_stream, stream);
    Py_RETURN_NONE;
}

using FastCall = PyObject* (*)(PyObject*, PyObject* const*, Py_ssize_t);
PyCFunction fast(FastCall f) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)); }

PyMethodDef kMethods[] = {{"bind", bind, METH_VARARGS, nullptr},
                          {kNames[0], fast(dense<true>), METH_FASTCALL, nullptr},
                          {kNames[1], fast(dense<false>), METH_FASTCALL, nullptr},
                          {kNames[2], fast(select_compact), METH_FASTCALL, nullptr},
                          {kNames[3], fast(select_compact_batch), METH_FASTCALL, nullptr},
                          {kNames[4], fast(apply_sparse), METH_FASTCALL, nullptr},
                          {kNames[5], fast(with_push), METH_FASTCALL, nullptr},
                          {kNames[6], fast(with_push_and_select), METH_FASTCALL, nullptr},
                          {kNames[7], fast(apply_pushes), METH_FASTCALL, nullptr},
                          {kNames[8], fast(apply_cached), METH_FASTCALL, nullptr},
                          {kNames[9], fast(apply_fetch), METH_FASTCALL, nullptr},
                          {kNames[10], fast(decide_segments), METH_FASTCALL, nullptr},
                          {kNames[11], fast(apply_segments), METH_FASTCALL, nullptr},
                          {"bind_client", bind_client, METH_O, nullptr},
                          {kClientNames[0], fast(client_dropout_call), METH_FASTCALL, nullptr},
                          {kClientNames[1], fast(norm_forward_call), METH_FASTCALL, nullptr},
                          {kClientNames[2], fast(norm_backward_call), METH_FASTCALL, nullptr},
                          {kClientNames[3], fast(quantize_call), METH_FASTCALL, nullptr},
                          {kClientNames[4], fast(matmul_call), METH_FASTCALL, nullptr},
                          {kClientNames[5], fast(linear_call), METH_FASTCALL, nullptr},
                          {kClientNames[6], fast(vocab_loss_forward_call), METH_FASTCALL, nullptr},
                          {kClientNames[7], fast(vocab_loss_backward_call), METH_FASTCALL, nullptr},
                          {kClientNames[8], fast(vocab_distill_forward_call), METH_FASTCALL, nullptr},
                          {kClientNames[9], fast(vocab_distill_backward_call), METH_FASTCALL, nullptr},
                          {nullptr, nullptr, 0, nullptr}};

PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal()
{
    PyObject* m = PyModule_Create(&kModule);
    if (!m) return nullptr;
    PyObject* names = PyTuple_New(kCount);
    if (!names) return nullptr;
    for (int i = 0; i < kCount; ++i) PyTuple_SET_ITEM(names, i, PyUnicode_FromString(kNames[i]));
    if (PyModule_AddObject(m, "ENTRY_POINTS", names) != 0) return nullptr;
    PyObject* client = PyTuple_New(kClientCount);
    if (!client) return nullptr;
    for (int i = 0; i < kClientCount; ++i) PyTuple_SET_ITEM(client, i, PyUnicode_FromString(kClientNames[i]));
    if (PyModule_AddObject(m, "CLIENT_ENTRY_POINTS", client) != 0) return nullptr;
    // at::Tensor's layout is that torch's alone
    if (PyModule_AddStringConstant(m, "TORCH_VERSION", FASGD_TORCH_VERSION) != 0) return nullptr;
    return m;
}
