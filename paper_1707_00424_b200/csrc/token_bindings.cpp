// The Python side of the token operators (module _token_ops): checks of the tensors and one call of the C ABI each.  In C++ because a
// call of a small operator is shorter than its checks are in Python: issuing a dropout of 77 x 1001 took 6.6 us with checks in Python
// and ctypes, 3.3 us here, nearly all of it
// the launch.  Arguments come by position from token_ops.py, which documents them.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <limits.h>

#include <initializer_list>
#include <string>
#include <vector>

#include "../../include/parle.h"

namespace {

PyObject *g_error = nullptr;                              // ParleError(code, what)

[[noreturn]] void fail(int code, const std::string &what) {
    PyObject *e = PyObject_CallFunction(g_error, "is", code, what.c_str());
    if (e) {
        PyErr_SetObject(g_error, e);
        Py_DECREF(e);
    }
    throw python_error();
}

// Without the interpreter's lock: an allocation may wait for the device, a launch for room in its queue.
struct Unlocked {
    PyThreadState *state = PyEval_SaveThread();
    ~Unlocked() { PyEval_RestoreThread(state); }
};

// One call: its name for messages, the device of its first tensor, the stream it runs on.
struct Call {
    const char *name;
    int index = -1;
    cudaStream_t stream = nullptr;
    c10::cuda::OptionalCUDAStreamGuard stream_guard;
    c10::cuda::OptionalCUDAGuard device_guard;

    explicit Call(const char *name_) : name(name_) {}
    [[noreturn]] void refuse(const std::string &why) const { fail(PARLE_EINVAL, std::string(name) + ": " + why); }
    template <class F>
    void run(F f) const {
        int rc;
        {
            const Unlocked u;
            rc = f();
        }
        if (rc != PARLE_OK) fail(rc, name);
    }

    // Behind the call: the given ones of these results have been written, which autograd's check of saved tensors has to see.  (An inference
    // tensor has no version; nothing saves it.)
    static void written(std::initializer_list<PyObject *> results) {
        for (PyObject *o : results) {
            if (o == Py_None) continue;
            const at::Tensor &t = THPVariable_Unpack(o);
            if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
        }
    }

    // The tensor that decides the device, and the stream: `stream` or the device's current one.
    const at::Tensor &first(const char *what, PyObject *o, PyObject *given_stream) {
        const at::Tensor &t = tensor(what, o);
        if (!t.is_cuda()) refuse(std::string(what) + " is on " + t.device().str() + ": a CUDA device is needed");
        index = t.get_device();
        if (given_stream == Py_None) {
            if (c10::cuda::current_device() != index) device_guard.set_index((c10::DeviceIndex)index);
            stream = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)index).stream();
        } else {
            const c10::cuda::CUDAStream s = c10::cuda::CUDAStream::unpack3(attribute(given_stream, "stream_id"), (c10::DeviceIndex)attribute(given_stream, "device_index"),
                                                                           (c10::DeviceType)attribute(given_stream, "device_type"));
            if (s.device_index() != index) refuse("the stream is on " + s.device().str() + ", the tensors on " + t.device().str());
            stream_guard.reset_stream(s);                 // (results are allocated for this stream, too)
            stream = s.stream();
        }
        return t;
    }
    long long attribute(PyObject *o, const char *what) const {
        PyObject *v = PyObject_GetAttrString(o, what);
        if (!v) throw python_error();
        const long long n = PyLong_AsLongLong(v);
        Py_DECREF(v);
        if (n == -1 && PyErr_Occurred()) throw python_error();
        return n;
    }
    const at::Tensor &tensor(const char *what, PyObject *o) const {
        if (!THPVariable_Check(o)) refuse(std::string(what) + " has to be a tensor, not " + Py_TYPE(o)->tp_name);
        return THPVariable_Unpack(o);
    }
    void here(const char *what, const at::Tensor &t) const {
        if (!t.is_cuda() || t.get_device() != index) refuse(std::string(what) + " is on " + t.device().str() + ", the other tensors on cuda:" + std::to_string(index));
    }
    static std::string describe(const at::Tensor &t) {
        std::string s = std::string(c10::toString(t.scalar_type())) + " [";
        for (int64_t i = 0; i < t.dim(); ++i) s += (i ? ", " : "") + std::to_string(t.size(i));
        s += "], strides [";
        for (int64_t i = 0; i < t.dim(); ++i) s += (i ? ", " : "") + std::to_string(t.stride(i));
        return s + "]";
    }
    int dtype(const char *what, const at::Tensor &t) const {
        switch (t.scalar_type()) {
            case at::kFloat: return PARLE_F32;
            case at::kBFloat16: return PARLE_BF16;
            case at::kHalf: return PARLE_F16;
            default: refuse(std::string(what) + " is " + describe(t) + ": fp32, bf16 and fp16 are supported");
        }
    }
    // A contiguous tensor of this shape and type.
    void *dense(const char *what, const at::Tensor &t, at::IntArrayRef shape, at::ScalarType type) const {
        if (t.sizes() != shape || t.scalar_type() != type || !t.is_contiguous()) {
            std::string s;
            for (const int64_t n : shape) s += (s.empty() ? "" : ", ") + std::to_string(n);
            refuse(std::string(what) + " has to be a contiguous " + c10::toString(type) + " tensor of shape [" + s + "], not " + describe(t));
        }
        here(what, t);
        return t.data_ptr();
    }
    void *dense_or_null(const char *what, PyObject *o, at::IntArrayRef shape, at::ScalarType type) const {
        return o == Py_None ? nullptr : dense(what, tensor(what, o), shape, type);
    }
    // A tensor of one element; NULL for None.
    void *word(const char *what, PyObject *o, at::ScalarType type, at::ScalarType other) const {
        if (o == Py_None) return nullptr;
        const at::Tensor &t = tensor(what, o);
        if (t.numel() != 1 || (t.scalar_type() != type && t.scalar_type() != other)) refuse(std::string(what) + " has to be one " + c10::toString(type) + ", not " + describe(t));
        here(what, t);
        return t.data_ptr();
    }
    // Dimensions first .. dim - 2 as rows of one pitch; the last dimension has to be dense.
    struct Rows {
        long long rows, cols, pitch;
    };
    Rows rows(const char *what, const at::Tensor &t, int64_t first) const {
        here(what, t);
        const int64_t d = t.dim();
        if (d < first + 1) refuse(std::string(what) + " has too few dimensions: " + describe(t));
        Rows r{1, t.size(d - 1), 0};
        if (r.cols > 1 && t.stride(d - 1) != 1) refuse(std::string("the last dimension of ") + what + " is not dense: " + describe(t));
        long long extent = 0;                             // of the dimensions behind, 0: none longer than 1
        for (int64_t i = d - 2; i >= first; --i) {
            const int64_t n = t.size(i);
            r.rows *= n;
            if (n == 1) continue;
            if (extent == 0) r.pitch = t.stride(i);
            else if (t.stride(i) != extent && t.numel() > 0) refuse(std::string(what) + " is no array of rows without a copy: " + describe(t));
            extent = t.stride(i) * n;
            if (extent == 0) extent = -1;                 // (a stride of 0 joins with nothing but 0)
            if (extent == -1 && i > first) {
                for (int64_t j = i - 1; j >= first; --j) {
                    r.rows *= t.size(j);
                    if (t.size(j) != 1 && t.stride(j) != 0 && t.numel() > 0) refuse(std::string(what) + " is no array of rows without a copy: " + describe(t));
                }
                break;
            }
        }
        if (r.rows <= 1) r.pitch = r.cols;                // the pitch of one row has no meaning
        return r;
    }
    long long integer(const char *what, PyObject *o, long long low, long long high) const {
        const long long v = PyLong_AsLongLong(o);
        if (v == -1 && PyErr_Occurred()) {
            PyErr_Clear();
            refuse(std::string(what) + " has to be an integer of " + std::to_string(low) + " .. " + std::to_string(high));
        }
        if (v < low || v > high) refuse(std::string(what) + " = " + std::to_string(v) + " is not in " + std::to_string(low) + " .. " + std::to_string(high));
        return v;
    }
    unsigned long long word64(const char *what, PyObject *o) const {
        PyObject *const i = PyNumber_Index(o);
        const unsigned long long v = i ? PyLong_AsUnsignedLongLong(i) : (unsigned long long)-1;
        Py_XDECREF(i);
        if (v == (unsigned long long)-1 && PyErr_Occurred()) {
            PyErr_Clear();
            refuse(std::string(what) + " has to be an unsigned 64-bit integer");
        }
        return v;
    }
    double number(const char *what, PyObject *o) const {
        const double v = PyFloat_AsDouble(o);
        if (v == -1.0 && PyErr_Occurred()) {
            PyErr_Clear();
            refuse(std::string(what) + " has to be a number");
        }
        return v;
    }
    at::Tensor make(at::IntArrayRef shape, at::ScalarType type) const {
        const Unlocked u;
        return at::empty(shape, at::TensorOptions().dtype(type).device(at::kCUDA, (c10::DeviceIndex)index));
    }
};

// A result: the given tensor, or a new one.
struct Result {
    PyObject *given;
    at::Tensor made;
    Result(PyObject *o) : given(o == Py_None ? nullptr : o) {}
    PyObject *take() {
        if (!given) return THPVariable_Wrap(std::move(made));
        Py_INCREF(given);
        return given;
    }
};

int int_size(const Call &c, const char *what, long long n) {
    if (n > INT_MAX) fail(PARLE_ETOOBIG, std::string(c.name) + ": " + what + " = " + std::to_string(n));
    return (int)n;
}

std::vector<int64_t> with(at::IntArrayRef shape, int64_t last) {
    std::vector<int64_t> v(shape.begin(), shape.end());
    v.push_back(last);
    return v;
}

bool expects(Py_ssize_t n, Py_ssize_t want) {
    if (n == want) return true;
    PyErr_Format(PyExc_TypeError, "%zd arguments are needed", want);
    return false;
}

// logits, tokens, k, scale, logprob, entropy, top_token, top_logprob, flags, stream
PyObject *token_logprobs(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!expects(n, 10)) return nullptr;
    Call c("parle_token_logprobs");
    const at::Tensor &logits = c.first("logits", a[0], a[9]);
    const int dtype = c.dtype("logits", logits);
    const Call::Rows x = c.rows("logits", logits, 0);
    const at::IntArrayRef lead = logits.sizes().slice(0, logits.dim() - 1);
    const int k = (int)c.integer("k", a[2], 0, PARLE_TOP_MAX);
    const double scale = c.number("scale", a[3]);
    const int32_t *tokens = (const int32_t *)c.dense_or_null("tokens", a[1], lead, at::kInt);
    Result logprob(a[4]), entropy(a[5]), top_token(a[6]), top_logprob(a[7]);
    if (!tokens && a[1] == Py_None && logprob.given) c.refuse("logprob needs tokens");
    const auto place = [&](const char *what, Result &r, at::IntArrayRef shape, at::ScalarType type) {
        if (!r.given) r.made = c.make(shape, type);
        return c.dense(what, r.given ? c.tensor(what, r.given) : r.made, shape, type);
    };
    const std::vector<int64_t> best = with(lead, k);
    float *logprob_at = a[1] != Py_None ? (float *)place("logprob", logprob, lead, at::kFloat) : nullptr;
    float *entropy_at = (float *)place("entropy", entropy, lead, at::kFloat);
    int32_t *top_token_at = (int32_t *)place("top_token", top_token, best, at::kInt);
    float *top_logprob_at = (float *)place("top_logprob", top_logprob, best, at::kFloat);
    int32_t *flags = (int32_t *)c.word("flags", a[8], at::kInt, at::kInt);
    const int vocab = int_size(c, "vocab", x.cols);
    const void *const logits_at = logits.data_ptr();
    c.run([&] { return parle_token_logprobs(logits_at, dtype, x.rows, vocab, x.pitch, tokens, scale, k, logprob_at, entropy_at,
                                 k ? top_token_at : nullptr, k ? top_logprob_at : nullptr, flags, c.stream); });
    c.written({a[4], a[5], a[6], a[7], a[8]});
    PyObject *first = Py_None;
    if (a[1] != Py_None) first = logprob.take(); else Py_INCREF(first);
    return Py_BuildValue("(NNNN)", first, entropy.take(), top_token.take(), top_logprob.take());
    END_HANDLE_TH_ERRORS
}

// logits, tokens, d_logprob, d_entropy, scale, dlogits, logprob, entropy, flags, stream
PyObject *token_logprobs_grad(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!expects(n, 10)) return nullptr;
    Call c("parle_token_logprobs_grad");
    const at::Tensor &logits = c.first("logits", a[0], a[9]);
    const int dtype = c.dtype("logits", logits);
    const Call::Rows x = c.rows("logits", logits, 0);
    const at::IntArrayRef lead = logits.sizes().slice(0, logits.dim() - 1);
    const int32_t *tokens = (const int32_t *)c.dense_or_null("tokens", a[1], lead, at::kInt);
    const float *d_logprob = (const float *)c.dense_or_null("d_logprob", a[2], lead, at::kFloat);
    const float *d_entropy = (const float *)c.dense_or_null("d_entropy", a[3], lead, at::kFloat);
    const double scale = c.number("scale", a[4]);
    float *logprob = (float *)c.dense_or_null("logprob", a[6], lead, at::kFloat), *entropy = (float *)c.dense_or_null("entropy", a[7], lead, at::kFloat);
    Result dlogits(a[5]);
    if (!dlogits.given) dlogits.made = c.make(logits.sizes(), logits.scalar_type());
    const at::Tensor &d = dlogits.given ? c.tensor("dlogits", dlogits.given) : dlogits.made;
    if (d.sizes() != logits.sizes() || d.scalar_type() != logits.scalar_type()) c.refuse("dlogits is " + Call::describe(d) + ", logits " + Call::describe(logits));
    const Call::Rows y = c.rows("dlogits", d, 0);
    int32_t *flags = (int32_t *)c.word("flags", a[8], at::kInt, at::kInt);
    const int vocab = int_size(c, "vocab", x.cols);
    const void *const logits_at = logits.data_ptr();
    void *const d_at = d.data_ptr();
    c.run([&] { return parle_token_logprobs_grad(logits_at, dtype, x.rows, vocab, x.pitch, tokens, scale, d_logprob, d_entropy, logprob, entropy,
                                      d_at, y.pitch, flags, c.stream); });
    c.written({a[5], a[6], a[7], a[8]});
    return dlogits.take();
    END_HANDLE_TH_ERRORS
}

// logits, u, scale, top_k, top_p, min_p, token, logprob, kept, flags, stream
PyObject *sample_tokens(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!expects(n, 11)) return nullptr;
    Call c("parle_sample_tokens");
    const at::Tensor &logits = c.first("logits", a[0], a[10]);
    const int dtype = c.dtype("logits", logits);
    const Call::Rows x = c.rows("logits", logits, 0);
    const at::IntArrayRef lead = logits.sizes().slice(0, logits.dim() - 1);
    const float *u = (const float *)c.dense("u", c.tensor("u", a[1]), lead, at::kFloat);
    parle_sampling h = {1.0, 1.0, 0.0, 0, nullptr, nullptr, nullptr, nullptr};
    const auto either = [&](const char *what, PyObject *o, double &number, const float *&array) {
        if (THPVariable_Check(o)) array = (const float *)c.dense(what, c.tensor(what, o), lead, at::kFloat);
        else number = c.number(what, o);
    };
    either("scale", a[2], h.scale, h.scales);
    if (THPVariable_Check(a[3])) h.top_ks = (const int32_t *)c.dense("top_k", c.tensor("top_k", a[3]), lead, at::kInt);
    else h.top_k = (int)c.integer("top_k", a[3], 0, INT_MAX);
    either("top_p", a[4], h.top_p, h.top_ps);
    either("min_p", a[5], h.min_p, h.min_ps);
    Result token(a[6]), logprob(a[7]), kept(a[8]);
    const auto place = [&](const char *what, Result &r, at::ScalarType type) {
        if (!r.given) r.made = c.make(lead, type);
        return c.dense(what, r.given ? c.tensor(what, r.given) : r.made, lead, type);
    };
    int32_t *token_at = (int32_t *)place("token", token, at::kInt);
    float *logprob_at = (float *)place("logprob", logprob, at::kFloat);
    int32_t *kept_at = (int32_t *)place("kept", kept, at::kInt);
    int32_t *flags = (int32_t *)c.word("flags", a[9], at::kInt, at::kInt);
    const int vocab = int_size(c, "vocab", x.cols);
    const void *const logits_at = logits.data_ptr();
    c.run([&] { return parle_sample_tokens(logits_at, dtype, x.rows, vocab, x.pitch, u, &h, token_at, logprob_at, kept_at, flags, c.stream); });
    c.written({a[6], a[7], a[8], a[9]});
    return Py_BuildValue("(NNN)", token.take(), logprob.take(), kept.take());
    END_HANDLE_TH_ERRORS
}

struct Tables {
    long long gs, ld;
};
// t as [n, rows, dim] (n: its first dimension; or one group of all its rows).
Tables grouped(const Call &c, const char *what, const at::Tensor &t, bool by_first, long long rows) {
    const Call::Rows r = c.rows(what, t, by_first ? 1 : 0);
    return {by_first && t.size(0) > 1 ? (long long)t.stride(0) : std::max(1LL, rows) * r.cols, r.pitch};
}

// table, tokens, scale, out, type as (None or a tensor's type), flags, stream
PyObject *embedding(PyObject *, PyObject *const *a, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    if (!expects(n_args, 7)) return nullptr;
    Call c("parle_embedding");
    const at::Tensor &table = c.first("table", a[0], a[6]);
    const int table_dtype = c.dtype("table", table);
    if (table.dim() != 2 && table.dim() != 3) c.refuse("table is " + Call::describe(table) + ", not [vocab, dim] or [n, vocab, dim]");
    const bool many = table.dim() == 3;
    const at::Tensor &tokens = c.tensor("tokens", a[1]);
    const long long n = many ? table.size(0) : 1;
    if (many && (tokens.dim() == 0 || tokens.size(0) != n)) c.refuse("tables " + Call::describe(table) + " and tokens " + Call::describe(tokens));
    const int32_t *tokens_at = (const int32_t *)c.dense("tokens", tokens, tokens.sizes(), at::kInt);
    const long long length = n ? tokens.numel() / n : 0;
    const std::vector<int64_t> shape = with(tokens.sizes(), table.size(-1));
    Result out(a[3]);
    at::ScalarType type = table.scalar_type();
    if (a[4] != Py_None) {
        if (!THPDtype_Check(a[4])) c.refuse("dtype has to be a torch type");
        type = reinterpret_cast<THPDtype *>(a[4])->scalar_type;
    }
    if (!out.given) out.made = c.make(shape, type);
    const at::Tensor &o = out.given ? c.tensor("out", out.given) : out.made;
    if (o.sizes() != at::IntArrayRef(shape) || (a[4] != Py_None && o.scalar_type() != type)) c.refuse("out is " + Call::describe(o) + ", tokens " + Call::describe(tokens) + ", table " + Call::describe(table));
    const int out_dtype = c.dtype("out", o);
    const Tables in = grouped(c, "table", table, many, table.size(-2)), to = grouped(c, "out", o, many, length);
    int32_t *flags = (int32_t *)c.word("flags", a[5], at::kInt, at::kInt);
    const double scale = c.number("scale", a[2]);
    const int n_int = int_size(c, "n", n), vocab = int_size(c, "vocab", table.size(-2)), dim = int_size(c, "dim", table.size(-1));
    const void *const table_at = table.data_ptr();
    void *const out_at = o.data_ptr();
    c.run([&] { return parle_embedding(table_at, table_dtype, in.gs, in.ld, n_int, vocab, dim, tokens_at, length, scale, out_at, out_dtype, to.gs, to.ld, flags, c.stream); });
    c.written({a[3], a[5]});
    return out.take();
    END_HANDLE_TH_ERRORS
}

// dout, tokens, vocab, scale, n, dtable, accumulate, workspace, flags, stream
PyObject *embedding_grad(PyObject *, PyObject *const *a, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    if (!expects(n_args, 10)) return nullptr;
    Call c("parle_embedding_grad");
    const at::Tensor &dout = c.first("dout", a[0], a[9]);
    const int dtype = c.dtype("dout", dout);
    const at::Tensor &tokens = c.tensor("tokens", a[1]);
    const int32_t *tokens_at = (const int32_t *)c.dense("tokens", tokens, tokens.sizes(), at::kInt);
    const int vocab = (int)c.integer("vocab", a[2], 1, INT_MAX);
    const double scale = c.number("scale", a[3]);
    if (dout.dim() != tokens.dim() + 1 || dout.sizes().slice(0, tokens.dim()) != tokens.sizes()) c.refuse("dout is " + Call::describe(dout) + ", tokens " + Call::describe(tokens));
    const long long dim = dout.size(-1);
    const bool asked = a[4] != Py_None;
    const long long n_asked = asked ? c.integer("n", a[4], 0, INT_MAX) : 1;
    const int accumulate = PyObject_IsTrue(a[6]);
    if (accumulate < 0) throw python_error();
    Result dtable(a[5]);
    if (!dtable.given) {
        if (accumulate) c.refuse("accumulate needs a dtable");
        dtable.made = asked ? c.make({n_asked, vocab, dim}, at::kFloat) : c.make({vocab, dim}, at::kFloat);
    }
    const at::Tensor &g = dtable.given ? c.tensor("dtable", dtable.given) : dtable.made;
    const bool many = g.dim() == 3;
    const long long n = many ? g.size(0) : 1;
    if ((g.dim() != 2 && !many) || g.scalar_type() != at::kFloat || g.size(-2) != vocab || g.size(-1) != dim || (asked && (!many || n != n_asked)) ||
        (many && (tokens.dim() == 0 || tokens.size(0) != n)))
        c.refuse("dtable is " + Call::describe(g) + ": fp32 [vocab, dim], or [n, vocab, dim] for tokens [n, ..], is needed with tokens " + Call::describe(tokens) +
                 " and dout " + Call::describe(dout));
    const long long length = n ? tokens.numel() / n : 0;
    const Tables in = grouped(c, "dout", dout, many, length), to = grouped(c, "dtable", g, many, vocab);
    const int n_int = int_size(c, "n", n), dim_int = int_size(c, "dim", dim);
    at::Tensor scratch;
    void *workspace = nullptr;
    size_t bytes = 0;
    if (a[7] == Py_None) {
        bytes = parle_embedding_grad_workspace_bytes(n_int, length, vocab, dim_int);
        if (bytes) {
            scratch = c.make({(int64_t)bytes}, at::kByte);
            workspace = scratch.data_ptr();
        }
    } else {
        const at::Tensor &w = c.tensor("workspace", a[7]);
        c.here("workspace", w);
        if (!w.is_contiguous()) c.refuse("workspace is not contiguous");
        workspace = w.data_ptr();
        bytes = w.nbytes();
    }
    int32_t *flags = (int32_t *)c.word("flags", a[8], at::kInt, at::kInt);
    const void *const dout_at = dout.data_ptr();
    float *const dtable_at = (float *)g.data_ptr();
    c.run([&] { return parle_embedding_grad(dout_at, dtype, in.gs, in.ld, tokens_at, n_int, length, vocab, dim_int, scale, dtable_at, to.gs, to.ld, accumulate,
                                 workspace, bytes, flags, c.stream); });
    c.written({a[5], a[7], a[8]});
    return dtable.take();
    END_HANDLE_TH_ERRORS
}

// x, p, seed, offset, residual, out, offset_dev, stream
PyObject *dropout(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!expects(n, 8)) return nullptr;
    Call c("parle_dropout");
    const at::Tensor &x = c.first("x", a[0], a[7]);
    const int dtype = c.dtype("x", x);
    const double p = c.number("p", a[1]);
    const unsigned long long seed = c.word64("seed", a[2]), offset = c.word64("offset", a[3]);
    const Call::Rows in = c.rows("x", x, 0);
    const auto same = [&](const char *what, const at::Tensor &t) {
        if (t.sizes() != x.sizes() || t.scalar_type() != x.scalar_type()) c.refuse(std::string(what) + " is " + Call::describe(t) + ", x " + Call::describe(x));
        return c.rows(what, t, 0);
    };
    const void *residual = nullptr;
    long long ld_r = 0;
    if (a[4] != Py_None) {
        const at::Tensor &r = c.tensor("residual", a[4]);
        ld_r = same("residual", r).pitch;
        residual = r.data_ptr();
    }
    Result out(a[5]);
    if (!out.given) out.made = c.make(x.sizes(), x.scalar_type());
    const at::Tensor &y = out.given ? c.tensor("out", out.given) : out.made;
    const long long ld_y = same("out", y).pitch;
    const uint64_t *offset_dev = (const uint64_t *)c.word("offset_dev", a[6], at::kLong, at::kUInt64);
    const void *const x_at = x.data_ptr();
    void *const out_at = y.data_ptr();
    c.run([&] { return parle_dropout(x_at, in.pitch, residual, ld_r, out_at, ld_y, dtype, in.rows, in.cols, p, seed, offset, offset_dev, c.stream); });
    c.written({a[5]});
    return out.take();
    END_HANDLE_TH_ERRORS
}

// A list or tuple of tensors; None: none.
struct Tensors {
    PyObject *source = nullptr, **items = nullptr;
    Py_ssize_t n = 0;
    Tensors(const Call &c, const char *what, PyObject *o, Py_ssize_t want = -1) {
        if (o == Py_None) return;
        if (!PyList_Check(o) && !PyTuple_Check(o)) c.refuse(std::string(what) + " has to be a list or tuple of tensors, not " + Py_TYPE(o)->tp_name);
        source = o;
        n = PySequence_Fast_GET_SIZE(o);
        static PyObject *none[1] = {nullptr};
        items = n ? PySequence_Fast_ITEMS(o) : none;
        if (want >= 0 && n != want) c.refuse(std::to_string(n) + " " + what + " for " + std::to_string(want) + " tensors");
    }
    explicit operator bool() const { return items; }
    PyObject *object(Py_ssize_t i) const { return items[i]; }
};

// The tensors of a list, checked: all of this type, contiguous, on the call's device, of the shapes of `like`'s if that is given; each
// goes to place(i, number of elements, tensor).  A list of some hundreds is checked faster than its kernel runs only if its objects, which lie
// anywhere, are fetched ahead.
template <class F> void members(const Call &c, const char *what, const Tensors &list, at::ScalarType type, const Tensors *like, F place) {
    const caffe2::TypeMeta meta = c10::scalarTypeToTypeMeta(type);
    const c10::Device device(at::kCUDA, (c10::DeviceIndex)c.index);
    constexpr Py_ssize_t kAhead = 4;
    for (Py_ssize_t i = 0; i < list.n; ++i) {
        if (i + 2 * kAhead < list.n) __builtin_prefetch(list.items[i + 2 * kAhead]);
        if (i + kAhead < list.n && THPVariable_Check(list.items[i + kAhead])) {
            const char *const next = reinterpret_cast<const char *>(THPVariable_Unpack(list.items[i + kAhead]).unsafeGetTensorImpl());
            for (size_t line = 0; line < sizeof(at::TensorImpl); line += 64) __builtin_prefetch(next + line);
        }
        const at::Tensor &t = c.tensor(what, list.items[i]);
        const at::TensorImpl *const impl = t.unsafeGetTensorImpl();
        const at::Tensor *const same = like ? &THPVariable_Unpack(like->items[i]) : nullptr;
        if (impl->dtype() != meta || !impl->is_contiguous() || impl->device() != device || (same && impl->sizes() != same->sizes())) {
            const std::string name = std::string(what) + "[" + std::to_string(i) + "]";
            c.here(name.c_str(), t);
            c.refuse(name + " is " + Call::describe(t) + ": a contiguous " + c10::toString(type) + " tensor" + (same ? " like " + Call::describe(*same) : "") + " is needed");
        }
        place(i, (long long)impl->numel(), t);
    }
}

// As Call::written(), for a list.  (Behind the call, during which another thread may have changed it: it is looked at anew.)
void written(const Tensors &list) {
    const Py_ssize_t n = list ? PySequence_Fast_GET_SIZE(list.source) : 0;
    for (Py_ssize_t i = 0; i < n; ++i) {
        PyObject *const o = PySequence_Fast_GET_ITEM(list.source, i);
        if (!THPVariable_Check(o)) continue;
        const at::Tensor &t = THPVariable_Unpack(o);
        if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
    }
}

// grads, out, workspace, stream
PyObject *grad_norm(PyObject *, PyObject *const *a, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    if (!expects(n_args, 4)) return nullptr;
    Call c("parle_grad_norm");
    const Tensors grads(c, "grads", a[0]);
    if (grads.n == 0) c.refuse("grads has to hold a tensor");
    if (grads.n > INT_MAX) c.refuse("too many tensors");
    const at::Tensor &first = c.first("grads[0]", grads.object(0), a[3]);
    const at::ScalarType type = first.scalar_type();
    const int dtype = c.dtype("grads[0]", first);
    std::vector<parle_grad_tensor> list((size_t)grads.n);
    members(c, "grads", grads, type, nullptr, [&](Py_ssize_t i, long long size, const at::Tensor &g) { list[i] = {g.const_data_ptr(), size}; });
    Result out(a[1]);
    if (!out.given) out.made = c.make({}, at::kFloat);
    float *const norm = (float *)c.word("out", out.given ? out.given : Py_None, at::kFloat, at::kFloat);
    float *const norm_at = out.given ? norm : (float *)out.made.data_ptr();
    at::Tensor scratch;
    void *workspace = nullptr;
    size_t bytes = 0;
    if (a[2] == Py_None) {
        bytes = parle_grad_norm_workspace_bytes(list.data(), (int)grads.n);
        if (bytes) {
            scratch = c.make({(int64_t)bytes}, at::kByte);
            workspace = scratch.data_ptr();
        }
    } else {
        const at::Tensor &w = c.tensor("workspace", a[2]);
        c.here("workspace", w);
        if (!w.is_contiguous()) c.refuse("workspace is not contiguous");
        workspace = w.data_ptr();
        bytes = w.nbytes();
    }
    c.run([&] { return parle_grad_norm(list.data(), (int)grads.n, dtype, norm_at, workspace, bytes, c.stream); });
    c.written({a[1], a[2]});
    return out.take();
    END_HANDLE_TH_ERRORS
}

// params, grads, exp_avg, exp_avg_sq, exp_avg_scales, exp_avg_sq_scales, copies, step, lr, beta1, beta2, eps, weight_decay, grad_scale,
// norm, max_norm, step_dev, lr_dev, flags, stream
PyObject *adamw(PyObject *, PyObject *const *a, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    if (!expects(n_args, 20)) return nullptr;
    Call c("parle_adamw");
    const Tensors params(c, "params", a[0]);
    if (params.n == 0) c.refuse("params has to hold a tensor");
    if (params.n > INT_MAX) c.refuse("too many tensors");
    const char *const names[7] = {"params", "grads", "exp_avg", "exp_avg_sq", "exp_avg_scales", "exp_avg_sq_scales", "copies"};
    const Tensors lists[7] = {params, {c, names[1], a[1], params.n}, {c, names[2], a[2], params.n}, {c, names[3], a[3], params.n}, {c, names[4], a[4], params.n},
                              {c, names[5], a[5], params.n}, {c, names[6], a[6], params.n}};
    const at::Tensor &first = c.first("params[0]", params.object(0), a[19]);
    at::ScalarType types[7];
    for (int k = 0; k < 4; ++k) {
        if (!lists[k]) c.refuse(std::string(names[k]) + " are needed");
        types[k] = k ? c.tensor(names[k], lists[k].object(0)).scalar_type() : first.scalar_type();
    }
    const int param_dtype = c.dtype("params[0]", first), grad_dtype = c.dtype("grads[0]", c.tensor("grads", lists[1].object(0)));
    if (types[2] != types[3] || (types[2] != at::kFloat && types[2] != at::kFloat8_e4m3fn))
        c.refuse(std::string("exp_avg is ") + c10::toString(types[2]) + ", exp_avg_sq " + c10::toString(types[3]) + ": both Float or both Float8_e4m3fn are needed");
    const int bits = types[2] == at::kFloat ? 32 : 8;
    types[4] = types[5] = at::kFloat;
    for (int k = 4; k < 6; ++k)
        if ((bool)lists[k] != (bits == 8)) c.refuse(std::string(names[k]) + (bits == 8 ? " are needed beside 8-bit moments" : " belong to 8-bit moments"));
    int copy_dtype = PARLE_NO_COPY;
    if (lists[6]) {
        const at::Tensor &t = c.tensor("copies", lists[6].object(0));
        types[6] = t.scalar_type();
        copy_dtype = c.dtype("copies[0]", t);
        if (copy_dtype == PARLE_F32 || param_dtype != PARLE_F32) c.refuse("copies are 16-bit ones of fp32 params");
    }
    std::vector<parle_adamw_tensor> list((size_t)params.n);
    members(c, names[0], params, types[0], nullptr, [&](Py_ssize_t i, long long size, const at::Tensor &p) {
        list[i] = {p.data_ptr(), nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, size};
    });
    members(c, names[1], lists[1], types[1], &params, [&](Py_ssize_t i, long long, const at::Tensor &g) { list[i].grad = g.const_data_ptr(); });
    members(c, names[2], lists[2], types[2], &params, [&](Py_ssize_t i, long long, const at::Tensor &m) { list[i].exp_avg = m.data_ptr(); });
    members(c, names[3], lists[3], types[3], &params, [&](Py_ssize_t i, long long, const at::Tensor &v) { list[i].exp_avg_sq = v.data_ptr(); });
    for (int k = 4; k < 6; ++k)
        members(c, names[k], lists[k], types[k], nullptr, [&](Py_ssize_t i, long long scales, const at::Tensor &s) {
            if (scales != (list[i].size + PARLE_ADAMW_BLOCK - 1) / PARLE_ADAMW_BLOCK)
                c.refuse(std::string(names[k]) + "[" + std::to_string(i) + "] has " + std::to_string(scales) + " numbers: one for each " + std::to_string(PARLE_ADAMW_BLOCK) + " of " +
                         std::to_string(list[i].size) + " elements is needed");
            (k == 4 ? list[i].exp_avg_scale : list[i].exp_avg_sq_scale) = (float *)s.data_ptr();
        });
    members(c, names[6], lists[6], lists[6] ? types[6] : at::kFloat, &params, [&](Py_ssize_t i, long long, const at::Tensor &copy) { list[i].copy = copy.data_ptr(); });
    parle_adamw_step h;
    h.step = c.integer("step", a[7], 0, LLONG_MAX);
    h.lr = c.number("lr", a[8]);
    h.beta1 = c.number("beta1", a[9]);
    h.beta2 = c.number("beta2", a[10]);
    h.eps = c.number("eps", a[11]);
    h.weight_decay = c.number("weight_decay", a[12]);
    h.grad_scale = c.number("grad_scale", a[13]);
    h.norm = (const float *)c.word("norm", a[14], at::kFloat, at::kFloat);
    h.max_norm = a[15] == Py_None ? std::numeric_limits<double>::infinity() : c.number("max_norm", a[15]);
    h.step_dev = (const int64_t *)c.word("step_dev", a[16], at::kLong, at::kLong);
    h.lr_dev = (const float *)c.word("lr_dev", a[17], at::kFloat, at::kFloat);
    int32_t *const flags = (int32_t *)c.word("flags", a[18], at::kInt, at::kInt);
    c.run([&] { return parle_adamw(list.data(), (int)params.n, param_dtype, grad_dtype, copy_dtype, bits, &h, flags, c.stream); });
    c.written({a[18]});
    for (int k = 0; k < 7; ++k)
        if (k != 1) written(lists[k]);
    Py_RETURN_NONE;
    END_HANDLE_TH_ERRORS
}

PyObject *set_error(PyObject *, PyObject *type) {
    Py_INCREF(type);
    Py_XDECREF(g_error);
    g_error = type;
    Py_RETURN_NONE;
}

#define FASTCALL(f) {#f, (PyCFunction)(void (*)(void))f, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FASTCALL(token_logprobs), FASTCALL(token_logprobs_grad), FASTCALL(embedding), FASTCALL(embedding_grad), FASTCALL(dropout), FASTCALL(sample_tokens), FASTCALL(grad_norm), FASTCALL(adamw),
                         {"set_error", set_error, METH_O, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_token_ops", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__token_ops() {
    PyObject *m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "built_from", BUILT_FROM) < 0) Py_CLEAR(m);
    return m;
}
