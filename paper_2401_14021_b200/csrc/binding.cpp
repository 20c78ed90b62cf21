// Marshalling of the generator's operators between torch tensors and the C ABI of include/ralm.h: argument
// checks, strides, the current stream. A decode step makes these calls hundreds of times per generated
// token; through ctypes the checks and conversions cost more than the kernels of a small batch.
// The library itself is found by Python, which hands its entry points over (bind).
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <exception>
#include <string>

#include "../../include/ralm.h"

namespace {

#define RALM_CALLS(X)                                                                                              \
    X(ralm_knn_mix) X(ralm_verify_tokens) X(ralm_pages_resize) X(ralm_pages_fork) X(ralm_pages_compact)            \
    X(ralm_pages_copy) X(ralm_kv_append) X(ralm_kv_read) X(ralm_kv_attend)
struct Calls {
#define X(name) decltype(&::name) name = nullptr;
    RALM_CALLS(X)
#undef X
} calls;
PyObject *error_class = nullptr;   // RalmError(status, where)

struct Refused : std::exception {   // becomes a TypeError
    std::string text;
    explicit Refused(std::string t) : text(std::move(t)) {}
    const char *what() const noexcept override { return text.c_str(); }
};

// Tensors of one call: the same device throughout.
struct Args {
    int device = -1;
    const at::Tensor *tensor(PyObject *o, const char *name, bool optional = false) {
        if (optional && o == Py_None) return nullptr;
        if (!THPVariable_Check(o)) throw Refused(std::string(name) + " must be a tensor");
        const at::Tensor &t = THPVariable_Unpack(o);
        if (!t.is_cuda()) throw Refused(std::string(name) + " must be a CUDA tensor");
        const int d = t.device().index();
        if (device >= 0 && d != device) throw Refused(std::string(name) + " is on another device");
        device = d;
        return &t;
    }
    static void type(const at::Tensor &t, at::ScalarType want, const char *name) {
        if (t.scalar_type() != want) throw Refused(std::string(name) + " must be of type " + c10::toString(want));
    }
    static void shape(const at::Tensor &t, at::IntArrayRef want, const char *name) {
        if (t.sizes() == want) return;
        std::string s = std::string(name) + " must have shape (";
        for (auto v : want) s += std::to_string(v) + ", ";
        s += "), got (";
        for (auto v : t.sizes()) s += std::to_string(v) + ", ";
        throw Refused(s + ")");
    }
    static void last_contiguous(const at::Tensor &t, const char *name) {
        if (t.dim() > 0 && t.size(-1) > 1 && t.stride(-1) != 1) throw Refused(std::string(name) + " must have a contiguous last dimension");
    }
    // a contiguous tensor of a shape and type; null for None where that is allowed
    template <typename P>
    P *dense(PyObject *o, at::IntArrayRef want, at::ScalarType st, const char *name, bool optional = false) {
        const at::Tensor *t = tensor(o, name, optional);
        if (!t) return nullptr;
        type(*t, st, name);
        shape(*t, want, name);
        if (!t->is_contiguous()) throw Refused(std::string(name) + " must be contiguous");
        return static_cast<P *>(t->data_ptr());
    }
};
int dtype_code(const at::Tensor &t, const char *name, bool f32) {
    switch (t.scalar_type()) {
        case at::kHalf: return RALM_F16;
        case at::kBFloat16: return RALM_BF16;
        case at::kFloat:
            if (f32) return RALM_F32;
            [[fallthrough]];
        default: throw Refused(std::string(name) + (f32 ? " must be float16, bfloat16 or float32" : " must be float16 or bfloat16"));
    }
}
// The call's stream on its tensors' device. Device and stream are current while it lives, so that a result
// made here belongs to the stream that writes it.
struct Where {
    c10::cuda::CUDAGuard guard;
    c10::cuda::OptionalCUDAStreamGuard stream_guard;
    void *stream;
    Where(const Args &a, PyObject *given) : guard(static_cast<c10::DeviceIndex>(a.device)) {
        if (given == Py_None) {
            stream = c10::cuda::getCurrentCUDAStream(static_cast<c10::DeviceIndex>(a.device)).stream();
            return;
        }
        PyObject *v = PyObject_GetAttrString(given, "cuda_stream");
        if (!v) {
            PyErr_Clear();
            throw Refused("stream must be a torch.cuda.Stream");
        }
        stream = PyLong_AsVoidPtr(v);
        Py_DECREF(v);
        if (PyErr_Occurred()) {
            PyErr_Clear();
            throw Refused("stream must be a torch.cuda.Stream");
        }
        stream_guard.reset_stream(c10::cuda::getStreamFromExternal(static_cast<cudaStream_t>(stream), static_cast<c10::DeviceIndex>(a.device)));
    }
};
void *pointer(PyObject *o) { return PyLong_AsVoidPtr(o); }
long long integer(PyObject *o, const char *name) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        throw Refused(std::string(name) + " must be an integer");
    }
    return v;
}
int32_t int32(PyObject *o, const char *name) {
    const long long v = integer(o, name);
    if (v < INT32_MIN || v > INT32_MAX) throw Refused(std::string(name) + " is out of range");
    return static_cast<int32_t>(v);
}
int32_t size32(int64_t v, const char *name) {
    if (v > INT32_MAX) throw Refused(std::string(name) + " is too large");
    return static_cast<int32_t>(v);
}
float real(PyObject *o, const char *name) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) {
        PyErr_Clear();
        throw Refused(std::string(name) + " must be a number");
    }
    return static_cast<float>(v);
}
bool failed(int status, const char *where) {
    if (status == RALM_OK) return false;
    PyObject *e = PyObject_CallFunction(error_class, "is", status, where);
    if (e) {
        PyErr_SetObject(error_class, e);
        Py_DECREF(e);
    }
    return true;
}
template <typename F> PyObject *guarded(Py_ssize_t n, Py_ssize_t want, F f) {
    if (n != want || !error_class) {
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments, or the module is not bound");
        return nullptr;
    }
    try {
        return f();
    } catch (const Refused &e) {
        PyErr_SetString(PyExc_TypeError, e.what());
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}
PyObject *same(PyObject *o) {
    Py_INCREF(o);
    return o;
}
at::Tensor fresh(at::IntArrayRef shape, at::ScalarType type, int device) {
    return at::empty(shape, at::TensorOptions().dtype(type).device(at::kCUDA, static_cast<c10::DeviceIndex>(device)));
}

// logits, ids, scores, values, lambda, temperature, knn_temperature, metric, probs, stream
PyObject *knn_mix(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 10, [&]() -> PyObject * {
        Args args;
        const at::Tensor &logits = *args.tensor(a[0], "logits");
        if (logits.dim() != 2) throw Refused("logits must be [R][V]");
        Args::last_contiguous(logits, "logits");
        const int dtype = dtype_code(logits, "logits", true);
        const int64_t R = logits.size(0), V = logits.size(1);
        const int64_t *ids = nullptr;
        const float *scores = nullptr;
        const int32_t *values = nullptr;
        int64_t k = 0, N = 0;
        if (a[1] != Py_None) {
            const at::Tensor &t = *args.tensor(a[1], "ids");
            if (t.dim() != 2) throw Refused("ids must be [R][k]");
            k = t.size(1);
            ids = args.dense<int64_t>(a[1], {R, k}, at::kLong, "ids");
            scores = args.dense<float>(a[2], {R, k}, at::kFloat, "scores");
            const at::Tensor &v = *args.tensor(a[3], "values");
            if (v.dim() != 1) throw Refused("values must be [N]");
            N = v.size(0);
            values = args.dense<int32_t>(a[3], {N}, at::kInt, "values");
        }
        const at::Tensor *probs = args.tensor(a[8], "probs", true);
        Where w(args, a[9]);
        at::Tensor made;
        if (!probs) {
            made = fresh({R, V}, at::kFloat, args.device);
            probs = &made;
        }
        Args::type(*probs, at::kFloat, "probs");
        Args::shape(*probs, {R, V}, "probs");
        Args::last_contiguous(*probs, "probs");
        const float lam = real(a[4], "lam"), temperature = real(a[5], "temperature"), tau = real(a[6], "knn_temperature");
        const int metric = int32(a[7], "metric");
        if (failed(calls.ralm_knn_mix(logits.data_ptr(), static_cast<ralm_dtype_t>(dtype), R > 1 ? logits.stride(0) : V, size32(R, "R"),
                                      size32(V, "V"), ids, scores, size32(k, "k"), static_cast<ralm_metric_t>(metric), values, N, lam,
                                      temperature, tau, static_cast<float *>(probs->data_ptr()), R > 1 ? probs->stride(0) : V, w.stream),
                   "ralm_knn_mix"))
            return nullptr;
        return made.defined() ? THPVariable_Wrap(made) : same(a[8]);
    });
}

// draft_tokens, draft_probs, target_probs, uniforms, draft_len, tokens, accepted, stream
PyObject *verify_tokens(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 8, [&]() -> PyObject * {
        Args args;
        const at::Tensor &draft = *args.tensor(a[0], "draft_tokens");
        const at::Tensor &target = *args.tensor(a[2], "target_probs");
        if (draft.dim() != 2 || target.dim() != 3) throw Refused("draft_tokens must be [R][S], target_probs [R][S + 1][V]");
        const int64_t R = draft.size(0), S = draft.size(1), V = target.size(2);
        const int64_t *dt = args.dense<int64_t>(a[0], {R, S}, at::kLong, "draft_tokens");
        Args::type(target, at::kFloat, "target_probs");
        Args::shape(target, {R, S + 1, V}, "target_probs");
        Args::last_contiguous(target, "target_probs");
        const at::Tensor *dp = args.tensor(a[1], "draft_probs", true);
        if (dp) {
            Args::type(*dp, at::kFloat, "draft_probs");
            Args::shape(*dp, {R, S, V}, "draft_probs");
            Args::last_contiguous(*dp, "draft_probs");
        }
        const float *u = args.dense<float>(a[3], {R, S + 1}, at::kFloat, "uniforms");
        const int32_t *len = args.dense<int32_t>(a[4], {R}, at::kInt, "draft_len", true);
        int64_t *tokens = args.dense<int64_t>(a[5], {R, S + 1}, at::kLong, "tokens", true);
        int32_t *accepted = args.dense<int32_t>(a[6], {R}, at::kInt, "accepted", true);
        Where w(args, a[7]);
        at::Tensor tokens_made, accepted_made;
        if (a[5] == Py_None) {
            tokens_made = fresh({R, S + 1}, at::kLong, args.device);
            tokens = static_cast<int64_t *>(tokens_made.data_ptr());
        }
        if (a[6] == Py_None) {
            accepted_made = fresh({R}, at::kInt, args.device);
            accepted = static_cast<int32_t *>(accepted_made.data_ptr());
        }
        if (failed(calls.ralm_verify_tokens(dt, dp ? static_cast<const float *>(dp->data_ptr()) : nullptr, dp ? dp->stride(0) : 0,
                                            dp ? dp->stride(1) : 0, static_cast<const float *>(target.data_ptr()), target.stride(0),
                                            target.stride(1), u, len, size32(R, "R"), size32(S, "S"), size32(V, "V"), tokens, accepted,
                                            w.stream),
                   "ralm_verify_tokens"))
            return nullptr;
        PyObject *first = tokens_made.defined() ? THPVariable_Wrap(tokens_made) : same(a[5]);
        PyObject *second = accepted_made.defined() ? THPVariable_Wrap(accepted_made) : same(a[6]);
        PyObject *both = PyTuple_Pack(2, first, second);
        Py_DECREF(first);
        Py_DECREF(second);
        return both;
    });
}

// pages (address of a ralm_pages_t), its table (for the device), new_lengths, stream
PyObject *pages_resize(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 4, [&]() -> PyObject * {
        const auto *p = static_cast<const ralm_pages_t *>(pointer(a[0]));
        Args args;
        args.tensor(a[1], "table");
        const int32_t *to = args.dense<int32_t>(a[2], {p->rows}, at::kInt, "new_lengths");
        Where w(args, a[3]);
        if (failed(calls.ralm_pages_resize(p, to, w.stream), "ralm_pages_resize")) return nullptr;
        Py_RETURN_NONE;
    });
}

// pages, table, src, dst, stream
PyObject *pages_fork(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 5, [&]() -> PyObject * {
        const auto *p = static_cast<const ralm_pages_t *>(pointer(a[0]));
        Args args;
        args.tensor(a[1], "table");
        const int64_t count = args.tensor(a[2], "src")->numel();
        const int32_t *src = args.dense<int32_t>(a[2], {count}, at::kInt, "src");
        const int32_t *dst = args.dense<int32_t>(a[3], {count}, at::kInt, "dst");
        Where w(args, a[4]);
        if (failed(calls.ralm_pages_fork(p, src, dst, size32(count, "n"), w.stream), "ralm_pages_fork")) return nullptr;
        Py_RETURN_NONE;
    });
}

// pages, live, stream
PyObject *pages_compact(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 3, [&]() -> PyObject * {
        const auto *p = static_cast<const ralm_pages_t *>(pointer(a[0]));
        Args args;
        int32_t *live = args.dense<int32_t>(a[1], {1}, at::kInt, "live");
        Where w(args, a[2]);
        if (failed(calls.ralm_pages_compact(p, live, w.stream), "ralm_pages_compact")) return nullptr;
        return same(a[1]);
    });
}

// source pages, from, destination pages, to, destination table, source table, stream
PyObject *pages_copy(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 7, [&]() -> PyObject * {
        const auto *s = static_cast<const ralm_pages_t *>(pointer(a[0]));
        const auto *d = static_cast<const ralm_pages_t *>(pointer(a[2]));
        Args args;
        args.tensor(a[4], "table");
        args.tensor(a[5], "the source's table");
        const int64_t count = args.tensor(a[1], "src")->numel();
        const int32_t *from = args.dense<int32_t>(a[1], {count}, at::kInt, "src");
        const int32_t *to = args.dense<int32_t>(a[3], {count}, at::kInt, "dst");
        Where w(args, a[6]);
        if (failed(calls.ralm_pages_copy(s, from, d, to, size32(count, "n"), w.stream), "ralm_pages_copy")) return nullptr;
        Py_RETURN_NONE;
    });
}

ralm_kv_tokens_t kv_tokens(Args &args, const ralm_kv_t *c, const at::Tensor &k, const at::Tensor &v, PyObject *starts, PyObject *count,
                           PyObject *rows) {
    if (k.dim() != 4 || k.size(2) != c->kv_heads || k.size(3) != c->head_dim) throw Refused("k must be [batch][n][kv_heads][head_dim]");
    Args::shape(v, k.sizes(), "v");
    Args::type(v, k.scalar_type(), "v");
    Args::last_contiguous(k, "k");
    Args::last_contiguous(v, "v");
    ralm_kv_tokens_t t;
    t.dtype = static_cast<ralm_dtype_t>(dtype_code(k, "k", false));
    t.k = k.data_ptr();
    t.v = v.data_ptr();
    t.k_stride_b = k.stride(0), t.k_stride_n = k.stride(1), t.k_stride_h = k.stride(2);
    t.v_stride_b = v.stride(0), t.v_stride_n = v.stride(1), t.v_stride_h = v.stride(2);
    t.batch = size32(k.size(0), "batch");
    t.n = size32(k.size(1), "n");
    const int64_t B = t.batch;
    t.rows = args.dense<int32_t>(rows, {B}, at::kInt, "rows", true);
    t.starts = args.dense<int32_t>(starts, {B}, at::kInt, "starts");
    t.count = args.dense<int32_t>(count, {B}, at::kInt, "count", true);
    if (!t.rows && t.batch > c->pages.rows) throw Refused("more entries than rows of the table");
    return t;
}

// cache (address of a ralm_kv_t), layer, k, v, starts, count, rows, stream, table
PyObject *kv_append(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 9, [&]() -> PyObject * {
        const auto *c = static_cast<const ralm_kv_t *>(pointer(a[0]));
        Args args;
        args.tensor(a[8], "table");
        const at::Tensor &k = *args.tensor(a[2], "k"), &v = *args.tensor(a[3], "v");
        const ralm_kv_tokens_t t = kv_tokens(args, c, k, v, a[4], a[5], a[6]);
        Where w(args, a[7]);
        if (failed(calls.ralm_kv_append(c, int32(a[1], "layer"), &t, w.stream), "ralm_kv_append")) return nullptr;
        Py_RETURN_NONE;
    });
}
// cache, layer, k or None, v or None, starts, count, rows, stream, table, positions per entry, dtype of a k that is made here
PyObject *kv_read(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 11, [&]() -> PyObject * {
        const auto *c = static_cast<const ralm_kv_t *>(pointer(a[0]));
        Args args;
        args.tensor(a[8], "table");
        const at::Tensor *k = args.tensor(a[2], "k", true), *v = args.tensor(a[3], "v", true);
        const at::Tensor &starts = *args.tensor(a[4], "starts");
        const int32_t positions = int32(a[9], "n");
        if (positions < 0) throw Refused("n must not be negative");
        if (!THPDtype_Check(a[10])) throw Refused("dtype must be a torch.dtype");
        if (starts.dim() != 1) throw Refused("starts must be [batch]");
        if (k && (k->dim() != 4 || k->size(1) != positions)) throw Refused("k must be [batch][n][kv_heads][head_dim]");
        Where w(args, a[7]);                                     // what is made here belongs to the call's stream
        const int64_t shape[4] = {starts.size(0), positions, c->kv_heads, c->head_dim};
        at::Tensor made_k, made_v;
        if (!k) {
            made_k = fresh(shape, reinterpret_cast<const THPDtype *>(a[10])->scalar_type, args.device);
            k = &made_k;
        }
        if (!v) {
            made_v = fresh(shape, k->scalar_type(), args.device);
            v = &made_v;
        }
        const ralm_kv_tokens_t t = kv_tokens(args, c, *k, *v, a[4], a[5], a[6]);
        if (failed(calls.ralm_kv_read(c, int32(a[1], "layer"), &t, w.stream), "ralm_kv_read")) return nullptr;
        PyObject *first = made_k.defined() ? THPVariable_Wrap(made_k) : same(a[2]);
        PyObject *second = made_v.defined() ? THPVariable_Wrap(made_v) : same(a[3]);
        PyObject *both = PyTuple_Pack(2, first, second);
        Py_DECREF(first);
        Py_DECREF(second);
        return both;
    });
}

// cache, layer, q, scale, q_len, rows, out, workspace, stream
PyObject *kv_attend(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 9, [&]() -> PyObject * {
        const auto *c = static_cast<const ralm_kv_t *>(pointer(a[0]));
        Args args;
        const at::Tensor &q = *args.tensor(a[2], "q");
        if (q.dim() != 4 || q.size(3) != c->head_dim) throw Refused("q must be [batch][n][q_heads][head_dim]");
        Args::last_contiguous(q, "q");
        ralm_attend_t t;
        t.dtype = static_cast<ralm_dtype_t>(dtype_code(q, "q", false));
        const at::Tensor *out = args.tensor(a[6], "out", true);
        const at::Tensor &work = *args.tensor(a[7], "workspace");
        const int64_t B = q.size(0);
        t.q_len = args.dense<int32_t>(a[4], {B}, at::kInt, "q_len", true);
        t.rows = args.dense<int32_t>(a[5], {B}, at::kInt, "rows", true);
        Where w(args, a[8]);
        at::Tensor made;
        if (!out) {
            made = fresh(q.sizes(), q.scalar_type(), args.device);
            out = &made;
        }
        Args::type(*out, q.scalar_type(), "out");
        Args::shape(*out, q.sizes(), "out");
        Args::last_contiguous(*out, "out");
        t.q = q.data_ptr();
        t.out = out->data_ptr();
        t.q_stride_b = q.stride(0), t.q_stride_n = q.stride(1), t.q_stride_h = q.stride(2);
        t.out_stride_b = out->stride(0), t.out_stride_n = out->stride(1), t.out_stride_h = out->stride(2);
        t.batch = size32(q.size(0), "batch");
        t.n = size32(q.size(1), "n");
        t.q_heads = size32(q.size(2), "q_heads");
        t.scale = real(a[3], "scale");
        if (!t.rows && t.batch > c->pages.rows) throw Refused("more entries than rows of the table");
        t.workspace = work.data_ptr();
        t.workspace_bytes = static_cast<int64_t>(work.nbytes());
        if (failed(calls.ralm_kv_attend(c, int32(a[1], "layer"), &t, w.stream), "ralm_kv_attend")) return nullptr;
        return made.defined() ? THPVariable_Wrap(made) : same(a[6]);
    });
}

// bind(entry points by name, the class to raise)
PyObject *bind(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 2 || !PyDict_Check(a[0])) {
        PyErr_SetString(PyExc_TypeError, "bind(dict, class)");
        return nullptr;
    }
#define X(name)                                                                           \
    {                                                                                     \
        PyObject *v = PyDict_GetItemString(a[0], #name);                                  \
        void *at = v ? PyLong_AsVoidPtr(v) : nullptr;                                     \
        if (!at) {                                                                        \
            PyErr_SetString(PyExc_RuntimeError, "the library does not export " #name);    \
            return nullptr;                                                               \
        }                                                                                 \
        calls.name = reinterpret_cast<decltype(calls.name)>(at);                          \
    }
    RALM_CALLS(X)
#undef X
    Py_XDECREF(error_class);
    error_class = same(a[1]);
    Py_RETURN_NONE;
}

#define METHOD(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(bind), METHOD(knn_mix), METHOD(verify_tokens), METHOD(pages_resize), METHOD(pages_fork),
                         METHOD(pages_compact), METHOD(pages_copy), METHOD(kv_append), METHOD(kv_read), METHOD(kv_attend),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native() { return PyModule_Create(&module); }
