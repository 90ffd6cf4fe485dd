// Python binding of the calls that are made once per token (stom_kv.h, stom_sample.h): checks the tensors of a call
// against one another and passes their addresses on.  Written against torch's C++ tensors because the same checks in
// Python, with ctypes for the call, take 10 us, several times what the smaller kernels run.
//
// The functions take their arguments by position (oqm.py gives them names and defaults) and return the library's status.
// A tensor of the wrong type, shape, layout or device raises ValueError, before anything is launched.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <sstream>
#include <stdexcept>

#include "stom_kv.h"
#include "stom_sample.h"

namespace {

// ---- the library's entry points, set by oqm.py from the library that it has loaded
struct Library {
    decltype(&stom_kv_attend) attend = nullptr;
    decltype(&stom_kv_rotate) rotate = nullptr;
    decltype(&stom_kv_append) append = nullptr;
    decltype(&stom_kv_reserve) reserve = nullptr;
    decltype(&stom_kv_fork) fork = nullptr;
    decltype(&stom_kv_free) free_pages = nullptr;
    decltype(&stom_kv_compact) compact = nullptr;
    decltype(&stom_sample_tokens) sample = nullptr;
} lib;

[[noreturn]] void refuse(const char *name, const std::string &needed, const at::Tensor *t) {
    std::ostringstream s;
    s << name << ": " << needed << " is needed";
    if (t) s << ", not " << t->dtype() << " " << t->sizes() << " with strides " << t->strides() << " on " << t->device();
    throw std::invalid_argument(s.str());
}

const at::Tensor *tensor(PyObject *o, const char *name) {
    if (o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) throw std::invalid_argument(std::string(name) + ": a tensor is needed");
    return &THPVariable_Unpack(o);
}
const at::Tensor &must(PyObject *o, const char *name) {
    const at::Tensor *t = tensor(o, name);
    if (!t) throw std::invalid_argument(std::string(name) + ": a tensor is needed");
    return *t;
}
bool on(const at::Tensor &t, int64_t dev) { return t.is_cuda() && t.get_device() == dev; }

int64_t integer(PyObject *o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw std::runtime_error("");
    return v;
}
int32_t int32(PyObject *o) {
    const int64_t v = integer(o);
    if (v < INT32_MIN || v > INT32_MAX) throw std::invalid_argument("an integer of 32 bits is needed");
    return (int32_t)v;
}
float number(PyObject *o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw std::runtime_error("");
    return (float)v;
}
template <typename P>
const P *at_address(PyObject *o) {
    return reinterpret_cast<const P *>(integer(o));
}

// Address of a contiguous tensor of this type and shape (cols < 0: one axis), or NULL for None
template <typename P>
P *dense(PyObject *o, at::ScalarType type, int64_t rows, int64_t cols, int64_t dev, const char *name) {
    const at::Tensor *t = tensor(o, name);
    if (!t) return nullptr;
    const bool shape = cols < 0 ? t->dim() == 1 && t->size(0) == rows : t->dim() == 2 && t->size(0) == rows && t->size(1) == cols;
    if (t->scalar_type() != type || !shape || !t->is_contiguous() || !on(*t, dev)) {
        std::ostringstream s;
        s << "a contiguous " << type << " tensor of shape [" << rows;
        if (cols >= 0) s << ", " << cols;
        s << "] on cuda:" << dev;
        refuse(name, s.str(), t);
    }
    return static_cast<P *>(t->data_ptr());
}

// An [n][heads][d] tensor with adjacent channels
struct Rows {
    void *at = nullptr;
    int64_t row = 0, head = 0;
    int32_t heads = 0;
};
Rows rows(PyObject *o, at::ScalarType type, int64_t n, int64_t heads, int64_t d, int64_t dev, const char *name) {
    const at::Tensor &t = must(o, name);
    if (t.scalar_type() != type || t.dim() != 3 || t.size(0) != n || (heads >= 0 && t.size(1) != heads) || t.size(2) != d ||
        t.stride(2) != 1 || !on(t, dev)) {
        std::ostringstream s;
        s << "a " << type << " tensor of shape [" << n << ", ";
        if (heads >= 0) s << heads;
        else s << "heads";
        s << ", " << d << "] with adjacent channels on cuda:" << dev;
        refuse(name, s.str(), &t);
    }
    return Rows{t.data_ptr(), t.stride(0), t.stride(1), (int32_t)t.size(1)};
}
void *workspace(PyObject *o, int64_t dev, int64_t &bytes) {
    const at::Tensor &t = must(o, "workspace");
    if (!on(t, dev) || !t.is_contiguous()) refuse("workspace", "a contiguous tensor on the device of the call", &t);
    bytes = (int64_t)t.nbytes();
    return t.data_ptr();
}
uint32_t *flags(PyObject *o, int64_t dev) {
    const at::Tensor *t = tensor(o, "dev_flags");
    if (!t) return nullptr;
    if (!on(*t, dev) || t->element_size() != 4 || t->numel() < 1) refuse("dev_flags", "one 32-bit word on the device of the call", t);
    return static_cast<uint32_t *>(t->data_ptr());
}
at::ScalarType type_of(int32_t dtype) {
    return dtype == STOM_BF16 ? at::kBFloat16 : dtype == STOM_FP16 ? at::kHalf : at::kFloat;
}
int32_t dtype_of(const at::Tensor &t, const char *name) {
    switch (t.scalar_type()) {
    case at::kBFloat16: return STOM_BF16;
    case at::kHalf: return STOM_FP16;
    case at::kFloat: return STOM_FP32;
    default: refuse(name, "a bfloat16, float16 or float32 tensor", &t);
    }
}

// The device of a call made current, and the stream to use: the one given by its handle, or the device's current one
struct On {
    c10::cuda::OptionalCUDAGuard guard;
    void *stream;
    On(int64_t dev, PyObject *given) {
        if (dev < 0) throw std::invalid_argument("the tensors of a call lie on a CUDA device");
        if (c10::cuda::current_device() != dev) guard.set_index((c10::DeviceIndex)dev);
        stream = given == Py_None ? (void *)c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)dev).stream()
                                  : reinterpret_cast<void *>(integer(given));
    }
};

template <typename F>
PyObject *guarded(Py_ssize_t got, Py_ssize_t wanted, F f) {
    try {
        if (got != wanted) throw std::invalid_argument("wrong number of arguments");
        return PyLong_FromLong(f());
    } catch (const std::exception &e) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, e.what());
    } catch (...) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, "unknown error");
    }
    return nullptr;
}

// pool, seqs, device, layer, q, out, scale, softcap, window, lse, workspace, dev_flags, stream
PyObject *attend(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 13, [&] {
        const auto *pool = at_address<stom_kv_pool>(a[0]);
        const auto *seqs = at_address<stom_kv_seqs>(a[1]);
        const int64_t dev = integer(a[2]);
        const at::ScalarType type = type_of(pool->dtype);
        const Rows q = rows(a[4], type, seqs->n_seqs, -1, pool->head_dim, dev, "q");
        const Rows out = rows(a[5], type, seqs->n_seqs, q.heads, pool->head_dim, dev, "out");
        float *lse = dense<float>(a[9], at::kFloat, seqs->n_seqs, q.heads, dev, "lse");
        int64_t bytes;
        void *ws = workspace(a[10], dev, bytes);
        uint32_t *fl = flags(a[11], dev);
        const On on(dev, a[12]);
        return lib.attend(pool, seqs, int32(a[3]), q.heads, q.at, q.row, q.head, number(a[6]), number(a[7]), int32(a[8]), out.at,
                          out.row, out.head, lse, ws, bytes, fl, on.stream);
    });
}

// rope, pos, q, q_out, k, k_out, q_weight, k_weight, eps, stream, device of the frequencies
PyObject *rotate(PyObject *, PyObject *const *a, Py_ssize_t count) {
    return guarded(count, 11, [&] {
        const auto *rope = at_address<stom_kv_rope>(a[0]);
        const at::Tensor &x = must(a[2] != Py_None ? a[2] : a[4], "q or k");
        if (x.dim() != 3) refuse("q or k", "a tensor of three axes", &x);
        const int64_t n = x.size(0), d = x.size(2), dev = x.is_cuda() ? x.get_device() : -1;
        const int32_t dtype = dtype_of(x, "q or k");
        if (n > INT32_MAX || d > INT32_MAX) refuse("q or k", "sizes of 32 bits", &x);
        if (a[10] != Py_None && integer(a[10]) != dev) throw std::invalid_argument("the frequencies lie on the device of the tensors");
        Rows q, qo, k, ko;
        const float *qw = nullptr, *kw = nullptr;
        if (a[2] != Py_None) {
            q = rows(a[2], type_of(dtype), n, -1, d, dev, "q");
            qo = rows(a[3], type_of(dtype), n, q.heads, d, dev, "q_out");
            qw = dense<float>(a[6], at::kFloat, d, -1, dev, "q_weight");
        }
        if (a[4] != Py_None) {
            k = rows(a[4], type_of(dtype), n, -1, d, dev, "k");
            ko = rows(a[5], type_of(dtype), n, k.heads, d, dev, "k_out");
            kw = dense<float>(a[7], at::kFloat, d, -1, dev, "k_weight");
        }
        const int32_t *pos = dense<int32_t>(a[1], at::kInt, n, -1, dev, "pos");
        const On on(dev, a[9]);
        return lib.rotate(rope, dtype, (int32_t)d, (int32_t)n, pos, q.at, q.heads, q.row, q.head, qo.at, qo.row, qo.head, qw, k.at,
                          k.heads, k.row, k.head, ko.at, ko.row, ko.head, kw, number(a[8]), on.stream);
    });
}

// pool, seqs, device, layer, rope, pos, slot, k, v, q, q_out, seq, q_weight, k_weight, eps, dev_flags, stream
PyObject *append(PyObject *, PyObject *const *a, Py_ssize_t count) {
    return guarded(count, 17, [&] {
        const auto *pool = at_address<stom_kv_pool>(a[0]);
        const auto *seqs = at_address<stom_kv_seqs>(a[1]);
        const int64_t dev = integer(a[2]), d = pool->head_dim;
        const at::ScalarType type = type_of(pool->dtype);
        const at::Tensor &x = must(a[7], "k");
        if (x.dim() != 3 || x.size(0) > INT32_MAX) refuse("k", "a tensor of three axes", &x);
        const int64_t n = x.size(0);
        const Rows k = rows(a[7], type, n, pool->n_kv_heads, d, dev, "k"), v = rows(a[8], type, n, pool->n_kv_heads, d, dev, "v");
        Rows q, qo;
        const float *qw = nullptr;
        if (a[9] != Py_None) {
            q = rows(a[9], type, n, -1, d, dev, "q");
            qo = rows(a[10], type, n, q.heads, d, dev, "q_out");
            qw = dense<float>(a[12], at::kFloat, d, -1, dev, "q_weight");
        }
        const float *kw = dense<float>(a[13], at::kFloat, d, -1, dev, "k_weight");
        const int32_t *pos = dense<int32_t>(a[5], at::kInt, n, -1, dev, "pos");
        const int32_t *slot = dense<int32_t>(a[6], at::kInt, n, -1, dev, "slot");
        const int32_t *seq = dense<int32_t>(a[11], at::kInt, n, -1, dev, "seq");
        uint32_t *fl = flags(a[15], dev);
        const On on(dev, a[16]);
        return lib.append(pool, seqs, int32(a[3]), at_address<stom_kv_rope>(a[4]), (int32_t)n, pos, slot, seq, q.at, q.heads, q.row,
                          q.head, qo.at, qo.row, qo.head, qw, k.at, k.row, k.head, kw, v.at, v.row, v.head, number(a[14]), fl,
                          on.stream);
    });
}

// pool, seqs, device, want, workspace, dev_flags, stream
PyObject *reserve(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 7, [&] {
        const auto *seqs = at_address<stom_kv_seqs>(a[1]);
        const int64_t dev = integer(a[2]);
        const int32_t *want = dense<int32_t>(a[3], at::kInt, seqs->n_seqs, -1, dev, "want");
        int64_t bytes;
        void *ws = workspace(a[4], dev, bytes);
        uint32_t *fl = flags(a[5], dev);
        const On on(dev, a[6]);
        return lib.reserve(at_address<stom_kv_pool>(a[0]), seqs, want, ws, bytes, fl, on.stream);
    });
}

// pool, seqs, device, parent or drop, dev_flags, stream
PyObject *fork_rows(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 6, [&] {
        const auto *seqs = at_address<stom_kv_seqs>(a[1]);
        const int64_t dev = integer(a[2]);
        const int32_t *wish = dense<int32_t>(a[3], at::kInt, seqs->n_seqs, -1, dev, "parent");
        uint32_t *fl = flags(a[4], dev);
        const On on(dev, a[5]);
        return lib.fork(at_address<stom_kv_pool>(a[0]), seqs, wish, fl, on.stream);
    });
}
PyObject *free_rows(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 6, [&] {
        const auto *seqs = at_address<stom_kv_seqs>(a[1]);
        const int64_t dev = integer(a[2]);
        const int32_t *wish = dense<int32_t>(a[3], at::kInt, seqs->n_seqs, -1, dev, "drop");
        uint32_t *fl = flags(a[4], dev);
        const On on(dev, a[5]);
        return lib.free_pages(at_address<stom_kv_pool>(a[0]), seqs, wish, fl, on.stream);
    });
}

// pool, seqs, device, table_out, refs_out, n_live, workspace, dev_flags, stream
PyObject *compact(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 9, [&] {
        const auto *pool = at_address<stom_kv_pool>(a[0]);
        const auto *seqs = at_address<stom_kv_seqs>(a[1]);
        const int64_t dev = integer(a[2]);
        const at::Tensor &t = must(a[3], "table_out");
        if (t.scalar_type() != at::kInt || t.dim() != 2 || t.size(0) != seqs->n_seqs || t.size(1) != seqs->max_pages ||
            (seqs->max_pages > 1 && t.stride(1) != 1) || (seqs->n_seqs > 1 && t.stride(0) != seqs->table_stride) || !on(t, dev))
            refuse("table_out", "a tensor like the sequences' table", &t);
        int32_t *refs = dense<int32_t>(a[4], at::kInt, pool->n_pages, -1, dev, "refs_out");
        int32_t *live = dense<int32_t>(a[5], at::kInt, 1, -1, dev, "n_live");
        int64_t bytes;
        void *ws = workspace(a[6], dev, bytes);
        uint32_t *fl = flags(a[7], dev);
        const On on(dev, a[8]);
        return lib.compact(pool, seqs, static_cast<int32_t *>(t.data_ptr()), refs, live, ws, bytes, fl, on.stream);
    });
}

// logits, u, token, temperature, top_k, top_p, min_p, logprob, kept, dev_flags, stream
PyObject *sample(PyObject *, PyObject *const *a, Py_ssize_t count) {
    return guarded(count, 11, [&] {
        const at::Tensor &x = must(a[0], "logits");
        if (x.dim() != 2 || (x.size(1) > 1 && x.stride(1) != 1) || x.size(0) > INT32_MAX || x.size(1) > INT32_MAX)
            refuse("logits", "a tensor of two axes whose rows have adjacent entries", &x);
        const int32_t dtype = dtype_of(x, "logits");
        const int64_t n = x.size(0), dev = x.is_cuda() ? x.get_device() : -1;
        const float *u = dense<float>(a[1], at::kFloat, n, -1, dev, "u");
        int32_t *token = dense<int32_t>(a[2], at::kInt, n, -1, dev, "token");
        const float *t = dense<float>(a[3], at::kFloat, n, -1, dev, "temperature");
        const int32_t *k = dense<int32_t>(a[4], at::kInt, n, -1, dev, "top_k");
        const float *p = dense<float>(a[5], at::kFloat, n, -1, dev, "top_p");
        const float *m = dense<float>(a[6], at::kFloat, n, -1, dev, "min_p");
        float *lp = dense<float>(a[7], at::kFloat, n, -1, dev, "logprob");
        int32_t *kept = dense<int32_t>(a[8], at::kInt, n, -1, dev, "kept");
        uint32_t *fl = flags(a[9], dev);
        const On on(dev, a[10]);
        return lib.sample(x.data_ptr(), dtype, (int32_t)n, (int32_t)x.size(1), x.stride(0), t, k, p, m, u, token, kept, lp, fl,
                          on.stream);
    });
}

// the addresses of the library's entry points, in the order of Library
PyObject *use(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 8, [&] {
        lib.attend = reinterpret_cast<decltype(lib.attend)>(integer(a[0]));
        lib.rotate = reinterpret_cast<decltype(lib.rotate)>(integer(a[1]));
        lib.append = reinterpret_cast<decltype(lib.append)>(integer(a[2]));
        lib.reserve = reinterpret_cast<decltype(lib.reserve)>(integer(a[3]));
        lib.fork = reinterpret_cast<decltype(lib.fork)>(integer(a[4]));
        lib.free_pages = reinterpret_cast<decltype(lib.free_pages)>(integer(a[5]));
        lib.compact = reinterpret_cast<decltype(lib.compact)>(integer(a[6]));
        lib.sample = reinterpret_cast<decltype(lib.sample)>(integer(a[7]));
        return 0;
    });
}

#define STOM_METHOD(name, f) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    STOM_METHOD("use", use), STOM_METHOD("attend", attend), STOM_METHOD("rotate", rotate), STOM_METHOD("append", append),
    STOM_METHOD("reserve", reserve), STOM_METHOD("fork", fork_rows), STOM_METHOD("free", free_rows),
    STOM_METHOD("compact", compact), STOM_METHOD("sample", sample), {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_stom_bind", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__stom_bind(void) { return PyModule_Create(&module); }
