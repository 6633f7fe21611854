// Python calls of the C ABI without ctypes: a step hands over some twenty tensors, and per call the marshalling in Python and
// ctypes took longer than the kernels' launches (26-node greedy step called one by one 15.9 -> 14.5 us; the first pass of a draft
// phase of six calls on new buffers 106 -> 67 us on one box).  What each argument has to be follows from the prototypes in fspad.h: a
// pointer to fspad_bf16, float, int32_t, uint64_t is a contiguous tensor of that type on the GPU (of the host entry point: in
// host memory, the cache apart) or None, a void pointer a uint8 tensor, an address or None, everything else a number.
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ATen.h>

#include <algorithm>
#include <climits>
#include <cstdarg>
#include <exception>
#include <string>
#include <tuple>
#include <utility>

#include "fspad.h"

namespace {

template <typename T> struct Wanted;
template <> struct Wanted<fspad_bf16> { static constexpr at::ScalarType type = at::kBFloat16; static constexpr const char *name = "torch.bfloat16"; };
template <> struct Wanted<float> { static constexpr at::ScalarType type = at::kFloat; static constexpr const char *name = "torch.float32"; };
template <> struct Wanted<int32_t> { static constexpr at::ScalarType type = at::kInt; static constexpr const char *name = "torch.int32"; };
template <> struct Wanted<uint64_t> { static constexpr at::ScalarType type = at::kLong; static constexpr const char *name = "torch.int64"; };
template <> struct Wanted<void> { static constexpr at::ScalarType type = at::kByte; static constexpr const char *name = "torch.uint8"; };

// Address of a tensor's data; a Python error is set and false returned where it is not what the call takes.
template <typename T>
bool tensor_address(PyObject *o, bool on_gpu, void **out)
{
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "expected a tensor of %s, got %R", Wanted<T>::name, (PyObject *)Py_TYPE(o));
        return false;
    }
    const at::Tensor &t = THPVariable_Unpack(o);
    if (t.scalar_type() != Wanted<T>::type) {
        PyObject *is = PyObject_GetAttrString(o, "dtype");
        if (is != nullptr) PyErr_Format(PyExc_TypeError, "expected %s, got %S", Wanted<T>::name, is);
        Py_XDECREF(is);
        return false;
    }
    if (!t.is_contiguous()) {
        PyErr_SetString(PyExc_ValueError, "tensor must be contiguous");
        return false;
    }
    if (on_gpu ? !t.is_cuda() : !t.is_cpu()) {
        PyErr_Format(PyExc_ValueError, "tensor must live on %s, not %s", on_gpu ? "cuda" : "cpu", t.device().str().c_str());
        return false;
    }
    *out = t.data_ptr();
    return true;
}

template <typename A>
bool convert(PyObject *o, bool on_gpu, A *out)
{
    if constexpr (std::is_pointer_v<A>) {
        using T = std::remove_cv_t<std::remove_pointer_t<A>>;
        void *p = nullptr;
        if (o == Py_None) {
        } else if constexpr (std::is_same_v<T, fspad_ctx> || std::is_same_v<T, void>) {
            if (PyLong_Check(o)) {
                p = PyLong_AsVoidPtr(o);
                if (p == nullptr && PyErr_Occurred()) return false;
            } else if constexpr (std::is_same_v<T, void>) {
                if (!tensor_address<T>(o, on_gpu, &p)) return false;
            } else {
                PyErr_SetString(PyExc_TypeError, "expected a context's address");
                return false;
            }
        } else if (!tensor_address<T>(o, on_gpu, &p)) {
            return false;
        }
        *out = static_cast<A>(p);
        return true;
    } else {
        const long long v = PyLong_AsLongLong(o);
        if (v == -1 && PyErr_Occurred()) return false;
        if (static_cast<long long>(static_cast<A>(v)) != v) {
            PyErr_SetString(PyExc_OverflowError, "number does not fit");
            return false;
        }
        *out = static_cast<A>(v);
        return true;
    }
}

// host_from: the first argument whose tensors lie in host memory.  A tensor may throw when it is asked for its strides or its address
// (one inside vmap or grad, for instance): by torch's own translation that becomes the Python exception.
template <typename... A, size_t... I>
PyObject *invoke(int (*fn)(A...), PyObject *const *args, Py_ssize_t n, size_t host_from, std::index_sequence<I...>)
{
    if (n != (Py_ssize_t)sizeof...(A)) {
        PyErr_Format(PyExc_TypeError, "%zd arguments, not %zd", (Py_ssize_t)sizeof...(A), n);
        return nullptr;
    }
    std::tuple<A...> a{};
    try {
        if (!(convert(args[I], I < host_from, &std::get<I>(a)) && ...)) return nullptr;
    } catch (...) {
        torch::translate_exception_to_python(std::current_exception());
        return nullptr;
    }
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = fn(std::get<I>(a)...);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}
template <typename... A>
PyObject *invoke(int (*fn)(A...), PyObject *const *args, Py_ssize_t n, size_t host_from = 99)
{
    return invoke(fn, args, n, host_from, std::index_sequence_for<A...>());
}

#define FSPAD_CALL(name, ...) \
    PyObject *call_##name(PyObject *, PyObject *const *args, Py_ssize_t n) { return invoke(fspad_##name, args, n, ##__VA_ARGS__); }
FSPAD_CALL(tree_attn)
FSPAD_CALL(tree_attn_paged)
FSPAD_CALL(tree_accept)
FSPAD_CALL(kv_compact)
FSPAD_CALL(kv_compact_paged)
FSPAD_CALL(kv_append)
FSPAD_CALL(lm_head_accept)
FSPAD_CALL(feature_sampler)
FSPAD_CALL(tree_build)
FSPAD_CALL(draft_expand)
FSPAD_CALL(verify_step)
FSPAD_CALL(verify_step_host, 2)
#undef FSPAD_CALL

// ---- the calls around the 4-bit cache: they know the context's sizes, look at every tensor's shape and device, and make the outputs that are
// not given (in Python that took longer than the launches: a single-token step 11.1 -> 7.5 us, rotary rows of a tree 13.8 -> 5.8) ----
// A tensor's address; an empty one has none, and nothing is read or written there: it gets one that is aligned.
alignas(16) char kNothing[16];
void *address(const at::Tensor &t) { return t.numel() ? t.data_ptr() : kNothing; }
template <typename T> T *as(const at::Tensor &t) { return static_cast<T *>(address(t)); }

struct Output {
    const char *name;
    PyObject *given;
    at::ScalarType type;
    std::initializer_list<long long> size;
    size_t bytes() const                                     // in whole steps of 256, so that each starts as an allocation does
    {
        size_t n = c10::elementSize(type);
        for (long long x : size) n *= (size_t)x;
        return n == 0 ? 256 : (n + 255) / 256 * 256;
    }
};

struct Call {
    fspad_ctx *ctx;
    int device;
    long long hq, hkv, layers, max_nodes;
    void *stream;
    bool ok = true;

    const at::Tensor *fail(PyObject *kind, const char *fmt, ...)
    {
        va_list ap;
        va_start(ap, fmt);
        if (ok) PyErr_FormatV(kind, fmt, ap);
        va_end(ap);
        ok = false;
        return nullptr;
    }
    long long whole(PyObject *o)
    {
        const long long v = ok ? PyLong_AsLongLong(o) : 0;
        if (v == -1 && PyErr_Occurred()) ok = false;
        return v;
    }
    int number(PyObject *o)
    {
        const long long v = whole(o);
        if (v != (int)v) fail(PyExc_OverflowError, "number does not fit");
        return (int)v;
    }
    // A tensor of this type on the context's device; its shape is looked at by `shaped`.
    const at::Tensor *tensor(const char *name, PyObject *o, at::ScalarType type, bool contiguous = true)
    {
        if (!ok) return nullptr;
        if (!THPVariable_Check(o)) return fail(PyExc_TypeError, "%s: expected a tensor, got %R", name, (PyObject *)Py_TYPE(o));
        const at::Tensor &t = THPVariable_Unpack(o);
        if (t.scalar_type() != type) return fail(PyExc_TypeError, "%s: expected %s, got %s", name, at::toString(type), at::toString(t.scalar_type()));
        if (!t.is_cuda() || (device >= 0 && t.get_device() != device))
            return fail(PyExc_ValueError, "%s: tensor must live on cuda:%d, not %s", name, device, t.device().str().c_str());
        if (contiguous && !t.is_contiguous()) return fail(PyExc_ValueError, "%s: tensor must be contiguous", name);
        return &t;
    }
    bool shaped(const char *name, const at::Tensor *t, std::initializer_list<long long> want)
    {
        if (!ok) return false;
        const auto is = t->sizes();
        bool same = is.size() == want.size();
        for (size_t i = 0; same && i < want.size(); ++i) same = is[i] == want.begin()[i];
        if (same) return true;
        std::string a, b;
        for (long long x : want) a += (a.empty() ? "" : ", ") + std::to_string(x);
        for (long long x : is) b += (b.empty() ? "" : ", ") + std::to_string(x);
        fail(PyExc_ValueError, "%s: expected shape (%s), got (%s)", name, a.c_str(), b.c_str());
        return false;
    }
    // ... or none: its address, or NULL
    void *data(const char *name, PyObject *o, at::ScalarType type, std::initializer_list<long long> want, bool optional = false)
    {
        if (!ok || (optional && o == Py_None)) return nullptr;
        const at::Tensor *t = tensor(name, o, type);
        return t && shaped(name, t, want) ? address(*t) : nullptr;
    }
    // Outputs: the tensors that were given; the others are new and share one allocation of the current stream's (on the current device, which
    // the library then checks).  An allocation for each took 0.9 us of a call's 8.
    void outputs(at::Tensor *to, std::initializer_list<Output> wanted)
    {
        size_t bytes = 0;
        at::Tensor *t = to;
        for (const Output &w : wanted) {
            if (!ok) return;
            if (w.given != Py_None) {
                const at::Tensor *x = tensor(w.name, w.given, w.type);
                if (x && shaped(w.name, x, w.size)) *t = *x;
            } else {
                bytes += w.bytes();
            }
            ++t;
        }
        if (!ok || bytes == 0) return;
        auto storage = c10::make_intrusive<c10::StorageImpl>(c10::StorageImpl::use_byte_size_t(), bytes, c10::GetAllocator(c10::kCUDA), true);
        size_t at = 0;
        t = to;
        for (const Output &w : wanted) {
            if (w.given == Py_None) {
                int64_t size[8];
                std::copy(w.size.begin(), w.size.end(), size);
                *t = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(storage), c10::DispatchKeySet(c10::DispatchKey::CUDA), caffe2::TypeMeta::fromScalarType(w.type));
                t->unsafeGetTensorImpl()->set_sizes_contiguous(at::IntArrayRef(size, w.size.size()));
                t->unsafeGetTensorImpl()->set_storage_offset((int64_t)(at / c10::elementSize(w.type)));
                at += w.bytes();
            }
            ++t;
        }
    }
    // Codes and scales of the cache: its blocks.
    int cache(PyObject *codes, PyObject *scales, uint8_t **c, uint8_t **s)
    {
        const at::Tensor *t = tensor("codes", codes, at::kByte);
        if (!t) return 0;
        const long long nb = t->dim() == 6 ? t->size(2) : 0;
        *c = static_cast<uint8_t *>(data("codes", codes, at::kByte, {layers, 2, nb, hkv, 128, 64}));
        *s = static_cast<uint8_t *>(data("scales", scales, at::kByte, {layers, 2, nb, hkv, 128, 8}));
        if (ok && nb > INT_MAX) fail(PyExc_OverflowError, "too many blocks");
        return (int)nb;
    }
};

// (handle, Hq, Hkv, layers, max_nodes, stream) come first.  `body` gives the arguments' checks and the call: its status, and what it returns.
template <typename F> PyObject *packed_call(PyObject *const *args, Py_ssize_t n, Py_ssize_t want, F body)
{
    if (n != want) {
        PyErr_Format(PyExc_TypeError, "%zd arguments, not %zd", want, n);
        return nullptr;
    }
    try {
        Call c{};
        c.ctx = PyLong_Check(args[0]) ? static_cast<fspad_ctx *>(PyLong_AsVoidPtr(args[0])) : nullptr;
        if (PyErr_Occurred()) return nullptr;
        c.device = fspad_device(c.ctx);
        c.hq = c.whole(args[1]); c.hkv = c.whole(args[2]); c.layers = c.whole(args[3]); c.max_nodes = c.whole(args[4]);
        c.stream = args[5] == Py_None ? nullptr : PyLong_AsVoidPtr(args[5]);
        if (PyErr_Occurred()) return nullptr;
        int rc = 0;
        PyObject *result = body(c, args + 6, rc);
        if (!c.ok) {
            Py_XDECREF(result);
            return nullptr;
        }
        if (rc != 0) {                               // the library's status, in place of a result
            Py_XDECREF(result);
            return PyLong_FromLong(rc);
        }
        return result;
    } catch (...) {
        torch::translate_exception_to_python(std::current_exception());
        return nullptr;
    }
}
template <typename F> int unlocked(F f)
{
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f();
    Py_END_ALLOW_THREADS
    return rc;
}
constexpr at::ScalarType kBf = at::kBFloat16, kI32 = at::kInt;

PyObject *call_rope_qkv(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return packed_call(args, n, 6 + 12, [](Call &c, PyObject *const *a, int &rc) -> PyObject * {
        const at::Tensor *qkv = c.tensor("qkv", a[0], kBf, false);
        const double theta = PyFloat_AsDouble(a[1]);
        if (theta == -1.0 && PyErr_Occurred()) c.ok = false;
        const int st = c.number(a[2]), sh = c.number(a[3]), sw = c.number(a[4]);
        if (!c.ok) return nullptr;
        const long long width = (c.hq + 2 * c.hkv) * 128;
        if (qkv->dim() != 3 || qkv->size(2) != width) {
            c.fail(PyExc_ValueError, "qkv: expected [batch][nodes][%lld]", width);
            return nullptr;
        }
        const long long B = qkv->size(0), N = qkv->size(1);
        long long row = N > 1 ? qkv->stride(1) : B > 1 ? qkv->stride(0) : width;
        if (qkv->stride(2) != 1 || (N > 1 && B > 1 && qkv->stride(0) != N * row)) {
            c.fail(PyExc_ValueError, "qkv: rows must be contiguous and evenly spaced");
            return nullptr;
        }
        if (B > INT_MAX || N > INT_MAX) c.fail(PyExc_OverflowError, "too many rows");
        const auto *parent = static_cast<const int32_t *>(c.data("parent", a[5], kI32, {B, N}, true));
        const auto *start = static_cast<const int32_t *>(c.data("start", a[6], kI32, {B, 3}, true));
        const auto *positions = static_cast<const int32_t *>(c.data("positions", a[7], kI32, {B, N, 3}, true));
        const int adjacent = c.ok ? PyObject_IsTrue(a[8]) : 0;
        at::Tensor o[3];
        c.outputs(o, {{"q", a[9], kBf, {B, N, c.hq, 128}}, {"k", a[10], kBf, {B, c.hkv, N, 128}}, {"v", a[11], kBf, {B, c.hkv, N, 128}}});
        if (!c.ok) return nullptr;
        const auto *x = as<fspad_bf16>(*qkv);
        rc = unlocked([&] { return fspad_rope_qkv(c.ctx, x, row, positions, start, parent, (int)N, (int)B, theta, st, sh, sw, adjacent, as<fspad_bf16>(o[0]), as<fspad_bf16>(o[1]), as<fspad_bf16>(o[2]), c.stream); });
        return rc ? nullptr : Py_BuildValue("(NNN)", THPVariable_Wrap(o[0]), THPVariable_Wrap(o[1]), THPVariable_Wrap(o[2]));
    });
}

PyObject *call_block_plan(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return packed_call(args, n, 6 + 12, [](Call &c, PyObject *const *a, int &rc) -> PyObject * {
        const at::Tensor *table = c.tensor("block_table", a[3], kI32), *free_blocks = c.tensor("free_blocks", a[5], kI32);
        const int max_rows = c.number(a[7]);
        if (!c.ok) return nullptr;
        if (table->dim() != 2 || free_blocks->dim() != 1 || table->numel() > (1ll << 40) || free_blocks->numel() > INT_MAX || max_rows < 0) {
            c.fail(PyExc_ValueError, "block_table: expected [batch][blocks]; free_blocks: [blocks]; max_rows: 0 or more");
            return nullptr;
        }
        const long long B = table->size(0), bps = table->size(1), nb = free_blocks->size(0);
        if (B > INT_MAX || bps > INT_MAX) c.fail(PyExc_OverflowError, "block_table is too large");
        const auto *len = static_cast<const int32_t *>(c.data("length", a[0], kI32, {B})), *add = static_cast<const int32_t *>(c.data("add", a[1], kI32, {B}));
        const auto *drop = static_cast<const int32_t *>(c.data("drop", a[2], kI32, {B}, true));
        auto *held = static_cast<int32_t *>(c.data("held", a[4], kI32, {B})), *n_free = static_cast<int32_t *>(c.data("n_free", a[6], kI32, {1}));
        at::Tensor o[4];
        c.outputs(o, {{"row_start", a[8], kI32, {B + 1}}, {"slots", a[9], at::kLong, {max_rows}}, {"row_seq", a[10], kI32, {max_rows}}, {"row_pos", a[11], kI32, {max_rows}}});
        if (!c.ok) return nullptr;
        rc = unlocked([&] { return fspad_block_plan(c.ctx, len, add, drop, (int)B, (int)bps, (int)nb, as<int32_t>(*table), held, as<int32_t>(*free_blocks), n_free, max_rows, as<int32_t>(o[0]),
                                                     as<int64_t>(o[1]), as<int32_t>(o[2]), as<int32_t>(o[3]), c.stream); });
        return rc ? nullptr : Py_BuildValue("(NNNN)", THPVariable_Wrap(o[0]), THPVariable_Wrap(o[1]), THPVariable_Wrap(o[2]), THPVariable_Wrap(o[3]));
    });
}

PyObject *call_kv_write_packed(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return packed_call(args, n, 6 + 8, [](Call &c, PyObject *const *a, int &rc) -> PyObject * {
        const at::Tensor *slots = c.tensor("slots", a[2], at::kLong);
        uint8_t *codes = nullptr, *scales = nullptr;
        const int nb = c.cache(a[3], a[4], &codes, &scales), layer = c.number(a[5]);
        if (!c.ok) return nullptr;
        if (slots->dim() != 1 || slots->numel() > INT_MAX) {
            c.fail(PyExc_ValueError, "slots: expected one axis");
            return nullptr;
        }
        const long long rows = slots->size(0);
        auto rows_of = [&](const char *name, PyObject *o, bool optional) -> fspad_bf16 * {       // [Hkv][rows][128], or that with an axis of one before it
            if (!c.ok || (optional && o == Py_None)) return nullptr;
            const at::Tensor *t = c.tensor(name, o, kBf);
            if (!t) return nullptr;
            if (!(t->dim() == 4 && t->size(0) == 1 && t->size(1) == c.hkv && t->size(2) == rows && t->size(3) == 128)) c.shaped(name, t, {c.hkv, rows, 128});
            return as<fspad_bf16>(*t);
        };
        const auto *k = rows_of("k", a[0], false), *v = rows_of("v", a[1], false);
        auto *kr = rows_of("k_rounded", a[6], true), *vr = rows_of("v_rounded", a[7], true);
        if (!c.ok) return nullptr;
        rc = unlocked([&] { return fspad_kv_write_packed(c.ctx, k, v, as<int64_t>(*slots), (int)rows, layer, codes, scales, nb, kr, vr, c.stream); });
        if (rc) return nullptr;
        Py_RETURN_NONE;
    });
}

// [batch][blocks] of a table of blocks
static const int32_t *block_table(Call &c, PyObject *o, long long *B, int *bps)
{
    const at::Tensor *t = c.tensor("block_table", o, kI32);
    if (!t) return nullptr;
    if (t->dim() != 2 || t->size(0) > INT_MAX || t->size(1) > INT_MAX) {
        c.fail(PyExc_ValueError, "block_table: expected [batch][blocks]");
        return nullptr;
    }
    *B = t->size(0);
    *bps = (int)t->size(1);
    return as<int32_t>(*t);
}

PyObject *call_kv_append_packed(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return packed_call(args, n, 6 + 9, [](Call &c, PyObject *const *a, int &rc) -> PyObject * {
        uint8_t *codes = nullptr, *scales = nullptr;
        const int nb = c.cache(a[0], a[1], &codes, &scales);
        long long B = 0;
        int bps = 0;
        const int32_t *table = block_table(c, a[2], &B, &bps);
        const at::Tensor *tree = c.tensor("tree_kv", a[3], kBf);
        if (!c.ok) return nullptr;
        const long long N = tree->dim() == 6 ? tree->size(4) : 0;
        const auto *kv = static_cast<const fspad_bf16 *>(c.data("tree_kv", a[3], kBf, {c.layers, 2, B, c.hkv, N, 128}));
        const auto *path = static_cast<const int32_t *>(c.data("accepted_path", a[4], kI32, {B, c.max_nodes}));
        const auto *count = static_cast<const int32_t *>(c.data("n_accepted", a[5], kI32, {B})), *len = static_cast<const int32_t *>(c.data("prefix_len", a[6], kI32, {B}));
        auto *rounded = static_cast<fspad_bf16 *>(c.data("rounded", a[7], kBf, {c.layers, 2, B, c.hkv, N, 128}, true));
        at::Tensor new_len;
        c.outputs(&new_len, {{"new_len", a[8], kI32, {B}}});
        if (!c.ok) return nullptr;
        rc = unlocked([&] { return fspad_kv_append_packed(c.ctx, codes, scales, table, bps, nb, kv, path, count, len, (int)N, (int)B, rounded, as<int32_t>(new_len), c.stream); });
        return rc ? nullptr : THPVariable_Wrap(new_len);
    });
}

PyObject *call_tree_attn_packed(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return packed_call(args, n, 6 + 11, [](Call &c, PyObject *const *a, int &rc) -> PyObject * {
        const at::Tensor *q = c.tensor("q", a[0], kBf);
        uint8_t *codes = nullptr, *scales = nullptr;
        const int nb = c.cache(a[1], a[2], &codes, &scales), layer = c.number(a[8]);
        long long B = 0;
        int bps = 0;
        const int32_t *table = block_table(c, a[3], &B, &bps);
        if (!c.ok) return nullptr;
        const long long N = q->dim() == 4 ? q->size(1) : 0;
        c.shaped("q", q, {B, N, c.hq, 128});
        const auto *tk = static_cast<const fspad_bf16 *>(c.data("tree_k", a[4], kBf, {B, c.hkv, N, 128})), *tv = static_cast<const fspad_bf16 *>(c.data("tree_v", a[5], kBf, {B, c.hkv, N, 128}));
        const auto *parent = static_cast<const int32_t *>(c.data("parent", a[6], kI32, {B, N})), *len = static_cast<const int32_t *>(c.data("prefix_len", a[7], kI32, {B}));
        at::Tensor out;
        c.outputs(&out, {{"out", a[9], kBf, {B, N, c.hq, 128}}});
        // none given: one is made, once everything else has been looked at, and goes back with the output (its size is the same for every call of a context;
        // a context that is none has none, and the library refuses the call)
        at::Tensor ws;
        const bool make = a[10] == Py_None;
        if (make) {
            const long long bytes = (long long)fspad_tree_attn_packed_workspace_bytes(c.ctx, (int)c.max_nodes, 0);
            if (bytes > 0) c.outputs(&ws, {{"workspace", Py_None, at::kByte, {bytes}}});
        } else if (const at::Tensor *t = c.tensor("workspace", a[10], at::kByte)) {
            ws = *t;
        }
        if (!c.ok) return nullptr;
        rc = unlocked([&] { return fspad_tree_attn_packed(c.ctx, as<fspad_bf16>(*q), codes, scales, layer, table, bps, nb, tk, tv, parent, len, (int)N, (int)B, as<fspad_bf16>(out),
                                                           ws.defined() ? address(ws) : nullptr, ws.defined() ? (size_t)ws.numel() : 0, c.stream); });
        if (rc) return nullptr;
        return make ? Py_BuildValue("(NN)", THPVariable_Wrap(out), THPVariable_Wrap(ws)) : THPVariable_Wrap(out);
    });
}

#define FSPAD_ENTRY(name) {#name, (PyCFunction)(void (*)(void))call_##name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FSPAD_ENTRY(tree_attn), FSPAD_ENTRY(tree_attn_paged), FSPAD_ENTRY(tree_accept), FSPAD_ENTRY(kv_compact),
                         FSPAD_ENTRY(kv_compact_paged), FSPAD_ENTRY(kv_append), FSPAD_ENTRY(lm_head_accept),
                         FSPAD_ENTRY(feature_sampler), FSPAD_ENTRY(tree_build), FSPAD_ENTRY(draft_expand),
                         FSPAD_ENTRY(verify_step), FSPAD_ENTRY(verify_step_host), FSPAD_ENTRY(rope_qkv),
                         FSPAD_ENTRY(block_plan), FSPAD_ENTRY(kv_write_packed), FSPAD_ENTRY(kv_append_packed),
                         FSPAD_ENTRY(tree_attn_packed), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_pycall", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__pycall() { return PyModule_Create(&module); }
