// The serving-step calls of the Python binding, from tensors to the C ABI: an
// extension module over libtl.  A serving step makes a few such calls per layer
// and token, each a few microseconds long on the GPU; taking shapes, types and
// addresses from a dozen tensors in Python took 4 - 10 us of the host's time,
// more than the kernels of a single token.
//
// A function returns the C entry point's status, or None for whatever is not a
// call with every tensor in hand, of the right type and size, without gaps, on
// the current device and stream: the caller then goes through its own checks,
// which say what is wrong or make the missing outputs.
#include <Python.h>

#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/tl.h"

namespace {

struct NotPlain {};

void need(bool ok) {
    if (!ok) throw NotPlain{};
}

const at::Tensor& tensor(PyObject* x, int device) {
    need(THPVariable_Check(x));
    const at::Tensor& t = THPVariable_Unpack(x);
    need(t.is_cuda() && t.get_device() == device && t.layout() == at::kStrided);
    return t;
}

// the address of a tensor without gaps
void* flat(const at::Tensor& t, at::ScalarType type, int64_t numel) {
    need(t.scalar_type() == type && t.numel() == numel && t.is_contiguous());
    return t.data_ptr();
}

int32_t* ints(const at::Tensor& t, int64_t numel) {
    need(t.scalar_type() == at::kInt || t.scalar_type() == at::kUInt32);
    return static_cast<int32_t*>(flat(t, t.scalar_type(), numel));
}

// [n, heads * size] or [n, heads, size] rows, each without gaps; elements between rows
int64_t rows(const at::Tensor& t, int64_t heads, int64_t size) {
    const auto shape = t.sizes(), stride = t.strides();
    const int64_t width = heads * size;
    need((t.dim() == 2 && shape[1] == width && stride[1] == 1) ||
         (t.dim() == 3 && shape[1] * shape[2] == width && stride[2] == 1 && (shape[1] == 1 || stride[1] == shape[2])));
    return shape[0] > 1 ? stride[0] : width;
}

int64_t heads_of(const at::Tensor& t, int64_t size) {
    need(t.dim() == 2 || t.dim() == 3);
    return t.dim() == 3 ? t.size(1) : t.size(1) / size;
}

int64_t number(PyObject* x) {
    const long long v = PyLong_AsLongLong(x);
    need(v != -1 || !PyErr_Occurred());
    return v;
}

int32_t number32(PyObject* x) {
    const int64_t v = number(x);
    need(v >= INT32_MIN && v <= INT32_MAX);
    return int32_t(v);
}

// a ctypes structure of the C ABI
template <typename T>
T structure(PyObject* x) {
    Py_buffer view;
    need(PyObject_GetBuffer(x, &view, PyBUF_SIMPLE) == 0);
    T out;
    const bool fits = view.len == Py_ssize_t(sizeof out);
    if (fits) memcpy(&out, view.buf, sizeof out);
    PyBuffer_Release(&view);
    need(fits);
    return out;
}

struct Attribute {
    PyObject* x;
    Attribute(PyObject* of, const char* name) : x(PyObject_GetAttrString(of, name)) { need(x != nullptr); }
    ~Attribute() { Py_XDECREF(x); }
    Attribute(const Attribute&) = delete;
};

// positions (int32 [axes][n]), inv_freq (float32), sections and interleaved of a binding's Rope
tl_rope rope_of(PyObject* x, int device, int64_t n) {
    const Attribute positions(x, "positions"), inv_freq(x, "inv_freq"), sections(x, "sections"), interleaved(x, "interleaved");
    tl_rope r{};
    need(PyTuple_Check(sections.x) && PyTuple_GET_SIZE(sections.x) >= 1 && PyTuple_GET_SIZE(sections.x) <= 3);
    r.axes = int32_t(PyTuple_GET_SIZE(sections.x));
    for (int i = 0; i < r.axes; ++i) r.sections[i] = number32(PyTuple_GET_ITEM(sections.x, i));
    r.positions = ints(tensor(positions.x, device), n * r.axes);
    const at::Tensor& f = tensor(inv_freq.x, device);
    r.inv_freq = static_cast<const float*>(flat(f, at::kFloat, f.numel()));
    need(f.numel() <= 4096);
    r.rot_dim = int32_t(2 * f.numel());
    const int truth = PyObject_IsTrue(interleaved.x);
    need(truth >= 0);
    r.interleaved = truth;
    return r;
}

int32_t in_dtype(const at::Tensor& t) {
    need(t.scalar_type() == at::kFloat || t.scalar_type() == at::kBFloat16);
    return t.scalar_type() == at::kFloat ? TL_IN_F32 : TL_IN_BF16;
}

struct Where {
    int device;
    void* stream;
    explicit Where(PyObject* given) {
        need(given == Py_None);
        const c10::hip::HIPStream s = c10::hip::getCurrentHIPStream();
        device = s.device_index();
        stream = s.stream();
    }
};

// q, k, v, cache descriptor, slots, rope, q_out, stream
int kv_append(PyObject* const* a) {
    const Where here(a[7]);
    const auto cache = structure<tl_kv_cache>(a[3]);
    const bool has_q = a[0] != Py_None, has_k = a[1] != Py_None;
    need((has_q || has_k) && has_k == (a[2] != Py_None) && cache.head_dim > 0);
    const at::Tensor& some = tensor(has_q ? a[0] : a[1], here.device);
    const int64_t n = some.dim() ? some.size(0) : 0, D = cache.head_dim;
    const void* at[3] = {nullptr, nullptr, nullptr};
    int64_t ld[3] = {0, 0, 0}, heads = 0;
    for (int i = 0; i < 3; ++i) {
        if (a[i] == Py_None) continue;
        const at::Tensor& x = tensor(a[i], here.device);
        need(x.dim() >= 2 && x.scalar_type() == some.scalar_type() && x.size(0) == n);
        if (i == 0) heads = heads_of(x, D);
        ld[i] = rows(x, i == 0 ? heads : cache.kv_heads, D);
        at[i] = x.data_ptr();
    }
    const int32_t* slots = has_k ? ints(tensor(a[4], here.device), n) : nullptr;
    tl_rope rope;
    if (a[5] != Py_None) rope = rope_of(a[5], here.device, n);
    void* out = has_q ? flat(tensor(a[6], here.device), at::kBFloat16, n * heads * D) : nullptr;
    need(has_q || a[6] == Py_None);
    need(heads <= INT32_MAX);
    const int32_t in = in_dtype(some);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = tl_kv_append(at[0], ld[0], at[1], ld[1], at[2], ld[2], in, n, int32_t(heads), slots, a[5] != Py_None ? &rope : nullptr, out, &cache, here.stream);
    Py_END_ALLOW_THREADS
    return rc;
}

// cache descriptor, slots, k_out, v_out, stream
int kv_read(PyObject* const* a) {
    const Where here(a[4]);
    const auto cache = structure<tl_kv_cache>(a[0]);
    const at::Tensor& s = tensor(a[1], here.device);
    const int64_t n = s.numel();
    const int32_t* slots = ints(s, n);
    void* out[2];
    for (int i = 0; i < 2; ++i) out[i] = flat(tensor(a[2 + i], here.device), at::kBFloat16, n * cache.kv_heads * cache.head_dim);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = tl_kv_read(&cache, slots, n, out[0], out[1], here.stream);
    Py_END_ALLOW_THREADS
    return rc;
}

// cache descriptor, page_table, starts, path, counts, stream
int kv_keep(PyObject* const* a) {
    const Where here(a[5]);
    const auto cache = structure<tl_kv_cache>(a[0]);
    const at::Tensor& table = tensor(a[1], here.device);
    const at::Tensor& path = tensor(a[3], here.device);
    need(table.dim() == 2 && path.dim() == 2 && path.size(0) == table.size(0) && table.size(0) <= INT32_MAX);
    const int64_t B = table.size(0), pages = table.size(1), most = path.size(1);
    const int32_t *t = ints(table, B * pages), *starts = ints(tensor(a[2], here.device), B), *p = ints(path, B * most),
                  *counts = ints(tensor(a[4], here.device), B);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = tl_kv_keep(&cache, t, pages, starts, p, most, counts, int32_t(B), here.stream);
    Py_END_ALLOW_THREADS
    return rc;
}

// int32 lists of n entries each, none of them missing
int32_t* list(PyObject* x, int device, int64_t n) { return ints(tensor(x, device), n); }

// pages descriptor, rows, lens, missing, stream
int kv_grow(PyObject* const* a) {
    const Where here(a[4]);
    const auto pages = structure<tl_kv_pages>(a[0]);
    const int64_t n = tensor(a[1], here.device).numel();
    need(n <= INT32_MAX);
    const int32_t *rows = list(a[1], here.device, n), *lens = list(a[2], here.device, n);
    int32_t* missing = list(a[3], here.device, 1);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = tl_kv_grow(&pages, rows, lens, int32_t(n), missing, here.stream);
    Py_END_ALLOW_THREADS
    return rc;
}

// pages descriptor, rows, lens, stream
int kv_free(PyObject* const* a) {
    const Where here(a[3]);
    const auto pages = structure<tl_kv_pages>(a[0]);
    const int64_t n = tensor(a[1], here.device).numel();
    need(n <= INT32_MAX);
    const int32_t *rows = list(a[1], here.device, n), *lens = a[2] == Py_None ? nullptr : list(a[2], here.device, n);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = tl_kv_free(&pages, rows, lens, int32_t(n), here.stream);
    Py_END_ALLOW_THREADS
    return rc;
}

// pages descriptor, parents, children, lens, src, dst, tokens, count, stream
int kv_fork(PyObject* const* a) {
    const Where here(a[8]);
    const auto pages = structure<tl_kv_pages>(a[0]);
    const int64_t n = tensor(a[2], here.device).numel();
    need(n <= INT32_MAX);
    int32_t* lists[6];
    for (int i = 0; i < 6; ++i) lists[i] = list(a[1 + i], here.device, n);
    int32_t* count = list(a[7], here.device, 2);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = tl_kv_fork(&pages, lists[0], lists[1], lists[2], int32_t(n), lists[3], lists[4], lists[5], count, here.stream);
    Py_END_ALLOW_THREADS
    return rc;
}

// pages descriptor, max_moves, src, dst, count, stream
int kv_compact(PyObject* const* a) {
    const Where here(a[5]);
    const auto pages = structure<tl_kv_pages>(a[0]);
    const int64_t n = number(a[1]);
    int32_t *src = list(a[2], here.device, n), *dst = list(a[3], here.device, n), *count = list(a[4], here.device, 2);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = tl_kv_compact(&pages, n, src, dst, count, here.stream);
    Py_END_ALLOW_THREADS
    return rc;
}

// cache descriptor, src, dst, tokens, count, stream
int kv_copy(PyObject* const* a) {
    const Where here(a[5]);
    const auto cache = structure<tl_kv_cache>(a[0]);
    const int64_t n = tensor(a[1], here.device).numel();
    const int32_t *src = list(a[1], here.device, n), *dst = list(a[2], here.device, n);
    const int32_t* tokens = a[3] == Py_None ? nullptr : list(a[3], here.device, n);
    const int32_t* count = nullptr;
    if (a[4] != Py_None) {
        const int64_t size = tensor(a[4], here.device).numel();
        need(size >= 1);
        count = list(a[4], here.device, size);
    }
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = tl_kv_copy(&cache, src, dst, tokens, count, n, here.stream);
    Py_END_ALLOW_THREADS
    return rc;
}

// q, cache descriptor, page_table, lens, q_offsets, max_q, max_len, scale, mask, out, stream
int attention(PyObject* const* a) {
    const Where here(a[10]);
    const auto cache = structure<tl_kv_cache>(a[1]);
    const at::Tensor& q = tensor(a[0], here.device);
    const at::Tensor& table = tensor(a[2], here.device);
    need(cache.head_dim > 0 && q.scalar_type() == at::kBFloat16 && table.dim() == 2 && table.size(0) <= INT32_MAX);
    const int64_t D = cache.head_dim, heads = heads_of(q, D), total = q.size(0), B = table.size(0), pages = table.size(1);
    need(heads <= INT32_MAX);
    const int64_t ld = rows(q, heads, D);
    const int32_t *t = ints(table, B * pages), *lens = ints(tensor(a[3], here.device), B), *offsets = ints(tensor(a[4], here.device), B + 1);
    const int64_t max_q = number(a[5]), max_len = number(a[6]);
    const double scale = PyFloat_AsDouble(a[7]);
    need(scale != -1.0 || !PyErr_Occurred());
    const uint32_t* mask = nullptr;
    int64_t words = 0;
    if (a[8] != Py_None) {
        const at::Tensor& m = tensor(a[8], here.device);
        need(m.dim() == 2 && m.size(0) == total && m.size(1) <= INT32_MAX);
        words = m.size(1);
        mask = reinterpret_cast<const uint32_t*>(ints(m, total * words));
    }
    void* out = flat(tensor(a[9], here.device), at::kBFloat16, total * heads * D);
    const void* from = q.data_ptr();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = tl_attn(from, ld, &cache, t, pages, lens, offsets, mask, int32_t(words), int32_t(B), total, max_q, max_len, int32_t(heads), float(scale), out, here.stream);
    Py_END_ALLOW_THREADS
    return rc;
}

// logits, node_offsets, parents, tokens, temperature, uniform, noise, max_nodes, draft, path, counts, next, stream
int verify(PyObject* const* a) {
    const Where here(a[12]);
    const at::Tensor& z = tensor(a[0], here.device);
    const at::Tensor& heat = tensor(a[4], here.device);
    need(z.dim() == 2 && heat.numel() <= INT32_MAX);
    const int64_t total = z.size(0), vocab = z.size(1), B = heat.numel();
    const int32_t max_nodes = number32(a[7]);
    const void* logits = flat(z, z.scalar_type(), total * vocab);
    const int32_t *offsets = ints(tensor(a[1], here.device), B + 1), *parents = ints(tensor(a[2], here.device), total),
                  *tokens = ints(tensor(a[3], here.device), total);
    const float* temperature = static_cast<const float*>(flat(heat, at::kFloat, B));
    const float* uniform = static_cast<const float*>(flat(tensor(a[5], here.device), at::kFloat, total));
    const float* noise = static_cast<const float*>(flat(tensor(a[6], here.device), at::kFloat, B * vocab));
    const void* draft = nullptr;
    const int32_t logits_type = in_dtype(z);
    int32_t draft_type = TL_IN_F32;
    if (a[8] != Py_None) {
        const at::Tensor& d = tensor(a[8], here.device);
        need(d.dim() == 2 && d.size(0) == total);
        draft = flat(d, d.scalar_type(), total * vocab);
        draft_type = in_dtype(d);
    }
    int32_t *path = ints(tensor(a[9], here.device), B * max_nodes), *counts = ints(tensor(a[10], here.device), B),
            *next = ints(tensor(a[11], here.device), B);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = tl_verify(logits, logits_type, vocab, offsets, parents, tokens, int32_t(B), total, max_nodes, draft, draft_type, temperature, uniform, noise, path, counts, next, here.stream);
    Py_END_ALLOW_THREADS
    return rc;
}

template <int (*F)(PyObject* const*), int COUNT>
PyObject* call(PyObject*, PyObject* const* args, Py_ssize_t count) {
    if (count != COUNT) return PyErr_Format(PyExc_TypeError, "%d arguments are needed", COUNT);
    try {
        return PyLong_FromLong(F(args));
    } catch (...) {     // also a tensor without storage, or no device: the caller's own checks name it
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

#define FUNCTION(name, count) \
    { #name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&call<name, count>)), METH_FASTCALL, nullptr }
PyMethodDef functions[] = {FUNCTION(kv_append, 8), FUNCTION(kv_read, 5), FUNCTION(kv_keep, 6), FUNCTION(kv_grow, 5), FUNCTION(kv_free, 4),
                           FUNCTION(kv_fork, 9), FUNCTION(kv_compact, 6), FUNCTION(kv_copy, 6), FUNCTION(attention, 11), FUNCTION(verify, 13), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tl_torch", nullptr, -1, functions, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tl_torch() { return PyModule_Create(&module); }
