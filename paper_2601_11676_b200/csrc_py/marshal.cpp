// Argument marshalling of the token-step entry points (CPython module _marshal): checks tensors against the shape and
// passes addresses, strides and the current stream on to libhalo.  In Python the same checks cost 8 to 15 us a call,
// several times the smallest kernels; here they cost a few hundred nanoseconds.  Nothing is computed here.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <exception>
#include <type_traits>

#include "halo.h"

namespace {

struct Entry {
    decltype(&halo_paged_kv_append) kv_append;
    decltype(&halo_paged_mha) paged_mha;
    decltype(&halo_norm_glue) norm_glue;
    decltype(&halo_quantize_rows_mx4) quantize;
    decltype(&halo_dequantize_rows_mx4) dequantize;
    decltype(&halo_product_mx4) product;
    decltype(&halo_paged_norm_append) norm_append;
    decltype(&halo_paged_kv_read) kv_read;
    decltype(&halo_paged_mha_f8) paged_mha_f8;
    decltype(&halo_paged_prompt_mha) prompt_mha;
} entry;
bool bound = false;

struct Refused : std::exception {};   // a Python error is set

[[noreturn]] void refuse(const char* what, const char* name, const char* why, PyObject* got = nullptr) {
    if (got && THPVariable_Check(got)) {
        const at::Tensor& t = THPVariable_Unpack(got);
        std::string s = c10::toString(t.scalar_type());
        s += " [";
        for (auto v : t.sizes()) s += std::to_string(v) + ",";
        s += "] strides [";
        for (auto v : t.strides()) s += std::to_string(v) + ",";
        s += "] on " + t.device().str();
        PyErr_Format(PyExc_ValueError, "%s: %s %s; got %s", what, name, why, s.c_str());
    } else {
        PyErr_Format(PyExc_ValueError, "%s: %s %s", what, name, why);
    }
    throw Refused();
}

long long integer(PyObject* o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Refused();
    return v;
}
int small(const char* what, const char* name, PyObject* o) {
    const long long v = integer(o);
    if (v < INT_MIN || v > INT_MAX) refuse(what, name, "is out of range");
    return static_cast<int>(v);
}
double real(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Refused();
    return v;
}
c10::ScalarType type_of(const char* what, int code) {
    if (code == HALO_F32) return c10::kFloat;
    if (code == HALO_BF16) return c10::kBFloat16;
    refuse(what, "the element type", "is unknown");
}
PyObject *paged_shape_type, *norm_shape_type;   // the binding's structures
// A ctypes structure: its bytes.  Compared by type, not by size: other shapes of the library have as many.
template <typename S>
S shape_of(const char* what, PyObject* o) {
    const int is = PyObject_IsInstance(o, std::is_same<S, halo_paged_shape>::value ? paged_shape_type : norm_shape_type);
    if (is < 0) throw Refused();
    if (is == 0) refuse(what, "the shape", "has another type");
    Py_buffer b;
    if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) throw Refused();
    S s;
    const bool ok = b.len == static_cast<Py_ssize_t>(sizeof(S));
    if (ok) memcpy(&s, b.buf, sizeof(S));
    PyBuffer_Release(&b);
    if (!ok) refuse(what, "the shape", "has another size");
    return s;
}

// One call's tensors: all on one device.
struct Call {
    const char* what;
    c10::Device device = c10::Device(c10::kCPU);

    const at::Tensor& tensor(const char* name, PyObject* o) const {
        if (!THPVariable_Check(o)) refuse(what, name, "has to be a tensor");
        return THPVariable_Unpack(o);
    }
    void lead(const char* name, PyObject* o) { device = tensor(name, o).device(); }
    // a dense tensor of `numel` elements (at least, if not exact); None stays
    void* dense(const char* name, PyObject* o, c10::ScalarType type, long long numel, bool exact = true) const {
        if (o == Py_None) return nullptr;
        const at::Tensor& t = tensor(name, o);
        if (t.scalar_type() != type) refuse(what, name, "has another element type", o);
        if (t.device() != device) refuse(what, name, "is on another device", o);
        if (!t.is_contiguous()) refuse(what, name, "has to be contiguous", o);
        if (exact ? t.numel() != numel : t.numel() < numel) refuse(what, name, "has another number of elements than the shape says", o);
        return t.data_ptr();
    }
    // n rows of `width` elements that are dense in themselves: [n][width] or [n][a][b]
    void* rows(const char* name, PyObject* o, c10::ScalarType type, long long n, long long width, long long& stride) const {
        const at::Tensor& t = tensor(name, o);
        if (t.scalar_type() != type) refuse(what, name, "has another element type", o);
        if (t.device() != device) refuse(what, name, "is on another device", o);
        const auto size = t.sizes(), step = t.strides();
        const size_t d = size.size();
        const bool fits = (d == 2 && size[1] == width) || (d == 3 && size[1] * size[2] == width && (size[1] == 1 || step[1] == size[2]));
        if (!fits || size[0] != n || (width > 1 && step[d - 1] != 1)) refuse(what, name, "has to be rows as wide as the shape says, dense in themselves", o);
        stride = n > 1 ? step[0] : width;
        return t.data_ptr();
    }
    // [n_pages][n_kv_heads][page_size][head_dim], dense or one page every page_stride elements
    void* cache(const char* name, PyObject* o, c10::ScalarType type, const halo_paged_shape& s) const {
        const at::Tensor& t = tensor(name, o);
        if (t.scalar_type() != type) refuse(what, name, "has another element type", o);
        if (t.device() != device) refuse(what, name, "is on another device", o);
        const long long row = static_cast<long long>(s.page_size) * s.head_dim, dense = row * s.n_kv_heads;
        const auto size = t.sizes(), step = t.strides();
        bool ok = size.size() == 4 && size[0] == s.n_pages && size[1] == s.n_kv_heads && size[2] == s.page_size && size[3] == s.head_dim;
        if (ok) {
            const long long want = s.page_stride ? s.page_stride : dense;
            ok = (size[3] == 1 || step[3] == 1) && (size[2] == 1 || step[2] == s.head_dim) && (size[1] == 1 || step[1] == row) &&
                 (size[0] == 1 || step[0] == want);
        }
        if (!ok) refuse(what, name, "does not fit the shape", o);
        return t.data_ptr();
    }
    // scale bytes of an 8-bit cache [n_pages][n_kv_heads][page_size], or None
    uint8_t* scales(const char* name, PyObject* o, const halo_paged_shape& s) const {
        return static_cast<uint8_t*>(dense(name, o, c10::kByte, static_cast<long long>(s.n_pages) * s.n_kv_heads * s.page_size));
    }
    cudaStream_t stream(PyObject* o) const {
        if (!device.is_cuda()) refuse(what, "the tensors", "have to be on a GPU");
        if (o == Py_None) return c10::cuda::getCurrentCUDAStream(device.index()).stream();
        PyObject* h = PyObject_GetAttrString(o, "cuda_stream");
        if (!h) throw Refused();
        void* p = PyLong_AsVoidPtr(h);
        Py_DECREF(h);
        if (!p && PyErr_Occurred()) throw Refused();
        return static_cast<cudaStream_t>(p);
    }
};

template <typename F>
PyObject* guarded(Py_ssize_t got, Py_ssize_t want, F f) {
    if (got != want || !bound) {
        PyErr_SetString(PyExc_TypeError, "_marshal: wrong number of arguments, or bind() was not called");
        return nullptr;
    }
    try {
        return PyLong_FromLong(f());
    } catch (const Refused&) {
        return nullptr;
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

PyObject* kv_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 14, [&]() -> halo_status {
        Call c{"halo_paged_kv_append"};
        const auto s = shape_of<halo_paged_shape>(c.what, a[0]);
        const auto type = type_of(c.what, s.dtype);
        c.lead("k", a[2]);
        const at::Tensor &k = c.tensor("k", a[2]), &table = c.tensor("block_table", a[6]);
        if (k.dim() < 1 || table.dim() < 1) refuse(c.what, "k and block_table", "have to have rows");
        const long long n_tok = k.size(0), n_seq = table.size(0);
        if (n_tok > INT_MAX || n_seq > INT_MAX) refuse(c.what, "k", "has too many rows");
        const long long qw = static_cast<long long>(s.n_heads) * s.head_dim, kw = static_cast<long long>(s.n_kv_heads) * s.head_dim;
        long long qs = 0, ks = 0, vs = 0, os = 0;
        void *q = nullptr, *qo = nullptr;
        if ((a[1] == Py_None) != (a[9] == Py_None)) refuse(c.what, "q and q_out", "go together");
        if (a[1] != Py_None) {
            q = c.rows("q", a[1], type, n_tok, qw, qs);
            qo = c.rows("q_out", a[9], type, n_tok, qw, os);
        }
        void* kp = c.rows("k", a[2], type, n_tok, kw, ks);
        void* vp = c.rows("v", a[3], type, n_tok, kw, vs);
        auto* pos = static_cast<const int32_t*>(c.dense("pos", a[4], c10::kInt, n_tok));
        auto* seq = static_cast<const int32_t*>(c.dense("seq_of_tok", a[5], c10::kInt, n_tok));
        auto* tab = static_cast<const int32_t*>(c.dense("block_table", a[6], c10::kInt, n_seq * s.max_pages));
        auto* inv = static_cast<const double*>(c.dense("inv_freq", a[7], c10::kDouble, 0, false));
        const long long pairs = inv ? c.tensor("inv_freq", a[7]).numel() : 0;
        if (pairs > 1 << 20) refuse(c.what, "inv_freq", "is too long", a[7]);
        void* K = c.cache("K_cache", a[10], type, s);
        void* V = c.cache("V_cache", a[11], type, s);
        auto* status = static_cast<uint32_t*>(c.dense("dev_status", a[12], c10::kInt, 1, false));
        const int inter = PyObject_IsTrue(a[8]);
        if (inter < 0) throw Refused();
        const cudaStream_t st = c.stream(a[13]);
        const c10::cuda::CUDAGuard guard(c.device);
        return entry.kv_append(&s, static_cast<int>(n_tok), static_cast<int>(n_seq), q, qs, kp, ks, vp, vs, pos, seq, tab, inv,
                               static_cast<int>(2 * pairs), inter, qo, os, K, V, status, st);
    });
}

PyObject* paged_mha(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 13, [&]() -> halo_status {
        Call c{"halo_paged_mha"};
        const auto s = shape_of<halo_paged_shape>(c.what, a[0]);
        const auto type = type_of(c.what, s.dtype);
        c.lead("q", a[1]);
        const at::Tensor& qt = c.tensor("q", a[1]);
        if (qt.dim() < 1) refuse(c.what, "q", "has to have rows");
        const long long n_seq = qt.size(0), width = static_cast<long long>(s.n_heads) * s.head_dim;
        if (n_seq > INT_MAX) refuse(c.what, "q", "has too many rows");
        long long qs = 0;
        void* q = c.rows("q", a[1], type, n_seq, width, qs);
        void* K = c.cache("K_cache", a[2], type, s);
        void* V = c.cache("V_cache", a[3], type, s);
        auto* tab = static_cast<const int32_t*>(c.dense("block_table", a[4], c10::kInt, n_seq * s.max_pages));
        auto* len = static_cast<const int32_t*>(c.dense("seq_len", a[5], c10::kInt, n_seq));
        const float scale = static_cast<float>(real(a[6]));
        void* out = c.dense("out", a[7], type, n_seq * width);
        void* ws = c.dense("workspace", a[8], c10::kByte, 0, false);
        const size_t ws_bytes = ws ? static_cast<size_t>(c.tensor("workspace", a[8]).numel()) : 0;
        auto* keep = static_cast<const uint8_t*>(c.dense("keep", a[9], c10::kByte, s.n_heads));
        auto* lse = static_cast<float*>(c.dense("lse", a[10], c10::kFloat, n_seq * s.n_heads));
        auto* status = static_cast<uint32_t*>(c.dense("dev_status", a[11], c10::kInt, 1, false));
        const cudaStream_t st = c.stream(a[12]);
        const c10::cuda::CUDAGuard guard(c.device);
        return entry.paged_mha(&s, static_cast<int>(n_seq), q, qs, K, V, tab, len, keep, scale, out, lse, ws, ws_bytes, status, st);
    });
}

// shape, q, k, v, w_q, w_k, eps, pos, seq, table, inv_freq, interleaved, turn_scale, q_out, K, V, K_scale, V_scale, status, stream
PyObject* norm_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 20, [&]() -> halo_status {
        Call c{"halo_paged_norm_append"};
        const auto s = shape_of<halo_paged_shape>(c.what, a[0]);
        const auto type = type_of(c.what, s.dtype);
        c.lead("k", a[2]);
        const at::Tensor &k = c.tensor("k", a[2]), &table = c.tensor("block_table", a[9]);
        if (k.dim() < 1 || table.dim() < 1) refuse(c.what, "k and block_table", "have to have rows");
        const long long n_tok = k.size(0), n_seq = table.size(0);
        if (n_tok > INT_MAX || n_seq > INT_MAX) refuse(c.what, "k", "has too many rows");
        const long long qw = static_cast<long long>(s.n_heads) * s.head_dim, kw = static_cast<long long>(s.n_kv_heads) * s.head_dim;
        long long qs = 0, ks = 0, vs = 0, os = 0;
        void *q = nullptr, *qo = nullptr;
        if ((a[1] == Py_None) != (a[13] == Py_None)) refuse(c.what, "q and q_out", "go together");
        if (a[1] != Py_None) {
            q = c.rows("q", a[1], type, n_tok, qw, qs);
            qo = c.rows("q_out", a[13], type, n_tok, qw, os);
        }
        void* kp = c.rows("k", a[2], type, n_tok, kw, ks);
        void* vp = c.rows("v", a[3], type, n_tok, kw, vs);
        void* wq = c.dense("w_q", a[4], type, s.head_dim);
        void* wk = c.dense("w_k", a[5], type, s.head_dim);
        const float eps = static_cast<float>(real(a[6]));
        auto* pos = static_cast<const int32_t*>(c.dense("pos", a[7], c10::kInt, n_tok));
        auto* seq = static_cast<const int32_t*>(c.dense("seq_of_tok", a[8], c10::kInt, n_tok));
        auto* tab = static_cast<const int32_t*>(c.dense("block_table", a[9], c10::kInt, n_seq * s.max_pages));
        auto* inv = static_cast<const double*>(c.dense("inv_freq", a[10], c10::kDouble, 0, false));
        const long long pairs = inv ? c.tensor("inv_freq", a[10]).numel() : 0;
        if (pairs > 1 << 20) refuse(c.what, "inv_freq", "is too long", a[10]);
        const int inter = PyObject_IsTrue(a[11]);
        if (inter < 0) throw Refused();
        const float turn_scale = static_cast<float>(real(a[12]));
        const auto row = a[16] == Py_None ? type : c10::kByte;
        void* K = c.cache("K_cache", a[14], row, s);
        void* V = c.cache("V_cache", a[15], row, s);
        uint8_t* Ks = c.scales("K_scale", a[16], s);
        uint8_t* Vs = c.scales("V_scale", a[17], s);
        auto* status = static_cast<uint32_t*>(c.dense("dev_status", a[18], c10::kInt, 1, false));
        const cudaStream_t st = c.stream(a[19]);
        const c10::cuda::CUDAGuard guard(c.device);
        return entry.norm_append(&s, static_cast<int>(n_tok), static_cast<int>(n_seq), q, qs, kp, ks, vp, vs, wq, wk, eps, pos, seq, tab,
                                 inv, static_cast<int>(2 * pairs), inter, turn_scale, qo, os, K, V, Ks, Vs, status, st);
    });
}

// shape, pos, seq, table, K, V, k_out, v_out, K_scale, V_scale, status, stream
PyObject* kv_read(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 12, [&]() -> halo_status {
        Call c{"halo_paged_kv_read"};
        const auto s = shape_of<halo_paged_shape>(c.what, a[0]);
        const auto type = type_of(c.what, s.dtype), row = a[8] == Py_None ? type : c10::kByte;
        c.lead("k_out", a[6]);
        const at::Tensor &k = c.tensor("k_out", a[6]), &table = c.tensor("block_table", a[3]);
        if (k.dim() < 1 || table.dim() < 1) refuse(c.what, "k_out and block_table", "have to have rows");
        const long long n_tok = k.size(0), n_seq = table.size(0), kw = static_cast<long long>(s.n_kv_heads) * s.head_dim;
        if (n_tok > INT_MAX || n_seq > INT_MAX) refuse(c.what, "k_out", "has too many rows");
        long long ks = 0, vs = 0;
        auto* pos = static_cast<const int32_t*>(c.dense("pos", a[1], c10::kInt, n_tok));
        auto* seq = static_cast<const int32_t*>(c.dense("seq_of_tok", a[2], c10::kInt, n_tok));
        auto* tab = static_cast<const int32_t*>(c.dense("block_table", a[3], c10::kInt, n_seq * s.max_pages));
        void* K = c.cache("K_cache", a[4], row, s);
        void* V = c.cache("V_cache", a[5], row, s);
        void* ko = c.rows("k_out", a[6], type, n_tok, kw, ks);
        void* vo = c.rows("v_out", a[7], type, n_tok, kw, vs);
        uint8_t* Ks = c.scales("K_scale", a[8], s);
        uint8_t* Vs = c.scales("V_scale", a[9], s);
        auto* status = static_cast<uint32_t*>(c.dense("dev_status", a[10], c10::kInt, 1, false));
        const cudaStream_t st = c.stream(a[11]);
        const c10::cuda::CUDAGuard guard(c.device);
        return entry.kv_read(&s, static_cast<int>(n_tok), static_cast<int>(n_seq), pos, seq, tab, K, V, Ks, Vs, ko, ks, vo, vs, status, st);
    });
}

// shape, q, K, V, K_scale, V_scale, table, seq_len, scale, out, workspace, keep, lse, status, stream
PyObject* paged_mha_f8(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 15, [&]() -> halo_status {
        Call c{"halo_paged_mha_f8"};
        const auto s = shape_of<halo_paged_shape>(c.what, a[0]);
        const auto type = type_of(c.what, s.dtype);
        c.lead("q", a[1]);
        const at::Tensor& qt = c.tensor("q", a[1]);
        if (qt.dim() < 1) refuse(c.what, "q", "has to have rows");
        const long long n_seq = qt.size(0), width = static_cast<long long>(s.n_heads) * s.head_dim;
        if (n_seq > INT_MAX) refuse(c.what, "q", "has too many rows");
        long long qs = 0;
        void* q = c.rows("q", a[1], type, n_seq, width, qs);
        void* K = c.cache("K_cache", a[2], c10::kByte, s);
        void* V = c.cache("V_cache", a[3], c10::kByte, s);
        uint8_t* Ks = c.scales("K_scale", a[4], s);
        uint8_t* Vs = c.scales("V_scale", a[5], s);
        auto* tab = static_cast<const int32_t*>(c.dense("block_table", a[6], c10::kInt, n_seq * s.max_pages));
        auto* len = static_cast<const int32_t*>(c.dense("seq_len", a[7], c10::kInt, n_seq));
        const float scale = static_cast<float>(real(a[8]));
        void* out = c.dense("out", a[9], type, n_seq * width);
        void* ws = c.dense("workspace", a[10], c10::kByte, 0, false);
        const size_t ws_bytes = ws ? static_cast<size_t>(c.tensor("workspace", a[10]).numel()) : 0;
        auto* keep = static_cast<const uint8_t*>(c.dense("keep", a[11], c10::kByte, s.n_heads));
        auto* lse = static_cast<float*>(c.dense("lse", a[12], c10::kFloat, n_seq * s.n_heads));
        auto* status = static_cast<uint32_t*>(c.dense("dev_status", a[13], c10::kInt, 1, false));
        const cudaStream_t st = c.stream(a[14]);
        const c10::cuda::CUDAGuard guard(c.device);
        return entry.paged_mha_f8(&s, static_cast<int>(n_seq), q, qs, K, V, Ks, Vs, tab, len, keep, scale, out, lse, ws, ws_bytes, status, st);
    });
}

// shape, q, q_start, K, V, table, seq_len, scale, out, workspace, K_scale, V_scale, keep, lse, status, stream
PyObject* prompt_mha(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 16, [&]() -> halo_status {
        Call c{"halo_paged_prompt_mha"};
        const auto s = shape_of<halo_paged_shape>(c.what, a[0]);
        const auto type = type_of(c.what, s.dtype), row = a[10] == Py_None ? type : c10::kByte;
        c.lead("q", a[1]);
        const at::Tensor &qt = c.tensor("q", a[1]), &lens = c.tensor("seq_len", a[6]);
        if (qt.dim() < 1) refuse(c.what, "q", "has to have rows");
        const long long n_tok = qt.size(0), n_seq = lens.numel(), width = static_cast<long long>(s.n_heads) * s.head_dim;
        if (n_tok > INT_MAX || n_seq > INT_MAX) refuse(c.what, "q", "has too many rows");
        long long qs = 0;
        void* q = c.rows("q", a[1], type, n_tok, width, qs);
        auto* start = static_cast<const int32_t*>(c.dense("q_start", a[2], c10::kInt, n_seq + 1));
        void* K = c.cache("K_cache", a[3], row, s);
        void* V = c.cache("V_cache", a[4], row, s);
        auto* tab = static_cast<const int32_t*>(c.dense("block_table", a[5], c10::kInt, n_seq * s.max_pages));
        auto* len = static_cast<const int32_t*>(c.dense("seq_len", a[6], c10::kInt, n_seq));
        const float scale = static_cast<float>(real(a[7]));
        void* out = c.dense("out", a[8], type, n_tok * width);
        void* ws = c.dense("workspace", a[9], c10::kByte, 0, false);
        const size_t ws_bytes = ws ? static_cast<size_t>(c.tensor("workspace", a[9]).numel()) : 0;
        uint8_t* Ks = c.scales("K_scale", a[10], s);
        uint8_t* Vs = c.scales("V_scale", a[11], s);
        auto* keep = static_cast<const uint8_t*>(c.dense("keep", a[12], c10::kByte, s.n_heads));
        auto* lse = static_cast<float*>(c.dense("lse", a[13], c10::kFloat, n_tok * s.n_heads));
        auto* status = static_cast<uint32_t*>(c.dense("dev_status", a[14], c10::kInt, 1, false));
        const cudaStream_t st = c.stream(a[15]);
        const c10::cuda::CUDAGuard guard(c.device);
        return entry.prompt_mha(&s, static_cast<int>(n_tok), static_cast<int>(n_seq), q, qs, start, K, V, Ks, Vs, tab, len, keep, scale, out,
                                lse, ws, ws_bytes, status, st);
    });
}

PyObject* norm_glue(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 10, [&]() -> halo_status {
        Call c{"halo_norm_glue"};
        const auto s = shape_of<halo_norm_shape>(c.what, a[0]);
        const auto yt = type_of(c.what, s.ydtype), xt = type_of(c.what, s.xdtype);
        c.lead("h", a[1]);
        const long long d = s.d_model, n_tok = d > 0 ? c.tensor("h", a[1]).numel() / d : 0;
        if (n_tok > INT_MAX) refuse(c.what, "h", "has too many rows");
        auto* h = static_cast<const float*>(c.dense("h", a[1], c10::kFloat, n_tok * d));
        void* y = c.dense("y", a[2], yt, n_tok * d);
        void* post = c.dense("w_post", a[3], xt, d);
        void* gate = nullptr;
        long long gs = 0;
        if (a[4] != Py_None) {
            const at::Tensor& g = c.tensor("gate", a[4]);
            if (g.numel() == d && (g.dim() == 1 || n_tok > 1))
                gate = c.dense("gate", a[4], xt, d);      // one row for all tokens
            else
                gate = c.rows("gate", a[4], xt, n_tok, d, gs);
        }
        const float res = static_cast<float>(real(a[5]));
        void* pre = c.dense("w_pre", a[6], xt, d);
        auto* h_out = static_cast<float*>(c.dense("h_out", a[7], c10::kFloat, n_tok * d));
        void* x_out = c.dense("x_out", a[8], xt, n_tok * d);
        const cudaStream_t st = c.stream(a[9]);
        const c10::cuda::CUDAGuard guard(c.device);
        return entry.norm_glue(&s, static_cast<int>(n_tok), h, y, post, gate, gs, res, pre, h_out, x_out, st);
    });
}

struct Rows {
    void *Q, *S;
};
Rows mx4_rows(const Call& c, long long d, long long n, const char* q_name, PyObject* Q, const char* s_name, PyObject* S) {
    if (d <= 0 || d % 128 != 0) refuse(c.what, "d_model", "has to be a positive multiple of 128");
    if (n <= 0) refuse(c.what, "the number of rows", "has to be positive");
    return {c.dense(q_name, Q, c10::kByte, n * (d / 2)), c.dense(s_name, S, c10::kByte, (n + 127) / 128 * (d / 128) * 512, false)};
}

template <bool BACK>
PyObject* rows_mx4(PyObject*, PyObject* const* a, Py_ssize_t n) {   // d, rows, type, W, Q, scales, stream
    return guarded(n, 7, [&]() -> halo_status {
        Call c{BACK ? "halo_dequantize_rows_mx4" : "halo_quantize_rows_mx4"};
        const int d = small(c.what, "d_model", a[0]), type = small(c.what, "the element type", a[2]);
        const long long rows = integer(a[1]);
        c.lead("W", a[3]);
        const Rows r = mx4_rows(c, d, rows, "Q", a[4], "scales", a[5]);
        void* W = c.dense("W", a[3], type_of(c.what, type), rows * d);
        const cudaStream_t st = c.stream(a[6]);
        const c10::cuda::CUDAGuard guard(c.device);
        return BACK ? entry.dequantize(d, rows, static_cast<halo_dtype>(type), r.Q, r.S, W, st)
                    : entry.quantize(d, rows, static_cast<halo_dtype>(type), W, r.Q, r.S, st);
    });
}

PyObject* product(PyObject*, PyObject* const* a, Py_ssize_t n) {   // d, n_tok, n_rows, Qx, Sx, Qw, Sw, type, y, status, stream
    return guarded(n, 11, [&]() -> halo_status {
        Call c{"halo_product_mx4"};
        const int d = small(c.what, "d_model", a[0]), n_tok = small(c.what, "n_tok", a[1]), n_rows = small(c.what, "n_rows", a[2]);
        const int type = small(c.what, "the element type", a[7]);
        c.lead("y", a[8]);
        const Rows x = mx4_rows(c, d, n_tok, "Qx", a[3], "Sx", a[4]), w = mx4_rows(c, d, n_rows, "Qw", a[5], "Sw", a[6]);
        void* y = c.dense("y", a[8], type_of(c.what, type), static_cast<long long>(n_tok) * n_rows);
        auto* status = static_cast<uint32_t*>(c.dense("dev_status", a[9], c10::kInt, 1, false));
        const cudaStream_t st = c.stream(a[10]);
        const c10::cuda::CUDAGuard guard(c.device);
        return entry.product(d, n_tok, n_rows, x.Q, x.S, w.Q, w.S, static_cast<halo_dtype>(type), y, status, st);
    });
}

PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {   // addresses, in the order of Entry, and the two types of shape
    constexpr int kEntries = 10;
    if (n != kEntries + 2) {
        PyErr_SetString(PyExc_TypeError, "_marshal.bind: ten addresses and two types");
        return nullptr;
    }
    void* p[kEntries];
    for (int i = 0; i < kEntries; ++i) {
        p[i] = PyLong_AsVoidPtr(a[i]);
        if (!p[i]) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "_marshal.bind: no address");
            return nullptr;
        }
    }
    entry.kv_append = reinterpret_cast<decltype(entry.kv_append)>(p[0]);
    entry.paged_mha = reinterpret_cast<decltype(entry.paged_mha)>(p[1]);
    entry.norm_glue = reinterpret_cast<decltype(entry.norm_glue)>(p[2]);
    entry.quantize = reinterpret_cast<decltype(entry.quantize)>(p[3]);
    entry.dequantize = reinterpret_cast<decltype(entry.dequantize)>(p[4]);
    entry.product = reinterpret_cast<decltype(entry.product)>(p[5]);
    entry.norm_append = reinterpret_cast<decltype(entry.norm_append)>(p[6]);
    entry.kv_read = reinterpret_cast<decltype(entry.kv_read)>(p[7]);
    entry.paged_mha_f8 = reinterpret_cast<decltype(entry.paged_mha_f8)>(p[8]);
    entry.prompt_mha = reinterpret_cast<decltype(entry.prompt_mha)>(p[9]);
    Py_INCREF(a[kEntries]);
    Py_INCREF(a[kEntries + 1]);
    paged_shape_type = a[kEntries];
    norm_shape_type = a[kEntries + 1];
    bound = true;
    Py_RETURN_NONE;
}

#define METHOD(name, f) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD("bind", bind),
                         METHOD("kv_append", kv_append),
                         METHOD("paged_mha", paged_mha),
                         METHOD("norm_glue", norm_glue),
                         METHOD("quantize_rows_mx4", rows_mx4<false>),
                         METHOD("dequantize_rows_mx4", rows_mx4<true>),
                         METHOD("product_mx4", product),
                         METHOD("norm_append", norm_append),
                         METHOD("kv_read", kv_read),
                         METHOD("paged_mha_f8", paged_mha_f8),
                         METHOD("prompt_mha", prompt_mha),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

#ifndef MARSHAL_MADE_FOR
#define MARSHAL_MADE_FOR ""
#endif
PyMODINIT_FUNC PyInit__marshal() {
    PyObject* m = PyModule_Create(&module_def);
    if (m && PyModule_AddStringConstant(m, "made_for", MARSHAL_MADE_FOR) != 0) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
