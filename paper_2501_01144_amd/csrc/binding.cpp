// Python calls of libdfp4 that allocate their results: arguments are unpacked, results and workspaces allocated and the C entry
// point called in one native call.  (paper_2501_01144_amd/dfp4.py; the entry points themselves are include/dfp4.h.)
// What bounds small products is the host: quantize + dfp4_gemm of 32 x 4096 x 4096 keeps the GPU busy for 14 us and took 21 us
// through ctypes structures and torch.empty calls, 13.4 so (a call that allocates its result: 8 to 12 us of host time, 5 to 7 so).
#include <Python.h>
#include <dlfcn.h>

#include <ATen/ATen.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/dfp4.h"

namespace {

PyObject* g_error = nullptr;          // Dfp4Error

#define DFP4_FUNCTIONS(F)                                                                                                  \
    F(dfp4_quantize) F(mxfp4_quantize) F(dfp4_quantize_block) F(dfp4_quantize_native) F(dfp4_dequantize) F(mxfp4_dequantize)  \
    F(dfp4_gemm) F(mxfp4_gemm) F(dfp4_gemm_batched) F(dfp4_gemm_workspace_bytes) F(dfp4_gemm_prepared_bytes)                \
    F(dfp4_gemm_prepare) F(mxfp4_gemm_prepare) F(dfp4_gemm_prepared_workspace_bytes) F(dfp4_gemm_prepared)                  \
    F(mxfp4_gemm_prepared) F(dfp4_native_packed_bytes) F(dfp4_native_pack) F(mxfp4_native_pack)                             \
    F(dfp4_gemm_native_packed) F(mxfp4_gemm_native_packed) F(dfp4_gemm_native_splitk_bytes) F(dfp4_strerror)         \
    F(dfp4_paged_write) F(dfp4_paged_read) F(dfp4_paged_attention_workspace_bytes) F(dfp4_paged_attention) F(dfp4_norm_rope)  \
    F(dfp4_route) F(dfp4_expert_plan_bytes) F(dfp4_expert_plan) F(dfp4_experts_workspace_bytes) F(dfp4_experts_up) F(dfp4_experts_down) F(dfp4_add_norm)
#define DFP4_DECLARE(NAME) decltype(&::NAME) p_##NAME = nullptr;
DFP4_FUNCTIONS(DFP4_DECLARE)
#undef DFP4_DECLARE

struct Failure {};                    // a Python exception is set

[[noreturn]] void fail(PyObject* type, const char* what) {
    PyErr_SetString(type, what);
    throw Failure{};
}

// Other Python threads run while memory is allocated (which may wait for the GPU) and while kernels are enqueued (a full queue waits)
struct Unlocked {
    PyThreadState* state = PyEval_SaveThread();
    ~Unlocked() { PyEval_RestoreThread(state); }
};

// an entry point of the library
template <class F, class... A>
void enqueue(const char* what, F* entry, A... a) {
    int rc;
    {
        Unlocked u;
        rc = entry(a...);
    }
    if (rc == DFP4_OK) return;
    PyErr_Format(g_error, "%s failed: %s (%d)", what, p_dfp4_strerror(rc), rc);
    throw Failure{};
}

const at::Tensor& tensor(PyObject* o) {
    if (!THPVariable_Check(o)) fail(PyExc_TypeError, "a tensor is expected");
    return THPVariable_Unpack(o);
}
int64_t number(PyObject* o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Failure{};
    return v;
}
uint8_t* data(const at::Tensor& t) { return t.numel() > 0 ? static_cast<uint8_t*>(t.data_ptr()) : nullptr; }
uint8_t* data(PyObject* o) { return o == Py_None ? nullptr : data(tensor(o)); }
void* stream() { return c10::hip::getCurrentHIPStream().stream(); }

at::Tensor empty(at::IntArrayRef shape, at::ScalarType type, const at::Device& dev) {
    Unlocked u;
    return at::empty(shape, at::TensorOptions().dtype(type).device(dev));
}
at::Tensor bytes(int64_t n, const at::Device& dev) { return empty({n}, at::kByte, dev); }
at::Tensor bytes(int64_t r, int64_t c, const at::Device& dev) { return empty({r, c}, at::kByte, dev); }
at::Tensor result(at::IntArrayRef shape, bool bf16, const at::Device& dev) { return empty(shape, bf16 ? at::kBFloat16 : at::kFloat, dev); }

int dtype(bool bf16) { return bf16 ? DFP4_BF16 : DFP4_F32; }

// codes, dialect, exponent, rows, K
dfp4_tensor quantized(PyObject* const* a) {
    return dfp4_tensor{data(a[0]), data(a[1]), data(a[2]), number(a[3]), number(a[4])};
}

const at::Tensor& dense(PyObject* o) {
    const at::Tensor& x = tensor(o);
    if (x.scalar_type() != at::kBFloat16 || x.dim() != 2 || !x.is_cuda() || x.stride(1) != 1)
        fail(PyExc_AssertionError, "a bf16 matrix on the device, contiguous along its rows, is expected");
    return x;
}

template <class F>
PyObject* call(Py_ssize_t given, Py_ssize_t wanted, F&& f) {
    if (given != wanted) {
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
        return nullptr;
    }
    try {
        return f();
    } catch (const Failure&) {
    } catch (...) {
        // as torch.empty raises them: an exhausted device is a torch.OutOfMemoryError
        torch::translate_exception_to_python(std::current_exception());
    }
    return nullptr;
}

// quantize(x, block, mx) -> codes, dialect, exponent, rows, K
PyObject* quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 3, [&]() -> PyObject* {
        const at::Tensor& x = dense(a[0]);
        const int64_t block = number(a[1]), rows = x.size(0), K = x.size(1), per = block == 16 ? 16 : 32;
        const bool mx = a[2] == Py_True;
        const at::Device dev = x.device();
        at::Tensor codes = bytes(rows, K / 2, dev), dialect, exponent = bytes(rows, K / per, dev);
        if (!mx) dialect = bytes(rows, K / per, dev);
        const dfp4_tensor q{data(codes), mx ? nullptr : data(dialect), data(exponent), rows, K};
        const int64_t ld = rows > 1 ? x.stride(0) : K;
        if (mx) enqueue("mxfp4_quantize", p_mxfp4_quantize, data(x), rows, K, ld, q, stream());
        else if (block == 32) enqueue("dfp4_quantize", p_dfp4_quantize, data(x), rows, K, ld, q, stream());
        else enqueue("dfp4_quantize_block", p_dfp4_quantize_block, data(x), rows, K, ld, (int)block, q, stream());
        PyObject* d = mx ? Py_NewRef(Py_None) : THPVariable_Wrap(std::move(dialect));
        return Py_BuildValue("NNNLL", THPVariable_Wrap(std::move(codes)), d, THPVariable_Wrap(std::move(exponent)), (long long)rows, (long long)K);
    });
}

// dequantize(codes, dialect, exponent, rows, K, bf16, mx) -> y
PyObject* dequantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 7, [&] {
        const dfp4_tensor q = quantized(a);
        const bool bf16 = a[5] == Py_True, mx = a[6] == Py_True;
        at::Tensor y = result({q.rows, q.K}, bf16, tensor(a[0]).device());
        enqueue(mx ? "mxfp4_dequantize" : "dfp4_dequantize", mx ? p_mxfp4_dequantize : p_dfp4_dequantize, q, data(y), dtype(bf16), q.K, stream());
        return THPVariable_Wrap(std::move(y));
    });
}

// gemm(a's five, w's five, bf16, mx) -> out
PyObject* gemm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 12, [&] {
        const dfp4_tensor A = quantized(a), W = quantized(a + 5);
        const bool bf16 = a[10] == Py_True, mx = a[11] == Py_True;
        const at::Device dev = tensor(a[0]).device();
        at::Tensor out = result({A.rows, W.rows}, bf16, dev), ws;
        const size_t need = p_dfp4_gemm_workspace_bytes(A.rows, W.rows, A.K);
        if (need > 0) ws = bytes((int64_t)need, dev);
        enqueue(mx ? "mxfp4_gemm" : "dfp4_gemm", mx ? p_mxfp4_gemm : p_dfp4_gemm, A, W, data(out), dtype(bf16), W.rows, need > 0 ? data(ws) : nullptr, need,
                stream());
        return THPVariable_Wrap(std::move(out));
    });
}

// gemm_batched(a's five, w's five, batch, M, N, bf16) -> out
PyObject* gemm_batched(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 14, [&] {
        dfp4_tensor A = quantized(a), W = quantized(a + 5);
        const int64_t batch = number(a[10]), M = number(a[11]), N = number(a[12]);
        const bool bf16 = a[13] == Py_True;
        const at::Device dev = tensor(a[0]).device();
        A.rows = M;
        W.rows = N;
        at::Tensor out = result({batch, M, N}, bf16, dev), ws;
        const size_t need = p_dfp4_gemm_workspace_bytes(M, N, A.K) * (size_t)batch;
        if (need > 0) ws = bytes((int64_t)need, dev);
        enqueue("dfp4_gemm_batched", p_dfp4_gemm_batched, A, W, data(out), dtype(bf16), N, batch, M, N, M * N, need > 0 ? data(ws) : nullptr, need,
                stream());
        return THPVariable_Wrap(std::move(out));
    });
}

// gemm_prepare(five, weight, mx) -> buffer, or None where nothing is prepared
PyObject* gemm_prepare(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 7, [&]() -> PyObject* {
        const dfp4_tensor q = quantized(a);
        const int weight = a[5] == Py_True ? 1 : 0;
        const size_t need = p_dfp4_gemm_prepared_bytes(q.rows, q.K, weight);
        if (need == 0) Py_RETURN_NONE;
        at::Tensor buf = bytes((int64_t)need, tensor(a[0]).device());
        enqueue("gemm_prepare", a[6] == Py_True ? p_mxfp4_gemm_prepare : p_dfp4_gemm_prepare, q, weight, data(buf), need, stream());
        return THPVariable_Wrap(std::move(buf));
    });
}

// gemm_prepared(a's five, its buffer, w's five, its buffer, bf16, mx) -> out
PyObject* gemm_prepared(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 14, [&] {
        const dfp4_tensor A = quantized(a), W = quantized(a + 6);
        const bool bf16 = a[12] == Py_True, mx = a[13] == Py_True;
        const at::Device dev = tensor(a[0]).device();
        at::Tensor out = result({A.rows, W.rows}, bf16, dev), ws;
        const size_t need = p_dfp4_gemm_prepared_workspace_bytes(A.rows, W.rows, A.K);
        if (need > 0) ws = bytes((int64_t)need, dev);
        enqueue("gemm_prepared", mx ? p_mxfp4_gemm_prepared : p_dfp4_gemm_prepared, A, data(a[5]), W, data(a[11]), data(out), dtype(bf16), W.rows,
                need > 0 ? data(ws) : nullptr, need, stream());
        return THPVariable_Wrap(std::move(out));
    });
}

// quantize_native(x) -> buffer (x not empty)
PyObject* quantize_native(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 1, [&] {
        const at::Tensor& x = dense(a[0]);
        const int64_t rows = x.size(0), K = x.size(1);
        at::Tensor buf = bytes((int64_t)p_dfp4_native_packed_bytes(rows, K), x.device());
        enqueue("dfp4_quantize_native", p_dfp4_quantize_native, data(x), rows, K, rows > 1 ? x.stride(0) : K, data(buf), (size_t)buf.numel(), stream());
        return THPVariable_Wrap(std::move(buf));
    });
}

// native_pack(five, mx) -> buffer
PyObject* native_pack(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 6, [&] {
        const dfp4_tensor q = quantized(a);
        const int64_t need = (int64_t)p_dfp4_native_packed_bytes(q.rows, q.K);
        at::Tensor buf = bytes(need > 256 ? need : 256, tensor(a[0]).device());
        enqueue("native_pack", a[5] == Py_True ? p_mxfp4_native_pack : p_dfp4_native_pack, q, data(buf), (size_t)buf.numel(), stream());
        return THPVariable_Wrap(std::move(buf));
    });
}

// gemm_native_packed(a's buffer, M, w's buffer, N, K, bf16, mx) -> out
PyObject* gemm_native_packed(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 7, [&] {
        const int64_t M = number(a[1]), N = number(a[3]), K = number(a[4]);
        const bool bf16 = a[5] == Py_True, mx = a[6] == Py_True;
        const at::Device dev = tensor(a[0]).device();
        at::Tensor out = result({M, N}, bf16, dev), ws;
        const size_t need = p_dfp4_gemm_native_splitk_bytes(M, N, K);
        if (need > 0) ws = bytes((int64_t)need, dev);
        enqueue("gemm_native_packed", mx ? p_mxfp4_gemm_native_packed : p_dfp4_gemm_native_packed, data(a[0]), M, data(a[2]), N, K, data(out), dtype(bf16), N,
                need > 0 ? data(ws) : nullptr, need, stream());
        return THPVariable_Wrap(std::move(out));
    });
}

// ---- serving operators.  Caches and batches come as the addresses of their C structures (kvcache.PagedCache, kvcache.PagedBatch keep
// them as long as they live); the rows of this call go into the copy.

double real(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Failure{};
    return v;
}
template <class T>
T structure(PyObject* o) {
    const void* at = PyLong_AsVoidPtr(o);
    if (!at) {
        if (PyErr_Occurred()) throw Failure{};
        fail(PyExc_ValueError, "a cache and a batch are expected");
    }
    return *static_cast<const T*>(at);
}
const at::Tensor& rows3(PyObject* o) {
    const at::Tensor& x = tensor(o);
    if (x.scalar_type() != at::kBFloat16 || x.dim() != 3 || !x.is_cuda() || (x.stride(2) != 1 && x.size(2) != 1))
        fail(PyExc_AssertionError, "bf16 [tokens, heads, head_dim] on the device, contiguous along head_dim, is expected");
    return x;
}
// stride of a dimension (a single token's, or a single head's, is nobody's concern: torch leaves anything there)
int64_t step(const at::Tensor& x, int64_t d) { return x.size(d) > 1 ? x.stride(d) : 0; }
// a contiguous tensor of `n` numbers on the device, or None
template <class T>
const T* numbers(PyObject* o, at::ScalarType type, int64_t n, const char* what) {
    if (o == Py_None) return nullptr;
    const at::Tensor& x = tensor(o);
    if (x.scalar_type() != type || !x.is_cuda() || !x.is_contiguous() || (n >= 0 && x.numel() != n)) fail(PyExc_AssertionError, what);
    return reinterpret_cast<const T*>(data(x));
}

// paged_write(k, v, cache, batch)
PyObject* paged_write(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 4, [&]() -> PyObject* {
        const at::Tensor &k = rows3(a[0]), &v = rows3(a[1]);
        const dfp4_cache cache = structure<dfp4_cache>(a[2]);
        dfp4_batch batch = structure<dfp4_batch>(a[3]);
        batch.tokens = k.size(0);
        if (k.sizes() != v.sizes() || k.size(1) != cache.kv_heads || k.size(2) != cache.head_dim)
            fail(PyExc_AssertionError, "k and v: [tokens, kv_heads, head_dim] of the cache");
        enqueue("dfp4_paged_write", p_dfp4_paged_write, data(k), step(k, 0), step(k, 1), data(v), step(v, 0), step(v, 1), cache, batch, stream());
        Py_RETURN_NONE;
    });
}

// paged_read(cache, batch, tokens, bf16, a tensor on the cache's device) -> k, v
PyObject* paged_read(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 5, [&]() -> PyObject* {
        const dfp4_cache cache = structure<dfp4_cache>(a[0]);
        dfp4_batch batch = structure<dfp4_batch>(a[1]);
        batch.tokens = number(a[2]);
        const bool bf16 = a[3] == Py_True;
        const at::Device dev = tensor(a[4]).device();
        at::Tensor k = result({batch.tokens, cache.kv_heads, cache.head_dim}, bf16, dev), v = result({batch.tokens, cache.kv_heads, cache.head_dim}, bf16, dev);
        enqueue("dfp4_paged_read", p_dfp4_paged_read, cache, batch, data(k), data(v), dtype(bf16), stream());
        return Py_BuildValue("NN", THPVariable_Wrap(std::move(k)), THPVariable_Wrap(std::move(v)));
    });
}

// paged_attention(q, cache, batch, scale, softcap, window, slopes or None, return_lse) -> out or (out, lse)
PyObject* paged_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 8, [&]() -> PyObject* {
        const at::Tensor& q = rows3(a[0]);
        const dfp4_cache cache = structure<dfp4_cache>(a[1]);
        dfp4_batch batch = structure<dfp4_batch>(a[2]);
        batch.tokens = q.size(0);
        const int64_t heads = q.size(1), window = number(a[5]);
        if (q.size(2) != cache.head_dim) fail(PyExc_AssertionError, "q: head_dim of the cache");
        const float* slopes = numbers<float>(a[6], at::kFloat, heads, "slopes: contiguous f32 [heads] on the device");
        const bool with_lse = a[7] == Py_True;
        const at::Device dev = q.device();
        at::Tensor out = result({batch.tokens, heads, cache.head_dim}, true, dev), lse, ws;
        if (with_lse) lse = result({batch.tokens, heads}, false, dev);
        const size_t need = p_dfp4_paged_attention_workspace_bytes(cache, batch, heads, window);
        if (need > 0) ws = bytes((int64_t)need, dev);
        enqueue("dfp4_paged_attention", p_dfp4_paged_attention, data(q), step(q, 0), step(q, 1), heads, cache, batch, (float)real(a[3]), (float)real(a[4]),
                window, slopes, data(out), step(out, 0), step(out, 1), with_lse ? reinterpret_cast<float*>(data(lse)) : nullptr,
                need > 0 ? data(ws) : nullptr, need, stream());
        if (!with_lse) return THPVariable_Wrap(std::move(out));
        return Py_BuildValue("NN", THPVariable_Wrap(std::move(out)), THPVariable_Wrap(std::move(lse)));
    });
}

// norm_rope(q, k or None, positions, inv_freq, q_weight or None, k_weight or None, eps, interleaved) -> q, k
PyObject* norm_rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 8, [&]() -> PyObject* {
        const at::Tensor& q = rows3(a[0]);
        const bool both = a[1] != Py_None;
        const at::Tensor& k = both ? rows3(a[1]) : q;
        const int64_t tokens = q.size(0), dim = q.size(2);
        if (k.size(0) != tokens || k.size(2) != dim) fail(PyExc_AssertionError, "q and k: the same tokens and head_dim");
        const int32_t* positions = numbers<int32_t>(a[2], at::kInt, tokens, "positions: contiguous int32 [tokens] on the device");
        const float* freq = numbers<float>(a[3], at::kFloat, -1, "inv_freq: contiguous f32 [rotary / 2] on the device");
        const float *qw = numbers<float>(a[4], at::kFloat, dim, "q_weight: contiguous f32 [head_dim] on the device"),
                    *kw = numbers<float>(a[5], at::kFloat, dim, "k_weight: contiguous f32 [head_dim] on the device");
        at::Tensor q_out = result(q.sizes(), true, q.device()), k_out;
        if (both) k_out = result(k.sizes(), true, q.device());
        enqueue("dfp4_norm_rope", p_dfp4_norm_rope, data(q), step(q, 0), step(q, 1), q.size(1), both ? data(k) : nullptr, step(k, 0), step(k, 1),
                both ? k.size(1) : 0, tokens, dim, qw, kw, (float)real(a[6]), positions, freq, a[3] == Py_None ? 0 : 2 * tensor(a[3]).numel(),
                a[7] == Py_True ? 1 : 0, data(q_out), both ? data(k_out) : nullptr, stream());
        PyObject* second = both ? THPVariable_Wrap(std::move(k_out)) : Py_NewRef(Py_None);
        return Py_BuildValue("NN", THPVariable_Wrap(std::move(q_out)), second);
    });
}

// ---- operators of a sparse layer

// route(logits, k, sigmoid, bias or None, groups, kept, best, renormalize, scale) -> ids, weights
PyObject* route(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 9, [&]() -> PyObject* {
        const at::Tensor& x = tensor(a[0]);
        const bool bf16 = x.scalar_type() == at::kBFloat16;
        if ((!bf16 && x.scalar_type() != at::kFloat) || x.dim() != 2 || !x.is_cuda() || (x.stride(1) != 1 && x.size(1) != 1))
            fail(PyExc_AssertionError, "logits: f32 or bf16 [tokens, experts] on the device, contiguous along the experts");
        const int64_t tokens = x.size(0), experts = x.size(1), k = number(a[1]);
        const float* bias = numbers<float>(a[3], at::kFloat, experts, "bias: contiguous f32 [experts] on the device");
        const int64_t cols = k >= 1 && k <= experts ? k : 0;              // (others are refused)
        at::Tensor ids = empty({tokens, cols}, at::kInt, x.device()), weights = result({tokens, cols}, false, x.device());
        enqueue("dfp4_route", p_dfp4_route, data(x), dtype(bf16), tokens > 1 ? x.stride(0) : experts, tokens, experts, k, a[2] == Py_True ? DFP4_SIGMOID : DFP4_SOFTMAX, bias,
                number(a[4]), number(a[5]), number(a[6]), a[7] == Py_True ? 1 : 0, (float)real(a[8]), reinterpret_cast<int32_t*>(data(ids)),
                reinterpret_cast<float*>(data(weights)), stream());
        return Py_BuildValue("NN", THPVariable_Wrap(std::move(ids)), THPVariable_Wrap(std::move(weights)));
    });
}

// data, tokens, k, experts
dfp4_plan plan_of(PyObject* const* a) { return dfp4_plan{reinterpret_cast<int32_t*>(data(a[0])), number(a[1]), number(a[2]), number(a[3])}; }
// packed, experts, rows, K, gated
dfp4_experts experts_of(PyObject* const* a) { return dfp4_experts{data(a[0]), number(a[1]), number(a[2]), number(a[3]), a[4] == Py_True ? 1 : 0}; }

// expert_plan(ids, experts) -> data
PyObject* expert_plan(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 2, [&]() -> PyObject* {
        const at::Tensor& ids = tensor(a[0]);
        if (ids.scalar_type() != at::kInt || ids.dim() != 2 || !ids.is_cuda() || !ids.is_contiguous()) fail(PyExc_AssertionError, "ids: contiguous int32 [tokens, k] on the device");
        dfp4_plan p{nullptr, ids.size(0), ids.size(1), number(a[1])};
        at::Tensor buf = empty({(int64_t)(p_dfp4_expert_plan_bytes(p.tokens, p.k, p.experts) / 4)}, at::kInt, ids.device());
        p.data = reinterpret_cast<int32_t*>(data(buf));
        enqueue("dfp4_expert_plan", p_dfp4_expert_plan, reinterpret_cast<const int32_t*>(data(ids)), p, stream());
        return THPVariable_Wrap(std::move(buf));
    });
}

// piece(tensor of one dimension, first, count) -> view
PyObject* piece(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 3, [&]() -> PyObject* { return THPVariable_Wrap(tensor(a[0]).narrow(0, number(a[1]), number(a[2]))); });
}

// experts_up(x, the plan's four, the weights' five) -> h
PyObject* experts_up(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 10, [&]() -> PyObject* {
        const at::Tensor& x = dense(a[0]);
        const dfp4_plan plan = plan_of(a + 1);
        const dfp4_experts w = experts_of(a + 5);
        if (x.size(0) != plan.tokens || x.size(1) != w.K) fail(PyExc_AssertionError, "x: [tokens of the plan, K of the weights]");
        at::Tensor h = result({plan.tokens * plan.k, w.rows}, true, x.device()), ws;
        const size_t need = p_dfp4_experts_workspace_bytes(plan, w);
        if (need > 0) ws = bytes((int64_t)need, x.device());
        enqueue("dfp4_experts_up", p_dfp4_experts_up, data(x), plan.tokens > 1 ? x.stride(0) : w.K, plan, w, data(h), need > 0 ? data(ws) : nullptr, need, stream());
        return THPVariable_Wrap(std::move(h));
    });
}

// experts_down(h, the plan's four, the weights' five, the router's weights, bf16) -> y
PyObject* experts_down(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 12, [&]() -> PyObject* {
        const at::Tensor& h = dense(a[0]);
        const dfp4_plan plan = plan_of(a + 1);
        const dfp4_experts w = experts_of(a + 5);
        if (h.size(0) != plan.tokens * plan.k || h.size(1) != w.K) fail(PyExc_AssertionError, "h: [tokens * k of the plan, K of the weights]");
        if (a[10] == Py_None) fail(PyExc_AssertionError, "weights: contiguous f32 [tokens, k] on the device");
        const float* weights = numbers<float>(a[10], at::kFloat, plan.tokens * plan.k, "weights: contiguous f32 [tokens, k] on the device");
        const bool bf16 = a[11] == Py_True;
        at::Tensor y = result({plan.tokens, w.rows}, bf16, h.device()), ws;
        const size_t need = p_dfp4_experts_workspace_bytes(plan, w);
        if (need > 0) ws = bytes((int64_t)need, h.device());
        enqueue("dfp4_experts_down", p_dfp4_experts_down, data(h), h.size(0) > 1 ? h.stride(0) : w.K, plan, w, weights, data(y), dtype(bf16), need > 0 ? data(ws) : nullptr, need,
                stream());
        return THPVariable_Wrap(std::move(y));
    });
}

// add_norm(y, residual, weight, post_weight or None, gate or None, scale, eps) -> residual, normed
PyObject* add_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 7, [&]() -> PyObject* {
        const at::Tensor &y = dense(a[0]), &r = tensor(a[1]);
        const int64_t tokens = y.size(0), dim = y.size(1);
        const bool bf16 = r.scalar_type() == at::kBFloat16;
        if ((!bf16 && r.scalar_type() != at::kFloat) || r.sizes() != y.sizes() || !r.is_cuda() || r.stride(1) != 1)
            fail(PyExc_AssertionError, "residual: f32 or bf16 [tokens, dim] on the device, contiguous along its rows");
        if (a[2] == Py_None) fail(PyExc_AssertionError, "weight: contiguous f32 [dim] on the device");
        const float *weight = numbers<float>(a[2], at::kFloat, dim, "weight: contiguous f32 [dim] on the device"),
                    *post = numbers<float>(a[3], at::kFloat, dim, "post_weight: contiguous f32 [dim] on the device");
        const uint8_t* gate = nullptr;
        int64_t gate_ld = 0;
        if (a[4] != Py_None) {
            const at::Tensor& g = tensor(a[4]);
            const bool one = g.dim() == 1;
            if (g.scalar_type() != at::kBFloat16 || !g.is_cuda() || (one ? g.size(0) != dim : g.sizes() != y.sizes()) || g.stride(-1) != 1)
                fail(PyExc_AssertionError, "gate: bf16 [dim] or [tokens, dim] on the device, contiguous along its rows");
            gate = data(g);
            gate_ld = one ? 0 : step(g, 0);
        }
        at::Tensor out = result(y.sizes(), bf16, y.device()), normed = result(y.sizes(), true, y.device());
        enqueue("dfp4_add_norm", p_dfp4_add_norm, data(y), step(y, 0), data(r), step(r, 0), dtype(bf16), gate, gate_ld, tokens, dim, post, weight, (float)real(a[5]), (float)real(a[6]),
                data(out), data(normed), stream());
        return Py_BuildValue("NN", THPVariable_Wrap(std::move(out)), THPVariable_Wrap(std::move(normed)));
    });
}

// bind(path of libdfp4.so, exception class)
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 2, [&]() -> PyObject* {
        const char* path = PyUnicode_AsUTF8(a[0]);
        if (!path) throw Failure{};
        void* lib = dlopen(path, RTLD_NOW | RTLD_LOCAL);
        if (!lib) fail(PyExc_OSError, dlerror());
#define DFP4_BIND(NAME)                                                          \
        p_##NAME = reinterpret_cast<decltype(&::NAME)>(dlsym(lib, #NAME));       \
        if (!p_##NAME) fail(PyExc_OSError, "libdfp4.so has no " #NAME);
        DFP4_FUNCTIONS(DFP4_BIND)
#undef DFP4_BIND
        Py_XSETREF(g_error, Py_NewRef(a[1]));
        Py_RETURN_NONE;
    });
}

#define DFP4_METHOD(NAME) {#NAME, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(NAME)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {DFP4_METHOD(bind), DFP4_METHOD(quantize), DFP4_METHOD(dequantize), DFP4_METHOD(gemm), DFP4_METHOD(gemm_batched),
                         DFP4_METHOD(gemm_prepare), DFP4_METHOD(gemm_prepared), DFP4_METHOD(quantize_native), DFP4_METHOD(native_pack),
                         DFP4_METHOD(gemm_native_packed), DFP4_METHOD(paged_write), DFP4_METHOD(paged_read), DFP4_METHOD(paged_attention),
                         DFP4_METHOD(norm_rope), DFP4_METHOD(route), DFP4_METHOD(expert_plan), DFP4_METHOD(piece), DFP4_METHOD(experts_up), DFP4_METHOD(experts_down),
                         DFP4_METHOD(add_norm), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&module); }
