// Argument marshalling of the layer operators for Python: looks at the tensors, makes the outputs, calls the C ABI of
// qil.h on the current stream.  Nothing is computed here.  (The calls of one decoding step are short: with ctypes and the
// tests of a dozen tensors in Python the host took 11 to 14 us a call, several times the device's work.)
// Each function takes its arguments by position and returns its result, or the qil_status as an int where that is not
// QIL_OK; wrong tensors raise ValueError.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <initializer_list>
#include <stdexcept>
#include <string>

#include "qil.h"

namespace {

using at::Tensor;
using Sizes = c10::IntArrayRef;

std::string type_name(c10::ScalarType t) {
    switch (t) {
        case c10::kFloat: return "float32";
        case c10::kBFloat16: return "bfloat16";
        case c10::kHalf: return "float16";
        case c10::kDouble: return "float64";
        case c10::kInt: return "int32";
        case c10::kLong: return "int64";
        case c10::kChar: return "int8";
        case c10::kByte: return "uint8";
        default: return c10::toString(t);
    }
}
std::string shape_name(Sizes s) {
    std::string text = "(";
    for (size_t i = 0; i < s.size(); ++i) text += (i ? ", " : "") + std::to_string(s[i]);
    return text + ")";
}

const Tensor& tensor(PyObject* o, const char* name) {
    if (!THPVariable_Check(o)) throw std::invalid_argument(std::string("qil: ") + name + " is not a tensor");
    return THPVariable_Unpack(o);
}
const Tensor& tensor(PyObject* o, const char* name, int64_t dims) {
    const Tensor& t = tensor(o, name);
    if (t.dim() != dims)
        throw std::invalid_argument(std::string("qil: ") + name + " has shape " + shape_name(t.sizes()) + ", expected " +
                                    std::to_string(dims) + " dimensions");
    return t;
}

void need_type_and_shape(const Tensor& t, const char* name, c10::ScalarType type, Sizes shape) {
    if (t.scalar_type() != type)
        throw std::invalid_argument(std::string("qil: ") + name + " is torch." + type_name(t.scalar_type()) + ", expected " + type_name(type));
    if (t.sizes() != shape)
        throw std::invalid_argument(std::string("qil: ") + name + " has shape " + shape_name(t.sizes()) + ", expected " + shape_name(shape));
}
// address of a contiguous CUDA tensor of this type and shape
void* arg(const Tensor& t, const char* name, c10::ScalarType type, Sizes shape) {
    need_type_and_shape(t, name, type, shape);
    if (!t.is_cuda() || !t.is_contiguous()) throw std::invalid_argument(std::string("qil: ") + name + " has to be a contiguous CUDA tensor");
    return t.data_ptr();
}
// the same for a bf16 matrix whose rows may be part of longer ones
void* arg_rows(const Tensor& t, const char* name, int64_t rows, int64_t cols, long long& stride) {
    need_type_and_shape(t, name, c10::kBFloat16, {rows, cols});
    if (!t.is_cuda() || (cols > 1 && t.stride(1) != 1))
        throw std::invalid_argument(std::string("qil: the rows of ") + name + " have to be contiguous, on a CUDA device");
    stride = rows > 1 ? t.stride(0) : cols;   // (the stride of a single row says nothing)
    return t.data_ptr();
}
int size32(int64_t n) {
    if (n > 0x7FFFFFFF || n < -0x7FFFFFFF) throw std::invalid_argument("qil: a size exceeds 32 bits");
    return (int)n;
}
qil_stream_t stream_of(const Tensor& t) {
    const c10::DeviceIndex dev = t.device().index();
    if (dev != c10::cuda::current_device()) throw std::invalid_argument("qil: the tensors are not on the current device");
    return reinterpret_cast<qil_stream_t>(c10::cuda::getCurrentCUDAStream(dev).stream());
}
// a caller's workspace, or a new one whose first `zeroed` bytes are zero (the rest needs no initialisation)
Tensor workspace_of(PyObject* o, size_t bytes, size_t zeroed, const Tensor& like) {
    if (o == Py_None) {
        const Tensor t = at::detail::empty_cuda({(int64_t)std::max<size_t>(bytes, 16)}, c10::kByte, like.device(), std::nullopt);
        if (zeroed && bytes) t.narrow(0, 0, (int64_t)std::min(zeroed, bytes)).zero_();
        return t;
    }
    const Tensor& t = tensor(o, "workspace");
    if (!t.is_cuda() || !t.is_contiguous()) throw std::invalid_argument("qil: the workspace has to be a contiguous CUDA tensor");
    return t;
}
double real(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw std::runtime_error("");
    return v;
}
long whole(PyObject* o) {
    const long v = PyLong_AsLong(o);
    if (v == -1 && PyErr_Occurred()) throw std::runtime_error("");
    return v;
}
// a new contiguous tensor on x's device (past the dispatcher: half the time of at::empty)
Tensor fresh(const Tensor& x, Sizes shape, c10::ScalarType type) {
    return at::detail::empty_cuda(shape, type, x.device(), std::nullopt);
}
PyObject* wrap(const Tensor& t) { return THPVariable_Wrap(t); }

// every tensor among the arguments has to be on the first one's device (a kernel would take any address)
void need_one_device(PyObject* const* args, std::initializer_list<const char*> names) {
    const Tensor* first = nullptr;
    const char* first_name = nullptr;
    for (const char* name : names) {
        PyObject* o = *args++;
        if (!THPVariable_Check(o)) continue;
        const Tensor& t = THPVariable_Unpack(o);
        if (!first) {
            first = &t;
            first_name = name;
        } else if (t.device() != first->device()) {
            throw std::invalid_argument(std::string("qil: ") + name + " is on " + t.device().str() + ", " + first_name + " on " +
                                        first->device().str());
        }
    }
}

// C++ exceptions end here
template <class F>
PyObject* guarded(PyObject* const* args, Py_ssize_t got, std::initializer_list<const char*> names, F body) {
    if (got != (Py_ssize_t)names.size()) {
        PyErr_Format(PyExc_TypeError, "expected %zu arguments, got %zd", names.size(), got);
        return nullptr;
    }
    try {
        need_one_device(args, names);
        return body();
    } catch (const std::invalid_argument& e) {
        PyErr_SetString(PyExc_ValueError, e.what());
    } catch (const std::exception& e) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, "qil: unknown C++ exception");
    }
    return nullptr;
}

// rmsnorm(x, weight, eps, residual, out, residual_out, a8)
PyObject* rmsnorm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(a, n, {"x", "weight", "eps", "residual", "out", "residual_out", "a8"}, [&]() -> PyObject* {
        const Tensor& x = tensor(a[0], "x", 2);
        const int64_t M = x.size(0), K = x.size(1);
        void* px = arg(x, "x", c10::kBFloat16, {M, K});
        void* pw = arg(tensor(a[1], "weight"), "weight", c10::kBFloat16, {K});
        const double eps = real(a[2]);
        const bool a8 = a[6] == Py_True;
        void *pr = nullptr, *ph = nullptr, *py = nullptr;
        Tensor h, y, codes, scales;
        if (a[3] != Py_None) {
            pr = arg(tensor(a[3], "residual"), "residual", c10::kBFloat16, {M, K});
            h = a[5] == Py_None ? fresh(x, {M, K}, c10::kBFloat16) : tensor(a[5], "residual_out");
            ph = arg(h, "residual_out", c10::kBFloat16, {M, K});
        } else if (a[5] != Py_None) {
            throw std::invalid_argument("qil: residual_out without a residual");
        }
        if (a[4] != Py_None) y = tensor(a[4], "out");
        else if (!a8) y = fresh(x, {M, K}, c10::kBFloat16);
        if (y.defined()) py = arg(y, "out", c10::kBFloat16, {M, K});
        if (a8) {
            codes = fresh(x, {M, K}, c10::kChar);
            scales = fresh(x, {M}, c10::kFloat);
        }
        const qil_status s = qil_rmsnorm(px, pr, pw, ph, py, a8 ? static_cast<int8_t*>(codes.data_ptr()) : nullptr,
                                         a8 ? static_cast<float*>(scales.data_ptr()) : nullptr, size32(M), size32(K), (float)eps, stream_of(x));
        if (s != QIL_OK) return PyLong_FromLong(s);
        if (a8) return h.defined() ? Py_BuildValue("(NNN)", wrap(codes), wrap(scales), wrap(h)) : Py_BuildValue("(NN)", wrap(codes), wrap(scales));
        return h.defined() ? Py_BuildValue("(NN)", wrap(y), wrap(h)) : wrap(y);
    });
}

// the paged cache and the requests: k_cache, v_cache, cu_q, kv_len, block_table
struct Paged {
    int64_t pages, kv_heads, page, dim, seqs, width;
    void *k, *v;
    int *cu, *len, *table;
    explicit Paged(PyObject* const* a) {
        const Tensor &kc = tensor(a[0], "k_cache", 4), &bt = tensor(a[4], "block_table", 2);
        pages = kc.size(0), kv_heads = kc.size(1), page = kc.size(2), dim = kc.size(3);
        seqs = bt.size(0), width = bt.size(1);
        k = arg(kc, "k_cache", c10::kBFloat16, kc.sizes());
        v = arg(tensor(a[1], "v_cache"), "v_cache", c10::kBFloat16, kc.sizes());
        cu = static_cast<int*>(arg(tensor(a[2], "cu_q"), "cu_q", c10::kInt, {seqs + 1}));
        len = static_cast<int*>(arg(tensor(a[3], "kv_len"), "kv_len", c10::kInt, {seqs}));
        table = static_cast<int*>(arg(bt, "block_table", c10::kInt, {seqs, width}));
    }
};

// rope_append(qkv, cos_sin, k_cache, v_cache, cu_q, kv_len, block_table, num_heads, out)
PyObject* rope_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(a, n, {"qkv", "cos_sin", "k_cache", "v_cache", "cu_q", "kv_len", "block_table", "num_heads", "out"}, [&]() -> PyObject* {
        const Tensor &qkv = tensor(a[0], "qkv", 2), &cs = tensor(a[1], "cos_sin", 2);
        const Paged c(a + 2);
        const int64_t heads = whole(a[7]), T = qkv.size(0);
        void* pq = arg(qkv, "qkv", c10::kBFloat16, {T, (heads + 2 * c.kv_heads) * c.dim});
        void* pcs = arg(cs, "cos_sin", c10::kFloat, {cs.size(0), c.dim});
        const Tensor out = a[8] == Py_None ? fresh(qkv, {T, heads, c.dim}, c10::kBFloat16) : tensor(a[8], "out");
        void* po = arg(out, "out", c10::kBFloat16, {T, heads, c.dim});
        const qil_status s = qil_rope_append(pq, static_cast<float*>(pcs), po, c.k, c.v, c.cu, c.len, c.table, size32(T), size32(c.seqs),
                                             size32(heads), size32(c.kv_heads), size32(c.dim), size32(c.page), size32(c.pages),
                                             size32(c.width), size32(cs.size(0)), stream_of(qkv));
        return s != QIL_OK ? PyLong_FromLong(s) : wrap(out);
    });
}

// attn_paged(q, k_cache, v_cache, cu_q, kv_len, block_table, max_q_len, max_kv_len, scale, out, workspace)
PyObject* attn_paged(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(a, n, {"q", "k_cache", "v_cache", "cu_q", "kv_len", "block_table", "max_q_len", "max_kv_len", "scale", "out",
                          "workspace"}, [&]() -> PyObject* {
        const Tensor& q = tensor(a[0], "q", 3);
        const Paged c(a + 1);
        const int64_t T = q.size(0), heads = q.size(1);
        void* pq = arg(q, "q", c10::kBFloat16, {T, heads, c.dim});
        const int max_q = size32(whole(a[6])), max_kv = size32(whole(a[7]));
        const double scale = a[8] == Py_None ? 1.0 / std::sqrt((double)c.dim) : real(a[8]);
        const Tensor out = a[9] == Py_None ? fresh(q, {T, heads, c.dim}, c10::kBFloat16) : tensor(a[9], "out");
        void* po = arg(out, "out", c10::kBFloat16, {T, heads, c.dim});
        const size_t bytes = a[10] != Py_None ? 0 : qil_attn_paged_workspace_size(size32(T), size32(c.seqs), size32(heads), size32(c.kv_heads),
                                                                                  size32(c.dim), max_q, max_kv);
        const Tensor ws = workspace_of(a[10], bytes, QIL_ATTN_PAGED_ZEROED_BYTES, q);
        const qil_status s = qil_attn_paged(pq, c.k, c.v, po, c.cu, c.len, c.table, size32(T), size32(c.seqs), size32(heads),
                                            size32(c.kv_heads), size32(c.dim), size32(c.page), size32(c.pages), size32(c.width), max_q, max_kv,
                                            (float)scale, ws.data_ptr(), ws.nbytes(), stream_of(q));
        return s != QIL_OK ? PyLong_FromLong(s) : wrap(out);
    });
}

// the quantised cache and the requests: k, v, k_scale, v_scale, cu, kv_len, block_table; the codes' type says how many bits
struct PagedQ {
    int64_t pages, kv_heads, page, dim, seqs, width;
    int bits;
    void *k, *v, *ks, *vs;
    int *cu, *len, *table;
    explicit PagedQ(PyObject* const* a) {
        const Tensor &kc = tensor(a[0], "k", 4), &bt = tensor(a[6], "block_table", 2);
        const c10::ScalarType type = kc.scalar_type();
        if (type != c10::kChar && type != c10::kInt)
            throw std::invalid_argument("qil: k is torch." + type_name(type) + ", expected int8 (8 bits) or int32 (4 bits)");
        bits = type == c10::kChar ? 8 : 4;
        pages = kc.size(0), kv_heads = kc.size(1), page = kc.size(2), dim = kc.size(3) * (bits == 8 ? 1 : 8);
        seqs = bt.size(0), width = bt.size(1);
        const int64_t of[4] = {pages, kv_heads, page, 2};
        const Sizes scales(of, bits == 8 ? 3 : 4);
        k = arg(kc, "k", type, kc.sizes());
        v = arg(tensor(a[1], "v"), "v", type, kc.sizes());
        ks = arg(tensor(a[2], "k_scale"), "k_scale", c10::kBFloat16, scales);
        vs = arg(tensor(a[3], "v_scale"), "v_scale", c10::kBFloat16, scales);
        cu = static_cast<int*>(arg(tensor(a[4], "cu_q"), "cu_q", c10::kInt, {seqs + 1}));
        len = static_cast<int*>(arg(tensor(a[5], "kv_len"), "kv_len", c10::kInt, {seqs}));
        table = static_cast<int*>(arg(bt, "block_table", c10::kInt, {seqs, width}));
    }
};

// rope_append_q(qkv, cos_sin, k, v, k_scale, v_scale, cu_q, kv_len, block_table, num_heads, out)
PyObject* rope_append_q(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(a, n, {"qkv", "cos_sin", "k", "v", "k_scale", "v_scale", "cu_q", "kv_len", "block_table", "num_heads", "out"}, [&]() -> PyObject* {
        const Tensor &qkv = tensor(a[0], "qkv", 2), &cs = tensor(a[1], "cos_sin", 2);
        const PagedQ c(a + 2);
        const int64_t heads = whole(a[9]), T = qkv.size(0);
        void* pq = arg(qkv, "qkv", c10::kBFloat16, {T, (heads + 2 * c.kv_heads) * c.dim});
        void* pcs = arg(cs, "cos_sin", c10::kFloat, {cs.size(0), c.dim});
        const Tensor out = a[10] == Py_None ? fresh(qkv, {T, heads, c.dim}, c10::kBFloat16) : tensor(a[10], "out");
        void* po = arg(out, "out", c10::kBFloat16, {T, heads, c.dim});
        const qil_status s = qil_rope_append_q(pq, static_cast<float*>(pcs), po, c.k, c.v, c.ks, c.vs, c.bits, c.cu, c.len, c.table, size32(T),
                                               size32(c.seqs), size32(heads), size32(c.kv_heads), size32(c.dim), size32(c.page),
                                               size32(c.pages), size32(c.width), size32(cs.size(0)), stream_of(qkv));
        return s != QIL_OK ? PyLong_FromLong(s) : wrap(out);
    });
}

// kv_read_q(k, v, k_scale, v_scale, cu_q, kv_len, block_table, total_rows, k_out, v_out)
PyObject* kv_read_q(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(a, n, {"k", "v", "k_scale", "v_scale", "cu_q", "kv_len", "block_table", "total_rows", "k_out", "v_out"}, [&]() -> PyObject* {
        const PagedQ c(a);
        const int64_t T = whole(a[7]);
        if (T <= 0) return PyLong_FromLong(QIL_ERR_SHAPE);
        const Tensor& kc = tensor(a[0], "k");
        const Tensor k = a[8] == Py_None ? fresh(kc, {T, c.kv_heads, c.dim}, c10::kBFloat16) : tensor(a[8], "k_out");
        const Tensor v = a[9] == Py_None ? fresh(kc, {T, c.kv_heads, c.dim}, c10::kBFloat16) : tensor(a[9], "v_out");
        void* pk = arg(k, "k_out", c10::kBFloat16, {T, c.kv_heads, c.dim});
        void* pv = arg(v, "v_out", c10::kBFloat16, {T, c.kv_heads, c.dim});
        const qil_status s = qil_kv_read_q(c.k, c.v, c.ks, c.vs, c.bits, pk, pv, c.cu, c.len, c.table, size32(T), size32(c.seqs),
                                           size32(c.kv_heads), size32(c.dim), size32(c.page), size32(c.pages), size32(c.width), stream_of(kc));
        return s != QIL_OK ? PyLong_FromLong(s) : Py_BuildValue("(NN)", wrap(k), wrap(v));
    });
}

// attn_paged_q(q, k, v, k_scale, v_scale, cu_q, kv_len, block_table, max_q_len, max_kv_len, scale, out, workspace)
PyObject* attn_paged_q(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(a, n, {"q", "k", "v", "k_scale", "v_scale", "cu_q", "kv_len", "block_table", "max_q_len", "max_kv_len", "scale", "out",
                          "workspace"}, [&]() -> PyObject* {
        const Tensor& q = tensor(a[0], "q", 3);
        const PagedQ c(a + 1);
        const int64_t T = q.size(0), heads = q.size(1);
        void* pq = arg(q, "q", c10::kBFloat16, {T, heads, c.dim});
        const int max_q = size32(whole(a[8])), max_kv = size32(whole(a[9]));
        const double scale = a[10] == Py_None ? 1.0 / std::sqrt((double)c.dim) : real(a[10]);
        const Tensor out = a[11] == Py_None ? fresh(q, {T, heads, c.dim}, c10::kBFloat16) : tensor(a[11], "out");
        void* po = arg(out, "out", c10::kBFloat16, {T, heads, c.dim});
        const size_t bytes = a[12] != Py_None ? 0 : qil_attn_paged_q_workspace_size(size32(T), size32(c.seqs), size32(heads), size32(c.kv_heads),
                                                                                    size32(c.dim), c.bits, max_q, max_kv);
        const Tensor ws = workspace_of(a[12], bytes, QIL_ATTN_PAGED_ZEROED_BYTES, q);
        const qil_status s = qil_attn_paged_q(pq, c.k, c.v, c.ks, c.vs, c.bits, po, c.cu, c.len, c.table, size32(T), size32(c.seqs),
                                              size32(heads), size32(c.kv_heads), size32(c.dim), size32(c.page), size32(c.pages),
                                              size32(c.width), max_q, max_kv, (float)scale, ws.data_ptr(), ws.nbytes(), stream_of(q));
        return s != QIL_OK ? PyLong_FromLong(s) : wrap(out);
    });
}

// sample(logits, u, temperature, top_k, top_p, min_p, out)
PyObject* sample(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(a, n, {"logits", "u", "temperature", "top_k", "top_p", "min_p", "out"}, [&]() -> PyObject* {
        const Tensor& x = tensor(a[0], "logits", 2);
        const int64_t B = x.size(0), V = x.size(1);
        const c10::ScalarType type = x.scalar_type();
        if (type != c10::kFloat && type != c10::kBFloat16 && type != c10::kHalf)
            throw std::invalid_argument("qil: logits is torch." + type_name(type) + ", expected float32, bfloat16 or float16");
        if (!x.is_cuda() || (V > 1 && x.stride(1) != 1)) throw std::invalid_argument("qil: the rows of logits have to be contiguous, on a CUDA device");
        const long long ld = B > 1 ? x.stride(0) : V;   // (the stride of a single row says nothing)
        const auto optional = [&](PyObject* o, const char* name, c10::ScalarType t) { return o == Py_None ? nullptr : arg(tensor(o, name), name, t, {B}); };
        float* u = static_cast<float*>(arg(tensor(a[1], "u"), "u", c10::kFloat, {B}));
        float* t = static_cast<float*>(arg(tensor(a[2], "temperature"), "temperature", c10::kFloat, {B}));
        int* k = static_cast<int*>(optional(a[3], "top_k", c10::kInt));
        float* p = static_cast<float*>(optional(a[4], "top_p", c10::kFloat));
        float* m = static_cast<float*>(optional(a[5], "min_p", c10::kFloat));
        const Tensor out = a[6] == Py_None ? fresh(x, {B}, c10::kInt) : tensor(a[6], "out");
        int* po = static_cast<int*>(arg(out, "out", c10::kInt, {B}));
        const qil_status s = qil_sample(x.data_ptr(), type == c10::kFloat ? QIL_F32 : type == c10::kBFloat16 ? QIL_BF16 : QIL_F16, ld, u, t, k, p, m,
                                        po, size32(B), size32(V), stream_of(x));
        return s != QIL_OK ? PyLong_FromLong(s) : wrap(out);
    });
}

// lora_batch_add(x, a, b, y, cu_q, adapter, scales, out, workspace)
PyObject* lora_batch_add(PyObject*, PyObject* const* p, Py_ssize_t n) {
    return guarded(p, n, {"x", "a", "b", "y", "cu_q", "adapter", "scales", "out", "workspace"}, [&]() -> PyObject* {
        const Tensor &x = tensor(p[0], "x", 2), &b = tensor(p[2], "b", 3), &y = tensor(p[3], "y", 2);
        const int64_t M = x.size(0), K = x.size(1), count = b.size(0), N = b.size(1), r = b.size(2);
        const Tensor& adapter = tensor(p[5], "adapter", 1);
        const int64_t seqs = adapter.size(0);
        long long ldx, ldy, ldo;
        void* px = arg_rows(x, "x", M, K, ldx);
        void* pa = arg(tensor(p[1], "a"), "a", c10::kBFloat16, {count, r, K});
        void* pb = arg(b, "b", c10::kBFloat16, {count, N, r});
        void* py = arg_rows(y, "y", M, N, ldy);
        const Tensor& out = p[7] == Py_None ? y : tensor(p[7], "out");
        void* po = arg_rows(out, "out", M, N, ldo);
        int* cu = static_cast<int*>(arg(tensor(p[4], "cu_q"), "cu_q", c10::kInt, {seqs + 1}));
        int* ad = static_cast<int*>(arg(adapter, "adapter", c10::kInt, {seqs}));
        float* sc = static_cast<float*>(arg(tensor(p[6], "scales"), "scales", c10::kFloat, {count}));
        const size_t bytes = p[8] != Py_None ? 0 : qil_lora_batch_workspace_size(size32(M), size32(seqs), size32(r));
        const Tensor ws = workspace_of(p[8], bytes, 0, x);
        const qil_status s = qil_lora_batch_add(px, pa, pb, py, po, cu, ad, sc, size32(M), size32(N), size32(K), size32(r), size32(seqs),
                                                size32(count), ldx, ldy, ldo, ws.data_ptr(), ws.nbytes(), stream_of(x));
        return s != QIL_OK ? PyLong_FromLong(s) : wrap(out);
    });
}

#define QIL_METHOD(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {QIL_METHOD(rmsnorm), QIL_METHOD(rope_append), QIL_METHOD(attn_paged), QIL_METHOD(lora_batch_add),
                         QIL_METHOD(rope_append_q), QIL_METHOD(kv_read_q), QIL_METHOD(attn_paged_q),
                         QIL_METHOD(sample),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_qil_torch", "Marshalling of the qil layer operators.", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__qil_torch() { return PyModule_Create(&module); }
