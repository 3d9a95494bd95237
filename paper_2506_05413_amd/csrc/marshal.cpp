// Argument marshalling of the per-token calls in native code: torch tensors in, the C ABI of include/ called
// on the current stream, tensors out.  No computation here.
//
// Why: a decode step's kernels run 5 - 10 us each, and marshalling through Python and ctypes cost 8.5 - 15 us per call
// (3 us of it torch.cuda.current_stream(), 1.7 us per torch.empty, 5.4 us for the fill kernel of a zeroed tile buffer),
// so the host, not the GPU, set the pace of everything below about 300 tokens.  Here a call costs the launch
// (~3.8 us per kernel) and about a microsecond.
//
// Every function takes positional arguments (binding.py has the signatures and their defaults) and returns its
// outputs, or the status as an int where the library refused the call.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/hip/EmptyTensor.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/smoothrot.h"
#include "../../include/smoothrot_attention.h"

#include <cmath>
#include <exception>

namespace {

struct Raised {};                                        // a Python exception is set

[[noreturn]] void value_error(const char *format, const char *a, const char *b = "")
{
    PyErr_Format(PyExc_ValueError, format, a, b);
    throw Raised();
}

const at::Tensor &tensor(PyObject *o, const char *name)
{
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "%s must be a tensor", name);
        throw Raised();
    }
    return THPVariable_Unpack(o);
}

// a device tensor of the given type, contiguous along its last dimension
const at::Tensor &device_tensor(PyObject *o, at::ScalarType type, const char *name)
{
    const at::Tensor &t = tensor(o, name);
    if (!t.is_cuda()) value_error("%s must be a device tensor", name);
    if (t.scalar_type() != type) value_error("%s must have dtype torch.%s", name, type == at::kHalf ? "float16" : type == at::kByte ? "uint8" : "float32");
    if ((t.dim() == 2 && t.stride(1) != 1) || (t.dim() == 1 && t.numel() > 1 && t.stride(0) != 1))
        value_error("%s must be contiguous along its last dimension", name);
    return t;
}
const at::Tensor &matrix(PyObject *o, at::ScalarType type, const char *name)
{
    const at::Tensor &t = device_tensor(o, type, name);
    if (t.dim() != 2) value_error("%s must have two dimensions", name);
    return t;
}

// Addresses are taken before the lock is released: data_ptr() throws for a tensor without memory of its own (inside vmap, ..).
void *pointer(PyObject *o, const char *name) { return o == Py_None ? nullptr : tensor(o, name).data_ptr(); }
float *floats(PyObject *o, const char *name) { return static_cast<float *>(pointer(o, name)); }
float *floats(const at::Tensor &t) { return static_cast<float *>(t.data_ptr()); }
uint8_t *bytes(const at::Tensor &t) { return static_cast<uint8_t *>(t.data_ptr()); }
int64_t integer(PyObject *o)
{
    const int64_t v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Raised();
    return v;
}
float real(PyObject *o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Raised();
    return (float)v;
}
bool truth(PyObject *o)
{
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw Raised();
    return v != 0;
}
int64_t row_stride(const at::Tensor &t) { return t.size(0) > 1 ? t.stride(0) : t.size(1); }

at::Tensor empty(at::IntArrayRef shape, at::ScalarType type, const at::Tensor &like)
{
    return at::detail::empty_cuda(shape, type, like.device(), std::nullopt);
}
// the caller's tensor, or a new one
at::Tensor output(PyObject *o, const char *name, at::IntArrayRef shape, at::ScalarType type, const at::Tensor &like)
{
    return o == Py_None ? empty(shape, type, like) : tensor(o, name);
}
void *stream() { return c10::hip::getCurrentHIPStream().stream(); }

PyObject *pair(const at::Tensor &a, const at::Tensor &b) { return Py_BuildValue("(NN)", THPVariable_Wrap(a), THPVariable_Wrap(b)); }

// calls into the library without holding the interpreter's lock (the library does not throw)
template <typename F> int released(F f)
{
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = f();
    Py_END_ALLOW_THREADS
    return status;
}

template <PyObject *(*F)(PyObject *const *), int N> PyObject *entry(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != N) {
        PyErr_Format(PyExc_TypeError, "%d arguments expected, %zd given", N, n);
        return nullptr;
    }
    try {
        return F(args);
    } catch (const Raised &) {
    } catch (...) {                                      // as torch raises them: out of memory, bad index, ..
        torch::translate_exception_to_python(std::current_exception());
    }
    return nullptr;
}

// X, inv_s, clip, Xq, x_scale
PyObject *fwht_quant_act(PyObject *const *a)
{
    const at::Tensor &X = matrix(a[0], at::kHalf, "X");
    const int64_t M = X.size(0), K = X.size(1);
    const at::Tensor Xq = output(a[3], "Xq", {M, K / 2}, at::kByte, X), xs = output(a[4], "x_scale", {M}, at::kFloat, X);
    const float clip = real(a[2]);
    const float *inv = floats(a[1], "inv_s");
    const void *x = X.data_ptr();
    uint8_t *q = bytes(Xq);
    float *scale = floats(xs);
    const int64_t ldx = row_stride(X);
    void *st = stream();
    const int status = released([&] { return sr_fwht_quant_act(x, M, K, ldx, inv, clip, q, scale, st); });
    return status ? PyLong_FromLong(status) : pair(Xq, xs);
}

// X, n_heads, across, inv_s, clip, Xq, x_scale
PyObject *fwht_quant_act_heads(PyObject *const *a)
{
    const at::Tensor &X = matrix(a[0], at::kHalf, "X");
    const int64_t M = X.size(0), K = X.size(1), heads = integer(a[1]);
    const int across = truth(a[2]);
    const at::Tensor Xq = output(a[5], "Xq", {M, K / 2}, at::kByte, X), xs = output(a[6], "x_scale", {M}, at::kFloat, X);
    const float clip = real(a[4]);
    const float *inv = floats(a[3], "inv_s");
    const void *x = X.data_ptr();
    uint8_t *q = bytes(Xq);
    float *scale = floats(xs);
    const int64_t ldx = row_stride(X);
    void *st = stream();
    const int status = released([&] { return sr_fwht_quant_act_heads(x, M, K, ldx, heads, across, inv, clip, q, scale, st); });
    return status ? PyLong_FromLong(status) : pair(Xq, xs);
}

// a buffer whose bytes the library may read as the next operand: (address, bytes)
void warm_region(PyObject *o, const void *&p, size_t &size)
{
    p = nullptr;
    size = 0;
    if (o == Py_None) return;
    const at::Tensor &t = tensor(o, "warm");
    if (!t.is_cuda() || !t.is_contiguous()) value_error("%s must be a contiguous device tensor", "warm");
    p = t.data_ptr();
    size = t.nbytes();
}

int64_t tile_bytes(int64_t M, int64_t K)
{
    const size_t n = sr_f6_tiles_bytes(M, K);
    return n > 16 ? (int64_t)n : 16;
}

// X, inv_s, clip, X6, x_scale, warm
PyObject *fwht_quant_act_f6(PyObject *const *a)
{
    const at::Tensor &X = matrix(a[0], at::kHalf, "X");
    const int64_t M = X.size(0), K = X.size(1);
    const at::Tensor X6 = output(a[3], "X6", {tile_bytes(M, K)}, at::kByte, X), xs = output(a[4], "x_scale", {M}, at::kFloat, X);
    const float clip = real(a[2]);
    const float *inv = floats(a[1], "inv_s");
    const void *warm;
    size_t warm_bytes;
    warm_region(a[5], warm, warm_bytes);
    const void *x = X.data_ptr();
    uint8_t *q = bytes(X6);
    float *scale = floats(xs);
    const int64_t ldx = row_stride(X);
    void *st = stream();
    const int status = released([&] { return sr_fwht_quant_act_f6_warm(x, M, K, ldx, inv, clip, q, scale, warm, warm_bytes, st); });
    return status ? PyLong_FromLong(status) : pair(X6, xs);
}

// G, U, inv_s, clip, Xq or X6, x_scale, tiles
PyObject *swiglu_fwht_quant_act(PyObject *const *a)
{
    const at::Tensor &G = matrix(a[0], at::kHalf, "G"), &U = matrix(a[1], at::kHalf, "U");
    const int64_t M = U.size(0), K = U.size(1);
    if (G.size(0) != M || G.size(1) != K) value_error("%s must have the same shape", "G and U");
    const bool tiles = truth(a[6]);
    const at::Tensor Q = tiles ? output(a[4], "X6", {tile_bytes(M, K)}, at::kByte, U) : output(a[4], "Xq", {M, K / 2}, at::kByte, U);
    const at::Tensor xs = output(a[5], "x_scale", {M}, at::kFloat, U);
    const float clip = real(a[3]);
    const float *inv = floats(a[2], "inv_s");
    const void *g = G.data_ptr(), *u = U.data_ptr();
    uint8_t *q = bytes(Q);
    float *scale = floats(xs);
    const int64_t ldg = row_stride(G), ldu = row_stride(U);
    void *st = stream();
    const auto f = tiles ? sr_swiglu_fwht_quant_act_f6 : sr_swiglu_fwht_quant_act;
    const int status = released([&] { return f(g, u, M, K, ldg, ldu, inv, clip, q, scale, st); });
    return status ? PyLong_FromLong(status) : pair(Q, xs);
}

// Xq, x_scale, Wq, w_scale, out_dtype, Y, workspace
PyObject *w4a4_gemm(PyObject *const *a)
{
    const at::Tensor &Xq = matrix(a[0], at::kByte, "Xq"), &Wq = matrix(a[2], at::kByte, "Wq");
    const int64_t M = Xq.size(0), Kb = Xq.size(1), N = Wq.size(0);
    if (Wq.size(1) != Kb) value_error("%s disagree on K", "Xq and Wq");
    const int type = (int)integer(a[4]);
    const at::Tensor Y = output(a[5], "Y", {M, N}, type == SR_F16 ? at::kHalf : at::kInt, Xq);
    const float *xs = floats(a[1], "x_scale"), *ws = floats(a[3], "w_scale");
    at::Tensor work;
    if (a[6] != Py_None) work = tensor(a[6], "workspace");
    else if (const size_t need = sr_gemm_workspace_bytes(M, N, 2 * Kb)) work = empty({(int64_t)need}, at::kByte, Xq);
    const int64_t ldy = M > 1 ? Y.stride(0) : N;
    const uint8_t *x = bytes(Xq), *w = bytes(Wq);
    void *y = Y.data_ptr(), *scratch = work.defined() ? work.data_ptr() : nullptr, *st = stream();
    const size_t scratch_bytes = work.defined() ? (size_t)work.numel() : 0;
    const int status = released([&] { return sr_w4a4_gemm(x, xs, w, ws, M, N, 2 * Kb, y, ldy, type, scratch, scratch_bytes, st); });
    return status ? PyLong_FromLong(status) : THPVariable_Wrap(Y);
}

// X6, x_scale, W6, w_scale, M, N, K, out_dtype, Y, warm
PyObject *w4a4_gemm_f6(PyObject *const *a)
{
    const at::Tensor &X6 = device_tensor(a[0], at::kByte, "X6"), &W6 = device_tensor(a[2], at::kByte, "W6");
    const int64_t M = integer(a[4]), N = integer(a[5]), K = integer(a[6]);
    if ((size_t)X6.numel() < sr_f6_tiles_bytes(M, K) || (size_t)W6.numel() < sr_f6_tiles_bytes(N, K))
        value_error("%s are smaller than sr_f6_tiles_bytes says", "tile buffers");
    const int type = (int)integer(a[7]);
    const at::Tensor Y = output(a[8], "Y", {M, N}, type == SR_F16 ? at::kHalf : at::kInt, X6);
    const float *xs = floats(a[1], "x_scale"), *ws = floats(a[3], "w_scale");
    const void *warm;
    size_t warm_bytes;
    warm_region(a[9], warm, warm_bytes);
    const int64_t ldy = M > 1 ? Y.stride(0) : N;
    const uint8_t *x = bytes(X6), *w = bytes(W6);
    void *y = Y.data_ptr(), *st = stream();
    const int status = released([&] { return sr_w4a4_gemm_f6_warm(x, xs, w, ws, M, N, K, y, ldy, type, warm, warm_bytes, nullptr, 0, st); });
    return status ? PyLong_FromLong(status) : THPVariable_Wrap(Y);
}

// X, inv_s, Wq, w_scale, clip, Y, Xq_out, x_scale_out, workspace
PyObject *w4a4_linear_decode(PyObject *const *a)
{
    const at::Tensor &X = matrix(a[0], at::kHalf, "X"), &Wq = matrix(a[2], at::kByte, "Wq");
    const int64_t M = X.size(0), K = X.size(1), N = Wq.size(0);
    if (Wq.size(1) * 2 != K) value_error("%s disagree on K", "X and Wq");
    const at::Tensor Y = output(a[5], "Y", {M, N}, at::kHalf, X);
    const float *inv = floats(a[1], "inv_s"), *ws = floats(a[3], "w_scale");
    uint8_t *xq = static_cast<uint8_t *>(pointer(a[6], "Xq_out"));
    float *xs = floats(a[7], "x_scale_out");
    const float clip = real(a[4]);
    at::Tensor work;
    if (a[8] != Py_None) work = tensor(a[8], "workspace");
    else if (const size_t need = sr_linear_decode_workspace_bytes(M, K)) work = empty({(int64_t)need}, at::kByte, X);
    const int64_t ldx = row_stride(X), ldy = M > 1 ? Y.stride(0) : N;
    const void *x = X.data_ptr();
    const uint8_t *w = bytes(Wq);
    void *y = Y.data_ptr(), *scratch = work.defined() ? work.data_ptr() : nullptr, *st = stream();
    const size_t scratch_bytes = work.defined() ? (size_t)work.numel() : 0;
    const int status = released([&] {
        return sr_w4a4_linear_decode(x, M, K, ldx, inv, clip, w, ws, N, y, ldy, xq, xs, scratch, scratch_bytes, st);
    });
    return status ? PyLong_FromLong(status) : THPVariable_Wrap(Y);
}

// X, group, clip, Q, scale, zero
PyObject *kv_quant_asym(PyObject *const *a)
{
    const at::Tensor &X = matrix(a[0], at::kHalf, "X");
    const int64_t rows = X.size(0), D = X.size(1), group = integer(a[1]);
    if (group <= 0) return PyLong_FromLong(SR_ERR_ARG);
    const int64_t groups = D / group > 1 ? D / group : 1;
    const at::Tensor Q = output(a[3], "Q", {rows, D / 2}, at::kByte, X), scale = output(a[4], "scale", {rows, groups}, at::kFloat, X),
                     zero = output(a[5], "zero", {rows, groups}, at::kFloat, X);
    const float clip = real(a[2]);
    const void *x = X.data_ptr();
    uint8_t *q = bytes(Q);
    float *scales = floats(scale), *zeros = floats(zero);
    const int64_t ldx = row_stride(X);
    void *st = stream();
    const int status = released([&] { return sr_kv_quant_asym(x, rows, D, ldx, group, clip, q, scales, zeros, st); });
    return status ? PyLong_FromLong(status)
                  : Py_BuildValue("(NNN)", THPVariable_Wrap(Q), THPVariable_Wrap(scale), THPVariable_Wrap(zero));
}

// ---- paged cache and attention: every tensor on the device that is current, sizes that follow from each other checked here ----

const at::Tensor &here(const at::Tensor &t, const char *name)
{
    if (t.device().index() != c10::hip::current_device()) value_error("%s is not on the current device", name);
    return t;
}
// rows of heads, [tokens, columns]
const at::Tensor &rows_of(PyObject *o, const char *name, int64_t tokens, int64_t columns)
{
    const at::Tensor &t = here(matrix(o, at::kHalf, name), name);
    if ((tokens >= 0 && t.size(0) != tokens) || (columns >= 0 && t.size(1) != columns)) value_error("%s has the wrong shape", name);
    return t;
}
at::Tensor rows_out(PyObject *o, const char *name, int64_t tokens, int64_t columns, const at::Tensor &like)
{
    return o == Py_None ? empty({tokens, columns}, at::kHalf, like) : rows_of(o, name, tokens, columns);
}
// a vector of whole numbers, [n] (n < 0: any)
const at::Tensor &indices(PyObject *o, const char *name, at::ScalarType type, int64_t n)
{
    const at::Tensor &t = tensor(o, name);
    if (!t.is_cuda()) value_error("%s must be a device tensor", name);
    here(t, name);
    if (t.scalar_type() != type) value_error("%s must have dtype torch.%s", name, type == at::kInt ? "int32" : "int64");
    if (t.dim() != 1 || (n >= 0 && t.size(0) != n) || (t.numel() > 1 && t.stride(0) != 1)) value_error("%s has the wrong shape", name);
    return t;
}
template <typename T> T *at_of(const at::Tensor &t) { return static_cast<T *>(t.data_ptr()); }

// (K, V, K_params, V_params): [pages, heads, page, head_dim] fp16, or uint8 with half as many columns and params [.., 2]
sr_kv_cache cache_of(PyObject *o)
{
    if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 4) {
        PyErr_SetString(PyExc_TypeError, "cache must be a tuple (K, V, K_params, V_params)");
        throw Raised();
    }
    sr_kv_cache c = {};
    const at::Tensor &K = tensor(PyTuple_GET_ITEM(o, 0), "cache K"), &V = tensor(PyTuple_GET_ITEM(o, 1), "cache V");
    const bool i4 = K.scalar_type() == at::kByte;
    if (!K.is_cuda() || !V.is_cuda()) value_error("%s must be device tensors", "cache K and V");
    if (!i4 && K.scalar_type() != at::kHalf) value_error("%s must have dtype torch.float16 or torch.uint8", "cache K");
    if (V.scalar_type() != K.scalar_type() || K.dim() != 4 || V.sizes() != K.sizes()) value_error("%s must have four dimensions and agree", "cache K and V");
    if (!here(K, "cache K").is_contiguous() || !here(V, "cache V").is_contiguous()) value_error("%s must be contiguous", "cache K and V");
    c.K = K.data_ptr(), c.V = V.data_ptr();
    c.n_pages = K.size(0), c.n_kv_heads = K.size(1), c.page_size = K.size(2), c.head_dim = i4 ? 2 * K.size(3) : K.size(3);
    c.type = i4 ? SR_KV_I4 : SR_KV_F16;
    for (int side = 0; side < 2; ++side) {
        PyObject *p = PyTuple_GET_ITEM(o, 2 + side);
        if (!i4) {
            if (p != Py_None) value_error("%s goes with 4-bit codes only", side ? "cache V_params" : "cache K_params");
            continue;
        }
        const char *name = side ? "cache V_params" : "cache K_params";
        const at::Tensor &t = here(device_tensor(p, at::kFloat, name), name);
        if (t.dim() != 4 || t.size(0) != c.n_pages || t.size(1) != c.n_kv_heads || t.size(2) != c.page_size || t.size(3) != 2 || !t.is_contiguous())
            value_error("%s has the wrong shape", name);
        (side ? c.V_params : c.K_params) = floats(t);
    }
    return c;
}

// Q, K, V, positions, slots, cos_sin, cache, hadamard, pairs, clip, Q_out, K_out
PyObject *rope_kv_append(PyObject *const *a)
{
    const sr_kv_cache c = cache_of(a[6]);
    const at::Tensor &K = rows_of(a[1], "K", -1, c.n_kv_heads * c.head_dim);
    const int64_t T = K.size(0);
    const at::Tensor &V = rows_of(a[2], "V", T, K.size(1));
    const bool any_q = a[0] != Py_None;
    at::Tensor Q, Qo, Ko;
    int64_t heads = 0;
    if (any_q) {
        Q = rows_of(a[0], "Q", T, -1);
        if (c.head_dim <= 0 || Q.size(1) == 0 || Q.size(1) % c.head_dim) value_error("%s is not made of heads of the cache's size", "Q");
        heads = Q.size(1) / c.head_dim;
        Qo = rows_out(a[10], "Q_out", T, Q.size(1), Q);
    }
    if (a[11] != Py_None) Ko = rows_of(a[11], "K_out", T, K.size(1));
    const int64_t *slots = at_of<int64_t>(indices(a[4], "slots", at::kLong, T));
    const float *table = nullptr;
    const int32_t *positions = nullptr;
    int64_t max_pos = 0;
    if (a[5] != Py_None) {
        const at::Tensor &t = here(matrix(a[5], at::kFloat, "cos_sin"), "cos_sin");
        // (one without a row has no address, which would read as "no rotation")
        if (t.size(0) < 1 || t.size(1) != c.head_dim || !t.is_contiguous()) value_error("%s has the wrong shape", "cos_sin");
        table = floats(t), max_pos = t.size(0);
        positions = at_of<int32_t>(indices(a[3], "positions", at::kInt, T));
    }
    const int flags = (truth(a[8]) ? SR_ROPE_PAIRS : 0) | (truth(a[7]) ? SR_ROPE_HADAMARD : 0);
    const float clip = real(a[9]);
    const void *q = any_q ? Q.data_ptr() : nullptr, *k = K.data_ptr(), *v = V.data_ptr();
    void *qo = any_q ? Qo.data_ptr() : nullptr, *ko = Ko.defined() ? Ko.data_ptr() : nullptr, *st = stream();
    const int64_t ldq = any_q ? row_stride(Q) : 0, ldqo = any_q ? row_stride(Qo) : 0, ldk = row_stride(K), ldv = row_stride(V),
                  ldko = Ko.defined() ? row_stride(Ko) : 0;
    const int status = released([&] {
        return sr_rope_kv_append(q, ldq, k, ldk, v, ldv, T, heads, positions, slots, table, max_pos, flags, clip, &c, qo, ldqo, ko, ldko, st);
    });
    if (status) return PyLong_FromLong(status);
    if (any_q) return THPVariable_Wrap(Qo);
    Py_RETURN_NONE;
}

// slots, cache, K_out, V_out
PyObject *kv_gather(PyObject *const *a)
{
    const sr_kv_cache c = cache_of(a[1]);
    const at::Tensor &S = indices(a[0], "slots", at::kLong, -1);
    const int64_t T = S.size(0), columns = c.n_kv_heads * c.head_dim;
    const at::Tensor Ko = rows_out(a[2], "K_out", T, columns, S), Vo = rows_out(a[3], "V_out", T, columns, S);
    const int64_t *slots = at_of<int64_t>(S);
    void *k = Ko.data_ptr(), *v = Vo.data_ptr(), *st = stream();
    const int64_t ldk = row_stride(Ko), ldv = row_stride(Vo);
    const int status = released([&] { return sr_kv_gather(slots, T, &c, k, ldk, v, ldv, st); });
    return status ? PyLong_FromLong(status) : pair(Ko, Vo);
}

// Q, cache, page_table, seq_lens, scale (None: 1 / sqrt(head_dim)), O, workspace
PyObject *attn_decode(PyObject *const *a)
{
    const sr_kv_cache c = cache_of(a[1]);
    const at::Tensor &Q = rows_of(a[0], "Q", -1, -1);
    const int64_t B = Q.size(0);
    if (c.head_dim <= 0 || Q.size(1) == 0 || Q.size(1) % c.head_dim) value_error("%s is not made of heads of the cache's size", "Q");
    const int64_t heads = Q.size(1) / c.head_dim;
    const at::Tensor &table = tensor(a[2], "page_table");
    if (!table.is_cuda()) value_error("%s must be a device tensor", "page_table");
    if (here(table, "page_table").scalar_type() != at::kInt) value_error("%s must have dtype torch.int32", "page_table");
    if (table.dim() != 2 || table.size(0) != B || (table.size(1) > 1 && table.stride(1) != 1)) value_error("%s has the wrong shape", "page_table");
    const int64_t pages = table.size(1), ld_table = B > 1 ? table.stride(0) : pages;
    const int32_t *lens = at_of<int32_t>(indices(a[3], "seq_lens", at::kInt, B)), *entries = at_of<int32_t>(table);
    const float scale = a[4] == Py_None ? 1.f / std::sqrt((float)c.head_dim) : real(a[4]);
    const at::Tensor O = rows_out(a[5], "O", B, Q.size(1), Q);
    at::Tensor work;
    if (a[6] != Py_None) {
        work = here(tensor(a[6], "workspace"), "workspace");
        if (!work.is_contiguous()) value_error("%s must be contiguous", "workspace");
    } else if (const size_t need = sr_attn_decode_workspace_bytes(B, heads, c.n_kv_heads, c.head_dim, pages, c.page_size, c.type)) {
        work = empty({(int64_t)need}, at::kByte, Q);
    }
    const void *q = Q.data_ptr();
    void *o = O.data_ptr(), *scratch = work.defined() ? work.data_ptr() : nullptr, *st = stream();
    const size_t scratch_bytes = work.defined() ? work.nbytes() : 0;
    const int64_t ldq = row_stride(Q), ldo = row_stride(O);
    const int status = released([&] {
        return sr_attn_decode(q, ldq, B, heads, &c, entries, pages, ld_table, lens, scale, o, ldo, scratch, scratch_bytes, st);
    });
    return status ? PyLong_FromLong(status) : THPVariable_Wrap(O);
}

// Q, K, V, cu_q, cu_k, head_dim, causal, scale (None: 1 / sqrt(head_dim)), O
PyObject *attn_prefill(PyObject *const *a)
{
    const int64_t d = integer(a[5]);
    if (d <= 0) return PyLong_FromLong(SR_ERR_ARG);
    const at::Tensor &Q = rows_of(a[0], "Q", -1, -1), &K = rows_of(a[1], "K", -1, -1), &V = rows_of(a[2], "V", K.size(0), K.size(1));
    if (Q.size(1) == 0 || Q.size(1) % d || K.size(1) == 0 || K.size(1) % d) value_error("%s are not made of heads of head_dim", "Q and K");
    const at::Tensor &cq = indices(a[3], "cu_q", at::kInt, -1);
    if (cq.size(0) < 1) value_error("%s has the wrong shape", "cu_q");
    const int64_t n = cq.size(0) - 1;
    const at::Tensor &ck = indices(a[4], "cu_k", at::kInt, n + 1);
    const int causal = truth(a[6]);
    const float scale = a[7] == Py_None ? 1.f / std::sqrt((float)d) : real(a[7]);
    const at::Tensor O = rows_out(a[8], "O", Q.size(0), Q.size(1), Q);
    const void *q = Q.data_ptr(), *k = K.data_ptr(), *v = V.data_ptr();
    const int32_t *cu_q = at_of<int32_t>(cq), *cu_k = at_of<int32_t>(ck);
    void *o = O.data_ptr(), *st = stream();
    const int64_t ldq = row_stride(Q), ldk = row_stride(K), ldv = row_stride(V), ldo = row_stride(O);
    const int64_t Tq = Q.size(0), Tk = K.size(0), heads = Q.size(1) / d, kv = K.size(1) / d;
    const int status = released([&] {
        return sr_attn_prefill(q, ldq, k, ldk, v, ldv, cu_q, cu_k, n, Tq, Tk, heads, kv, d, causal, scale, o, ldo, st);
    });
    return status ? PyLong_FromLong(status) : THPVariable_Wrap(O);
}

PyObject *current_stream(PyObject *const *) { return PyLong_FromVoidPtr(stream()); }

#define SR_ENTRY(F, N) {#F, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(entry<F, N>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {SR_ENTRY(fwht_quant_act, 5), SR_ENTRY(fwht_quant_act_heads, 7), SR_ENTRY(fwht_quant_act_f6, 6),
                         SR_ENTRY(swiglu_fwht_quant_act, 7), SR_ENTRY(w4a4_gemm, 7), SR_ENTRY(w4a4_gemm_f6, 10),
                         SR_ENTRY(w4a4_linear_decode, 9), SR_ENTRY(kv_quant_asym, 6), SR_ENTRY(rope_kv_append, 12), SR_ENTRY(kv_gather, 4),
                         SR_ENTRY(attn_decode, 7), SR_ENTRY(attn_prefill, 9), SR_ENTRY(current_stream, 0), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void)
{
    PyObject *m = PyModule_Create(&module_def);
    if (m && PyModule_AddStringConstant(m, "torch_version", SR_TORCH_VERSION) < 0) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
