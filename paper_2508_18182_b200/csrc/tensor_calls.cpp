// Python entry points of the operators between the linear layers: the arguments of adloco.h's calls from torch tensors.
// The rest of the binding marshals in Python; these calls run once a layer or a token, where ten tensors' shapes,
// strides, types and pointers read one Python attribute at a time cost more (3 to 8 us) than the launch they are for.
// Each function takes the context's handle, the call's tensors (None where absent) and numbers, and the stream (None:
// the current one); it returns the call's status, or (status, text) where the arguments cannot be passed on.
#include <Python.h>
#include <ATen/ops/empty.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <string>

#include "../../include/adloco.h"

namespace {

struct Refused {
    int status;
    std::string text;
};

[[noreturn]] void refuse(int status, const std::string& text) { throw Refused{status, text}; }

const at::Tensor* tensor(PyObject* o, const char* what, bool optional) {
    if (o == Py_None && optional) return nullptr;
    if (!THPVariable_Check(o)) refuse(ADLOCO_ERR_INVALID_ARG, std::string(what) + ": expected a tensor");
    return &THPVariable_Unpack(o);
}
const at::Tensor& need(PyObject* o, const char* what) { return *tensor(o, what, false); }

std::string described(const at::Tensor& t) {
    std::string s = "[";
    for (int64_t i = 0; i < t.dim(); ++i) s += (i ? ", " : "") + std::to_string(t.size(i));
    return s + "] " + c10::toString(t.scalar_type()) + " on " + t.device().str();
}

adloco_dtype code(const at::Tensor& t, const char* what) {
    if (t.scalar_type() == at::kFloat) return ADLOCO_F32;
    if (t.scalar_type() == at::kBFloat16) return ADLOCO_BF16;
    refuse(ADLOCO_ERR_UNSUPPORTED, std::string(what) + ": unsupported dtype " + c10::toString(t.scalar_type()));
}

void on(const at::Tensor& t, const char* what, int64_t dev) {
    if (!t.is_cuda() || t.device().index() != dev)
        refuse(ADLOCO_ERR_INVALID_ARG, std::string(what) + " is on " + t.device().str() + ", the context on cuda:" + std::to_string(dev));
}

// A tensor [..., d] whose leading dimensions are one run of evenly spaced rows.
struct Rows {
    int64_t rows = 0, d = 0, pitch = 0;
    void* p = nullptr;
};
Rows rows_of(const at::Tensor& t, const char* what) {
    Rows r;
    const int64_t n = t.dim();
    if (n < 1) refuse(ADLOCO_ERR_INVALID_ARG, std::string(what) + ": a tensor of rows is needed");
    r.p = t.data_ptr();
    r.d = r.pitch = t.size(n - 1);
    if (t.stride(n - 1) != 1 && r.d > 1) refuse(ADLOCO_ERR_INVALID_ARG, std::string(what) + ": the last dimension must be contiguous");
    r.rows = 1;
    for (int64_t i = n - 2; i >= 0; --i) {          // a dimension of extent one puts no demand on its stride
        if (t.size(i) == 1) continue;
        if (r.rows == 1) r.pitch = t.stride(i);
        else if (t.stride(i) != r.rows * r.pitch) refuse(ADLOCO_ERR_INVALID_ARG, std::string(what) + ": rows must be evenly spaced");
        r.rows *= t.size(i);
    }
    return r;
}
Rows rows_like(const at::Tensor* t, const char* what, int64_t rows, int64_t d, at::ScalarType type, int64_t dev) {
    if (!t) return Rows();
    on(*t, what, dev);
    const Rows r = rows_of(*t, what);
    if (r.rows != rows || r.d != d || t->scalar_type() != type)
        refuse(ADLOCO_ERR_INVALID_ARG, std::string(what) + ": expected " + std::to_string(rows) + " rows of " + std::to_string(d) + " " +
                                           c10::toString(type) + ", got " + described(*t));
    return r;
}
void* vector(const at::Tensor* t, const char* what, int64_t n, at::ScalarType type, int64_t dev) {
    if (!t) return nullptr;
    on(*t, what, dev);
    if (t->numel() != n || t->scalar_type() != type || !t->is_contiguous())
        refuse(ADLOCO_ERR_INVALID_ARG, std::string(what) + ": expected " + std::to_string(n) + " contiguous " + c10::toString(type) + ", got " + described(*t));
    return t->data_ptr();
}
// an 8-bit matrix: float8_e4m3fn, or its bytes
Rows bytes_like(const at::Tensor* t, const char* what, int64_t rows, int64_t d, int64_t dev) {
    if (!t) return Rows();
    Rows r = rows_like(t, what, rows, d, t->scalar_type() == at::kByte ? at::kByte : at::kFloat8_e4m3fn, dev);
    if (rows == 1) r.pitch = (d + 15) / 16 * 16;      // a single row has no pitch: any that fits the rules will do
    return r;
}
Rows row_scales_like(const at::Tensor* t, const char* what, int64_t rows, int64_t d, int64_t dev) {
    if (!t) return Rows();
    Rows r = rows_like(t, what, rows, (d + 127) / 128, at::kByte, dev);
    if (rows == 1) r.pitch = (r.pitch + 3) / 4 * 4;
    return r;
}

// numbers
int64_t whole(PyObject* o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) { PyErr_Clear(); refuse(ADLOCO_ERR_INVALID_ARG, "expected a whole number of 64 bits"); }
    return v;
}
uint64_t unsigned_whole(PyObject* o, const char* what) {
    const unsigned long long v = PyLong_AsUnsignedLongLong(o);
    if (v == (unsigned long long)-1 && PyErr_Occurred()) { PyErr_Clear(); refuse(ADLOCO_ERR_INVALID_ARG, std::string(what) + " is an unsigned 64-bit number"); }
    return v;
}
double real(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) { PyErr_Clear(); refuse(ADLOCO_ERR_INVALID_ARG, "expected a number"); }
    return v;
}
bool truth(PyObject* o, const char* what) {
    const int v = PyObject_IsTrue(o);
    if (v < 0) { PyErr_Clear(); refuse(ADLOCO_ERR_INVALID_ARG, std::string(what) + ": expected True or False"); }
    return v != 0;
}
struct Mask {
    double p = 0.0;
    uint64_t seed = 0, offset = 0;
};
Mask mask_of(PyObject* o) {                            // (p, seed, offset) or None
    Mask m;
    if (o == Py_None) return m;
    PyObject* seq = PySequence_Fast(o, "");
    if (!seq || PySequence_Fast_GET_SIZE(seq) != 3) {
        PyErr_Clear();
        Py_XDECREF(seq);
        refuse(ADLOCO_ERR_INVALID_ARG, "dropout: expected (p, seed, offset)");
    }
    PyObject** v = PySequence_Fast_ITEMS(seq);
    PyObject *p = v[0], *s = v[1], *f = v[2];
    Py_INCREF(p); Py_INCREF(s); Py_INCREF(f);
    Py_DECREF(seq);
    struct Drop { PyObject *a, *b, *c; ~Drop() { Py_DECREF(a); Py_DECREF(b); Py_DECREF(c); } } drop{p, s, f};
    m.p = real(p);
    m.seed = unsigned_whole(s, "seed");
    m.offset = unsigned_whole(f, "offset");
    return m;
}
adloco_ctx* handle(PyObject* o) { return reinterpret_cast<adloco_ctx*>(static_cast<uintptr_t>(unsigned_whole(o, "handle"))); }
void* stream_of(PyObject* o, int64_t dev) {
    if (o == Py_None) return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)dev).stream();
    PyObject* v = PyObject_GetAttrString(o, "cuda_stream");
    if (!v) { PyErr_Clear(); refuse(ADLOCO_ERR_INVALID_ARG, "stream: expected a torch.cuda.Stream"); }
    const unsigned long long s = PyLong_AsUnsignedLongLong(v);
    Py_DECREF(v);
    if (PyErr_Occurred()) { PyErr_Clear(); refuse(ADLOCO_ERR_INVALID_ARG, "stream: expected a torch.cuda.Stream"); }
    return reinterpret_cast<void*>(static_cast<uintptr_t>(s));
}

// A call of the library with the interpreter's lock released, as the rest of the binding makes them: a launch waits where the
// queue to the device is full.  The arguments are formed before.
template <typename F, typename... Args>
int unlocked(F f, Args... args) {
    struct Released {
        PyThreadState* state = PyEval_SaveThread();
        ~Released() { PyEval_RestoreThread(state); }
    } released;
    return f(args...);
}

// handle, device, x, gain, residual, h, y, rstd, q, q_scale, eps, dropout, stream
int add_rmsnorm(PyObject* const* v) {
    const int64_t dev = whole(v[1]);
    const at::Tensor& x = need(v[2], "x");
    on(x, "x", dev);
    const Rows xr = rows_of(x, "x");
    const at::Tensor& gain = need(v[3], "gain");
    const at::Tensor *res = tensor(v[4], "residual", true), *h = tensor(v[5], "h", true);
    const at::Tensor& stream = res ? *res : h ? *h : x;
    adloco_rmsnorm_args a = {};
    a.dtype = code(x, "x");
    a.stream_dtype = code(stream, "residual");
    a.gain_dtype = code(gain, "gain");
    a.eps = (float)real(v[10]);
    a.rows = xr.rows; a.d = xr.d; a.x = xr.p; a.x_stride = xr.pitch;
    const Rows rr = rows_like(res, "residual", a.rows, a.d, stream.scalar_type(), dev), hr = rows_like(h, "h", a.rows, a.d, stream.scalar_type(), dev);
    const Rows yr = rows_like(tensor(v[6], "y", true), "y", a.rows, a.d, x.scalar_type(), dev);
    const at::Tensor *q = tensor(v[8], "q", true), *s = tensor(v[9], "q_scale", true);
    if (!q != !s) refuse(ADLOCO_ERR_INVALID_ARG, "q and its scales go together");
    const Rows qr = bytes_like(q, "q", a.rows, a.d, dev), sr = row_scales_like(s, "q_scale", a.rows, a.d, dev);
    a.residual = rr.p; a.residual_stride = rr.pitch;
    a.gain = vector(&gain, "gain", a.d, gain.scalar_type(), dev);
    a.h = hr.p; a.h_stride = hr.pitch;
    a.y = yr.p; a.y_stride = yr.pitch;
    a.rstd = static_cast<float*>(vector(tensor(v[7], "rstd", true), "rstd", a.rows, at::kFloat, dev));
    a.q = qr.p; a.q_stride = qr.pitch;
    a.q_scale = static_cast<uint8_t*>(sr.p); a.q_scale_stride = sr.pitch;
    const Mask m = mask_of(v[11]);
    a.dropout_p = m.p; a.seed = m.seed; a.offset = m.offset;
    return unlocked(adloco_add_rmsnorm, handle(v[0]), &a, stream_of(v[12], dev));
}

// handle, device, dy, h, rstd, gain, dh, dh_residual, dx, dropout, norms, accumulate_norms, sum, accumulate_sum, workspace, stream
int add_rmsnorm_backward(PyObject* const* v) {
    const int64_t dev = whole(v[1]);
    const at::Tensor &dy = need(v[2], "dy"), &h = need(v[3], "h"), &gain = need(v[5], "gain");
    on(dy, "dy", dev);
    const Rows yr = rows_of(dy, "dy");
    adloco_rmsnorm_backward_args a = {};
    a.dtype = code(dy, "dy");
    a.stream_dtype = code(h, "h");
    a.gain_dtype = code(gain, "gain");
    a.d = yr.d;
    a.B = dy.dim() == 3 ? dy.size(0) : 1;
    a.T = a.B ? yr.rows / a.B : 0;
    a.dy = yr.p; a.dy_stride = yr.pitch;
    const at::ScalarType ht = h.scalar_type();
    const Rows hr = rows_like(&h, "h", yr.rows, a.d, ht, dev), rr = rows_like(tensor(v[7], "dh_residual", true), "dh_residual", yr.rows, a.d, ht, dev);
    const Rows or_ = rows_like(&need(v[6], "dh"), "dh", yr.rows, a.d, ht, dev), xr = rows_like(tensor(v[8], "dx", true), "dx", yr.rows, a.d, dy.scalar_type(), dev);
    a.h = hr.p; a.h_stride = hr.pitch;
    a.rstd = static_cast<const float*>(vector(&need(v[4], "rstd"), "rstd", yr.rows, at::kFloat, dev));
    a.gain = vector(&gain, "gain", a.d, gain.scalar_type(), dev);
    a.dh_residual = rr.p; a.dh_residual_stride = rr.pitch;
    a.dh = or_.p; a.dh_stride = or_.pitch;
    a.dx = xr.p; a.dx_stride = xr.pitch;
    const Mask m = mask_of(v[9]);
    a.dropout_p = m.p; a.seed = m.seed; a.offset = m.offset;
    a.per_sample_sqnorm = static_cast<float*>(vector(tensor(v[10], "per_sample_sqnorm", true), "per_sample_sqnorm", a.B, at::kFloat, dev));
    a.accumulate_norms = truth(v[11], "accumulate_norms");
    a.grad_sum = static_cast<float*>(vector(tensor(v[12], "grad_sum", true), "grad_sum", a.d, at::kFloat, dev));
    a.accumulate_sum = truth(v[13], "accumulate_sum");
    at::Tensor own;                                    // from torch's allocator, on the current stream
    if (a.per_sample_sqnorm || a.grad_sum) {
        const at::Tensor* ws = tensor(v[14], "workspace", true);
        if (!ws) {
            if (v[15] != Py_None) refuse(ADLOCO_ERR_INVALID_ARG, "workspace: needed beside a stream");
            own = at::empty({adloco_add_rmsnorm_backward_workspace(handle(v[0]), a.B, a.T, a.d)}, dy.options().dtype(at::kByte));
            ws = &own;
        }
        a.workspace = vector(ws, "workspace", ws->numel(), at::kByte, dev);
        a.workspace_bytes = ws->numel();
    }
    return unlocked(adloco_add_rmsnorm_backward, handle(v[0]), &a, stream_of(v[15], dev));
}

// handle, device, x, out, residual, p, seed, offset, stream
int dropout(PyObject* const* v) {
    const int64_t dev = whole(v[1]);
    const at::Tensor& x = need(v[2], "x");
    on(x, "x", dev);
    const Rows xr = rows_of(x, "x");
    const Rows yr = rows_like(&need(v[3], "out"), "out", xr.rows, xr.d, x.scalar_type(), dev);
    const Rows rr = rows_like(tensor(v[4], "residual", true), "residual", xr.rows, xr.d, x.scalar_type(), dev);
    return unlocked(adloco_dropout, handle(v[0]), code(x, "x"), xr.rows, xr.d, xr.p, xr.pitch, rr.p, rr.pitch, yr.p, yr.pitch, real(v[5]),
                          unsigned_whole(v[6], "seed"), unsigned_whole(v[7], "offset"), stream_of(v[8], dev));
}

// handle, device, tensors, outs, turns, rot_dim, magnitude, positions, first_position, interleaved, inverse, stream
int rope(PyObject* const* v) {
    const int64_t dev = whole(v[1]);
    struct Hold { PyObject* o; ~Hold() { Py_XDECREF(o); } };
    Hold in{PySequence_Fast(v[2], "")}, out{PySequence_Fast(v[3], "")};
    PyErr_Clear();
    if (!in.o || !out.o || PySequence_Fast_GET_SIZE(in.o) < 1 || PySequence_Fast_GET_SIZE(in.o) != PySequence_Fast_GET_SIZE(out.o))
        refuse(ADLOCO_ERR_INVALID_ARG, "tensors and outs are two sequences of one length");
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(in.o);
    if (n > 4) refuse(ADLOCO_ERR_UNSUPPORTED, "at most four tensors go in one call");
    adloco_rope_tensor t[4];
    const at::Tensor& x = need(PySequence_Fast_ITEMS(in.o)[0], "tensors[0]");
    on(x, "tensors[0]", dev);
    if (x.dim() != 4) refuse(ADLOCO_ERR_INVALID_ARG, "tensors are [B, T, heads, head_dim]");
    const int64_t B = x.size(0), T = x.size(1), D = x.size(3);
    for (Py_ssize_t i = 0; i < n; ++i) {
        const at::Tensor &a = need(PySequence_Fast_ITEMS(in.o)[i], "tensors"), &o = need(PySequence_Fast_ITEMS(out.o)[i], "outs");
        on(a, "tensors", dev);
        on(o, "outs", dev);
        if (a.dim() != 4 || a.size(0) != B || a.size(1) != T || a.size(3) != D || o.sizes() != a.sizes() || a.scalar_type() != x.scalar_type() ||
            o.scalar_type() != x.scalar_type() || (D > 1 && (a.stride(3) != 1 || o.stride(3) != 1)))
            refuse(ADLOCO_ERR_INVALID_ARG, "tensors and outs must share B, T, head_dim and type, with head_dim contiguous");
        t[i] = adloco_rope_tensor{a.data_ptr(), o.data_ptr(), a.size(2), a.stride(0), a.stride(1), a.stride(2), o.stride(0), o.stride(1), o.stride(2)};
    }
    const at::Tensor* pos = tensor(v[7], "positions", true);
    int64_t pitch = 0;
    if (pos) {
        on(*pos, "positions", dev);
        if (pos->scalar_type() != at::kInt || pos->dim() != 2 || pos->size(0) != B || pos->size(1) != T || (T > 1 && pos->stride(1) != 1))
            refuse(ADLOCO_ERR_INVALID_ARG, "positions must be int32 [B, T] with contiguous rows, got " + described(*pos));
        pitch = B > 1 ? pos->stride(0) : T;
    }
    const at::Tensor& turns = need(v[4], "table");
    on(turns, "the table", dev);
    return unlocked(adloco_rope, handle(v[0]), code(x, "tensors"), t, (int32_t)n, B, T, D, whole(v[5]), static_cast<const uint64_t*>(turns.data_ptr()),
                       (float)real(v[6]), pos ? static_cast<const int32_t*>(pos->data_ptr()) : nullptr, pitch, whole(v[8]),
                       truth(v[9], "interleaved"), truth(v[10], "inverse"), stream_of(v[11], dev));
}

// handle, device, x, q, scale, stream
int blockscale_quantize(PyObject* const* v) {
    const int64_t dev = whole(v[1]);
    const at::Tensor& x = need(v[2], "x");
    on(x, "x", dev);
    const Rows xr = rows_of(x, "x"), qr = bytes_like(&need(v[3], "q"), "q", xr.rows, xr.d, dev);
    const Rows sr = row_scales_like(&need(v[4], "scale"), "scale", xr.rows, xr.d, dev);
    return unlocked(adloco_blockscale_quantize, handle(v[0]), code(x, "x"), xr.rows, xr.d, xr.p, xr.pitch, qr.p, qr.pitch, static_cast<uint8_t*>(sr.p),
                                      sr.pitch, stream_of(v[5], dev));
}

// handle, device, W, q, scale, q_t, stream
int blockscale_quantize_weight(PyObject* const* v) {
    const int64_t dev = whole(v[1]);
    const at::Tensor& W = need(v[2], "W");
    on(W, "W", dev);
    const Rows wr = rows_of(W, "W"), qr = bytes_like(&need(v[3], "q"), "q", wr.rows, wr.d, dev);
    const Rows tr = bytes_like(tensor(v[5], "q_t", true), "q_t", wr.d, wr.rows, dev);
    const Rows sr = rows_like(&need(v[4], "scale"), "scale", (wr.rows + 127) / 128, (wr.d + 127) / 128, at::kByte, dev);
    return unlocked(adloco_blockscale_quantize_weight, handle(v[0]), code(W, "W"), wr.rows, wr.d, wr.p, wr.pitch, qr.p, qr.pitch, tr.p, tr.pitch,
                                             static_cast<uint8_t*>(sr.p), sr.pitch, stream_of(v[6], dev));
}

// handle, device, a, a_scale, b, b_scale, out, scale_transposed, bias, stream
int blockscale_matmul(PyObject* const* v) {
    const int64_t dev = whole(v[1]);
    const at::Tensor &at_ = need(v[2], "a"), &bt = need(v[4], "b"), &ot = need(v[6], "out");
    adloco_blockscale_matmul_args a = {};
    const Rows shape = rows_of(at_, "a");
    a.M = shape.rows; a.K = shape.d;
    if (bt.dim() != 2) refuse(ADLOCO_ERR_INVALID_ARG, "b: expected [N, K], got " + described(bt));
    a.N = bt.size(0);
    const Rows ar = bytes_like(&at_, "a", a.M, a.K, dev), sr = row_scales_like(&need(v[3], "a_scale"), "a_scale", a.M, a.K, dev);
    const Rows br = bytes_like(&bt, "b", a.N, a.K, dev);
    const int64_t nb = (a.N + 127) / 128, kb = (a.K + 127) / 128;
    const bool transposed = truth(v[7], "scale_transposed");
    const Rows bs = rows_like(&need(v[5], "b_scale"), "b_scale", transposed ? kb : nb, transposed ? nb : kb, at::kByte, dev);
    const Rows orow = rows_like(&ot, "out", a.M, a.N, ot.scalar_type(), dev);
    a.a = ar.p; a.a_stride = ar.pitch;
    a.a_scale = static_cast<const uint8_t*>(sr.p); a.a_scale_stride = sr.pitch;
    a.b = br.p; a.b_stride = br.pitch;
    a.b_scale = static_cast<const uint8_t*>(bs.p);
    a.b_scale_stride_n = transposed ? 1 : bs.pitch;
    a.b_scale_stride_k = transposed ? bs.pitch : 1;
    a.bias = static_cast<const float*>(vector(tensor(v[8], "bias", true), "bias", a.N, at::kFloat, dev));
    a.out = orow.p; a.out_stride = orow.pitch; a.out_dtype = code(ot, "out");
    return unlocked(adloco_blockscale_matmul, handle(v[0]), &a, stream_of(v[9], dev));
}

// handle, device, q, scale, x, stream
int blockscale_dequantize(PyObject* const* v) {
    const int64_t dev = whole(v[1]);
    const at::Tensor& x = need(v[4], "x");
    on(x, "x", dev);
    const Rows xr = rows_of(x, "x"), qr = bytes_like(&need(v[2], "q"), "q", xr.rows, xr.d, dev);
    const Rows sr = row_scales_like(&need(v[3], "scale"), "scale", xr.rows, xr.d, dev);
    return unlocked(adloco_blockscale_dequantize, handle(v[0]), code(x, "x"), xr.rows, xr.d, qr.p, qr.pitch, static_cast<uint8_t*>(sr.p), sr.pitch,
                    xr.p, xr.pitch, stream_of(v[5], dev));
}

// bf16 rows that a product takes
Rows operand(const at::Tensor& t, const char* what, int64_t rows, int64_t d, int64_t dev) {
    Rows r = rows_like(&t, what, rows, d, at::kBFloat16, dev);
    if (rows == 1) r.pitch = (d + 7) / 8 * 8;         // a single row has no pitch
    return r;
}
Rows weight(const at::Tensor& t, const char* what, int64_t rows, int64_t d, int64_t dev) {
    if (t.dim() != 2) refuse(ADLOCO_ERR_INVALID_ARG, std::string(what) + ": expected a matrix, got " + described(t));
    return operand(t, what, rows < 0 ? t.size(0) : rows, d < 0 ? t.size(1) : d, dev);
}
// what is kept for the backward pass, in bf16 or in bytes with their scales
adloco_kept kept(PyObject* t, PyObject* s, const char* what, int64_t rows, int64_t d, int64_t dev) {
    const at::Tensor *x = tensor(t, what, true), *scale = tensor(s, what, true);
    adloco_kept k = {};
    if (!x) {
        if (scale) refuse(ADLOCO_ERR_INVALID_ARG, std::string(what) + ": scales without values");
        return k;
    }
    if (!scale) {
        const Rows r = operand(*x, what, rows, d, dev);
        k.p = r.p; k.stride = r.pitch;
        return k;
    }
    const Rows r = bytes_like(x, what, rows, d, dev), sr = row_scales_like(scale, what, rows, d, dev);
    k.p = r.p; k.stride = r.pitch;
    k.scale = static_cast<uint8_t*>(sr.p); k.scale_stride = sr.pitch;
    return k;
}
int32_t activation(PyObject* o) {
    static const char* const names[] = {"none", "relu", "gelu", "gelu_tanh", "silu"};
    if (o == Py_None) return ADLOCO_ACT_NONE;
    if (PyUnicode_Check(o))
        for (int32_t i = 0; i < 5; ++i)
            if (PyUnicode_CompareWithASCIIString(o, names[i]) == 0) return i;
    refuse(ADLOCO_ERR_INVALID_ARG, "activation: expected none, relu, gelu, gelu_tanh or silu");
}

// handle, device, x, w, y, bias, activation, residual, z, z_scale, stream
int linear(PyObject* const* v) {
    const int64_t dev = whole(v[1]);
    const at::Tensor &x = need(v[2], "x"), &w = need(v[3], "w"), &y = need(v[4], "y");
    on(x, "x", dev);
    adloco_linear_args a = {};
    const Rows shape = rows_of(x, "x"), wr = weight(w, "w", -1, shape.d, dev);
    a.M = shape.rows; a.K = shape.d; a.N = w.size(0);
    const Rows xr = operand(x, "x", a.M, a.K, dev), yr = rows_like(&y, "y", a.M, a.N, y.scalar_type(), dev);
    const Rows rr = rows_like(tensor(v[7], "residual", true), "residual", a.M, a.N, y.scalar_type(), dev);
    a.x = xr.p; a.x_stride = xr.pitch;
    a.w = wr.p; a.w_stride = wr.pitch;
    a.bias = static_cast<const float*>(vector(tensor(v[5], "bias", true), "bias", a.N, at::kFloat, dev));
    a.residual = rr.p; a.residual_stride = rr.pitch;
    a.y = yr.p; a.y_stride = yr.pitch; a.out_dtype = code(y, "y");
    a.z = kept(v[8], v[9], "z", a.M, a.N, dev);
    a.activation = activation(v[6]);
    return unlocked(adloco_linear, handle(v[0]), &a, stream_of(v[10], dev));
}

// handle, device, dy, w, dx, activation, z, z_scale, a, residual, stream
int linear_backward(PyObject* const* v) {
    const int64_t dev = whole(v[1]);
    const at::Tensor &dy = need(v[2], "dy"), &w = need(v[3], "w"), &dx = need(v[4], "dx");
    on(dy, "dy", dev);
    adloco_linear_backward_args a = {};
    const Rows shape = rows_of(dy, "dy"), wr = weight(w, "w", shape.d, -1, dev);
    a.M = shape.rows; a.N = shape.d; a.K = w.size(1);
    const Rows dr = operand(dy, "dy", a.M, a.N, dev), xr = rows_like(&dx, "dx", a.M, a.K, dx.scalar_type(), dev);
    const Rows rr = rows_like(tensor(v[9], "residual", true), "residual", a.M, a.K, dx.scalar_type(), dev);
    const Rows ar = rows_like(tensor(v[8], "a", true), "a", a.M, a.K, at::kBFloat16, dev);
    a.dy = dr.p; a.dy_stride = dr.pitch;
    a.w = wr.p; a.w_stride = wr.pitch;
    a.z = kept(v[6], v[7], "z", a.M, a.K, dev);
    a.residual = rr.p; a.residual_stride = rr.pitch;
    a.dx = xr.p; a.dx_stride = xr.pitch; a.out_dtype = code(dx, "dx");
    a.a = ar.p; a.a_stride = ar.pitch;
    a.activation = activation(v[5]);
    return unlocked(adloco_linear_backward, handle(v[0]), &a, stream_of(v[10], dev));
}

// handle, device, x, w_gate, w_up, a, activation, gate, up, gate_scale, up_scale, stream
int gated_linear(PyObject* const* v) {
    const int64_t dev = whole(v[1]);
    const at::Tensor &x = need(v[2], "x"), &wg = need(v[3], "w_gate");
    on(x, "x", dev);
    adloco_gated_linear_args a = {};
    const Rows shape = rows_of(x, "x"), gr = weight(wg, "w_gate", -1, shape.d, dev);
    a.M = shape.rows; a.d = shape.d; a.f = wg.size(0);
    const Rows ur = weight(need(v[4], "w_up"), "w_up", a.f, a.d, dev), xr = operand(x, "x", a.M, a.d, dev);
    const Rows ar = rows_like(&need(v[5], "a"), "a", a.M, a.f, at::kBFloat16, dev);
    a.x = xr.p; a.x_stride = xr.pitch;
    a.w_gate = gr.p; a.w_gate_stride = gr.pitch;
    a.w_up = ur.p; a.w_up_stride = ur.pitch;
    a.a = ar.p; a.a_stride = ar.pitch;
    a.activation = activation(v[6]);
    a.gate = kept(v[7], v[9], "gate", a.M, a.f, dev);
    a.up = kept(v[8], v[10], "up", a.M, a.f, dev);
    return unlocked(adloco_gated_linear, handle(v[0]), &a, stream_of(v[11], dev));
}

// handle, device, dy, w_down, gate, up, d_gate, d_up, activation, gate_scale, up_scale, a, stream
int gated_linear_backward(PyObject* const* v) {
    const int64_t dev = whole(v[1]);
    const at::Tensor &dy = need(v[2], "dy"), &w = need(v[3], "w_down");
    on(dy, "dy", dev);
    adloco_gated_linear_backward_args a = {};
    const Rows shape = rows_of(dy, "dy"), wr = weight(w, "w_down", shape.d, -1, dev);
    a.M = shape.rows; a.d = shape.d; a.f = w.size(1);
    const Rows dr = operand(dy, "dy", a.M, a.d, dev);
    a.dy = dr.p; a.dy_stride = dr.pitch;
    a.w_down = wr.p; a.w_down_stride = wr.pitch;
    need(v[4], "gate"); need(v[5], "up");
    a.gate = kept(v[4], v[9], "gate", a.M, a.f, dev);
    a.up = kept(v[5], v[10], "up", a.M, a.f, dev);
    const Rows gr = rows_like(&need(v[6], "d_gate"), "d_gate", a.M, a.f, at::kBFloat16, dev), ur = rows_like(&need(v[7], "d_up"), "d_up", a.M, a.f, at::kBFloat16, dev);
    const Rows ar = rows_like(tensor(v[11], "a", true), "a", a.M, a.f, at::kBFloat16, dev);
    a.d_gate = gr.p; a.d_gate_stride = gr.pitch;
    a.d_up = ur.p; a.d_up_stride = ur.pitch;
    a.a = ar.p; a.a_stride = ar.pitch;
    a.activation = activation(v[8]);
    return unlocked(adloco_gated_linear_backward, handle(v[0]), &a, stream_of(v[12], dev));
}

// handle, device, logits, targets, logp, entropy, lse, top_values, top_ids, stream
int token_logprobs(PyObject* const* v) {
    const int64_t dev = whole(v[1]);
    const at::Tensor& l = need(v[2], "logits");
    on(l, "logits", dev);
    const Rows lr = rows_of(l, "logits");
    adloco_token_logprobs_args a = {};
    a.rows = lr.rows; a.V = lr.d; a.logits = lr.p; a.logits_stride = lr.pitch; a.dtype = code(l, "logits");
    a.targets = static_cast<const int32_t*>(vector(tensor(v[3], "targets", true), "targets", a.rows, at::kInt, dev));
    a.logp = static_cast<float*>(vector(tensor(v[4], "logp", true), "logp", a.rows, at::kFloat, dev));
    a.entropy = static_cast<float*>(vector(tensor(v[5], "entropy", true), "entropy", a.rows, at::kFloat, dev));
    a.lse = static_cast<float*>(vector(tensor(v[6], "lse", true), "lse", a.rows, at::kFloat, dev));
    const at::Tensor *tv = tensor(v[7], "top_values", true), *ti = tensor(v[8], "top_ids", true);
    if (!tv != !ti) refuse(ADLOCO_ERR_INVALID_ARG, "top_values and top_ids go together");
    if (tv) {
        const int64_t top = tv->dim() ? tv->size(tv->dim() - 1) : 0;
        if (top < 1 || top > 64) refuse(ADLOCO_ERR_UNSUPPORTED, "top_values: 1 to 64 tokens a row, got " + described(*tv));
        a.top = (int32_t)top;
        a.top_values = static_cast<float*>(vector(tv, "top_values", a.rows * top, at::kFloat, dev));
        a.top_ids = static_cast<int32_t*>(vector(ti, "top_ids", a.rows * top, at::kInt, dev));
    }
    return unlocked(adloco_token_logprobs, handle(v[0]), &a, stream_of(v[9], dev));
}

// handle, device, logits, targets, lse, d_logp, d_logits, entropy, d_entropy, stream
int token_logprobs_backward(PyObject* const* v) {
    const int64_t dev = whole(v[1]);
    const at::Tensor& l = need(v[2], "logits");
    on(l, "logits", dev);
    const Rows lr = rows_of(l, "logits"), dr = rows_like(&need(v[6], "d_logits"), "d_logits", lr.rows, lr.d, l.scalar_type(), dev);
    adloco_token_logprobs_backward_args a = {};
    a.rows = lr.rows; a.V = lr.d; a.logits = lr.p; a.logits_stride = lr.pitch; a.dtype = code(l, "logits");
    a.d_logits = dr.p; a.d_logits_stride = dr.pitch;
    a.targets = static_cast<const int32_t*>(vector(&need(v[3], "targets"), "targets", a.rows, at::kInt, dev));
    a.lse = static_cast<const float*>(vector(&need(v[4], "lse"), "lse", a.rows, at::kFloat, dev));
    a.d_logp = static_cast<const float*>(vector(&need(v[5], "d_logp"), "d_logp", a.rows, at::kFloat, dev));
    a.entropy = static_cast<const float*>(vector(tensor(v[7], "entropy", true), "entropy", a.rows, at::kFloat, dev));
    a.d_entropy = static_cast<const float*>(vector(tensor(v[8], "d_entropy", true), "d_entropy", a.rows, at::kFloat, dev));
    return unlocked(adloco_token_logprobs_backward, handle(v[0]), &a, stream_of(v[9], dev));
}

template <int (*F)(PyObject* const*), int N>
PyObject* call(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != N) {
        PyErr_Format(PyExc_TypeError, "expected %d arguments, got %zd", N, n);
        return nullptr;
    }
    try {
        return PyLong_FromLong(F(args));
    } catch (const Refused& r) {
        return Py_BuildValue("(is)", r.status, r.text.c_str());
    } catch (const std::exception& e) {               // torch's allocator, or a tensor without storage
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}
#define ADLOCO_METHOD(f, n) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&call<f, n>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ADLOCO_METHOD(add_rmsnorm, 13), ADLOCO_METHOD(add_rmsnorm_backward, 16), ADLOCO_METHOD(dropout, 9),
                         ADLOCO_METHOD(rope, 12), ADLOCO_METHOD(blockscale_quantize, 6), ADLOCO_METHOD(blockscale_quantize_weight, 7),
                         ADLOCO_METHOD(blockscale_matmul, 10), ADLOCO_METHOD(blockscale_dequantize, 6), ADLOCO_METHOD(linear, 11),
                         ADLOCO_METHOD(linear_backward, 11), ADLOCO_METHOD(gated_linear, 12), ADLOCO_METHOD(gated_linear_backward, 13),
                         ADLOCO_METHOD(token_logprobs, 10), ADLOCO_METHOD(token_logprobs_backward, 10), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensor_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensor_calls() { return PyModule_Create(&module); }
