// policy_binding.cpp -- Python binding of the policy operators (module _policy).
//
// Argument marshalling between torch tensors and the library's C functions:
// checks what it is given (ValueError), makes the outputs, takes the current
// stream, calls av_*.  It is written against torch's C++ interface because on
// small inputs a call's time is the host's: a layer norm of one row of 256 took
// 17.3 us through ctypes and torch's Python functions and takes 5.9 here, some
// four of them the library's call.
// The functions take positional arguments only; policy.py is their face.
#include <ATen/core/grad_mode.h>
#include <ATen/cuda/EmptyTensor.h>
#include <Python.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstring>
#include <stdexcept>
#include <string>

#include "autoverse.h"

namespace {

using at::Tensor;

PyObject *g_error = nullptr;  // AvError

struct Refused : std::runtime_error {
    using std::runtime_error::runtime_error;
};
struct Failed {
    const char *fn;
    int status;
};

[[noreturn]] void refuse(const char *name, const std::string &why) { throw Refused(std::string(name) + ": " + why); }

void check(const char *fn, int status)
{
    if (status != AV_OK)
        throw Failed{fn, status};
}

std::string shape_text(at::IntArrayRef s)
{
    std::string t = "(";
    for (size_t i = 0; i < s.size(); ++i)
        t += (i ? ", " : "") + std::to_string(s[i]);
    return t + (s.size() == 1 ? ",)" : ")");
}

// The interpreter's lock let go, as ctypes does: others run while this thread allocates and launches.
class Unlocked {
public:
    Unlocked() : state_(PyEval_SaveThread()) {}
    Unlocked(const Unlocked &) = delete;
    Unlocked &operator=(const Unlocked &) = delete;
    ~Unlocked() { end(); }
    void end()
    {
        if (state_)
            PyEval_RestoreThread(state_);
        state_ = nullptr;
    }

private:
    PyThreadState *state_;
};

// ------------------------------------------------------------ arguments

bool given(PyObject *o) { return o != Py_None; }

const Tensor &tensor(const char *name, PyObject *o)
{
    if (!THPVariable_Check(o))
        refuse(name, "expected a CUDA tensor");
    const Tensor &t = THPVariable_Unpack(o);
    if (!t.is_cuda())
        refuse(name, "expected a CUDA tensor");
    return t;
}

int type_of(const char *name, const Tensor &t)
{
    switch (t.scalar_type()) {
    case at::kFloat: return AV_F32;
    case at::kBFloat16: return AV_BF16;
    case at::kHalf: return AV_F16;
    default: refuse(name, "expected float32, bfloat16 or float16");
    }
}

void on_device(const char *name, const Tensor &t, const Tensor &ref)
{
    if (t.device() != ref.device())
        refuse(name, "expected a tensor on " + ref.device().str());
}
void of_type(const char *name, const Tensor &t, at::ScalarType type)
{
    if (t.scalar_type() != type)
        refuse(name, std::string("expected ") + c10::toString(type) + ", got " + c10::toString(t.scalar_type()));
}
void of_shape(const char *name, const Tensor &t, at::IntArrayRef shape)
{
    if (t.sizes() != shape)
        refuse(name, "expected shape " + shape_text(shape) + ", got " + shape_text(t.sizes()));
}

// A contiguous tensor on ref's device, of that type and shape.
const Tensor &dense(const char *name, PyObject *o, const Tensor &ref, at::ScalarType type, at::IntArrayRef shape)
{
    const Tensor &t = tensor(name, o);
    on_device(name, t, ref);
    of_type(name, t, type);
    of_shape(name, t, shape);
    if (!t.is_contiguous())
        refuse(name, "expected a contiguous tensor");
    return t;
}
float *floats(const char *name, PyObject *o, const Tensor &ref, at::IntArrayRef shape)
{
    return given(o) ? static_cast<float *>(dense(name, o, ref, at::kFloat, shape).data_ptr()) : nullptr;
}

// t [..., n] as evenly spaced rows.
struct Rows {
    int64_t rows, n, stride;
};
Rows rows_of(const char *name, const Tensor &t)
{
    const int64_t dims = t.dim();
    if (dims < 1)
        refuse(name, "expected at least 1 axis");
    const auto size = t.sizes(), stride = t.strides();
    Rows r{1, size[dims - 1], 0};
    if (r.n > 1 && stride[dims - 1] != 1)
        refuse(name, "the last axis is not contiguous");
    for (int64_t d = dims - 2; d >= 0; --d) {
        if (size[d] != 1 && t.numel() > 0) {
            if (r.rows == 1)
                r.stride = stride[d];
            else if (stride[d] != r.stride * r.rows)
                refuse(name, "the rows are not evenly spaced");
        }
        r.rows *= size[d];
    }
    if (r.rows <= 1 || t.numel() == 0)
        r.stride = r.n;
    return r;
}

at::IntArrayRef lead_of(const Tensor &t) { return t.sizes().slice(0, t.dim() - 1); }

Tensor make(at::IntArrayRef shape, at::ScalarType type, const Tensor &ref)
{
    return at::Tensor(at::detail::empty_cuda(shape, type, ref.device(), std::nullopt));
}

uintptr_t stream_of(const Tensor &t)
{
    return reinterpret_cast<uintptr_t>(c10::cuda::getCurrentCUDAStream(t.get_device()).stream());
}

PyObject *tuple(std::initializer_list<Tensor> list)
{
    PyObject *out = PyTuple_New((Py_ssize_t)list.size());
    if (!out)
        return nullptr;
    Py_ssize_t i = 0;
    for (const Tensor &t : list) {
        PyObject *v = THPVariable_Wrap(t);
        if (!v) {
            Py_DECREF(out);
            return nullptr;
        }
        PyTuple_SET_ITEM(out, i++, v);
    }
    return out;
}

double number(PyObject *o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred())
        throw python_error();
    return v;
}
long whole(PyObject *o)
{
    const long v = PyLong_AsLong(o);
    if (v == -1 && PyErr_Occurred())
        throw python_error();
    return v;
}

// ------------------------------------------------------------ layer norm

PyObject *layer_norm(PyObject *const *a)
{
    const Tensor &x = tensor("x", a[0]);
    const int dtype = type_of("x", x);
    const Rows r = rows_of("x", x);
    const void *w = nullptr, *b = nullptr;
    at::ScalarType params = x.scalar_type();
    int ptype = dtype;
    if (given(a[1])) {
        const Tensor &t = tensor("weight", a[1]);
        ptype = type_of("weight", t);
        params = t.scalar_type();
        w = dense("weight", a[1], x, params, {r.n}).data_ptr();
    }
    if (given(a[2])) {
        if (!given(a[1])) {
            ptype = type_of("bias", tensor("bias", a[2]));
            params = tensor("bias", a[2]).scalar_type();
        }
        b = dense("bias", a[2], x, params, {r.n}).data_ptr();
    }
    const float eps = (float)number(a[3]);
    if (r.n > INT32_MAX)
        refuse("x", "rows too long");
    Unlocked unlocked;
    const c10::cuda::CUDAGuard guard(x.device());
    const Tensor y = make(x.sizes(), x.scalar_type(), x), mean = make(lead_of(x), at::kFloat, x),
                 rstd = make(lead_of(x), at::kFloat, x);
    check("av_layer_norm", av_layer_norm(r.rows, (int32_t)r.n, dtype, ptype, eps, x.data_ptr(), r.stride, w, b,
                                         y.data_ptr(), r.n, (float *)mean.data_ptr(), (float *)rstd.data_ptr(),
                                         stream_of(x)));
    unlocked.end();
    return tuple({y, mean, rstd});
}

PyObject *layer_norm_grad(PyObject *const *a)
{
    const Tensor &dy = tensor("dy", a[0]), &x = tensor("x", a[1]);
    const int dtype = type_of("x", x);
    const Rows r = rows_of("x", x);
    on_device("dy", dy, x);
    of_type("dy", dy, x.scalar_type());
    of_shape("dy", dy, x.sizes());
    at::ScalarType params = at::kFloat;
    int ptype = AV_F32;
    const void *w = nullptr;
    if (given(a[2])) {
        const Tensor &t = tensor("weight", a[2]);
        ptype = type_of("weight", t);
        params = t.scalar_type();
        w = dense("weight", a[2], x, params, {r.n}).data_ptr();
    }
    const Tensor &mean = dense("mean", a[3], x, at::kFloat, lead_of(x)),
                 &rstd = dense("rstd", a[4], x, at::kFloat, lead_of(x));
    if (r.n > INT32_MAX)
        refuse("x", "rows too long");
    int64_t need = 0;
    check("av_layer_norm_work", av_layer_norm_work(r.rows, (int32_t)r.n, &need));
    Unlocked unlocked;
    const c10::cuda::CUDAGuard guard(x.device());
    const Tensor dx = make(x.sizes(), x.scalar_type(), x), dw = make({r.n}, params, x), db = make({r.n}, params, x),
                 work = make({need}, at::kByte, x);
    check("av_layer_norm_grad",
          av_layer_norm_grad(r.rows, (int32_t)r.n, dtype, ptype, dy.data_ptr(), rows_of("dy", dy).stride, x.data_ptr(),
                             r.stride, w, (const float *)mean.data_ptr(), (const float *)rstd.data_ptr(), dx.data_ptr(),
                             r.n, dw.data_ptr(), db.data_ptr(), work.data_ptr(), need, stream_of(x)));
    unlocked.end();
    return tuple({dx, dw, db});
}

// ------------------------------------------------------------ recurrence

// A [T, B, D] tensor with D contiguous: strides of steps and sequences.
struct Seq {
    const void *p;
    int64_t t, b;
};
Seq seq_of(const char *name, const Tensor &x)
{
    if (x.size(2) > 1 && x.stride(2) != 1)
        refuse(name, "the last axis is not contiguous");
    return {x.data_ptr(), x.stride(0), x.stride(1)};
}

struct ScanInputs {
    int dtype;
    int64_t T, B, D, states, work;
    Seq gate, value, reset;
};
ScanInputs scan_inputs(const Tensor &gate, PyObject *value_o, PyObject *reset_o)
{
    ScanInputs s;
    s.dtype = type_of("gate", gate);
    if (gate.dim() != 3)
        refuse("gate", "expected [T, B, D]");
    const Tensor &value = tensor("value", value_o);
    on_device("value", value, gate);
    of_type("value", value, gate.scalar_type());
    of_shape("value", value, gate.sizes());
    s.T = gate.size(0), s.B = gate.size(1), s.D = gate.size(2);
    s.gate = seq_of("gate", gate);
    s.value = seq_of("value", value);
    s.reset = {nullptr, 0, 0};
    if (given(reset_o)) {
        const Tensor &reset = tensor("reset", reset_o);
        on_device("reset", reset, gate);
        if (reset.scalar_type() != at::kBool)
            of_type("reset", reset, at::kByte);
        of_shape("reset", reset, gate.sizes().slice(0, 2));
        s.reset = {reset.data_ptr(), reset.stride(0), reset.stride(1)};
    }
    check("av_scan_sizes", av_scan_sizes(s.T, s.B, s.D, s.dtype, &s.states, &s.work));
    return s;
}

PyObject *scan(PyObject *const *a)
{
    const Tensor &gate = tensor("gate", a[0]);
    const ScanInputs s = scan_inputs(gate, a[1], a[2]);
    const float *h0 = floats("h0", a[3], gate, {s.B, s.D});
    const int save = PyObject_IsTrue(a[4]);
    if (save < 0)
        throw python_error();
    Unlocked unlocked;
    const c10::cuda::CUDAGuard guard(gate.device());
    const Tensor h = make(gate.sizes(), gate.scalar_type(), gate), last = make({s.B, s.D}, at::kFloat, gate);
    Tensor states, work;
    if (save)
        states = make({s.states}, at::kFloat, gate);
    if (s.work)
        work = make({s.work}, at::kByte, gate);
    check("av_scan", av_scan(s.T, s.B, s.D, s.dtype, s.gate.p, s.gate.t, s.gate.b, s.value.p, s.value.t, s.value.b,
                             (const uint8_t *)s.reset.p, s.reset.t, s.reset.b, h0, h.data_ptr(), s.B * s.D, s.D,
                             (float *)last.data_ptr(), save ? (float *)states.data_ptr() : nullptr,
                             s.work ? work.data_ptr() : nullptr, s.work, stream_of(gate)));
    unlocked.end();
    return save ? tuple({h, last, states}) : tuple({h, last});
}

PyObject *scan_grad(PyObject *const *a)
{
    const Tensor &dh = tensor("dh", a[0]), &gate = tensor("gate", a[1]);
    const ScanInputs s = scan_inputs(gate, a[2], a[3]);
    on_device("dh", dh, gate);
    of_type("dh", dh, gate.scalar_type());
    of_shape("dh", dh, gate.sizes());
    const Seq up = seq_of("dh", dh);
    const Tensor &states = dense("states", a[4], gate, at::kFloat, {s.states});
    const float *dlast = floats("dlast", a[5], gate, {s.B, s.D});
    Unlocked unlocked;
    const c10::cuda::CUDAGuard guard(gate.device());
    const Tensor dgate = make(gate.sizes(), gate.scalar_type(), gate),
                 dvalue = make(gate.sizes(), gate.scalar_type(), gate), dh0 = make({s.B, s.D}, at::kFloat, gate);
    Tensor work;
    if (s.work)
        work = make({s.work}, at::kByte, gate);
    const int64_t t = s.B * s.D, b = s.D;
    check("av_scan_grad",
          av_scan_grad(s.T, s.B, s.D, s.dtype, up.p, up.t, up.b, s.gate.p, s.gate.t, s.gate.b, s.value.p, s.value.t,
                       s.value.b, (const uint8_t *)s.reset.p, s.reset.t, s.reset.b, (const float *)states.data_ptr(),
                       dlast, dgate.data_ptr(), t, b, dvalue.data_ptr(), t, b, (float *)dh0.data_ptr(),
                       s.work ? work.data_ptr() : nullptr, s.work, stream_of(gate)));
    unlocked.end();
    return tuple({dgate, dvalue, dh0});
}

// ------------------------------------------------------------ log probabilities

struct LogpInputs {
    int dtype, token_bytes;
    Rows r;
    const void *tokens;
    const uint8_t *mask;
    int64_t mask_stride;
};
LogpInputs logp_inputs(const Tensor &logits, PyObject *tokens_o, PyObject *mask_o)
{
    LogpInputs s{};
    s.dtype = type_of("logits", logits);
    s.r = rows_of("logits", logits);
    if (s.r.n > INT32_MAX)
        refuse("logits", "rows too long");
    const Tensor &tokens = tensor("tokens", tokens_o);
    on_device("tokens", tokens, logits);
    of_shape("tokens", tokens, lead_of(logits));
    switch (tokens.scalar_type()) {
    case at::kByte: s.token_bytes = 1; break;
    case at::kInt: s.token_bytes = 4; break;
    case at::kLong: s.token_bytes = 8; break;
    default: refuse("tokens", "expected uint8, int32 or int64");
    }
    if (!tokens.is_contiguous())
        refuse("tokens", "expected a contiguous tensor");
    s.tokens = tokens.data_ptr();
    if (given(mask_o)) {
        const Tensor &mask = tensor("mask", mask_o);
        on_device("mask", mask, logits);
        if (mask.scalar_type() != at::kBool)
            of_type("mask", mask, at::kByte);
        if (mask.sizes() == logits.sizes())
            s.mask_stride = rows_of("mask", mask).stride;
        else if (mask.dim() != 1 || mask.size(0) != s.r.n || !mask.is_contiguous())
            refuse("mask", "expected shape " + shape_text(logits.sizes()) + " or " + shape_text({s.r.n}));
        s.mask = (const uint8_t *)mask.data_ptr();
    }
    return s;
}

bool put(PyObject *dict, const char *key, const Tensor &t)
{
    PyObject *v = THPVariable_Wrap(t);
    if (!v)
        return false;
    const int rc = PyDict_SetItemString(dict, key, v);
    Py_DECREF(v);
    return rc == 0;
}

PyObject *log_probs(PyObject *const *a)
{
    const Tensor &logits = tensor("logits", a[0]);
    const LogpInputs s = logp_inputs(logits, a[1], a[2]);
    const long top = whole(a[3]), most = s.r.n < AV_MAX_TOP ? s.r.n : AV_MAX_TOP;
    if (top < 0 || top > most)
        refuse("top", "expected 0.." + std::to_string(most));
    Unlocked unlocked;
    const c10::cuda::CUDAGuard guard(logits.device());
    const at::IntArrayRef lead = lead_of(logits);
    const Tensor logp = make(lead, at::kFloat, logits), entropy = make(lead, at::kFloat, logits),
                 peak = make(lead, at::kFloat, logits), logz = make(lead, at::kFloat, logits);
    Tensor best, which;
    if (top) {
        at::DimVector shape(lead.begin(), lead.end());
        shape.push_back(top);
        best = make(shape, at::kFloat, logits);
        which = make(shape, at::kInt, logits);
    }
    check("av_log_probs",
          av_log_probs(s.r.rows, (int32_t)s.r.n, s.dtype, logits.data_ptr(), s.r.stride, s.tokens, s.token_bytes, s.mask,
                       s.mask_stride, (int32_t)top, (float *)logp.data_ptr(), (float *)entropy.data_ptr(),
                       (float *)peak.data_ptr(), (float *)logz.data_ptr(), top ? (float *)best.data_ptr() : nullptr,
                       top ? (int32_t *)which.data_ptr() : nullptr, stream_of(logits)));
    unlocked.end();
    PyObject *out = PyDict_New();
    if (!out || !put(out, "logp", logp) || !put(out, "entropy", entropy) || !put(out, "peak", peak) ||
        !put(out, "logz", logz) || (top && (!put(out, "top_logp", best) || !put(out, "top_index", which)))) {
        Py_XDECREF(out);
        return nullptr;
    }
    return out;
}

PyObject *log_probs_grad(PyObject *const *a)
{
    const Tensor &logits = tensor("logits", a[2]);
    const LogpInputs s = logp_inputs(logits, a[3], a[7]);
    const at::IntArrayRef lead = lead_of(logits);
    const float *dlogp = floats("dlogp", a[0], logits, lead), *dentropy = floats("dentropy", a[1], logits, lead);
    const Tensor &peak = dense("peak", a[4], logits, at::kFloat, lead), &logz = dense("logz", a[5], logits, at::kFloat, lead);
    const float *entropy = floats("entropy", a[6], logits, lead);
    Unlocked unlocked;
    const c10::cuda::CUDAGuard guard(logits.device());
    const Tensor dx = make(logits.sizes(), logits.scalar_type(), logits);
    check("av_log_probs_grad",
          av_log_probs_grad(s.r.rows, (int32_t)s.r.n, s.dtype, logits.data_ptr(), s.r.stride, s.tokens, s.token_bytes,
                            s.mask, s.mask_stride, dlogp, dentropy, (const float *)peak.data_ptr(),
                            (const float *)logz.data_ptr(), entropy, dx.data_ptr(), s.r.n, stream_of(logits)));
    unlocked.end();
    return THPVariable_Wrap(dx);
}

// ------------------------------------------------------------ gated feed-forward

struct FfnInputs {
    int dtype, act;
    Rows r;
    int64_t H;
};
FfnInputs ffn_inputs(const Tensor &x, const Tensor &w, PyObject *act)
{
    FfnInputs s;
    s.dtype = type_of("x", x);
    if (s.dtype == AV_F32)
        refuse("x", "expected bfloat16 or float16");
    const char *name = PyUnicode_Check(act) ? PyUnicode_AsUTF8(act) : nullptr;
    if (name && !strcmp(name, "silu"))
        s.act = AV_SILU;
    else if (name && !strcmp(name, "gelu"))
        s.act = AV_GELU;
    else
        refuse("act", "expected \"silu\" or \"gelu\"");
    s.r = rows_of("x", x);
    on_device("w", w, x);
    of_type("w", w, x.scalar_type());
    if (w.dim() != 3 || w.size(0) != 2 || w.size(2) != s.r.n || !w.is_contiguous())
        refuse("w", "expected a contiguous [2, H, " + std::to_string(s.r.n) + "] tensor");
    s.H = w.size(1);
    return s;
}

PyObject *gated_ffn(PyObject *const *a)
{
    const Tensor &x = tensor("x", a[0]), &w = tensor("w", a[1]);
    const FfnInputs s = ffn_inputs(x, w, a[2]);
    Unlocked unlocked;
    const c10::cuda::CUDAGuard guard(x.device());
    at::DimVector shape(x.sizes().begin(), x.sizes().end());
    shape.back() = s.H;
    const Tensor h = make(shape, x.scalar_type(), x);
    check("av_gated_ffn", av_gated_ffn(s.r.rows, s.r.n, s.H, s.dtype, s.act, x.data_ptr(), s.r.stride, w.data_ptr(),
                                       h.data_ptr(), s.H, stream_of(x)));
    unlocked.end();
    return THPVariable_Wrap(h);
}

PyObject *gated_ffn_grad(PyObject *const *a)
{
    const Tensor &dh = tensor("dh", a[0]), &x = tensor("x", a[1]), &w = tensor("w", a[2]);
    const FfnInputs s = ffn_inputs(x, w, a[3]);
    at::DimVector shape(x.sizes().begin(), x.sizes().end());
    shape.back() = s.H;
    on_device("dh", dh, x);
    of_type("dh", dh, x.scalar_type());
    of_shape("dh", dh, shape);
    int64_t need = 0;
    check("av_gated_ffn_work", av_gated_ffn_work(s.r.rows, s.r.n, s.H, &need));
    Unlocked unlocked;
    const c10::cuda::CUDAGuard guard(x.device());
    const Tensor dx = make(x.sizes(), x.scalar_type(), x), dw = make(w.sizes(), w.scalar_type(), w),
                 work = make({need}, at::kByte, x);
    check("av_gated_ffn_grad",
          av_gated_ffn_grad(s.r.rows, s.r.n, s.H, s.dtype, s.act, dh.data_ptr(), rows_of("dh", dh).stride, x.data_ptr(),
                            s.r.stride, w.data_ptr(), dx.data_ptr(), s.r.n, dw.data_ptr(), work.data_ptr(), need,
                            stream_of(x)));
    unlocked.end();
    return tuple({dx, dw});
}

// ------------------------------------------------------------ module

// Results are detached.  Where autograd would have recorded the call, it says so;
// false: the warning was made an error.
bool warn_detached(PyObject *const *args, Py_ssize_t n)
{
    if (!c10::GradMode::is_enabled())
        return true;
    for (Py_ssize_t k = 0; k < n; ++k)
        if (THPVariable_Check(args[k]) && THPVariable_Unpack(args[k]).requires_grad())
            return PyErr_WarnEx(PyExc_UserWarning,
                                "policy operators are not recorded by autograd: the results are detached from arguments "
                                "that require gradients (call them under torch.no_grad() or in a torch.autograd.Function)",
                                2) == 0;
    return true;
}

// A function of exactly kArgs arguments; no exception leaves it.
template <PyObject *(*fn)(PyObject *const *), Py_ssize_t kArgs>
PyObject *call(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != kArgs) {
        PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", kArgs, n);
        return nullptr;
    }
    HANDLE_TH_ERRORS
    if (!warn_detached(args, n))
        return nullptr;
    try {
        return fn(args);
    } catch (const Refused &e) {
        PyErr_SetString(PyExc_ValueError, e.what());
    } catch (const Failed &e) {
        if (PyObject *v = PyObject_CallFunction(g_error, "sis", e.fn, e.status, av_strerror(e.status))) {
            PyErr_SetObject(g_error, v);
            Py_DECREF(v);
        }
    }
    return nullptr;
    END_HANDLE_TH_ERRORS
}

PyObject *set_error(PyObject *, PyObject *type)
{
    Py_INCREF(type);
    Py_XDECREF(g_error);
    g_error = type;
    Py_RETURN_NONE;
}

#define AV_METHOD(name, args) \
    {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(&call<name, args>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {AV_METHOD(layer_norm, 4),
                         AV_METHOD(layer_norm_grad, 5),
                         AV_METHOD(scan, 5),
                         AV_METHOD(scan_grad, 6),
                         AV_METHOD(log_probs, 4),
                         AV_METHOD(log_probs_grad, 8),
                         AV_METHOD(gated_ffn, 3),
                         AV_METHOD(gated_ffn_grad, 4),
                         {"set_error", set_error, METH_O, nullptr},
                         {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_policy", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__policy() { return PyModule_Create(&module); }
