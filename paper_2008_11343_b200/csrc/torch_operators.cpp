// The operators beside the step as functions of torch tensors: checks, output allocation and the C call, without an interpreter's
// overhead per tensor and attribute (a forward norm of one row: 16 us through ctypes, of which the launch is 3; the addresses
// and checks of 400 gradients: 95 us).  A CPython extension, loaded by operators.py, which hands it the addresses of the C entry points
// of the library it has loaded.  Nothing here computes.

#include <Python.h>
#include <ATen/ATen.h>
#include <ATen/cuda/CUDAEvent.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAGraphsC10Utils.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <memory>
#include <sstream>
#include <stdexcept>
#include <string>
#include <vector>

#include "apms.h"

namespace {

// The library's entry points (bind()), and the exception for a status that is not APMS_OK.
decltype(&apms_tensors_create) c_create;
decltype(&apms_tensors_workspace_bytes) c_workspace_bytes;
decltype(&apms_tensors_bind) c_bind;
decltype(&apms_tensors_destroy) c_destroy;
decltype(&apms_tensors_scratch_bytes) c_scratch_bytes;
decltype(&apms_tensors_use_scratch) c_use_scratch;
decltype(&apms_grad_norm) c_grad_norm;
decltype(&apms_clip_grads) c_clip_grads;
decltype(&apms_rms_norm) c_rms_norm;
decltype(&apms_rms_norm_backward_workspace_bytes) c_backward_bytes;
decltype(&apms_rms_norm_backward) c_rms_norm_backward;
decltype(&apms_embedding) c_embedding;
decltype(&apms_embedding_backward_workspace_bytes) c_embedding_bytes;
decltype(&apms_embedding_backward) c_embedding_backward;
decltype(&apms_dropout) c_dropout;
decltype(&apms_gated_scan_workspace_bytes) c_scan_bytes;
decltype(&apms_gated_scan_starts_bytes) c_starts_bytes;
decltype(&apms_gated_scan) c_gated_scan;
decltype(&apms_gated_scan_backward) c_gated_scan_backward;
decltype(&apms_gated_scan_step) c_gated_scan_step;
decltype(&apms_last_error) c_last_error;
PyObject* g_error;

struct Refused : std::runtime_error { using std::runtime_error::runtime_error; };   // a ValueError
struct Raised {};                                                                     // the Python error is set

template <class... Parts>
[[noreturn]] void refuse(const Parts&... parts)
{
    std::ostringstream s;
    (s << ... << parts);
    throw Refused(s.str());
}

[[noreturn]] void fail(apms_status st, const std::string& message)
{
    PyObject* e = PyObject_CallFunction(g_error, "is", (int)st, message.c_str());
    if (e) { PyErr_SetObject(g_error, e); Py_DECREF(e); }
    throw Raised();
}

void check(apms_status st)
{
    if (st != APMS_OK) fail(st, c_last_error(nullptr));
}

template <class Body>
PyObject* guarded(Body body)
{
    try {
        at::AutoDispatchBelowADInplaceOrView below;                                   // outputs are plain memory
        return body();
    } catch (const Refused& e) {
        PyErr_SetString(PyExc_ValueError, e.what());
    } catch (const Raised&) {
    } catch (const c10::Error& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what_without_backtrace());
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

const at::Tensor& tensor(PyObject* o, const char* what)
{
    if (!THPVariable_Check(o)) refuse(what, " must be a torch tensor");
    return THPVariable_Unpack(o);
}

int type_of(const at::Tensor& t, const char* what)
{
    switch (t.scalar_type()) {
        case at::kFloat: return APMS_GRAD_F32;
        case at::kBFloat16: return APMS_GRAD_BF16;
        case at::kHalf: return APMS_GRAD_F16;
        default: refuse(what, " is ", t.scalar_type(), ": float32, bfloat16 or float16 is needed");
    }
}

// A tensor as rows of `width` consecutive elements (copied only where its strides cannot be read that way).
struct Rows {
    at::Tensor kept;
    const void* p;
    int64_t stride;
};
Rows rows_of(const at::Tensor& t, const char* what, int64_t width, const at::Device& device, int64_t rows)
{
    if (t.device() != device) refuse(what, " lies on ", t.device(), ", not on ", device);
    if (t.dim() == 0 || t.size(-1) != width || t.numel() != rows * width) refuse(what, " of shape ", t.sizes(), " does not fit ", rows, " rows of width ", width);
    if (t.is_contiguous()) return {at::Tensor(), t.const_data_ptr(), width};
    at::Tensor m = t.reshape({-1, width});
    if ((width > 1 && m.stride(1) != 1) || (m.size(0) > 1 && m.stride(0) < width)) m = m.contiguous();
    const void* p = m.const_data_ptr();
    const int64_t stride = m.size(0) > 1 ? m.stride(0) : width;
    return {std::move(m), p, stride};
}

void check_weight(const at::Tensor& w, int64_t width, const at::Tensor& x)
{
    if (w.device() != x.device() || w.dim() != 1 || w.size(0) != width || !w.is_contiguous() || (w.scalar_type() != x.scalar_type() && w.scalar_type() != at::kFloat))
        refuse("weight must be ", width, " contiguous elements on ", x.device(), ", of ", x.scalar_type(), " or float32");
}

int64_t width_of(const at::Tensor& x, const char* what)
{
    if (!x.is_cuda()) refuse(what, " must be a CUDA tensor; there is no CPU path");
    if (x.dim() == 0 || x.size(-1) == 0) refuse(what, " of shape ", x.sizes(), " has no rows of at least one element");
    return x.size(-1);
}

// at::empty without the dispatcher's share of its time
at::Tensor empty(at::IntArrayRef sizes, at::ScalarType type, const at::Device& device) { return at::Tensor(at::detail::empty_cuda(sizes, type, device, std::nullopt)); }

// Whether the current stream's work is being captured into a graph.
bool capturing() { return c10::cuda::currentStreamCaptureStatusMayInitCtx() != c10::cuda::CaptureStatus::None; }

PyObject* wrap(at::Tensor t) { return THPVariable_Wrap(std::move(t)); }

PyObject* tuple_of(std::initializer_list<PyObject*> items)
{
    PyObject* r = PyTuple_New((Py_ssize_t)items.size());
    Py_ssize_t k = 0;
    for (PyObject* o : items) PyTuple_SET_ITEM(r, k++, o);
    return r;
}

// rms_norm(x, weight, residual or None, eps, group or -1): (y, h, rstd), or with a group (q, scales, h, rstd)
PyObject* rms_norm(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject* {
        if (n != 5) refuse("rms_norm takes 5 arguments");
        const at::Tensor& x = tensor(args[0], "x");
        const at::Tensor& weight = tensor(args[1], "weight");
        const double eps = PyFloat_AsDouble(args[3]);
        const int64_t group = PyLong_AsLongLong(args[4]);
        if (PyErr_Occurred()) throw Raised();
        apms_rms_norm_args a = {};
        a.width = width_of(x, "x");
        a.rows = x.numel() / a.width;
        a.x_type = (apms_grad_type)type_of(x, "x");
        check_weight(weight, a.width, x);
        const c10::cuda::OptionalCUDAGuard on(x.device());
        const Rows xr = rows_of(x, "x", a.width, x.device(), a.rows);
        a.x = xr.p; a.x_stride = xr.stride;
        a.weight = weight.const_data_ptr(); a.weight_type = (apms_grad_type)type_of(weight, "weight");
        a.eps = (float)eps;
        Rows rr;
        at::Tensor h;
        if (args[2] != Py_None) {
            const at::Tensor& residual = tensor(args[2], "residual");
            if (residual.sizes() != x.sizes() || (residual.scalar_type() != x.scalar_type() && residual.scalar_type() != at::kFloat))
                refuse("residual must have x's shape ", x.sizes(), ", and its type or float32: ", residual.sizes(), ", ", residual.scalar_type());
            rr = rows_of(residual, "residual", a.width, x.device(), a.rows);
            h = empty(x.sizes(), residual.scalar_type(), x.device());
            a.residual = rr.p; a.residual_stride = rr.stride; a.residual_type = (apms_grad_type)type_of(residual, "residual");
            a.h = h.data_ptr();
        }
        at::Tensor rstd = empty(x.sizes().slice(0, x.dim() - 1), at::kFloat, x.device()), scales;
        at::Tensor y = empty(x.sizes(), group < 0 ? x.scalar_type() : at::kFloat8_e4m3fn, x.device());
        if (group >= 0) {
            std::vector<int64_t> shape(x.sizes().begin(), x.sizes().end());
            const int64_t size = group ? group : a.width;
            shape.back() = (a.width + size - 1) / size;
            scales = empty(shape, at::kFloat, x.device());
            a.scales = (float*)scales.data_ptr();
            a.group = group;
        }
        a.rstd = (float*)rstd.data_ptr();
        a.y = y.data_ptr();
        if (a.rows) check(c_rms_norm(&a, c10::cuda::getCurrentCUDAStream(x.get_device()).stream()));
        if (args[2] == Py_None) Py_INCREF(args[0]);
        PyObject* kept = args[2] == Py_None ? args[0] : wrap(std::move(h));
        if (group < 0) return tuple_of({wrap(std::move(y)), kept, wrap(std::move(rstd))});
        return tuple_of({wrap(std::move(y)), wrap(std::move(scales)), kept, wrap(std::move(rstd))});
    });
}

// rms_norm_backward(dy, h, weight, rstd, dh or None): (dx, dweight), and the residual's gradient where h's type is not dy's
PyObject* rms_norm_backward(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject* {
        if (n != 5) refuse("rms_norm_backward takes 5 arguments");
        const at::Tensor& dy = tensor(args[0], "dy");
        const at::Tensor& h = tensor(args[1], "h");
        const at::Tensor& weight = tensor(args[2], "weight");
        const at::Tensor& rstd = tensor(args[3], "rstd");
        apms_rms_norm_backward_args a = {};
        a.width = width_of(dy, "dy");
        a.rows = dy.numel() / a.width;
        a.dy_type = (apms_grad_type)type_of(dy, "dy");
        const bool wide = h.scalar_type() != dy.scalar_type();
        if (wide && h.scalar_type() != at::kFloat) refuse("h must have dy's type or float32, not ", h.scalar_type());
        check_weight(weight, a.width, dy);
        if (rstd.scalar_type() != at::kFloat || rstd.numel() != a.rows || !rstd.is_contiguous() || rstd.device() != dy.device())
            refuse("rstd must be ", a.rows, " contiguous float32 values on ", dy.device());
        const c10::cuda::OptionalCUDAGuard on(dy.device());
        const Rows dyr = rows_of(dy, "dy", a.width, dy.device(), a.rows), hr = rows_of(h, "h", a.width, dy.device(), a.rows);
        Rows dhr;
        a.dy = dyr.p; a.dy_stride = dyr.stride;
        a.h = hr.p; a.h_stride = hr.stride; a.h_type = (apms_grad_type)type_of(h, "h");
        a.weight = weight.const_data_ptr(); a.weight_type = (apms_grad_type)type_of(weight, "weight");
        a.rstd = (const float*)rstd.const_data_ptr();
        if (args[4] != Py_None) {
            const at::Tensor& dh = tensor(args[4], "dh");
            if (dh.scalar_type() != h.scalar_type()) refuse("dh must have h's type ", h.scalar_type(), ", not ", dh.scalar_type());
            dhr = rows_of(dh, "dh", a.width, dy.device(), a.rows);
            a.dh = dhr.p; a.dh_stride = dhr.stride;
        }
        at::Tensor dx = empty(dy.sizes(), dy.scalar_type(), dy.device()), dweight = empty(weight.sizes(), weight.scalar_type(), dy.device()), dresidual;
        if (wide) dresidual = empty(dy.sizes(), h.scalar_type(), dy.device());
        a.workspace_bytes = c_backward_bytes(a.rows, a.width);
        at::Tensor workspace = empty({(int64_t)a.workspace_bytes}, at::kByte, dy.device());
        a.dx = dx.data_ptr(); a.dweight = dweight.data_ptr(); a.dresidual = wide ? dresidual.data_ptr() : nullptr;
        a.workspace_dev = workspace.data_ptr();
        check(c_rms_norm_backward(&a, c10::cuda::getCurrentCUDAStream(dy.get_device()).stream()));
        if (wide) return tuple_of({wrap(std::move(dx)), wrap(std::move(dweight)), wrap(std::move(dresidual))});
        return tuple_of({wrap(std::move(dx)), wrap(std::move(dweight))});
    });
}

// ------------------------------------------------------------------------------------------ layers

// Autograd's notice that a tensor was written: a graph that has saved it raises in its backward pass.  (Inference tensors have no version, and
// no graph can save them.)
void note_write(at::TensorImpl* t)
{
    if (!t->is_inference()) t->bump_version();
}

// None, or the element type that a torch.dtype names.
at::ScalarType dtype_of(PyObject* o, at::ScalarType otherwise)
{
    if (o == Py_None) return otherwise;
    if (!THPDtype_Check(o)) refuse("dtype must be a torch.dtype");
    const at::ScalarType t = reinterpret_cast<THPDtype*>(o)->scalar_type;
    if (t != at::kFloat && t != at::kBFloat16 && t != at::kHalf) refuse("dtype is ", t, ": float32, bfloat16 or float16 is needed");
    return t;
}
apms_grad_type type_of(at::ScalarType t) { return t == at::kFloat ? APMS_GRAD_F32 : t == at::kBFloat16 ? APMS_GRAD_BF16 : APMS_GRAD_F16; }

// Tokens as consecutive numbers.
at::Tensor tokens_of(PyObject* o, const at::Device& device)
{
    const at::Tensor& t = tensor(o, "tokens");
    if (t.scalar_type() != at::kLong && t.scalar_type() != at::kInt) refuse("tokens are ", t.scalar_type(), ": int64 or int32 is needed");
    if (t.device() != device) refuse("tokens lie on ", t.device(), ", not on ", device);
    return t.contiguous();
}

// embedding(tokens, weight, scale, dtype or None): out
PyObject* embedding(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject* {
        if (n != 4) refuse("embedding takes 4 arguments");
        const at::Tensor& weight = tensor(args[1], "weight");
        const double scale = PyFloat_AsDouble(args[2]);
        if (PyErr_Occurred()) throw Raised();
        apms_embedding_args a = {};
        a.width = width_of(weight, "weight");
        if (weight.dim() != 2 || weight.size(0) == 0) refuse("weight must have the shape (vocabulary, width), not ", weight.sizes());
        a.vocab = weight.size(0);
        a.weight_type = (apms_grad_type)type_of(weight, "weight");
        const at::ScalarType type = dtype_of(args[3], weight.scalar_type());
        const c10::cuda::OptionalCUDAGuard on(weight.device());
        const at::Tensor tokens = tokens_of(args[0], weight.device());
        const Rows w = rows_of(weight, "weight", a.width, weight.device(), a.vocab);
        std::vector<int64_t> shape(tokens.sizes().begin(), tokens.sizes().end());
        shape.push_back(a.width);
        at::Tensor out = empty(shape, type, weight.device());
        a.count = tokens.numel(); a.tokens = tokens.const_data_ptr(); a.token_bytes = (int)tokens.element_size();
        a.weight = w.p; a.weight_stride = w.stride; a.scale = (float)scale;
        a.out = out.data_ptr(); a.out_type = type_of(type);
        check(c_embedding(&a, c10::cuda::getCurrentCUDAStream(weight.get_device()).stream()));
        return wrap(std::move(out));
    });
}

// embedding_backward(dout, tokens, vocabulary, scale, dtype or None, out or None): dweight
PyObject* embedding_backward(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject* {
        if (n != 6) refuse("embedding_backward takes 6 arguments");
        const at::Tensor& dout = tensor(args[0], "dout");
        apms_embedding_backward_args a = {};
        a.vocab = PyLong_AsLongLong(args[2]);
        const double scale = PyErr_Occurred() ? 0.0 : PyFloat_AsDouble(args[3]);
        if (PyErr_Occurred()) throw Raised();
        a.width = width_of(dout, "dout");
        if (a.vocab < 1) refuse("the vocabulary has at least one row, not ", a.vocab);
        a.dout_type = (apms_grad_type)type_of(dout, "dout");
        const c10::cuda::OptionalCUDAGuard on(dout.device());
        const at::Tensor tokens = tokens_of(args[1], dout.device());
        a.count = tokens.numel(); a.tokens = tokens.const_data_ptr(); a.token_bytes = (int)tokens.element_size();
        if (dout.sizes().slice(0, dout.dim() - 1) != tokens.sizes()) refuse("dout of shape ", dout.sizes(), " does not fit tokens of shape ", tokens.sizes());
        const Rows d = rows_of(dout, "dout", a.width, dout.device(), a.count);
        a.dout = d.p; a.dout_stride = d.stride; a.scale = (float)scale;
        at::Tensor out;
        if (args[5] != Py_None) {
            out = tensor(args[5], "out");
            if (out.device() != dout.device() || !out.is_contiguous() || out.dim() != 2 || out.size(0) != a.vocab || out.size(1) != a.width)
                refuse("out must be contiguous, of shape (", a.vocab, ", ", a.width, ") on ", dout.device(), ", not ", out.sizes());
            const char *o0 = static_cast<const char*>(out.const_data_ptr()), *o1 = o0 + out.nbytes();
            const char *t0 = static_cast<const char*>(a.tokens), *d0 = static_cast<const char*>(a.dout);
            if (a.count && ((t0 < o1 && o0 < t0 + tokens.nbytes()) || (d0 < o1 && o0 < d0 + ((a.count - 1) * a.dout_stride + a.width) * (int64_t)dout.element_size())))
                refuse("out shares memory with dout or tokens");
            type_of(out, "out");
            if (args[4] != Py_None && dtype_of(args[4], out.scalar_type()) != out.scalar_type()) refuse("out is ", out.scalar_type(), ", not of dtype");
        } else {
            out = empty({a.vocab, a.width}, dtype_of(args[4], dout.scalar_type()), dout.device());
        }
        a.dweight = out.data_ptr(); a.dweight_type = type_of(out.scalar_type());
        a.workspace_bytes = c_embedding_bytes(a.count, a.vocab, a.width);
        at::Tensor workspace = empty({(int64_t)a.workspace_bytes}, at::kByte, dout.device());
        a.workspace_dev = workspace.data_ptr();
        check(c_embedding_backward(&a, c10::cuda::getCurrentCUDAStream(dout.get_device()).stream()));
        if (args[5] != Py_None) note_write(out.unsafeGetTensorImpl());
        return wrap(std::move(out));
    });
}

// dropout(x, p, rng, site, residual or None, dtype or None, keep): h, or with keep (h, the numbers used)
PyObject* dropout(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject* {
        if (n != 7) refuse("dropout takes 7 arguments");
        const at::Tensor& x = tensor(args[0], "x");
        const at::Tensor& rng = tensor(args[2], "rng");
        apms_dropout_args a = {};
        a.p = PyFloat_AsDouble(args[1]);
        a.site = PyErr_Occurred() ? 0 : PyLong_AsLongLong(args[3]);
        const int keep = PyErr_Occurred() ? 0 : PyObject_IsTrue(args[6]);
        if (PyErr_Occurred()) throw Raised();
        a.width = width_of(x, "x");
        a.rows = x.numel() / a.width;
        a.x_type = (apms_grad_type)type_of(x, "x");
        if (rng.scalar_type() != at::kLong || rng.numel() != 2 || !rng.is_contiguous() || rng.device() != x.device()) refuse("rng must be two contiguous int64 numbers (seed, step) on ", x.device());
        const c10::cuda::OptionalCUDAGuard on(x.device());
        const Rows xr = rows_of(x, "x", a.width, x.device(), a.rows);
        a.x = xr.p; a.x_stride = xr.stride;
        a.rng_dev = static_cast<const int64_t*>(rng.const_data_ptr());
        at::ScalarType type = dtype_of(args[5], x.scalar_type());
        Rows rr;
        if (args[4] != Py_None) {
            const at::Tensor& residual = tensor(args[4], "residual");
            if (residual.sizes() != x.sizes() || (residual.scalar_type() != x.scalar_type() && residual.scalar_type() != at::kFloat))
                refuse("residual must have x's shape ", x.sizes(), ", and its type or float32: ", residual.sizes(), ", ", residual.scalar_type());
            rr = rows_of(residual, "residual", a.width, x.device(), a.rows);
            a.residual = rr.p; a.residual_stride = rr.stride;
            type = residual.scalar_type();
        }
        at::Tensor h = empty(x.sizes(), type, x.device()), used;
        a.h = h.data_ptr(); a.h_type = type_of(type);
        if (keep) {
            used = empty({2}, at::kLong, x.device());
            a.used_dev = static_cast<int64_t*>(used.data_ptr());
        }
        check(c_dropout(&a, c10::cuda::getCurrentCUDAStream(x.get_device()).stream()));
        if (!keep) return wrap(std::move(h));
        return tuple_of({wrap(std::move(h)), wrap(std::move(used))});
    });
}

// A tensor (batch, steps, width) with consecutive channels, copied only where its last stride is not 1.
struct Sequences {
    at::Tensor kept;
    const void* p;
    int64_t batch, step;
};
Sequences sequences_of(const at::Tensor& t, const char* what, const at::Tensor& like)
{
    if (t.device() != like.device() || t.sizes() != like.sizes() || t.scalar_type() != like.scalar_type())
        refuse(what, " must have the shape ", like.sizes(), ", type ", like.scalar_type(), " and device ", like.device(), ": ", t.sizes(), ", ", t.scalar_type(), ", ", t.device());
    Sequences s = {t.size(2) == 1 || t.stride(2) == 1 ? t : t.contiguous(), nullptr, 0, 0};
    s.p = s.kept.const_data_ptr(); s.batch = s.kept.stride(0); s.step = s.kept.stride(1);
    return s;
}

// A state (batch, width): contiguous float32.
at::Tensor state_of(PyObject* o, const char* what, int64_t batch, int64_t width, const at::Device& device)
{
    const at::Tensor& t = tensor(o, what);
    if (t.scalar_type() != at::kFloat || t.dim() != 2 || t.size(0) != batch || t.size(1) != width || t.device() != device)
        refuse(what, " must be float32 of shape (", batch, ", ", width, ") on ", device, ": ", t.sizes(), ", ", t.scalar_type(), ", ", t.device());
    return t.contiguous();
}

void check_sequences(const at::Tensor& x)
{
    if (!x.is_cuda()) refuse("x must be a CUDA tensor; there is no CPU path");
    if (x.dim() != 3 || x.size(2) == 0) refuse("x must have the shape (batch, steps, width), not ", x.sizes());
}

// The rows of starts hold whole slabs of channels.
std::vector<int64_t> starts_shape(const at::Tensor& x)
{
    const int64_t row = (int64_t)(c_starts_bytes(1, 1, x.size(2)) / sizeof(float)), bytes = (int64_t)c_starts_bytes(1, x.size(1), x.size(2));
    return {x.size(0), row ? bytes / (int64_t)sizeof(float) / row : 0, row};
}

// The call's workspace, where it needs one.
template <class Args>
at::Tensor workspace_of(Args& a, const at::Device& device)
{
    a.workspace_bytes = c_scan_bytes(a.batch, a.steps, a.width, a.type);
    if (!a.workspace_bytes) return at::Tensor();
    at::Tensor w = empty({(int64_t)a.workspace_bytes}, at::kByte, device);
    a.workspace_dev = w.data_ptr();
    return w;
}

// gated_scan(x, gate, state or None, keep): (h, last, starts or None)
PyObject* gated_scan(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject* {
        if (n != 4) refuse("gated_scan takes 4 arguments");
        const at::Tensor& x = tensor(args[0], "x");
        const int keep = PyObject_IsTrue(args[3]);
        if (PyErr_Occurred()) throw Raised();
        check_sequences(x);
        apms_gated_scan_args a = {};
        a.batch = x.size(0); a.steps = x.size(1); a.width = x.size(2);
        a.type = (apms_grad_type)type_of(x, "x");
        const c10::cuda::OptionalCUDAGuard on(x.device());
        const Sequences xs = sequences_of(x, "x", x), gs = sequences_of(tensor(args[1], "gate"), "gate", x);
        a.x = xs.p; a.x_batch_stride = xs.batch; a.x_step_stride = xs.step;
        a.gate = gs.p; a.gate_batch_stride = gs.batch; a.gate_step_stride = gs.step;
        at::Tensor state, starts;
        if (args[2] != Py_None) {
            state = state_of(args[2], "state", a.batch, a.width, x.device());
            a.state = static_cast<const float*>(state.const_data_ptr());
        }
        at::Tensor h = empty(x.sizes(), x.scalar_type(), x.device()), last = empty({a.batch, a.width}, at::kFloat, x.device());
        if (keep) {
            starts = empty(starts_shape(x), at::kFloat, x.device());
            a.starts = static_cast<float*>(starts.data_ptr());
        }
        a.h = h.data_ptr(); a.last = static_cast<float*>(last.data_ptr());
        const at::Tensor workspace = workspace_of(a, x.device());
        check(c_gated_scan(&a, c10::cuda::getCurrentCUDAStream(x.get_device()).stream()));
        if (!keep) { Py_INCREF(Py_None); return tuple_of({wrap(std::move(h)), wrap(std::move(last)), Py_None}); }
        return tuple_of({wrap(std::move(h)), wrap(std::move(last)), wrap(std::move(starts))});
    });
}

// gated_scan_backward(dh, x, gate, starts, dlast or None): (dx, dgate, dstate)
PyObject* gated_scan_backward(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject* {
        if (n != 5) refuse("gated_scan_backward takes 5 arguments");
        const at::Tensor& x = tensor(args[1], "x");
        const at::Tensor& starts = tensor(args[3], "starts");
        check_sequences(x);
        apms_gated_scan_backward_args a = {};
        a.batch = x.size(0); a.steps = x.size(1); a.width = x.size(2);
        a.type = (apms_grad_type)type_of(x, "x");
        const c10::cuda::OptionalCUDAGuard on(x.device());
        const Sequences xs = sequences_of(x, "x", x), gs = sequences_of(tensor(args[2], "gate"), "gate", x), ds = sequences_of(tensor(args[0], "dh"), "dh", x);
        a.x = xs.p; a.x_batch_stride = xs.batch; a.x_step_stride = xs.step;
        a.gate = gs.p; a.gate_batch_stride = gs.batch; a.gate_step_stride = gs.step;
        a.dh = ds.p; a.dh_batch_stride = ds.batch; a.dh_step_stride = ds.step;
        if (starts.scalar_type() != at::kFloat || starts.device() != x.device() || !starts.is_contiguous() || starts.sizes() != at::IntArrayRef(starts_shape(x)))
            refuse("starts must be what gated_scan_forward kept for x of shape ", x.sizes());
        a.starts = static_cast<const float*>(starts.const_data_ptr());
        at::Tensor dlast;
        if (args[4] != Py_None) {
            dlast = state_of(args[4], "dlast", a.batch, a.width, x.device());
            a.dlast = static_cast<const float*>(dlast.const_data_ptr());
        }
        at::Tensor dx = empty(x.sizes(), x.scalar_type(), x.device()), dgate = empty(x.sizes(), x.scalar_type(), x.device()), dstate = empty({a.batch, a.width}, at::kFloat, x.device());
        a.dx = dx.data_ptr(); a.dgate = dgate.data_ptr(); a.dstate = static_cast<float*>(dstate.data_ptr());
        const at::Tensor workspace = workspace_of(a, x.device());
        check(c_gated_scan_backward(&a, c10::cuda::getCurrentCUDAStream(x.get_device()).stream()));
        return tuple_of({wrap(std::move(dx)), wrap(std::move(dgate)), wrap(std::move(dstate))});
    });
}

// gated_scan_step(x, gate, state, out or None): h; the new states in out, or in state
PyObject* gated_scan_step(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject* {
        if (n != 4) refuse("gated_scan_step takes 4 arguments");
        const at::Tensor& x = tensor(args[0], "x");
        const at::Tensor& gate = tensor(args[1], "gate");
        const at::Tensor& state = tensor(args[2], "state");
        const at::Tensor& next = args[3] == Py_None ? state : tensor(args[3], "out");
        apms_gated_scan_step_args a = {};
        a.width = width_of(x, "x");
        if (x.dim() != 2) refuse("x must have the shape (batch, width), not ", x.sizes());
        a.batch = x.size(0);
        a.type = (apms_grad_type)type_of(x, "x");
        if (gate.scalar_type() != x.scalar_type()) refuse("gate must have x's type ", x.scalar_type(), ", not ", gate.scalar_type());
        for (const at::Tensor* t : {&state, &next})
            if (t->scalar_type() != at::kFloat || t->sizes() != x.sizes() || !t->is_contiguous() || t->device() != x.device())
                refuse("state and out must be contiguous float32 of shape ", x.sizes(), " on ", x.device());
        const c10::cuda::OptionalCUDAGuard on(x.device());
        const Rows xr = rows_of(x, "x", a.width, x.device(), a.batch), gr = rows_of(gate, "gate", a.width, x.device(), a.batch);
        a.x = xr.p; a.x_stride = xr.stride; a.gate = gr.p; a.gate_stride = gr.stride;
        at::Tensor h = empty(x.sizes(), x.scalar_type(), x.device());
        a.state = static_cast<const float*>(state.const_data_ptr());
        a.next = static_cast<float*>(next.data_ptr());
        if (a.state != a.next && a.state < a.next + next.numel() && a.next < a.state + state.numel()) refuse("out shares part of state's memory");
        auto meets = [&](const Rows& r) {
            const char *p0 = static_cast<const char*>(r.p), *n0 = reinterpret_cast<const char*>(a.next);
            return a.batch && p0 < n0 + next.nbytes() && n0 < p0 + ((a.batch - 1) * r.stride + a.width) * (int64_t)x.element_size();
        };
        if (meets(xr) || meets(gr)) refuse("the new states share memory with x or gate");
        a.h = h.data_ptr();
        check(c_gated_scan_step(&a, c10::cuda::getCurrentCUDAStream(x.get_device()).stream()));
        note_write(next.unsafeGetTensorImpl());
        return wrap(std::move(h));
    });
}

// ------------------------------------------------------------------------------------------ many tensors

struct Layout {
    int64_t numel;
    at::ScalarType type;
    std::vector<int64_t> sizes, strides;             // empty: contiguous
    bool turned;                                     // one run of memory, its elements in another order than their indexes'
};

struct TensorList {
    apms_tensors* list = nullptr;
    std::vector<Layout> layout;
    std::vector<void*> addresses;                    // of the running call
    std::vector<at::TensorImpl*> written;            // ... and the tensors that it writes in place
    int64_t numel = 0;
    bool turned = false;                             // some tensor's layout is
    at::Device device{at::kCUDA, 0};
    at::Tensor workspace;
    c10::cuda::CUDAStream stream = c10::cuda::getDefaultCUDAStream(0);
    ~TensorList() { if (list) c_destroy(list); }
};

constexpr const char* kListName = "apms tensor list";

struct Sequence {
    PyObject* fast;
    explicit Sequence(PyObject* o) : fast(PySequence_Fast(o, "the tensors must be a sequence")) { if (!fast) throw Raised(); }
    ~Sequence() { Py_DECREF(fast); }
    Py_ssize_t size() const { return PySequence_Fast_GET_SIZE(fast); }
    const at::Tensor& operator[](Py_ssize_t k) const { return tensor(PySequence_Fast_GET_ITEM(fast, k), "each of the tensors"); }
};

// (elements of a row, distance between rows) of a tensor that is contiguous or rows of consecutive elements
std::pair<int64_t, int64_t> row_layout(const at::Tensor& t)
{
    if (t.is_contiguous()) { const int64_t n = std::max<int64_t>(1, t.numel()); return {n, n}; }
    const int64_t cols = t.size(-1);
    int64_t step = -1, rows = 1;                     // distance between rows (-1: one row so far), rows it has been seen to reach
    bool fits = t.stride(-1) == 1 || cols == 1;
    for (int64_t d = t.dim() - 2; d >= 0; --d) {
        if (t.size(d) == 1) continue;
        if (step < 0) step = t.stride(d);
        else fits = fits && t.stride(d) == step * rows;
        rows *= t.size(d);
    }
    if (step < 0) step = cols;
    if (!fits || step < cols) refuse("a tensor of shape ", t.sizes(), " and strides ", t.strides(), " is no rows of consecutive elements; use .contiguous()");
    return {cols, step};
}

PyObject* row_layout_of(PyObject*, PyObject* o)
{
    return guarded([&]() -> PyObject* {
        const auto r = row_layout(tensor(o, "t"));
        return Py_BuildValue("LL", (long long)r.first, (long long)r.second);
    });
}

PyObject* list_create(PyObject*, PyObject* tensors)
{
    return guarded([&]() -> PyObject* {
        const Sequence ts(tensors);
        if (ts.size() == 0) refuse("a TensorList needs at least one tensor");
        if (!ts[0].is_cuda()) refuse("the tensors must be CUDA tensors; there is no CPU path");
        std::unique_ptr<TensorList> self(new TensorList());
        self->device = ts[0].device();
        std::vector<int64_t> numel, cols, strides;
        std::vector<apms_grad_type> types;
        for (Py_ssize_t k = 0; k < ts.size(); ++k) {
            const at::Tensor& t = ts[k];
            if (t.device() != self->device) refuse("the tensors of a TensorList lie on one CUDA device: ", t.device(), " and ", self->device);
            const bool turned = !t.is_contiguous() && t.is_non_overlapping_and_dense();
            const auto r = turned ? std::pair<int64_t, int64_t>(t.numel(), t.numel()) : row_layout(t);
            numel.push_back(t.numel()); cols.push_back(r.first); strides.push_back(r.second);
            types.push_back((apms_grad_type)type_of(t, "a tensor"));
            Layout l = {t.numel(), t.scalar_type(), {}, {}, turned};
            if (!t.is_contiguous()) { l.sizes = t.sizes().vec(); l.strides = t.strides().vec(); }
            self->layout.push_back(std::move(l));
            self->numel += t.numel();
            self->turned |= turned;
        }
        self->addresses.resize(numel.size());
        check(c_create(&self->list, (int)numel.size(), numel.data(), types.data(), cols.data(), strides.data()));
        const c10::cuda::OptionalCUDAGuard on(self->device);
        if (capturing()) refuse("a TensorList is built before a graph's capture, not within it");
        self->stream = c10::cuda::getCurrentCUDAStream(self->device.index());
        const size_t bytes = c_workspace_bytes(self->list);
        self->workspace = empty({(int64_t)bytes}, at::kByte, self->device);
        check(c_bind(self->list, self->workspace.data_ptr(), bytes, self->stream.stream()));
        const int64_t total = self->numel;
        PyObject* capsule = PyCapsule_New(self.get(), kListName, [](PyObject* c) { delete static_cast<TensorList*>(PyCapsule_GetPointer(c, kListName)); });
        if (!capsule) throw Raised();
        self.release();
        return Py_BuildValue("NL", capsule, (long long)total);
    });
}

TensorList& list_of(PyObject* capsule)
{
    void* p = PyCapsule_GetPointer(capsule, kListName);
    if (!p) throw Raised();
    return *static_cast<TensorList*>(p);
}

// The tensors' addresses, once they are found to be laid out as the list's are.
void take_addresses(TensorList& self, const Sequence& ts, bool written)
{
    if (ts.size() != (Py_ssize_t)self.layout.size()) refuse("the list has ", self.layout.size(), " tensors, not ", ts.size());
    self.written.clear();
    for (Py_ssize_t k = 0; k < ts.size(); ++k) {
        const at::Tensor& t = ts[k];
        const Layout& l = self.layout[k];
        if (t.numel() != l.numel || t.scalar_type() != l.type) refuse("tensor ", k, " has ", t.numel(), " elements of ", t.scalar_type(), ", the list's ", l.numel, " of ", l.type);
        if (l.sizes.empty() ? !t.is_contiguous() : t.sizes() != at::IntArrayRef(l.sizes) || t.strides() != at::IntArrayRef(l.strides))
            refuse("tensor ", k, " has other strides than the list's: ", t.strides());
        if (t.device() != self.device) refuse("tensor ", k, " lies on ", t.device(), ", the list on ", self.device);
        self.addresses[k] = written ? t.data_ptr() : const_cast<void*>(t.const_data_ptr());
        if (written) self.written.push_back(t.unsafeGetTensorImpl());
    }
}

// For the flat gradient, which has the elements in their indexes' order: copies in that order of the tensors that lie in another.
std::vector<at::Tensor> in_order(TensorList& self, const Sequence& ts, const at::Tensor& out)
{
    std::vector<at::Tensor> copies;
    const char *f0 = static_cast<const char*>(out.const_data_ptr()), *f1 = f0 + out.nbytes();
    for (Py_ssize_t k = 0; k < ts.size(); ++k) {
        if (!self.layout[k].turned) continue;
        const char* p = static_cast<const char*>(self.addresses[k]);
        if (p < f1 && f0 < p + ts[k].nbytes()) fail(APMS_ERR_INVALID_ARG, "clip_grads: tensor " + std::to_string(k) + " overlaps the flat gradient without being in its place there");
        copies.push_back(ts[k].contiguous());
        self.addresses[k] = const_cast<void*>(copies.back().const_data_ptr());
    }
    return copies;
}

// The stream of one call, and the memory it writes to on the way.  The list's own memory is shared by its calls, so one on another stream than the last
// one's waits for that one.  A call that is being captured cannot wait for what is outside its graph, and no stream order holds the
// graph's replays apart from the list's other calls: it works in memory of its own, which comes from the graph's pool.
class Turn {
public:
    explicit Turn(TensorList& list) : list_(list)
    {
        const c10::cuda::CUDAStream now = c10::cuda::getCurrentCUDAStream(list.device.index());
        stream = now.stream();
        if (capturing()) {
            const size_t bytes = c_scratch_bytes(list.list);
            scratch_ = empty({(int64_t)bytes}, at::kByte, list.device);
            check(c_use_scratch(list.list, scratch_.data_ptr(), bytes, stream));
        } else if (now != list.stream) {
            at::cuda::CUDAEvent done;
            done.record(list.stream);
            done.block(now);
            list.workspace.record_stream(now);
            list.stream = now;
        }
    }
    ~Turn() { if (scratch_.defined()) c_use_scratch(list_.list, nullptr, 0, nullptr); }
    Turn(const Turn&) = delete;
    cudaStream_t stream;

private:
    TensorList& list_;
    at::Tensor scratch_;
};

PyObject* grad_norm(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject* {
        if (n != 2) refuse("grad_norm takes 2 arguments");
        TensorList& self = list_of(args[0]);
        take_addresses(self, Sequence(args[1]), false);
        const c10::cuda::OptionalCUDAGuard on(self.device);
        at::Tensor norm = empty({}, at::kFloat, self.device), norms = empty({(int64_t)self.layout.size()}, at::kFloat, self.device);
        const Turn turn(self);
        check(c_grad_norm(self.list, self.addresses.data(), (float*)norm.data_ptr(), (float*)norms.data_ptr(), turn.stream));
        return tuple_of({wrap(std::move(norm)), wrap(std::move(norms))});
    });
}

PyObject* clip_grads(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject* {
        if (n != 4) refuse("clip_grads takes 4 arguments");
        TensorList& self = list_of(args[0]);
        const double max_norm = PyFloat_AsDouble(args[2]);
        if (PyErr_Occurred()) throw Raised();
        void* flat = nullptr;
        apms_grad_type type = APMS_GRAD_F32;
        const Sequence ts(args[1]);
        take_addresses(self, ts, args[3] == Py_None);
        if (args[3] != Py_None) {
            const at::Tensor& out = tensor(args[3], "out");
            if (out.device() != self.device || !out.is_contiguous() || out.numel() != self.numel) refuse("out must be ", self.numel, " contiguous elements on ", self.device);
            type = (apms_grad_type)type_of(out, "out");
            flat = self.numel ? out.data_ptr() : self.workspace.data_ptr();       // an empty tensor has no address, and nothing is written
        }
        const c10::cuda::OptionalCUDAGuard on(self.device);
        const std::vector<at::Tensor> copies = flat && self.turned ? in_order(self, ts, tensor(args[3], "out")) : std::vector<at::Tensor>();
        at::Tensor norm = empty({}, at::kFloat, self.device);
        const Turn turn(self);
        check(c_clip_grads(self.list, self.addresses.data(), (float)max_norm, flat, type, (float*)norm.data_ptr(), turn.stream));
        if (flat) note_write(tensor(args[3], "out").unsafeGetTensorImpl());
        for (at::TensorImpl* t : self.written) note_write(t);
        return wrap(std::move(norm));
    });
}

// bind(error class, {name: address of the C function})
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject* {
        if (n != 2 || !PyDict_Check(args[1])) refuse("bind takes the error class and a dict of addresses");
        auto address = [&](const char* name) {
            PyObject* v = PyDict_GetItemString(args[1], name);
            void* p = v ? PyLong_AsVoidPtr(v) : nullptr;
            if (!p) refuse("no address for ", name);
            return p;
        };
        c_create = (decltype(c_create))address("apms_tensors_create");
        c_workspace_bytes = (decltype(c_workspace_bytes))address("apms_tensors_workspace_bytes");
        c_bind = (decltype(c_bind))address("apms_tensors_bind");
        c_destroy = (decltype(c_destroy))address("apms_tensors_destroy");
        c_scratch_bytes = (decltype(c_scratch_bytes))address("apms_tensors_scratch_bytes");
        c_use_scratch = (decltype(c_use_scratch))address("apms_tensors_use_scratch");
        c_grad_norm = (decltype(c_grad_norm))address("apms_grad_norm");
        c_clip_grads = (decltype(c_clip_grads))address("apms_clip_grads");
        c_rms_norm = (decltype(c_rms_norm))address("apms_rms_norm");
        c_backward_bytes = (decltype(c_backward_bytes))address("apms_rms_norm_backward_workspace_bytes");
        c_rms_norm_backward = (decltype(c_rms_norm_backward))address("apms_rms_norm_backward");
        c_embedding = (decltype(c_embedding))address("apms_embedding");
        c_embedding_bytes = (decltype(c_embedding_bytes))address("apms_embedding_backward_workspace_bytes");
        c_embedding_backward = (decltype(c_embedding_backward))address("apms_embedding_backward");
        c_dropout = (decltype(c_dropout))address("apms_dropout");
        c_scan_bytes = (decltype(c_scan_bytes))address("apms_gated_scan_workspace_bytes");
        c_starts_bytes = (decltype(c_starts_bytes))address("apms_gated_scan_starts_bytes");
        c_gated_scan = (decltype(c_gated_scan))address("apms_gated_scan");
        c_gated_scan_backward = (decltype(c_gated_scan_backward))address("apms_gated_scan_backward");
        c_gated_scan_step = (decltype(c_gated_scan_step))address("apms_gated_scan_step");
        c_last_error = (decltype(c_last_error))address("apms_last_error");
        Py_INCREF(args[0]);
        Py_XDECREF(g_error);
        g_error = args[0];
        Py_RETURN_NONE;
    });
}

#define FASTCALL(f) (PyCFunction)(void (*)(void))f, METH_FASTCALL, nullptr
PyMethodDef methods[] = {
    {"bind", FASTCALL(bind)},
    {"rms_norm", FASTCALL(rms_norm)},
    {"rms_norm_backward", FASTCALL(rms_norm_backward)},
    {"embedding", FASTCALL(embedding)},
    {"embedding_backward", FASTCALL(embedding_backward)},
    {"dropout", FASTCALL(dropout)},
    {"gated_scan", FASTCALL(gated_scan)},
    {"gated_scan_backward", FASTCALL(gated_scan_backward)},
    {"gated_scan_step", FASTCALL(gated_scan_step)},
    {"row_layout", row_layout_of, METH_O, nullptr},
    {"list_create", list_create, METH_O, nullptr},
    {"grad_norm", FASTCALL(grad_norm)},
    {"clip_grads", FASTCALL(clip_grads)},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_operators", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__operators() { return PyModule_Create(&module); }
