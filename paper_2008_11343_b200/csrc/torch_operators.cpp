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

// Autograd's notice that a tensor was written: a graph that has saved it raises in its backward pass.  (Inference tensors have no version, and
// no graph can save them.)
void note_write(at::TensorImpl* t)
{
    if (!t->is_inference()) t->bump_version();
}

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
    {"row_layout", row_layout_of, METH_O, nullptr},
    {"list_create", list_create, METH_O, nullptr},
    {"grad_norm", FASTCALL(grad_norm)},
    {"clip_grads", FASTCALL(clip_grads)},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_operators", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__operators() { return PyModule_Create(&module); }
