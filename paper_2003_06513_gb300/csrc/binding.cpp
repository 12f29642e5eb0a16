// Python's way to the operators of masked retraining: what a call does on the host, in one native
// function each -- the checks of its tensors, its outputs' allocation, the C entry point.  Through
// ctypes the same took 25 to 40 us a call (fifty gradients to look at, three outputs to make), several
// times what the small calls take on the GPU; here it is 5 to 8 us.
//
// The functions take positional arguments from norm.py, distill.py and optim.py, which hold the defaults and the
// documentation, and return the entry point's status where that is not 0; arguments that are no fit raise
// ValueError.  Tensors are only looked at and allocated: no operator of torch runs here.
#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <memory>
#include <optional>
#include <stdexcept>
#include <string>
#include <vector>

#include "patconv.h"

namespace {

struct Refused : std::runtime_error {       // becomes ValueError
    using std::runtime_error::runtime_error;
};
struct Raised {};                           // a Python error is set already
struct Status {                             // of a C entry point, where there is no result to return it as
    int e;
};

[[noreturn]] void refuse(const std::string& why) { throw Refused(why); }

const at::Tensor& tensor(PyObject* o, const char* what) {
    if (!THPVariable_Check(o)) refuse(std::string(what) + " must be a tensor");
    return THPVariable_Unpack(o);
}
const at::Tensor* maybe(PyObject* o, const char* what) { return o == Py_None ? nullptr : &tensor(o, what); }

int64_t integer(PyObject* o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Raised();
    return v;
}
double real(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Raised();
    return v;
}

// A new tensor on x's device, by the allocator without the dispatcher: a backward pass of block norm makes nine.
at::Tensor fresh(at::IntArrayRef shape, at::ScalarType type, const at::Tensor& x, at::MemoryFormat order = at::MemoryFormat::Contiguous) {
    return at::Tensor(at::detail::empty_cuda(shape, type, x.device(), order));
}

int dtype_of(const at::Tensor& t) {         // pp_dtype, or -1
    switch (t.scalar_type()) {
        case at::kFloat: return PP_F32;
        case at::kHalf: return PP_F16;
        case at::kBFloat16: return PP_BF16;
        default: return -1;
    }
}

// A tensor that a kernel writes: what torch has kept of it for a backward pass is no longer good.
void changed(const at::Tensor& t) {
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

// The device and, where one is given (a stream's handle, None for the current one), the stream are
// current while this lives; outputs and workspaces belong to that stream.
struct Place {
    c10::cuda::OptionalCUDAGuard device;
    std::optional<c10::cuda::CUDAStreamGuard> guard;
    void* stream;
    Place(at::Device d, PyObject* handle) {
        if (d.index() != c10::cuda::current_device()) device.set_device(d);
        if (handle == Py_None) {
            stream = c10::cuda::getCurrentCUDAStream(d.index()).stream();
        } else {
            cudaStream_t s = reinterpret_cast<cudaStream_t>(PyLong_AsVoidPtr(handle));
            if (PyErr_Occurred()) throw Raised();
            guard.emplace(s ? c10::cuda::getStreamFromExternal(s, d.index()) : c10::cuda::getDefaultCUDAStream(d.index()));
            stream = s;
        }
    }
};

// ---------------------------------------------------------------------------------- group norm

struct Layout {
    int64_t pixel = 0, sample = 0;
};

// Elements between pixels and between samples of a channels-last tensor; false for another order.
bool layout_of(const at::Tensor& t, Layout& l) {
    const auto size = t.sizes(), stride = t.strides();
    const int64_t n = size[0], c = size[1], h = size[2], w = size[3];
    if (c > 1 && stride[1] != 1) return false;
    if (w > 1) {
        l.pixel = stride[3];
        if (h > 1 && stride[2] != w * stride[3]) return false;
    } else {
        l.pixel = h > 1 ? stride[2] : c;
    }
    l.sample = n > 1 ? stride[0] : 0;
    return l.pixel >= c;
}

Layout input(const at::Tensor& t, const char* what) {
    if (!t.is_cuda() || dtype_of(t) < 0 || t.dim() != 4)
        refuse(std::string(what) + " must be a 4-d CUDA float32, float16 or bfloat16 tensor");
    Layout l;
    if (t.numel() && !layout_of(t, l)) refuse(std::string(what) + " must be channels last");
    return l;
}

const float* values(PyObject* o, int64_t count, const at::Tensor& x, const char* what) {
    const at::Tensor* t = maybe(o, what);
    if (!t) return nullptr;
    if (t->scalar_type() != at::kFloat || t->numel() != count || !t->is_contiguous() || t->device() != x.device())
        refuse(std::string(what) + " must be " + std::to_string(count) + " contiguous float32 values on the activations' device");
    return static_cast<const float*>(t->const_data_ptr());
}

at::Tensor like(const at::Tensor& x, PyObject* o) {
    const at::Tensor* out = maybe(o, "out");
    if (!out) return fresh(x.sizes(), x.scalar_type(), x, at::MemoryFormat::ChannelsLast);
    if (out->sizes() != x.sizes() || out->scalar_type() != x.scalar_type() || out->device() != x.device() ||
        !out->is_contiguous(at::MemoryFormat::ChannelsLast))
        refuse("out must be a dense channels-last tensor of x's shape, type and device");
    return *out;
}

struct Workspace {
    at::Tensor held;
    void* p = nullptr;
    size_t bytes = 0;
    Workspace(const at::Tensor& x, PyObject* o, int dtype, int64_t pixels, int groups, int backward) {
        if (const at::Tensor* w = maybe(o, "workspace")) {
            if (!w->is_contiguous() || w->device() != x.device())
                refuse("workspace must be a contiguous CUDA tensor on x's device");
            p = w->data_ptr();
            bytes = w->nbytes();
            return;
        }
        if (pp_group_norm_workspace_size(dtype, (int)x.size(0), pixels, (int)x.size(1), groups, backward, &bytes) != PP_OK)
            return;                          // the call says what is wrong
        if (bytes) {
            held = fresh({(int64_t)bytes}, at::kByte, x);
            p = held.data_ptr();
        }
    }
};

at::Tensor floats(at::IntArrayRef shape, const at::Tensor& x) {
    return fresh(shape, at::kFloat, x);
}

PyObject* triple(const at::Tensor& a, const at::Tensor& b, const at::Tensor& c) {
    PyObject* t = PyTuple_New(3);
    if (!t) throw Raised();
    PyTuple_SET_ITEM(t, 0, THPVariable_Wrap(a));
    PyTuple_SET_ITEM(t, 1, THPVariable_Wrap(b));
    PyTuple_SET_ITEM(t, 2, THPVariable_Wrap(c));
    return t;
}

void want(Py_ssize_t given, Py_ssize_t wanted) {
    if (given != wanted) refuse("wrong number of arguments");
}

int checked_groups(int64_t groups, int64_t channels) {
    if (groups < 1 || groups > channels || channels % groups)
        refuse(std::to_string(channels) + " channels do not make " + std::to_string(groups) + " groups");
    return (int)groups;
}

bool too_large(const at::Tensor& x) { return x.size(0) > INT32_MAX || x.size(1) > INT32_MAX; }

// x, groups, weight, bias, eps, act, out, stream, workspace
PyObject* group_norm(PyObject* const* a, Py_ssize_t n_args) {
    want(n_args, 9);
    const at::Tensor& x = tensor(a[0], "x");
    const Layout l = input(x, "x");
    if (too_large(x)) return PyLong_FromLong(PP_ERR_SHAPE);
    const int64_t n = x.size(0), c = x.size(1), pixels = x.size(2) * x.size(3);
    const int groups = checked_groups(integer(a[1]), c), dtype = dtype_of(x), act = (int)integer(a[5]);
    const float *gamma = values(a[2], c, x, "weight"), *beta = values(a[3], c, x, "bias");
    const float eps = (float)real(a[4]);
    const Place at(x.device(), a[7]);
    const at::Tensor y = like(x, a[6]), mean = floats({n, groups}, x), rstd = floats({n, groups}, x);
    const Workspace w(x, a[8], dtype, pixels, groups, 0);
    const int e = pp_group_norm(x.const_data_ptr(), l.pixel, l.sample, dtype, (int)n, pixels, (int)c, groups, gamma, beta, eps,
                                act, y.data_ptr(), mean.data_ptr<float>(), rstd.data_ptr<float>(), w.p, w.bytes, at.stream);
    if (!e && a[6] != Py_None) changed(y);
    return e ? PyLong_FromLong(e) : triple(y, mean, rstd);
}

// dy, x, mean, rstd, groups, weight, bias, act, out, stream, workspace
PyObject* group_norm_backward(PyObject* const* a, Py_ssize_t n_args) {
    want(n_args, 11);
    const at::Tensor &dy = tensor(a[0], "dy"), &x = tensor(a[1], "x");
    const Layout l = input(x, "x"), d = input(dy, "dy");
    if (dy.sizes() != x.sizes() || dy.scalar_type() != x.scalar_type() || dy.device() != x.device())
        refuse("dy must have x's shape, type and device");
    if (too_large(x)) return PyLong_FromLong(PP_ERR_SHAPE);
    const int64_t n = x.size(0), c = x.size(1), pixels = x.size(2) * x.size(3);
    const int groups = checked_groups(integer(a[4]), c), dtype = dtype_of(x), act = (int)integer(a[7]);
    const float *gamma = values(a[5], c, x, "weight"), *beta = values(a[6], c, x, "bias");
    const float *mean = values(a[2], n * groups, x, "mean"), *rstd = values(a[3], n * groups, x, "rstd");
    const Place at(x.device(), a[9]);
    const at::Tensor dx = like(x, a[8]), dgamma = floats({c}, x), dbeta = floats({c}, x);
    const Workspace w(x, a[10], dtype, pixels, groups, 1);
    const int e = pp_group_norm_backward(dy.const_data_ptr(), d.pixel, d.sample, x.const_data_ptr(), l.pixel, l.sample, dtype,
                                         (int)n, pixels, (int)c, groups, gamma, beta, mean, rstd, act, dx.data_ptr(),
                                         dgamma.data_ptr<float>(), dbeta.data_ptr<float>(), w.p, w.bytes, at.stream);
    if (!e && a[8] != Py_None) changed(dx);
    return e ? PyLong_FromLong(e) : triple(dx, dgamma, dbeta);
}

// tensor -> (elements between pixels, elements between samples), or None
PyObject* layout(PyObject* const* a, Py_ssize_t n_args) {
    want(n_args, 1);
    const at::Tensor& t = tensor(a[0], "tensor");
    if (t.dim() != 4) refuse("a 4-d tensor is wanted");
    Layout l;
    if (!layout_of(t, l)) Py_RETURN_NONE;
    return Py_BuildValue("(LL)", (long long)l.pixel, (long long)l.sample);
}

// ---------------------------------------------------------------------------------- block norm

// an input like x in shape and device, of a type
Layout alike(const at::Tensor& t, const at::Tensor& x, at::ScalarType type, const char* what) {
    const Layout l = input(t, what);
    if (t.sizes() != x.sizes() || t.device() != x.device() || t.scalar_type() != type)
        refuse(std::string(what) + " must have the stream's shape and device, and be " + c10::toString(type));
    return l;
}
// a dense channels-last result like x, of a type: the one that is given, or a new one
at::Tensor result(PyObject* o, const at::Tensor& x, at::ScalarType type, const char* what) {
    const at::Tensor* out = maybe(o, what);
    if (!out) return fresh(x.sizes(), type, x, at::MemoryFormat::ChannelsLast);
    if (out->sizes() != x.sizes() || out->scalar_type() != type || out->device() != x.device() ||
        !out->is_contiguous(at::MemoryFormat::ChannelsLast))
        refuse(std::string(what) + " must be a dense channels-last tensor of the stream's shape and device, " + c10::toString(type));
    return *out;
}
struct Parameters {
    int post, pre, act;
    const float *post_weight, *post_bias, *scale, *gate, *weight, *bias;
    float eps;
    // post, post_weight, post_bias, scale, gate, pre, weight, bias, act, eps
    Parameters(PyObject* const* a, const at::Tensor& x) {
        const int64_t n = x.size(0), c = x.size(1);
        post = (int)integer(a[0]);
        post_weight = values(a[1], c, x, "post_weight");
        post_bias = values(a[2], c, x, "post_bias");
        scale = values(a[3], c, x, "scale");
        gate = values(a[4], n * c, x, "gate");
        if (gate && (tensor(a[4], "gate").dim() != 2 || tensor(a[4], "gate").size(1) != c)) refuse("gate must be [N, C]");
        pre = (int)integer(a[5]);
        weight = values(a[6], c, x, "weight");
        bias = values(a[7], c, x, "bias");
        act = (int)integer(a[8]);
        eps = (float)real(a[9]);
    }
};

// x, block, then Parameters' ten, out_h, out_y, stream -> (h, y or None)
PyObject* block_norm(PyObject* const* a, Py_ssize_t n_args) {
    want(n_args, 15);
    const at::Tensor& x = tensor(a[0], "x");
    const Layout l = input(x, "x");
    const at::Tensor* b = maybe(a[1], "block");
    if (b && x.scalar_type() != b->scalar_type() && x.scalar_type() != at::kFloat) refuse("x must have the block's type, or be float32");
    const at::ScalarType type = b ? b->scalar_type() : x.scalar_type();
    const Layout lb = b ? alike(*b, x, type, "block") : Layout();
    if (too_large(x)) return PyLong_FromLong(PP_ERR_SHAPE);
    const Parameters p(a + 2, x);
    const Place at(x.device(), a[14]);
    const at::Tensor h = b ? result(a[12], x, x.scalar_type(), "h") : x;
    const bool normed = p.pre != PP_NORM_NONE;
    const at::Tensor y = normed ? result(a[13], x, type, "y") : at::Tensor();
    const int e = pp_block_norm(x.const_data_ptr(), l.pixel, l.sample, dtype_of(x), b ? b->const_data_ptr() : nullptr, lb.pixel, lb.sample,
                                b ? dtype_of(*b) : dtype_of(x), (int)x.size(0), x.size(2) * x.size(3), (int)x.size(1), p.post,
                                p.post_weight, p.post_bias, p.scale, p.gate, p.pre, p.weight, p.bias, p.act, p.eps,
                                b ? h.data_ptr() : nullptr, normed ? y.data_ptr() : nullptr, at.stream);
    if (e) return PyLong_FromLong(e);
    if (b && a[12] != Py_None) changed(h);
    if (normed && a[13] != Py_None) changed(y);
    PyObject* t = PyTuple_New(2);
    if (!t) throw Raised();
    if (b) {
        PyTuple_SET_ITEM(t, 0, THPVariable_Wrap(h));
    } else {
        Py_INCREF(a[0]);
        PyTuple_SET_ITEM(t, 0, a[0]);
    }
    if (normed) {
        PyTuple_SET_ITEM(t, 1, THPVariable_Wrap(y));
    } else {
        Py_INCREF(Py_None);
        PyTuple_SET_ITEM(t, 1, Py_None);
    }
    return t;
}

// dh, dy, h, block, then Parameters' ten, out_dx, out_dblock, stream, workspace -> (dx, dblock, dpost_weight, dpost_bias, dscale, dgate, dweight, dbias),
// None for what is not there
PyObject* block_norm_backward(PyObject* const* a, Py_ssize_t n_args) {
    want(n_args, 18);
    const at::Tensor& h = tensor(a[2], "h");
    const Layout l = input(h, "h");
    const at::Tensor *dh = maybe(a[0], "dh"), *dy = maybe(a[1], "dy"), *b = maybe(a[3], "block");
    if (b && h.scalar_type() != b->scalar_type() && h.scalar_type() != at::kFloat) refuse("h must have the block's type, or be float32");
    const at::ScalarType type = b ? b->scalar_type() : h.scalar_type();
    const Layout lb = b ? alike(*b, h, type, "block") : Layout(), ld = dh ? alike(*dh, h, h.scalar_type(), "dh") : Layout(),
                 ly = dy ? alike(*dy, h, type, "dy") : Layout();
    if (too_large(h)) return PyLong_FromLong(PP_ERR_SHAPE);
    const Parameters p(a + 4, h);
    const int n = (int)h.size(0), c = (int)h.size(1), dtype = b ? dtype_of(*b) : dtype_of(h);
    const int64_t pixels = h.size(2) * h.size(3);
    const Place at(h.device(), a[16]);
    at::Tensor grads[8];                        // in the order of the result
    grads[0] = result(a[14], h, h.scalar_type(), "dx");
    if (b) grads[1] = result(a[15], h, type, "dblock");
    const int of[6] = {5, 6, 7, 8, 10, 11};     // the parameters among the arguments
    float* sums[6];
    for (int i = 0; i < 6; ++i) {
        const bool given = a[of[i]] != Py_None;
        if (given) grads[2 + i] = i == 3 ? floats({n, c}, h) : floats({c}, h);
        sums[i] = given ? grads[2 + i].data_ptr<float>() : nullptr;
    }
    size_t bytes = 0;
    void* space = nullptr;
    at::Tensor held;
    if (const at::Tensor* w = maybe(a[17], "workspace")) {
        if (!w->is_contiguous() || w->device() != h.device()) refuse("workspace must be a contiguous CUDA tensor on the stream's device");
        space = w->data_ptr();
        bytes = w->nbytes();
    } else if (pp_block_norm_workspace_size(n, pixels, c, &bytes) == PP_OK && bytes) {
        held = fresh({(int64_t)bytes}, at::kByte, h);
        space = held.data_ptr();
    }
    const int e = pp_block_norm_backward(
        dh ? dh->const_data_ptr() : nullptr, ld.pixel, ld.sample, dy ? dy->const_data_ptr() : nullptr, ly.pixel, ly.sample, h.const_data_ptr(),
        l.pixel, l.sample, dtype_of(h), b ? b->const_data_ptr() : nullptr, lb.pixel, lb.sample, dtype, n, pixels, c, p.post,
        p.post_weight, p.post_bias, p.scale, p.gate, p.pre, p.weight, p.bias, p.act, p.eps, grads[0].data_ptr(),
        b ? grads[1].data_ptr() : nullptr, sums[0], sums[1], sums[2], sums[3], sums[4], sums[5], space, bytes, at.stream);
    if (e) return PyLong_FromLong(e);
    if (a[14] != Py_None) changed(grads[0]);
    if (b && a[15] != Py_None) changed(grads[1]);
    PyObject* t = PyTuple_New(8);
    if (!t) throw Raised();
    for (int i = 0; i < 8; ++i) {
        PyObject* o = grads[i].defined() ? THPVariable_Wrap(grads[i]) : Py_None;
        if (o == Py_None) Py_INCREF(o);
        PyTuple_SET_ITEM(t, i, o);
    }
    return t;
}

// ---------------------------------------------------------------------------------- distillation

int64_t row_stride(const at::Tensor& t, const char* what) {
    if (!t.is_cuda() || t.layout() != at::kStrided || dtype_of(t) < 0 || t.dim() != 2)
        refuse(std::string(what) + " must be a 2-d CUDA float32, float16 or bfloat16 tensor");
    if ((t.size(1) > 1 && t.stride(1) != 1) || (t.size(0) > 1 && t.stride(0) < t.size(1)))
        refuse(std::string(what) + " must have its classes adjacent, and rows that do not overlap");
    return t.size(0) > 1 ? t.stride(0) : t.size(1);
}

// logits, k, temperature, stream -> (values, indices, rest)
PyObject* top_logits(PyObject* const* a, Py_ssize_t n_args) {
    want(n_args, 4);
    const at::Tensor& s = tensor(a[0], "logits");
    const int64_t stride = row_stride(s, "logits"), k = integer(a[1]);
    const double temperature = real(a[2]);
    if (k < 1 || k > PP_MOST_KEPT || k > s.size(1))
        refuse("k must be 1 to " + std::to_string(PP_MOST_KEPT) + " and no more than the classes");
    const Place at(s.device(), a[3]);
    const at::Tensor values = fresh({s.size(0), k}, s.scalar_type(), s), rest = floats({s.size(0)}, s);
    const at::Tensor indices = fresh({s.size(0), k}, at::kInt, s);
    const int e = pp_top_logits(s.const_data_ptr(), stride, dtype_of(s), s.size(0), s.size(1), (int)k, temperature, values.data_ptr(),
                                indices.data_ptr<int>(), rest.data_ptr<float>(), at.stream);
    return e ? PyLong_FromLong(e) : triple(values, indices, rest);
}

struct Teacher {
    const at::Tensor *values, *indices, *rest, *labels;
    double temperature, alpha;
    // values, indices, rest, labels, temperature, alpha
    Teacher(PyObject* const* a, const at::Tensor& s) {
        values = &tensor(a[0], "values"), indices = &tensor(a[1], "indices"), rest = maybe(a[2], "rest"), labels = maybe(a[3], "labels");
        const int64_t n = s.size(0);
        if (values->dim() != 2 || values->size(0) != n || dtype_of(*values) < 0 || !values->is_contiguous() || values->device() != s.device())
            refuse("values must be a contiguous [rows, kept] float32, float16 or bfloat16 tensor on the logits' device");
        if (indices->sizes() != values->sizes() || indices->scalar_type() != at::kInt || !indices->is_contiguous() || indices->device() != s.device())
            refuse("indices must be a contiguous int32 tensor of values' shape on the logits' device");
        if (rest && (rest->dim() != 1 || rest->size(0) != n || rest->scalar_type() != at::kFloat || !rest->is_contiguous() || rest->device() != s.device()))
            refuse("rest must be a contiguous float32 tensor [rows] on the logits' device");
        if (labels && (labels->dim() != 1 || labels->size(0) != n || labels->scalar_type() != at::kLong || !labels->is_contiguous() || labels->device() != s.device()))
            refuse("labels must be a contiguous int64 tensor [rows] on the logits' device");
        if (values->size(1) < 1 || values->size(1) > PP_MOST_KEPT || values->size(1) > s.size(1))
            refuse("kept logits must be 1 to " + std::to_string(PP_MOST_KEPT) + " a row and no more than the classes");
        temperature = real(a[4]);
        alpha = real(a[5]);
    }
    int kept() const { return (int)values->size(1); }
    const float* rest_ptr() const { return rest ? rest->const_data_ptr<float>() : nullptr; }
    const int64_t* labels_ptr() const { return labels ? labels->const_data_ptr<int64_t>() : nullptr; }
};

// logits, then Teacher's six, stream -> (loss, stats)
PyObject* distill(PyObject* const* a, Py_ssize_t n_args) {
    want(n_args, 8);
    const at::Tensor& s = tensor(a[0], "logits");
    const int64_t stride = row_stride(s, "logits");
    const Teacher t(a + 1, s);
    const Place at(s.device(), a[7]);
    const at::Tensor loss = floats({s.size(0)}, s), stats = floats({s.size(0), 5}, s);
    const int e = pp_distill(s.const_data_ptr(), stride, dtype_of(s), s.size(0), s.size(1), t.values->const_data_ptr(), dtype_of(*t.values),
                             t.indices->const_data_ptr<int>(), t.kept(), t.rest_ptr(), t.labels_ptr(), t.temperature, t.alpha,
                             loss.data_ptr<float>(), stats.data_ptr<float>(), at.stream);
    if (e) return PyLong_FromLong(e);
    PyObject* r = PyTuple_New(2);
    if (!r) throw Raised();
    PyTuple_SET_ITEM(r, 0, THPVariable_Wrap(loss));
    PyTuple_SET_ITEM(r, 1, THPVariable_Wrap(stats));
    return r;
}

// dloss, logits, stats, then Teacher's six, out, stream -> dlogits
PyObject* distill_backward(PyObject* const* a, Py_ssize_t n_args) {
    want(n_args, 11);
    const at::Tensor &d = tensor(a[0], "dloss"), &s = tensor(a[1], "logits"), &stats = tensor(a[2], "stats");
    const int64_t stride = row_stride(s, "logits"), n = s.size(0);
    if (d.dim() != 1 || d.size(0) != n || d.scalar_type() != at::kFloat || d.device() != s.device())
        refuse("dloss must be a float32 tensor [rows] on the logits' device");
    if (stats.dim() != 2 || stats.size(0) != n || stats.size(1) != 5 || stats.scalar_type() != at::kFloat || !stats.is_contiguous() || stats.device() != s.device())
        refuse("stats must be the contiguous float32 [rows, 5] of the forward pass");
    const Teacher t(a + 3, s);
    const Place at(s.device(), a[10]);
    const at::Tensor* given = maybe(a[9], "out");
    if (given && (given->sizes() != s.sizes() || given->scalar_type() != s.scalar_type() || given->device() != s.device() || !given->is_contiguous()))
        refuse("out must be a contiguous tensor of the logits' shape, type and device");
    const at::Tensor out = given ? *given : fresh(s.sizes(), s.scalar_type(), s);
    const int e = pp_distill_backward(d.const_data_ptr<float>(), n > 1 ? d.stride(0) : 0, s.const_data_ptr(), stride, dtype_of(s), n, s.size(1),
                                      stats.const_data_ptr<float>(), t.values->const_data_ptr(), dtype_of(*t.values),
                                      t.indices->const_data_ptr<int>(), t.kept(), t.rest_ptr(), t.labels_ptr(), t.temperature, t.alpha,
                                      out.data_ptr(), at.stream);
    if (e) return PyLong_FromLong(e);
    if (given) changed(out);
    return THPVariable_Wrap(out);
}

// The loss as one differentiable operation.  Its backward pass runs on a thread of torch's engine: there is no Python in it.
struct DistillLoss : torch::autograd::Function<DistillLoss> {
    using Context = torch::autograd::AutogradContext;
    static at::Tensor forward(Context* ctx, const at::Tensor& s, const at::Tensor& values, const at::Tensor& indices,
                              const std::optional<at::Tensor>& rest, const std::optional<at::Tensor>& labels, double temperature, double alpha,
                              int64_t stride) {
        const c10::cuda::CUDAGuard guard(s.device());
        const at::Tensor loss = floats({s.size(0)}, s), stats = floats({s.size(0), 5}, s);
        const int e = pp_distill(s.const_data_ptr(), stride, dtype_of(s), s.size(0), s.size(1), values.const_data_ptr(), dtype_of(values),
                                 indices.const_data_ptr<int>(), (int)values.size(1), rest ? rest->const_data_ptr<float>() : nullptr,
                                 labels ? labels->const_data_ptr<int64_t>() : nullptr, temperature, alpha, loss.data_ptr<float>(),
                                 stats.data_ptr<float>(), c10::cuda::getCurrentCUDAStream(s.get_device()).stream());
        if (e) throw Status{e};
        ctx->save_for_backward({s, stats, values, indices, rest.value_or(at::Tensor()), labels.value_or(at::Tensor())});
        ctx->saved_data["temperature"] = temperature;
        ctx->saved_data["alpha"] = alpha;
        return loss;
    }
    static torch::autograd::variable_list backward(Context* ctx, torch::autograd::variable_list grads) {
        TORCH_CHECK(!at::GradMode::is_enabled(), "distill_loss is differentiable once: its gradient has no graph (create_graph)");
        const auto saved = ctx->get_saved_variables();
        const at::Tensor &s = saved[0], &stats = saved[1], &values = saved[2], &indices = saved[3], &rest = saved[4], &labels = saved[5];
        const c10::cuda::CUDAGuard guard(s.device());
        const at::Tensor d = grads[0].to(at::kFloat), out = fresh(s.sizes(), s.scalar_type(), s);
        const int64_t n = s.size(0);
        const int e = pp_distill_backward(d.const_data_ptr<float>(), n > 1 ? d.stride(0) : 0, s.const_data_ptr(), n > 1 ? s.stride(0) : s.size(1),
                                          dtype_of(s), n, s.size(1), stats.const_data_ptr<float>(), values.const_data_ptr(), dtype_of(values),
                                          indices.const_data_ptr<int>(), (int)values.size(1),
                                          rest.defined() ? rest.const_data_ptr<float>() : nullptr,
                                          labels.defined() ? labels.const_data_ptr<int64_t>() : nullptr, ctx->saved_data["temperature"].toDouble(),
                                          ctx->saved_data["alpha"].toDouble(), out.data_ptr(),
                                          c10::cuda::getCurrentCUDAStream(s.get_device()).stream());
        TORCH_CHECK(e == PP_OK, "pp_distill_backward failed: ", pp_status_string(e));
        torch::autograd::variable_list r(8);
        r[0] = out;
        return r;
    }
};

// logits, then Teacher's six -> loss
PyObject* distill_loss(PyObject* const* a, Py_ssize_t n_args) {
    want(n_args, 7);
    const at::Tensor& s = tensor(a[0], "logits");
    const int64_t stride = row_stride(s, "logits");
    const Teacher t(a + 1, s);
    const auto given = [](const at::Tensor* p) { return p ? std::optional<at::Tensor>(*p) : std::nullopt; };
    return THPVariable_Wrap(DistillLoss::apply(s, *t.values, *t.indices, given(t.rest), given(t.labels), t.temperature, t.alpha, stride));
}

// ---------------------------------------------------------------------------------- many tensors

struct Wanted {                             // of one tensor's gradient, and of the tensor itself
    std::vector<int64_t> shape, strides;
    at::ScalarType type;
};
struct Written {                            // a parameter or a copy, as it was when the handle was made
    const void* at;
    at::ScalarType type;
    size_t tensor;                          // whose shape and strides it has
};
struct List {
    pp_tensors_handle handle;
    at::Device device;
    std::vector<Wanted> wanted;
    std::vector<Written> written;
    int64_t state_elements;
    std::vector<int64_t> missed;            // steps at which each tensor had no gradient
};
constexpr const char* kList = "patconv.tensors";

void drop(PyObject* capsule) { delete static_cast<List*>(PyCapsule_GetPointer(capsule, kList)); }

// whether a tensor has the strides, as far as they matter
bool in_order(const at::Tensor& t, const std::vector<int64_t>& shape, const std::vector<int64_t>& strides) {
    if (t.strides() == at::IntArrayRef(strides) || !t.numel()) return true;
    for (size_t k = 0; k < shape.size(); ++k)
        if (shape[k] > 1 && t.stride((int64_t)k) != strides[k]) return false;
    return true;
}

// handle, device index, [(shape, strides, pp_dtype)], [(parameter or copy, its tensor's number)] -> what a call's
// gradients, and the tensors that it writes, are checked against
PyObject* tensors(PyObject* const* a, Py_ssize_t n_args) {
    want(n_args, 4);
    auto list = std::make_unique<List>(List{static_cast<pp_tensors_handle>(PyLong_AsVoidPtr(a[0])),
                                            at::Device(at::kCUDA, (int8_t)integer(a[1])), {}, {}, 0, {}});
    if (PyErr_Occurred()) throw Raised();
    if (pp_tensors_query(list->handle, PP_TQ_STATE_ELEMENTS, &list->state_elements) != PP_OK) refuse("a handle is wanted");
    if (!PyList_Check(a[2]) || !PyList_Check(a[3])) refuse("a list is wanted");
    for (Py_ssize_t i = 0; i < PyList_GET_SIZE(a[2]); ++i) {
        PyObject *shape, *strides;
        int dtype;
        if (!PyArg_ParseTuple(PyList_GET_ITEM(a[2], i), "O!O!i", &PyTuple_Type, &shape, &PyTuple_Type, &strides, &dtype))
            throw Raised();
        Wanted w;
        for (Py_ssize_t k = 0; k < PyTuple_GET_SIZE(shape); ++k) w.shape.push_back(integer(PyTuple_GET_ITEM(shape, k)));
        for (Py_ssize_t k = 0; k < PyTuple_GET_SIZE(strides); ++k) w.strides.push_back(integer(PyTuple_GET_ITEM(strides, k)));
        w.type = dtype == PP_F32 ? at::kFloat : dtype == PP_F16 ? at::kHalf : at::kBFloat16;
        list->wanted.push_back(std::move(w));
    }
    for (Py_ssize_t i = 0; i < PyList_GET_SIZE(a[3]); ++i) {
        PyObject* o;
        Py_ssize_t k;
        if (!PyArg_ParseTuple(PyList_GET_ITEM(a[3], i), "On", &o, &k)) throw Raised();
        const at::Tensor& t = tensor(o, "a parameter");
        if (k < 0 || (size_t)k >= list->wanted.size()) refuse("there is no such tensor");
        list->written.push_back({t.const_data_ptr(), t.scalar_type(), (size_t)k});
    }
    list->missed.assign(list->wanted.size(), 0);
    PyObject* capsule = PyCapsule_New(list.get(), kList, drop);
    if (capsule) list.release();
    return capsule;
}

List& list_of(PyObject* o) {
    List* l = static_cast<List*>(PyCapsule_GetPointer(o, kList));
    if (!l) throw Raised();
    return *l;
}

// The gradients' addresses, each checked against its tensor: type, shape, order, device.
std::vector<const void*> addresses(const List& list, PyObject* grads) {
    PyObject* fast = PySequence_Fast(grads, "the gradients must be a sequence");
    if (!fast) throw Raised();
    struct Release {
        PyObject* o;
        ~Release() { Py_DECREF(o); }
    } release{fast};
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(fast);
    if ((size_t)n != list.wanted.size())
        refuse(std::to_string(n) + " gradients for " + std::to_string(list.wanted.size()) + " tensors");
    std::vector<const void*> at(n ? n : 1, nullptr);
    for (Py_ssize_t i = 0; i < n; ++i) {
        PyObject* o = PySequence_Fast_GET_ITEM(fast, i);
        if (o == Py_None) continue;
        const at::Tensor& g = tensor(o, "a gradient");
        const Wanted& w = list.wanted[i];
        if (g.scalar_type() != w.type || g.device() != list.device || g.layout() != at::kStrided || g.sizes() != at::IntArrayRef(w.shape))
            refuse("gradient " + std::to_string(i) + " is not of its tensor's shape, on its device or of the type it was announced as");
        if (!in_order(g, w.shape, w.strides)) refuse("gradient " + std::to_string(i) + " is not in its tensor's memory order");
        at[i] = g.const_data_ptr();
    }
    return at;
}

// tensors, grads, max_norm, out, stream
PyObject* grad_norm(PyObject* const* a, Py_ssize_t n_args) {
    want(n_args, 5);
    const List& list = list_of(a[0]);
    const std::vector<const void*> grads = addresses(list, a[1]);
    const Place at(list.device, a[4]);
    const at::Tensor* given = maybe(a[3], "out");
    if (given && (given->scalar_type() != at::kFloat || given->numel() != 2 || !given->is_contiguous() || given->device() != list.device))
        refuse("out must be a contiguous float32 tensor of two values on the tensors' device");
    const at::Tensor out = given ? given->detach().view({2}) : at::empty({2}, at::TensorOptions().dtype(at::kFloat).device(list.device));
    const int e = pp_grad_norm(list.handle, grads.data(), real(a[2]), out.data_ptr<float>(), at.stream);
    if (e) return PyLong_FromLong(e);
    if (given) changed(*given);
    PyObject* t = PyTuple_New(2);
    if (!t) throw Raised();
    PyTuple_SET_ITEM(t, 0, THPVariable_Wrap(out.narrow(0, 0, 1)));
    PyTuple_SET_ITEM(t, 1, THPVariable_Wrap(out.narrow(0, 1, 1)));
    return t;
}

// The parameters and copies are still the memory whose addresses the handle holds: a tensor that was given other
// memory since (by its `data`, by a module's move to another order or type) has left that memory to others.
void check_written(const List& list, PyObject* tensors) {
    if (!PyList_Check(tensors) || (size_t)PyList_GET_SIZE(tensors) != list.written.size())
        refuse("the parameters and copies must be those that the handle was made with");
    for (size_t i = 0; i < list.written.size(); ++i) {
        const Written& w = list.written[i];
        const Wanted& like = list.wanted[w.tensor];
        const at::Tensor& t = tensor(PyList_GET_ITEM(tensors, (Py_ssize_t)i), "a parameter");
        if (t.scalar_type() != w.type || t.device() != list.device || t.layout() != at::kStrided ||
            t.sizes() != at::IntArrayRef(like.shape) || t.const_data_ptr() != w.at || !in_order(t, like.shape, like.strides))
            refuse("parameter " + std::to_string(w.tensor) + ", or its copy, has been given other memory: make a new AdamW, "
                   "with this one's state_dict() as its state");
    }
}

// A state of the handle's tensors: `count` values of a type.
void* state_of(const List& list, PyObject* o, const char* what, at::ScalarType type, int64_t count) {
    const at::Tensor& t = tensor(o, what);
    if (t.scalar_type() != type || t.layout() != at::kStrided || t.numel() != count || !t.is_contiguous() || t.device() != list.device)
        refuse(std::string(what) + " must be " + std::to_string(count) + " contiguous " + c10::toString(type) + " values on the parameters' device");
    return t.data_ptr();
}

// tensors, grads, parameters and copies, state_bits, m, v, m_scale, v_scale, lr, beta1, beta2, eps, step, seed, grad_scale, stream
PyObject* adamw_step(PyObject* const* a, Py_ssize_t n_args) {
    want(n_args, 16);
    List& list = list_of(a[0]);
    const std::vector<const void*> grads = addresses(list, a[1]);
    const at::Tensor* scale = maybe(a[14], "grad_scale");
    if (scale && (scale->scalar_type() != at::kFloat || scale->numel() != 1 || scale->device() != list.device))
        refuse("grad_scale must be one float32 on the parameters' device");
    check_written(list, a[2]);
    const int bits = (int)integer(a[3]);
    const int64_t count = list.state_elements, blocks = count / PP_STATE_BLOCK;
    const at::ScalarType type = bits == 8 ? at::kFloat8_e4m3fn : at::kFloat;
    void *m = state_of(list, a[4], "m", type, count), *v = state_of(list, a[5], "v", type, count);
    void* ms = bits == 8 ? state_of(list, a[6], "m_scale", at::kFloat, blocks) : nullptr;
    void* vs = bits == 8 ? state_of(list, a[7], "v_scale", at::kFloat, blocks) : nullptr;
    const Place at(list.device, a[15]);
    const double lr = real(a[8]), b1 = real(a[9]), b2 = real(a[10]), eps = real(a[11]);
    const int64_t step = integer(a[12]);
    const uint32_t seed = (uint32_t)integer(a[13]);
    // A tensor's step number counts the steps at which it had a gradient.  It is one for all as a rule; tensors that
    // have missed some take launches of their own, those that have missed as many together.
    std::vector<int64_t> apart;
    for (size_t i = 0; i < list.missed.size(); ++i)
        if (grads[i]) {
            if (list.missed[i] >= step) refuse("tensor " + std::to_string(i) + " has missed more steps than were taken");
            if (std::find(apart.begin(), apart.end(), list.missed[i]) == apart.end()) apart.push_back(list.missed[i]);
        }
    if (apart.empty()) apart.push_back(0);
    std::vector<const void*> some;
    for (const int64_t missed : apart) {
        if (apart.size() > 1) {
            some = grads;
            for (size_t i = 0; i < list.missed.size(); ++i)
                if (list.missed[i] != missed) some[i] = nullptr;
        }
        const int e = pp_adamw_step(list.handle, apart.size() > 1 ? some.data() : grads.data(), bits, m, v, static_cast<float*>(ms),
                                    static_cast<float*>(vs), lr, b1, b2, eps, step - missed, seed,
                                    scale ? scale->const_data_ptr<float>() : nullptr, at.stream);
        if (e) return PyLong_FromLong(e);
    }
    for (size_t i = 0; i < list.missed.size(); ++i) list.missed[i] += !grads[i];
    for (Py_ssize_t i = 0; i < PyList_GET_SIZE(a[2]); ++i) changed(tensor(PyList_GET_ITEM(a[2], i), "a parameter"));
    return PyLong_FromLong(PP_OK);
}

// tensors, None -> the steps that each tensor has missed, a list; tensors, list -> sets them
PyObject* missed(PyObject* const* a, Py_ssize_t n_args) {
    want(n_args, 2);
    List& list = list_of(a[0]);
    if (a[1] == Py_None) {
        PyObject* out = PyList_New((Py_ssize_t)list.missed.size());
        if (!out) throw Raised();
        for (size_t i = 0; i < list.missed.size(); ++i) PyList_SET_ITEM(out, (Py_ssize_t)i, PyLong_FromLongLong(list.missed[i]));
        return out;
    }
    if (!PyList_Check(a[1]) || (size_t)PyList_GET_SIZE(a[1]) != list.missed.size()) refuse("missed must be a list of one count a tensor");
    std::vector<int64_t> to;
    for (Py_ssize_t i = 0; i < PyList_GET_SIZE(a[1]); ++i) to.push_back(integer(PyList_GET_ITEM(a[1], i)));
    for (const int64_t k : to)
        if (k < 0) refuse("missed must be counts");
    list.missed = std::move(to);
    Py_RETURN_NONE;
}

template <PyObject* (*F)(PyObject* const*, Py_ssize_t)>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
    try {
        return F(args, n);
    } catch (const Raised&) {
    } catch (const Status& s) {
        return PyLong_FromLong(s.e);
    } catch (const Refused& e) {
        PyErr_SetString(PyExc_ValueError, e.what());
    } catch (const std::exception& e) {      // an allocation that failed, for one
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}
template <PyObject* (*F)(PyObject* const*, Py_ssize_t)>
constexpr PyCFunction fast() {
    return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&entry<F>));
}

PyMethodDef methods[] = {{"group_norm", fast<group_norm>(), METH_FASTCALL, nullptr},
                         {"group_norm_backward", fast<group_norm_backward>(), METH_FASTCALL, nullptr},
                         {"block_norm", fast<block_norm>(), METH_FASTCALL, nullptr},
                         {"block_norm_backward", fast<block_norm_backward>(), METH_FASTCALL, nullptr},
                         {"top_logits", fast<top_logits>(), METH_FASTCALL, nullptr},
                         {"distill", fast<distill>(), METH_FASTCALL, nullptr},
                         {"distill_loss", fast<distill_loss>(), METH_FASTCALL, nullptr},
                         {"distill_backward", fast<distill_backward>(), METH_FASTCALL, nullptr},
                         {"layout", fast<layout>(), METH_FASTCALL, nullptr},
                         {"tensors", fast<tensors>(), METH_FASTCALL, nullptr},
                         {"grad_norm", fast<grad_norm>(), METH_FASTCALL, nullptr},
                         {"adamw_step", fast<adamw_step>(), METH_FASTCALL, nullptr},
                         {"missed", fast<missed>(), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_patconv", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__patconv() { return PyModule_Create(&module); }
