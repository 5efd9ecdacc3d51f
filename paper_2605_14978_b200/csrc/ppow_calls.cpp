// One call from Python for each training-end operator: checks, allocations and the library call of binding.py's wrappers, for
// the case that all is as it should be (tensors on the current device, current stream).  The operators take 4 to 10 us on the
// device for one window of tokens; marshalled in Python a call takes 13 to 26 us.
//
// Marshalling only: the functions of the library are handed over as addresses (so that every build of it can be used), nothing
// is computed here, and a call whose arguments do not pass the checks returns None -- the Python wrapper then takes its own
// path, which says what is wrong or handles the case (another stream, another device).
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <ATen/record_function.h>
#include <c10/core/impl/LocalDispatchKeySet.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/pybind.h>

#include <string>
#include <vector>

#include "../../include/ppow.h"

namespace py = pybind11;

namespace {

struct Library {
    decltype(&ppow_head_workspace_bytes) head_workspace_bytes = nullptr;
    decltype(&ppow_head_logprob) head_logprob = nullptr;
    decltype(&ppow_head_logprob_backward) head_logprob_backward = nullptr;
    decltype(&ppow_layer_norm) layer_norm = nullptr;
    decltype(&ppow_layer_norm_workspace_bytes) layer_norm_workspace_bytes = nullptr;
    decltype(&ppow_layer_norm_backward) layer_norm_backward = nullptr;
    decltype(&ppow_pack_activation) pack_activation = nullptr;
    decltype(&ppow_unpack_activation) unpack_activation = nullptr;
    decltype(&ppow_rms_norm) rms_norm = nullptr;
    decltype(&ppow_rms_norm_workspace_bytes) rms_norm_workspace_bytes = nullptr;
    decltype(&ppow_rms_norm_backward) rms_norm_backward = nullptr;
    decltype(&ppow_clip_workspace_bytes) clip_workspace_bytes = nullptr;
    decltype(&ppow_clip_gradients) clip_gradients = nullptr;
    decltype(&ppow_sample_tokens) sample_tokens = nullptr;
} lib;

void bind(const py::dict &addresses)
{
    auto set = [&](const char *name, auto &fn) { fn = reinterpret_cast<std::decay_t<decltype(fn)>>(addresses[name].cast<uintptr_t>()); };
    set("ppow_head_workspace_bytes", lib.head_workspace_bytes);
    set("ppow_head_logprob", lib.head_logprob);
    set("ppow_head_logprob_backward", lib.head_logprob_backward);
    set("ppow_layer_norm", lib.layer_norm);
    set("ppow_layer_norm_workspace_bytes", lib.layer_norm_workspace_bytes);
    set("ppow_layer_norm_backward", lib.layer_norm_backward);
    set("ppow_pack_activation", lib.pack_activation);
    set("ppow_unpack_activation", lib.unpack_activation);
    set("ppow_rms_norm", lib.rms_norm);
    set("ppow_rms_norm_workspace_bytes", lib.rms_norm_workspace_bytes);
    set("ppow_rms_norm_backward", lib.rms_norm_backward);
    set("ppow_clip_workspace_bytes", lib.clip_workspace_bytes);
    set("ppow_clip_gradients", lib.clip_gradients);
    set("ppow_sample_tokens", lib.sample_tokens);
}

int code_of(at::ScalarType t)
{
    return t == at::kFloat ? PPOW_F32 : t == at::kBFloat16 ? PPOW_BF16 : t == at::kHalf ? PPOW_F16 : -1;
}

bool on_device(const at::Tensor &t, int dev) { return t.defined() && t.is_cuda() && t.get_device() == dev && t.layout() == at::kStrided; }
bool vector_ok(const at::Tensor &t, int64_t n, at::ScalarType type, int dev)
{
    return on_device(t, dev) && t.scalar_type() == type && t.dim() == 1 && t.size(0) == n && t.is_contiguous();
}
bool rows_ok(const at::Tensor &t, int64_t r, int64_t d, at::ScalarType type, int dev)
{
    return on_device(t, dev) && t.scalar_type() == type && t.dim() == 2 && t.size(0) == r && t.size(1) == d && (d <= 1 || t.stride(1) == 1);
}
bool packed_ok(const at::Tensor &q, const at::Tensor &s, int64_t r, int64_t d, int dev)
{
    return on_device(q, dev) && on_device(s, dev) && q.scalar_type() == at::kFloat8_e4m3fn && s.scalar_type() == at::kByte && q.dim() == 2 &&
           s.dim() == 2 && q.size(0) == r && q.size(1) == d && s.size(0) == r && s.size(1) == (d + 127) / 128 && q.is_contiguous() &&
           s.is_contiguous();
}
int64_t row_stride(const at::Tensor &t) { return t.size(0) > 1 ? t.stride(0) : t.size(1); }
bool fits(int64_t n) { return n >= 0 && n <= INT32_MAX; }

struct Place {
    int dev;
    void *stream;
    at::TensorOptions options;
    bool here;           // the tensor's device is the current one
    explicit Place(const at::Tensor &t)
        : dev(t.is_cuda() ? t.get_device() : -1), stream(nullptr), options(t.options().requires_grad(false)),
          here(dev >= 0 && dev == c10::cuda::current_device())
    {
        if (here) stream = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)dev).stream();
    }
    // Whether somebody is to see, or fill, what is allocated: dispatch modes and other changes of this thread's dispatch keys, observers of
    // operators (the profiler), deterministic algorithms, which fill memory.
    static bool watched()
    {
        const c10::impl::LocalDispatchKeySet keys = c10::impl::tls_local_dispatch_key_set();
        return keys.included_ != c10::default_included_set || keys.excluded_ != c10::default_excluded_set || at::hasCallbacks() ||
               at::globalContext().deterministicAlgorithms();
    }
    // Unwatched, without the dispatcher, which the type and device would only lead back here (3 tensors: 0.9 us less).
    at::Tensor empty(at::IntArrayRef sizes, at::ScalarType type) const
    {
        if (watched()) return at::empty(sizes, options.dtype(type));
        return at::detail::empty_cuda(sizes, type, c10::Device(c10::kCUDA, (c10::DeviceIndex)dev), c10::nullopt);
    }
    at::Tensor scratch(size_t bytes) const { return empty({(int64_t)(bytes ? bytes : 256)}, at::kByte); }
};

py::object status_of(ppow_status st) { return py::int_((int)st); }
py::object to_python(const at::Tensor &t) { return t.defined() ? py::cast(t) : py::none(); }

bool head_params(ppow_head_params &p, const at::Tensor &hidden, const at::Tensor &weight, const at::Tensor &tokens, double temperature,
                 const Place &at)
{
    if (!at.here || hidden.dim() != 2 || weight.dim() != 2) return false;
    const auto type = hidden.scalar_type();
    const int64_t T = hidden.size(0), D = hidden.size(1), V = weight.size(0);
    if ((type != at::kBFloat16 && type != at::kHalf) || !fits(T) || !fits(D) || !fits(V) || !rows_ok(hidden, T, D, type, at.dev) ||
        !rows_ok(weight, V, D, type, at.dev) || !vector_ok(tokens, T, at::kInt, at.dev))
        return false;
    p = {(int32_t)T, (int32_t)V, (int32_t)D, code_of(type), row_stride(hidden), row_stride(weight), (float)temperature};
    return true;
}

// Each returns (status, outputs...), or None where the Python path is to be taken.
py::object head_logprob(const at::Tensor &hidden, const at::Tensor &weight, const at::Tensor &tokens, double temperature, bool want_workspace)
{
    const Place at(hidden);
    ppow_head_params p;
    if (!head_params(p, hidden, weight, tokens, temperature, at)) return py::none();
    const at::Tensor logp = at.empty({p.T}, at::kFloat), lse = at.empty({p.T}, at::kFloat);
    const size_t bytes = lib.head_workspace_bytes(&p, 0);
    const at::Tensor ws = at.scratch(bytes);
    const ppow_status st = lib.head_logprob(&p, hidden.data_ptr(), weight.data_ptr(), tokens.data_ptr<int32_t>(), logp.data_ptr<float>(),
                                            lse.data_ptr<float>(), ws.data_ptr(), bytes, at.stream);
    return py::make_tuple(status_of(st), to_python(logp), to_python(lse), to_python(want_workspace ? ws : at::Tensor()));
}

py::object head_logprob_backward(const at::Tensor &hidden, const at::Tensor &weight, const at::Tensor &tokens, const at::Tensor &lse,
                                 const at::Tensor &grad_logp, double temperature, bool want_hidden, bool want_weight, bool want_workspace)
{
    const Place at(hidden);
    ppow_head_params p;
    if (!head_params(p, hidden, weight, tokens, temperature, at) || !vector_ok(lse, p.T, at::kFloat, at.dev) ||
        !vector_ok(grad_logp, p.T, at::kFloat, at.dev))
        return py::none();
    const at::Tensor gh = want_hidden ? at.empty({p.T, p.D}, hidden.scalar_type()) : at::Tensor();
    const at::Tensor gw = want_weight ? at.empty({p.V, p.D}, hidden.scalar_type()) : at::Tensor();
    const size_t bytes = lib.head_workspace_bytes(&p, 1);
    const at::Tensor ws = at.scratch(bytes);
    const ppow_status st = lib.head_logprob_backward(&p, hidden.data_ptr(), weight.data_ptr(), tokens.data_ptr<int32_t>(),
                                                     lse.data_ptr<float>(), grad_logp.data_ptr<float>(), want_hidden ? gh.data_ptr() : nullptr,
                                                     want_weight ? gw.data_ptr() : nullptr, ws.data_ptr(), bytes, at.stream);
    return py::make_tuple(status_of(st), to_python(gh), to_python(gw), to_python(want_workspace ? ws : at::Tensor()));
}

bool norm_params(ppow_norm_params &p, const at::Tensor &rows, const at::Tensor &weight, double eps, const Place &at)
{
    if (!at.here || rows.dim() != 2) return false;
    const int64_t R = rows.size(0), D = rows.size(1);
    if (!fits(R) || !fits(D) || code_of(rows.scalar_type()) < 0 || code_of(weight.scalar_type()) < 0 ||
        !rows_ok(rows, R, D, rows.scalar_type(), at.dev) || !vector_ok(weight, D, weight.scalar_type(), at.dev))
        return false;
    p = {(int32_t)R, (int32_t)D, code_of(rows.scalar_type()), code_of(weight.scalar_type()), (float)eps};
    return true;
}

py::object layer_norm(const at::Tensor &x, const at::Tensor &weight, const c10::optional<at::Tensor> &bias, double eps, bool checkpoint)
{
    const Place at(x);
    ppow_norm_params p;
    if (!norm_params(p, x, weight, eps, at) || (bias && !vector_ok(*bias, p.D, weight.scalar_type(), at.dev))) return py::none();
    const at::Tensor y = at.empty({p.R, p.D}, x.scalar_type()), mean = at.empty({p.R}, at::kFloat), rstd = at.empty({p.R}, at::kFloat);
    at::Tensor packed, scale;
    if (checkpoint) {
        packed = at.empty({p.R, p.D}, at::kFloat8_e4m3fn);
        scale = at.empty({p.R, (p.D + 127) / 128}, at::kByte);
    }
    const ppow_status st = lib.layer_norm(&p, x.data_ptr(), row_stride(x), weight.data_ptr(), bias ? bias->data_ptr() : nullptr, y.data_ptr(),
                                          mean.data_ptr<float>(), rstd.data_ptr<float>(), checkpoint ? (uint8_t *)packed.data_ptr() : nullptr,
                                          checkpoint ? scale.data_ptr<uint8_t>() : nullptr, at.stream);
    return py::make_tuple(status_of(st), to_python(y), to_python(mean), to_python(rstd), to_python(packed), to_python(scale));
}

py::object layer_norm_backward(const at::Tensor &grad_y, const c10::optional<at::Tensor> &x, const c10::optional<at::Tensor> &packed,
                               const c10::optional<at::Tensor> &scale, const at::Tensor &weight, const at::Tensor &mean,
                               const at::Tensor &rstd, bool want_bias)
{
    const Place at(grad_y);
    ppow_norm_params p;
    if (!norm_params(p, grad_y, weight, 1e-5, at) || !vector_ok(mean, p.R, at::kFloat, at.dev) || !vector_ok(rstd, p.R, at::kFloat, at.dev))
        return py::none();
    if (x ? !rows_ok(*x, p.R, p.D, grad_y.scalar_type(), at.dev) : !packed || !scale || !packed_ok(*packed, *scale, p.R, p.D, at.dev))
        return py::none();
    const at::Tensor gx = at.empty({p.R, p.D}, grad_y.scalar_type()), gw = at.empty({p.D}, weight.scalar_type());
    const at::Tensor gb = want_bias ? at.empty({p.D}, weight.scalar_type()) : at::Tensor();
    const size_t bytes = lib.layer_norm_workspace_bytes(&p);
    const at::Tensor ws = at.scratch(bytes);
    const ppow_status st = lib.layer_norm_backward(
        &p, grad_y.data_ptr(), row_stride(grad_y), x ? x->data_ptr() : nullptr, x ? row_stride(*x) : p.D,
        x ? nullptr : (const uint8_t *)packed->data_ptr(), x ? nullptr : scale->data_ptr<uint8_t>(), weight.data_ptr(), mean.data_ptr<float>(),
        rstd.data_ptr<float>(), gx.data_ptr(), gw.data_ptr(), want_bias ? gb.data_ptr() : nullptr, ws.data_ptr(), bytes, at.stream);
    return py::make_tuple(status_of(st), to_python(gx), to_python(gw), to_python(gb));
}

py::object pack_activation(const at::Tensor &x)
{
    const Place at(x);
    if (!at.here || x.dim() != 2 || code_of(x.scalar_type()) < 0) return py::none();
    const int64_t R = x.size(0), D = x.size(1);
    if (!fits(R) || !fits(D) || !rows_ok(x, R, D, x.scalar_type(), at.dev)) return py::none();
    const at::Tensor packed = at.empty({R, D}, at::kFloat8_e4m3fn), scale = at.empty({R, (D + 127) / 128}, at::kByte);
    const ppow_status st = lib.pack_activation(x.data_ptr(), row_stride(x), (int32_t)R, (int32_t)D, code_of(x.scalar_type()),
                                               (uint8_t *)packed.data_ptr(), scale.data_ptr<uint8_t>(), at.stream);
    return py::make_tuple(status_of(st), to_python(packed), to_python(scale));
}

py::object unpack_activation(const at::Tensor &packed, const at::Tensor &scale, int code)
{
    const Place at(packed);
    if (!at.here || packed.dim() != 2) return py::none();
    const int64_t R = packed.size(0), D = packed.size(1);
    if (!fits(R) || !fits(D) || !packed_ok(packed, scale, R, D, at.dev)) return py::none();
    const auto type = code == PPOW_F32 ? at::kFloat : code == PPOW_BF16 ? at::kBFloat16 : at::kHalf;
    const at::Tensor x = at.empty({R, D}, type);
    const ppow_status st = lib.unpack_activation((const uint8_t *)packed.data_ptr(), scale.data_ptr<uint8_t>(), (int32_t)R, (int32_t)D, code,
                                                 x.data_ptr(), at.stream);
    return py::make_tuple(status_of(st), to_python(x));
}

py::object rms_norm(const at::Tensor &x, const at::Tensor &weight, const c10::optional<at::Tensor> &residual, double eps, bool checkpoint,
                    bool packed_output)
{
    const Place at(x);
    ppow_norm_params p;
    if (!norm_params(p, x, weight, eps, at) || (residual && !rows_ok(*residual, p.R, p.D, x.scalar_type(), at.dev))) return py::none();
    at::Tensor sum, y, y_packed, y_scale, packed, scale;
    if (residual) sum = at.empty({p.R, p.D}, x.scalar_type());
    if (packed_output) {
        y_packed = at.empty({p.R, p.D}, at::kFloat8_e4m3fn);
        y_scale = at.empty({p.R, (p.D + 127) / 128}, at::kByte);
    } else {
        y = at.empty({p.R, p.D}, x.scalar_type());
    }
    const at::Tensor rstd = at.empty({p.R}, at::kFloat);
    if (checkpoint) {
        packed = at.empty({p.R, p.D}, at::kFloat8_e4m3fn);
        scale = at.empty({p.R, (p.D + 127) / 128}, at::kByte);
    }
    const ppow_status st = lib.rms_norm(
        &p, x.data_ptr(), row_stride(x), residual ? residual->data_ptr() : nullptr, residual ? row_stride(*residual) : p.D, weight.data_ptr(),
        residual ? sum.data_ptr() : nullptr, packed_output ? nullptr : y.data_ptr(), rstd.data_ptr<float>(),
        packed_output ? (uint8_t *)y_packed.data_ptr() : nullptr, packed_output ? y_scale.data_ptr<uint8_t>() : nullptr,
        checkpoint ? (uint8_t *)packed.data_ptr() : nullptr, checkpoint ? scale.data_ptr<uint8_t>() : nullptr, at.stream);
    return py::make_tuple(status_of(st), to_python(sum), to_python(y), to_python(rstd), to_python(y_packed), to_python(y_scale), to_python(packed),
                          to_python(scale));
}

py::object rms_norm_backward(const at::Tensor &grad_y, const c10::optional<at::Tensor> &x, const c10::optional<at::Tensor> &packed,
                             const c10::optional<at::Tensor> &scale, const at::Tensor &weight, const at::Tensor &rstd,
                             const c10::optional<at::Tensor> &grad_sum)
{
    const Place at(grad_y);
    ppow_norm_params p;
    if (!norm_params(p, grad_y, weight, 1e-5, at) || !vector_ok(rstd, p.R, at::kFloat, at.dev) ||
        (grad_sum && !rows_ok(*grad_sum, p.R, p.D, grad_y.scalar_type(), at.dev)))
        return py::none();
    if (x ? !rows_ok(*x, p.R, p.D, grad_y.scalar_type(), at.dev) : !packed || !scale || !packed_ok(*packed, *scale, p.R, p.D, at.dev))
        return py::none();
    const at::Tensor gx = at.empty({p.R, p.D}, grad_y.scalar_type()), gw = at.empty({p.D}, weight.scalar_type());
    const size_t bytes = lib.rms_norm_workspace_bytes(&p);
    const at::Tensor ws = at.scratch(bytes);
    const ppow_status st = lib.rms_norm_backward(
        &p, grad_y.data_ptr(), row_stride(grad_y), grad_sum ? grad_sum->data_ptr() : nullptr, grad_sum ? row_stride(*grad_sum) : p.D,
        x ? x->data_ptr() : nullptr, x ? row_stride(*x) : p.D, x ? nullptr : (const uint8_t *)packed->data_ptr(),
        x ? nullptr : scale->data_ptr<uint8_t>(), weight.data_ptr(), rstd.data_ptr<float>(), gx.data_ptr(), gw.data_ptr(), ws.data_ptr(), bytes,
        at.stream);
    return py::make_tuple(status_of(st), to_python(gx), to_python(gw));
}

// The tensors of a list, without a reference each: the list holds them.  False if something else is in it.
bool tensors_of(const py::list &list, std::vector<const at::Tensor *> &tensors)
{
    const size_t n = list.size();
    tensors.resize(n);
    for (size_t i = 0; i < n; ++i) {
        PyObject *item = PyList_GET_ITEM(list.ptr(), (Py_ssize_t)i);
        if (!THPVariable_Check(item)) return false;
        tensors[i] = &THPVariable_Unpack(item);
    }
    return true;
}

bool alike(const c10::TensorImpl *a, const c10::TensorImpl *b)
{
    return a->key_set() == b->key_set() && a->dtype() == b->dtype() && a->device() == b->device();
}

py::object clip_gradients(const py::list &grad_list, const py::object &out_list, double max_norm)
{
    std::vector<const at::Tensor *> grads, out;
    const size_t n = grad_list.size();
    if (n == 0 || n > 65536 || !tensors_of(grad_list, grads)) return py::none();
    if (!out_list.is_none() && (!py::isinstance<py::list>(out_list) || !tensors_of(py::reinterpret_borrow<py::list>(out_list), out) || out.size() != n))
        return py::none();
    const bool write = !out_list.is_none();
    const Place at(*grads[0]);
    if (!at.here) return py::none();
    std::vector<const void *> from(n);
    std::vector<void *> to(write ? n : 0);
    std::vector<int64_t> sizes(n);
    std::vector<int32_t> dtypes(n);
    // tensors with the dispatch keys, the device and the type of one that was looked at are like it
    const c10::TensorImpl *like = nullptr;
    int32_t like_code = -1;
    for (size_t i = 0; i < n; ++i) {
        const at::Tensor &g = *grads[i];
        const c10::TensorImpl *impl = g.unsafeGetTensorImpl();
        if (!like || !alike(impl, like)) {
            if (!on_device(g, at.dev) || (like_code = code_of(g.scalar_type())) < 0) return py::none();
            like = impl;
        }
        if (!g.is_non_overlapping_and_dense()) return py::none();
        dtypes[i] = like_code;
        from[i] = g.data_ptr();                              // in place it has to be the address that is written
        sizes[i] = g.numel();
        if (!write) continue;
        const at::Tensor &o = *out[i];
        if (&o != &g && (!o.defined() || !alike(o.unsafeGetTensorImpl(), like) || o.sizes() != g.sizes() || o.strides() != g.strides())) return py::none();
        to[i] = o.data_ptr();
    }
    const at::Tensor norm = at.empty({}, at::kFloat);
    const size_t bytes = lib.clip_workspace_bytes((int32_t)n);
    const at::Tensor ws = at.scratch(bytes);
    const ppow_status st = lib.clip_gradients((int32_t)n, from.data(), write ? to.data() : nullptr, sizes.data(), dtypes.data(), max_norm,
                                              norm.data_ptr<float>(), ws.data_ptr(), bytes, at.stream);
    if (st == PPOW_OK)
        for (const at::Tensor *t : out)                      // for autograd, modified in place (inference tensors keep no version)
            if (!t->is_inference()) t->unsafeGetTensorImpl()->bump_version();
    return py::make_tuple(status_of(st), to_python(norm));
}

py::object sample_tokens(const at::Tensor &logits, const at::Tensor &uniforms, double temperature, int64_t top_k, double top_p, double min_p)
{
    const Place at(logits);
    if (!at.here || logits.dim() != 2 || code_of(logits.scalar_type()) < 0 || top_k < INT32_MIN || top_k > INT32_MAX) return py::none();
    const int64_t R = logits.size(0), V = logits.size(1);
    if (!fits(R) || !fits(V) || !rows_ok(logits, R, V, logits.scalar_type(), at.dev) || !vector_ok(uniforms, R, at::kFloat, at.dev)) return py::none();
    const ppow_sample_params p = {(int32_t)R, (int32_t)V, code_of(logits.scalar_type()), (int32_t)top_k, row_stride(logits), temperature, top_p, min_p};
    const at::Tensor tokens = at.empty({R}, at::kInt), logp = at.empty({R}, at::kFloat), kept = at.empty({R}, at::kInt);
    const ppow_status st = lib.sample_tokens(&p, logits.data_ptr(), uniforms.data_ptr<float>(), tokens.data_ptr<int32_t>(), logp.data_ptr<float>(),
                                             kept.data_ptr<int32_t>(), at.stream);
    return py::make_tuple(status_of(st), to_python(tokens), to_python(logp), to_python(kept));
}

// Out of memory is the Python path's to report: its allocations raise torch's own exception.
template <typename... Args> auto guarded(py::object (*f)(Args...))
{
    return [f](Args... args) -> py::object {
        try {
            return f(args...);
        } catch (const c10::OutOfMemoryError &) {
            return py::none();
        }
    };
}

}  // namespace

PYBIND11_MODULE(_calls, m)
{
    const std::string mark = PPOW_TORCH_MARK;        // "ppow_calls for torch <version>"
    m.attr("torch_version") = mark.substr(mark.rfind(' ') + 1);
    m.def("bind", &bind);
    m.def("head_logprob", guarded(&head_logprob));
    m.def("head_logprob_backward", guarded(&head_logprob_backward));
    m.def("layer_norm", guarded(&layer_norm));
    m.def("layer_norm_backward", guarded(&layer_norm_backward));
    m.def("pack_activation", guarded(&pack_activation));
    m.def("unpack_activation", guarded(&unpack_activation));
    m.def("rms_norm", guarded(&rms_norm));
    m.def("rms_norm_backward", guarded(&rms_norm_backward));
    m.def("clip_gradients", guarded(&clip_gradients));
    m.def("sample_tokens", guarded(&sample_tokens));
}
