// One call from Python for each training-end operator: checks, allocations and the library call of binding.py's wrappers, for
// the case that all is as it should be (tensors on the current device, current stream).  The operators take 4 to 10 us on the
// device for one window of tokens; marshalled in Python a call takes 13 to 26 us.
//
// Marshalling only: the functions of the library are handed over as addresses (so that every build of it can be used), nothing
// is computed here, and a call whose arguments do not pass the checks returns None -- the Python wrapper then takes its own
// path, which says what is wrong or handles the case (another stream, another device).
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/utils/pybind.h>

#include <string>

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
    at::Tensor empty(at::IntArrayRef sizes, at::ScalarType type) const { return at::empty(sizes, options.dtype(type)); }
    at::Tensor scratch(size_t bytes) const { return at::empty({(int64_t)(bytes ? bytes : 256)}, options.dtype(at::kByte)); }
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
}
