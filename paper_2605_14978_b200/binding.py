"""ctypes binding of ``libppow.so``: the same entry points as ``include/ppow.h``, marshalling only.

Every step of the scoring path runs in the CUDA library.  There is no CPU or PyTorch fallback: if
the library has not been built, or a tensor is not on a CUDA device, the call raises.
PyTorch is used for device memory and streams only.
"""
from __future__ import annotations

import contextlib
import ctypes
import os
import warnings
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
# PPOW_LIBRARY=checked loads the bounds-checked build of the same sources (see ppow_checked_failures)
#                        timeline loads the build whose row kernel records a per-warp timeline (ppow_timeline_read)
LIB_PATH = os.path.join(_HERE, {"checked": "libppow_checked.so", "timeline": "libppow_timeline.so"}.get(
    os.environ.get("PPOW_LIBRARY", ""), "libppow.so"))

PPOW_OK = 0
PPOW_ERR_INVALID_ARG, PPOW_ERR_UNSUPPORTED, PPOW_ERR_WORKSPACE, PPOW_ERR_CUDA, PPOW_ERR_DEVICE_TIMEOUT = 1, 2, 3, 4, 5
PPOW_GREEDY, PPOW_STOCHASTIC = 0, 1
PPOW_F32, PPOW_BF16, PPOW_F16 = 0, 1, 2
LOGIT_DTYPES = {PPOW_F32: torch.float32, PPOW_BF16: torch.bfloat16, PPOW_F16: torch.float16}
DTYPE_CODES = {v: k for k, v in LOGIT_DTYPES.items()}
PPOW_FLAG_TOKEN_RANGE, PPOW_FLAG_DEVICE_TIMEOUT, PPOW_FLAG_BOUNDS = 1, 2, 4

EXPORTS = ("ppow_score_workspace_bytes", "ppow_score_windows", "ppow_score_windows_traced", "ppow_read_error_flags",
           "ppow_select_workspace_bytes", "ppow_select_windows", "ppow_host_scratch_bytes",
           "ppow_score_and_select_host", "ppow_noalloc_scratch_bytes", "ppow_score_windows_noalloc",
           "ppow_noalloc_read_error_flags",
           "ppow_group_advantage", "ppow_sequence_windows", "ppow_sequence_windows_mixed", "ppow_expected_acceptance",
           "ppow_reference_logprob", "ppow_selftest_wait_timeout", "ppow_stream_read_probe", "ppow_score_kernel_launches",
           "ppow_head_workspace_bytes", "ppow_head_plan", "ppow_head_logprob", "ppow_head_logprob_backward",
           "ppow_layer_norm", "ppow_layer_norm_workspace_bytes", "ppow_layer_norm_backward", "ppow_pack_activation",
           "ppow_unpack_activation", "ppow_rms_norm", "ppow_rms_norm_workspace_bytes", "ppow_rms_norm_backward",
           "ppow_clip_workspace_bytes", "ppow_clip_gradients", "ppow_sample_tokens",
           "ppow_checked_failures", "ppow_timeline_read", "ppow_status_string", "ppow_version")

POSITION_OUTPUTS = {"accept_flag": torch.uint8, "kl": torch.float32, "conf": torch.float32, "crit": torch.float32,
                    "logp_tok": torch.float32, "logq_tok": torch.float32, "target_argmax": torch.int32}
WINDOW_OUTPUTS = {"accepted_len": torch.int32, "reward_speedup": torch.float32, "reward_dist": torch.float32,
                  "reward": torch.float32, "delta": torch.float32, "score": torch.float32}
# training-side outputs of the scoring pass, written only when asked for
TRAIN_POSITION_OUTPUTS = {"kl_rev": torch.float32, "nabla": torch.float32, "lse_p": torch.float32,
                          "lse_q": torch.float32}
TRAIN_WINDOW_OUTPUTS = {"kl_rev_mean": torch.float32}
_ALL_OUTPUTS = {**POSITION_OUTPUTS, **WINDOW_OUTPUTS, **TRAIN_POSITION_OUTPUTS, **TRAIN_WINDOW_OUTPUTS}


class ppow_params(ctypes.Structure):
    _fields_ = [("N", ctypes.c_int32), ("K", ctypes.c_int32), ("V", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("mode", ctypes.c_int32),
                ("c", ctypes.c_float), ("temperature", ctypes.c_float),
                ("eta", ctypes.c_float), ("eps", ctypes.c_float)]


class ppow_outputs(ctypes.Structure):
    # field order is the order of the C struct
    _fields_ = [(n, ctypes.c_void_p) for n in
                ("accept_flag", "accepted_len", "reward_speedup", "reward_dist", "reward", "delta", "score",
                 "kl", "conf", "crit", "logp_tok", "logq_tok", "target_argmax",
                 "kl_rev", "kl_rev_mean", "nabla", "lse_p", "lse_q")]


class ppow_head_params(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int32), ("V", ctypes.c_int32), ("D", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("hidden_stride", ctypes.c_int64), ("weight_stride", ctypes.c_int64), ("temperature", ctypes.c_float)]


class ppow_norm_params(ctypes.Structure):
    _fields_ = [("R", ctypes.c_int32), ("D", ctypes.c_int32), ("dtype", ctypes.c_int32), ("param_dtype", ctypes.c_int32),
                ("eps", ctypes.c_float)]


class ppow_sample_params(ctypes.Structure):
    _fields_ = [("R", ctypes.c_int32), ("V", ctypes.c_int32), ("dtype", ctypes.c_int32), ("top_k", ctypes.c_int32),
                ("logits_stride", ctypes.c_int64), ("temperature", ctypes.c_double), ("top_p", ctypes.c_double), ("min_p", ctypes.c_double)]


class PpowError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__("%s failed: %s (status %d)" % (where, ppow_status_string(status), status))


_lib = None


def load_library():
    """Load libppow.so; raises if it was not built (there is no fallback path)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError("libppow.so is missing: build it with `python -m paper_2605_14978_b200.build` "
                           "(the scoring path has no CPU or PyTorch fallback)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    lib.ppow_score_workspace_bytes.restype = sz
    lib.ppow_score_workspace_bytes.argtypes = [ctypes.POINTER(ppow_params)]
    lib.ppow_score_windows.restype = ctypes.c_int
    lib.ppow_score_windows.argtypes = [ctypes.POINTER(ppow_params), vp, vp, vp, vp, vp, vp,
                                       ctypes.POINTER(ppow_outputs), vp, sz, vp]
    lib.ppow_score_windows_traced.restype = ctypes.c_int
    lib.ppow_score_windows_traced.argtypes = lib.ppow_score_windows.argtypes + [vp, vp]
    lib.ppow_read_error_flags.restype = ctypes.c_int
    lib.ppow_read_error_flags.argtypes = [vp, ctypes.POINTER(ctypes.c_uint32), vp]
    lib.ppow_select_workspace_bytes.restype = sz
    lib.ppow_select_workspace_bytes.argtypes = [i32]
    lib.ppow_select_windows.restype = ctypes.c_int
    lib.ppow_select_windows.argtypes = [vp, i32, i32, vp, vp, vp, sz, vp]
    lib.ppow_host_scratch_bytes.restype = sz
    lib.ppow_host_scratch_bytes.argtypes = [ctypes.POINTER(ppow_params), i32]
    lib.ppow_score_and_select_host.restype = ctypes.c_int
    lib.ppow_score_and_select_host.argtypes = [ctypes.POINTER(ppow_params), vp, vp, vp, vp, vp, vp,
                                               ctypes.POINTER(ppow_outputs), i32, vp, vp, vp, sz, vp]
    lib.ppow_noalloc_scratch_bytes.restype = sz
    lib.ppow_noalloc_scratch_bytes.argtypes = []
    lib.ppow_score_windows_noalloc.restype = ctypes.c_int
    lib.ppow_score_windows_noalloc.argtypes = [ctypes.POINTER(ppow_params), vp, vp, vp, vp, vp, vp,
                                               ctypes.POINTER(ppow_outputs), vp]
    lib.ppow_noalloc_read_error_flags.restype = ctypes.c_int
    lib.ppow_noalloc_read_error_flags.argtypes = [ctypes.POINTER(ctypes.c_uint32), vp]
    lib.ppow_group_advantage.restype = ctypes.c_int
    lib.ppow_group_advantage.argtypes = [vp, i32, i32, ctypes.c_float, vp, vp]
    lib.ppow_sequence_windows.restype = ctypes.c_int
    lib.ppow_sequence_windows.argtypes = [vp, vp, i32, i32, vp, vp, vp, vp]
    lib.ppow_sequence_windows_mixed.restype = ctypes.c_int
    lib.ppow_sequence_windows_mixed.argtypes = [vp, vp, i32, i32, ctypes.c_float, vp, vp, vp, vp, vp]
    lib.ppow_expected_acceptance.restype = ctypes.c_int
    lib.ppow_expected_acceptance.argtypes = [ctypes.POINTER(ppow_params), vp, vp, vp, vp, vp, vp, vp]
    lib.ppow_reference_logprob.restype = ctypes.c_int
    lib.ppow_reference_logprob.argtypes = [ctypes.POINTER(ppow_params), vp, vp, vp, vp, vp]
    lib.ppow_selftest_wait_timeout.restype = ctypes.c_int
    lib.ppow_selftest_wait_timeout.argtypes = [vp, sz, ctypes.c_uint32, vp]
    lib.ppow_stream_read_probe.restype = ctypes.c_int
    lib.ppow_stream_read_probe.argtypes = [vp, sz, vp, vp]
    lib.ppow_score_kernel_launches.restype = ctypes.c_int
    lib.ppow_score_kernel_launches.argtypes = [ctypes.POINTER(ppow_params)]
    lib.ppow_head_workspace_bytes.restype = sz
    lib.ppow_head_workspace_bytes.argtypes = [ctypes.POINTER(ppow_head_params), ctypes.c_int]
    lib.ppow_head_plan.restype = ctypes.c_int
    lib.ppow_head_plan.argtypes = [ctypes.POINTER(ppow_head_params), i32, i32] + [ctypes.POINTER(i32)] * 3
    lib.ppow_head_logprob.restype = ctypes.c_int
    lib.ppow_head_logprob.argtypes = [ctypes.POINTER(ppow_head_params), vp, vp, vp, vp, vp, vp, sz, vp]
    lib.ppow_head_logprob_backward.restype = ctypes.c_int
    lib.ppow_head_logprob_backward.argtypes = [ctypes.POINTER(ppow_head_params), vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.ppow_layer_norm.restype = ctypes.c_int
    i64 = ctypes.c_int64
    lib.ppow_layer_norm.argtypes = [ctypes.POINTER(ppow_norm_params), vp, i64, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.ppow_layer_norm_workspace_bytes.restype = sz
    lib.ppow_layer_norm_workspace_bytes.argtypes = [ctypes.POINTER(ppow_norm_params)]
    lib.ppow_layer_norm_backward.restype = ctypes.c_int
    lib.ppow_layer_norm_backward.argtypes = [ctypes.POINTER(ppow_norm_params), vp, i64, vp, i64, vp, vp, vp, vp, vp, vp, vp, vp,
                                             vp, sz, vp]
    lib.ppow_pack_activation.restype = ctypes.c_int
    lib.ppow_pack_activation.argtypes = [vp, i64, i32, i32, i32, vp, vp, vp]
    lib.ppow_unpack_activation.restype = ctypes.c_int
    lib.ppow_unpack_activation.argtypes = [vp, vp, i32, i32, i32, vp, vp]
    lib.ppow_rms_norm.restype = ctypes.c_int
    lib.ppow_rms_norm.argtypes = [ctypes.POINTER(ppow_norm_params), vp, i64, vp, i64] + [vp] * 9
    lib.ppow_rms_norm_workspace_bytes.restype = sz
    lib.ppow_rms_norm_workspace_bytes.argtypes = [ctypes.POINTER(ppow_norm_params)]
    lib.ppow_rms_norm_backward.restype = ctypes.c_int
    lib.ppow_rms_norm_backward.argtypes = [ctypes.POINTER(ppow_norm_params), vp, i64, vp, i64, vp, i64] + [vp] * 7 + [sz, vp]
    lib.ppow_clip_workspace_bytes.restype = sz
    lib.ppow_clip_workspace_bytes.argtypes = [i32]
    lib.ppow_clip_gradients.restype = ctypes.c_int
    lib.ppow_clip_gradients.argtypes = [i32, vp, vp, vp, vp, ctypes.c_double, vp, vp, sz, vp]
    lib.ppow_sample_tokens.restype = ctypes.c_int
    lib.ppow_sample_tokens.argtypes = [ctypes.POINTER(ppow_sample_params)] + [vp] * 6
    lib.ppow_checked_failures.restype = ctypes.c_int
    lib.ppow_checked_failures.argtypes = [ctypes.POINTER(ctypes.c_uint32), ctypes.POINTER(ctypes.c_uint32)]
    lib.ppow_timeline_read.restype = ctypes.c_int
    lib.ppow_timeline_read.argtypes = [vp, sz]
    lib.ppow_status_string.restype = ctypes.c_char_p
    lib.ppow_status_string.argtypes = [ctypes.c_int]
    lib.ppow_version.restype = ctypes.c_int
    lib.ppow_version.argtypes = []
    _bind_calls(lib)
    _lib = lib
    return lib


class _NoCalls:
    """In the place of the extension module where that does not load: every call goes the wrappers' Python way."""

    def __getattr__(self, name):
        return lambda *args: None


_calls = None
CALLED = ("ppow_head_workspace_bytes", "ppow_head_logprob", "ppow_head_logprob_backward", "ppow_layer_norm",
          "ppow_layer_norm_workspace_bytes", "ppow_layer_norm_backward", "ppow_pack_activation", "ppow_unpack_activation", "ppow_rms_norm",
          "ppow_rms_norm_workspace_bytes", "ppow_rms_norm_backward", "ppow_clip_workspace_bytes", "ppow_clip_gradients", "ppow_sample_tokens")


def _bind_calls(lib) -> None:
    """Hand the addresses of the training-end entry points to the extension module that marshals their calls.  A module that is
    missing or was built against another torch costs those calls 5 to 15 us each and nothing else."""
    global _calls
    try:
        from . import _calls as module
        if module.torch_version != torch.__version__:
            raise ImportError("built against torch %s, this is %s" % (module.torch_version, torch.__version__))
        module.bind({n: ctypes.cast(getattr(lib, n), ctypes.c_void_p).value for n in CALLED})
    except ImportError as e:
        warnings.warn("_calls.so does not load (%s): training-end calls are marshalled in Python, which is slower; build it with "
                      "`python -m paper_2605_14978_b200.build`" % e, RuntimeWarning, stacklevel=3)
        module = _NoCalls()
    _calls = module


def ppow_status_string(status: int) -> str:
    return load_library().ppow_status_string(int(status)).decode()


def ppow_version() -> int:
    return int(load_library().ppow_version())


def _dev_ptr(t: Optional[torch.Tensor], dtype=None, name="tensor"):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("%s must live on a CUDA device (no CPU path exists)" % name)
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    if dtype is not None and t.dtype != dtype:
        raise ValueError("%s must have dtype %s, got %s" % (name, dtype, t.dtype))
    return ctypes.c_void_p(t.data_ptr())


def _stream_ptr(stream):
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


def make_params(N, K, V, dtype, mode, c, temperature=1.0, eta=1.0, eps=0.5) -> ppow_params:
    return ppow_params(int(N), int(K), int(V), int(dtype), int(mode), float(c), float(temperature),
                       float(eta), float(eps))


def ppow_score_workspace_bytes(params: ppow_params) -> int:
    return int(load_library().ppow_score_workspace_bytes(ctypes.byref(params)))


def ppow_score_kernel_launches(params: ppow_params) -> int:
    return int(load_library().ppow_score_kernel_launches(ctypes.byref(params)))


def ppow_stream_read_probe(data: torch.Tensor, checksum: torch.Tensor, stream=None) -> None:
    """One read-only streaming pass over ``data`` (any dtype, contiguous, a multiple of 16 bytes); XOR of its
    32-bit words into ``checksum`` (one int32/uint32-sized CUDA element)."""
    lib = load_library()
    st = lib.ppow_stream_read_probe(_dev_ptr(data, None, "data"), data.numel() * data.element_size(),
                                    _dev_ptr(checksum, None, "checksum"), _stream_ptr(stream))
    if st != PPOW_OK:
        raise PpowError(st, "ppow_stream_read_probe")


def ppow_checked_failures():
    """(status, failed checks, first failing site) of the bounds-checked build; status PPOW_ERR_UNSUPPORTED and
    zeros from the ordinary library."""
    f, site = ctypes.c_uint32(0), ctypes.c_uint32(0)
    st = load_library().ppow_checked_failures(ctypes.byref(f), ctypes.byref(site))
    return int(st), int(f.value), int(site.value)


def ppow_timeline_read(warps: int):
    """(status, array [warps, 11] of uint64) from the timeline build; status PPOW_ERR_UNSUPPORTED otherwise."""
    import numpy as np
    buf = np.zeros((int(warps), 11), dtype=np.uint64)
    st = load_library().ppow_timeline_read(ctypes.c_void_p(buf.ctypes.data), int(warps))
    return int(st), buf


def ppow_select_workspace_bytes(N: int) -> int:
    return int(load_library().ppow_select_workspace_bytes(int(N)))


def alloc_outputs(N: int, K: int, device) -> dict:
    out = {k: torch.empty((N, K), dtype=dt, device=device) for k, dt in POSITION_OUTPUTS.items()}
    out.update({k: torch.empty((N,), dtype=dt, device=device) for k, dt in WINDOW_OUTPUTS.items()})
    return out


def alloc_train_outputs(N: int, K: int, device) -> dict:
    out = {k: torch.empty((N, K), dtype=dt, device=device) for k, dt in TRAIN_POSITION_OUTPUTS.items()}
    out.update({k: torch.empty((N,), dtype=dt, device=device) for k, dt in TRAIN_WINDOW_OUTPUTS.items()})
    return out


def alloc_workspace(nbytes: int, device) -> torch.Tensor:
    # torch's caching allocator returns 512-byte aligned blocks
    return torch.empty((max(int(nbytes), 256),), dtype=torch.uint8, device=device)


def _event_ptr(ev):
    """cudaEvent_t of a torch.cuda.Event (created on first record), or NULL."""
    if ev is None:
        return None
    if not ev.cuda_event:
        ev.record()           # torch creates the CUDA event lazily; the library re-records it
    return ctypes.c_void_p(ev.cuda_event)


def ppow_score_windows(params: ppow_params, draft_logits, target_logits, draft_tokens, uniforms, valid_len,
                       ref_logp, outputs: dict, workspace: torch.Tensor, stream=None) -> None:
    """Enqueue the scoring pass; raises PpowError on a non-OK status.  ``outputs`` maps output names
    to preallocated CUDA tensors (absent or None = not written; ``accepted_len`` is required)."""
    ppow_score_windows_traced(params, draft_logits, target_logits, draft_tokens, uniforms, valid_len, ref_logp,
                              outputs, workspace, stream, None, None)


def ppow_score_windows_traced(params: ppow_params, draft_logits, target_logits, draft_tokens, uniforms, valid_len,
                              ref_logp, outputs: dict, workspace: torch.Tensor, stream=None,
                              event_reduce_begin=None, event_reduce_end=None) -> None:
    """ppow_score_windows plus two optional torch.cuda.Event objects recorded around the row-reduction kernel."""
    lib = load_library()
    lt = LOGIT_DTYPES[params.dtype]
    o = ppow_outputs()
    for name, _ in ppow_outputs._fields_:
        t = outputs.get(name)
        want = _ALL_OUTPUTS[name]
        p = _dev_ptr(t, want, name)
        setattr(o, name, p.value if p is not None else None)
    traced = event_reduce_begin is not None or event_reduce_end is not None
    fn = lib.ppow_score_windows_traced if traced else lib.ppow_score_windows
    extra = (_event_ptr(event_reduce_begin), _event_ptr(event_reduce_end)) if traced else ()
    st = fn(
        ctypes.byref(params),
        _dev_ptr(draft_logits, lt, "draft_logits"), _dev_ptr(target_logits, lt, "target_logits"),
        _dev_ptr(draft_tokens, torch.int32, "draft_tokens"), _dev_ptr(uniforms, torch.float32, "uniforms"),
        _dev_ptr(valid_len, torch.int32, "valid_len"), _dev_ptr(ref_logp, torch.float32, "ref_logp"),
        ctypes.byref(o), _dev_ptr(workspace, torch.uint8, "workspace"),
        workspace.numel() if workspace is not None else 0, _stream_ptr(stream), *extra)
    if st != PPOW_OK:
        raise PpowError(st, "ppow_score_windows")


class ScoreCall:
    """The arguments of ``ppow_score_windows`` marshalled once.  ``launch()`` repeats the foreign call without
    rebuilding them, which matters when the same buffers are scored step after step and the problem is small
    enough for argument marshalling to show.  Holds references to the tensors; nothing is computed here."""

    def __init__(self, params: ppow_params, draft_logits, target_logits, draft_tokens, uniforms, valid_len, ref_logp,
                 outputs: dict, workspace: torch.Tensor):
        self._lib = load_library()
        lt = LOGIT_DTYPES[params.dtype]
        self._keep = (params, draft_logits, target_logits, draft_tokens, uniforms, valid_len, ref_logp, outputs, workspace)
        self._out = ppow_outputs()
        for name, _ in ppow_outputs._fields_:
            ptr = _dev_ptr(outputs.get(name), _ALL_OUTPUTS[name], name)
            setattr(self._out, name, ptr.value if ptr is not None else None)
        self._args = (ctypes.byref(params),
                      _dev_ptr(draft_logits, lt, "draft_logits"), _dev_ptr(target_logits, lt, "target_logits"),
                      _dev_ptr(draft_tokens, torch.int32, "draft_tokens"), _dev_ptr(uniforms, torch.float32, "uniforms"),
                      _dev_ptr(valid_len, torch.int32, "valid_len"), _dev_ptr(ref_logp, torch.float32, "ref_logp"),
                      ctypes.byref(self._out), _dev_ptr(workspace, torch.uint8, "workspace"),
                      workspace.numel() if workspace is not None else 0)

    def launch(self, stream=None, event_reduce_begin=None, event_reduce_end=None) -> None:
        if event_reduce_begin is None and event_reduce_end is None:
            st = self._lib.ppow_score_windows(*self._args, _stream_ptr(stream))
        else:
            st = self._lib.ppow_score_windows_traced(*self._args, _stream_ptr(stream), _event_ptr(event_reduce_begin),
                                                     _event_ptr(event_reduce_end))
        if st != PPOW_OK:
            raise PpowError(st, "ppow_score_windows")


class SelectCall:
    """The arguments of ``ppow_select_windows`` marshalled once (see ScoreCall)."""

    def __init__(self, score, n_keep: int, selected, mask, workspace):
        self._lib = load_library()
        self._keep = (score, selected, mask, workspace)
        self._args = (_dev_ptr(score, torch.float32, "score"), int(score.numel()) if score is not None else 0, int(n_keep),
                      _dev_ptr(selected, torch.int32, "selected"), _dev_ptr(mask, torch.uint8, "mask"),
                      _dev_ptr(workspace, torch.uint8, "workspace"), workspace.numel() if workspace is not None else 0)

    def launch(self, stream=None) -> None:
        st = self._lib.ppow_select_windows(*self._args, _stream_ptr(stream))
        if st != PPOW_OK:
            raise PpowError(st, "ppow_select_windows")


def ppow_read_error_flags(workspace: torch.Tensor, stream=None) -> int:
    lib = load_library()
    flags = ctypes.c_uint32(0)
    st = lib.ppow_read_error_flags(_dev_ptr(workspace, torch.uint8, "workspace"), ctypes.byref(flags),
                                   _stream_ptr(stream))
    if st not in (PPOW_OK, PPOW_ERR_DEVICE_TIMEOUT):
        raise PpowError(st, "ppow_read_error_flags")
    return int(flags.value)


def ppow_selftest_wait_timeout(workspace: torch.Tensor, probes: int = 64, stream=None) -> None:
    """Makes the bounded device-side wait run out on purpose (harmlessly); see include/ppow.h."""
    lib = load_library()
    st = lib.ppow_selftest_wait_timeout(_dev_ptr(workspace, torch.uint8, "workspace"), workspace.numel(), int(probes),
                                        _stream_ptr(stream))
    if st != PPOW_OK:
        raise PpowError(st, "ppow_selftest_wait_timeout")


def ppow_read_error_status(workspace: torch.Tensor, stream=None):
    """(status, flags) of ppow_read_error_flags without raising on PPOW_ERR_DEVICE_TIMEOUT."""
    lib = load_library()
    flags = ctypes.c_uint32(0)
    st = lib.ppow_read_error_flags(_dev_ptr(workspace, torch.uint8, "workspace"), ctypes.byref(flags), _stream_ptr(stream))
    return int(st), int(flags.value)


def ppow_select_windows(score, n_keep: int, selected, mask, workspace, stream=None) -> None:
    lib = load_library()
    N = int(score.numel()) if score is not None else 0
    st = lib.ppow_select_windows(
        _dev_ptr(score, torch.float32, "score"), N, int(n_keep), _dev_ptr(selected, torch.int32, "selected"),
        _dev_ptr(mask, torch.uint8, "mask"), _dev_ptr(workspace, torch.uint8, "workspace"),
        workspace.numel() if workspace is not None else 0, _stream_ptr(stream))
    if st != PPOW_OK:
        raise PpowError(st, "ppow_select_windows")


def ppow_noalloc_scratch_bytes() -> int:
    return int(load_library().ppow_noalloc_scratch_bytes())


def ppow_score_windows_noalloc(params: ppow_params, draft_logits, target_logits, draft_tokens, uniforms, valid_len,
                               ref_logp, outputs: dict, stream=None) -> None:
    """ppow_score_windows for callers that cannot hand over a workspace: the library's built-in 4 MiB
    scratch array is used instead.  The binding itself allocates nothing here; ``outputs`` must hold
    preallocated CUDA tensors.  Calls on one device must not overlap (they share the array)."""
    lib = load_library()
    lt = LOGIT_DTYPES[params.dtype]
    o = ppow_outputs()
    for name, _ in ppow_outputs._fields_:
        want = _ALL_OUTPUTS[name]
        p = _dev_ptr(outputs.get(name), want, name)
        setattr(o, name, p.value if p is not None else None)
    st = lib.ppow_score_windows_noalloc(
        ctypes.byref(params),
        _dev_ptr(draft_logits, lt, "draft_logits"), _dev_ptr(target_logits, lt, "target_logits"),
        _dev_ptr(draft_tokens, torch.int32, "draft_tokens"), _dev_ptr(uniforms, torch.float32, "uniforms"),
        _dev_ptr(valid_len, torch.int32, "valid_len"), _dev_ptr(ref_logp, torch.float32, "ref_logp"),
        ctypes.byref(o), _stream_ptr(stream))
    if st != PPOW_OK:
        raise PpowError(st, "ppow_score_windows_noalloc")


def ppow_noalloc_read_error_flags(stream=None):
    """(status, flags) left by the last ppow_score_windows_noalloc call on the current device."""
    flags = ctypes.c_uint32(0)
    st = load_library().ppow_noalloc_read_error_flags(ctypes.byref(flags), _stream_ptr(stream))
    return int(st), int(flags.value)


def ppow_group_advantage(reward, group_size: int, delta: float, advantage, stream=None) -> None:
    lib = load_library()
    N = int(reward.numel()) if reward is not None else 0
    st = lib.ppow_group_advantage(_dev_ptr(reward, torch.float32, "reward"), N, int(group_size), float(delta),
                                  _dev_ptr(advantage, torch.float32, "advantage"), _stream_ptr(stream))
    if st != PPOW_OK:
        raise PpowError(st, "ppow_group_advantage")


def ppow_sequence_windows(crit, seq_offsets, K: int, scores, uniforms, starts, stream=None) -> None:
    lib = load_library()
    B = int(seq_offsets.numel()) - 1 if seq_offsets is not None else 0
    st = lib.ppow_sequence_windows(_dev_ptr(crit, torch.float32, "crit"), _dev_ptr(seq_offsets, torch.int32, "seq_offsets"),
                                   B, int(K), _dev_ptr(scores, torch.float32, "scores"),
                                   _dev_ptr(uniforms, torch.float32, "uniforms"), _dev_ptr(starts, torch.int32, "starts"),
                                   _stream_ptr(stream))
    if st != PPOW_OK:
        raise PpowError(st, "ppow_sequence_windows")


def ppow_sequence_windows_mixed(crit, seq_offsets, K: int, hard_frac: float, scores, uniforms_mix, uniforms_draw,
                                starts, stream=None) -> None:
    lib = load_library()
    B = int(seq_offsets.numel()) - 1 if seq_offsets is not None else 0
    st = lib.ppow_sequence_windows_mixed(
        _dev_ptr(crit, torch.float32, "crit"), _dev_ptr(seq_offsets, torch.int32, "seq_offsets"), B, int(K),
        float(hard_frac), _dev_ptr(scores, torch.float32, "scores"), _dev_ptr(uniforms_mix, torch.float32, "uniforms_mix"),
        _dev_ptr(uniforms_draw, torch.float32, "uniforms_draw"), _dev_ptr(starts, torch.int32, "starts"),
        _stream_ptr(stream))
    if st != PPOW_OK:
        raise PpowError(st, "ppow_sequence_windows_mixed")


def ppow_expected_acceptance(params: ppow_params, draft_logits, target_logits, valid_len, lse_p, lse_q,
                             expected_accept, stream=None) -> None:
    lib = load_library()
    lt = LOGIT_DTYPES[params.dtype]
    st = lib.ppow_expected_acceptance(
        ctypes.byref(params), _dev_ptr(draft_logits, lt, "draft_logits"), _dev_ptr(target_logits, lt, "target_logits"),
        _dev_ptr(valid_len, torch.int32, "valid_len"), _dev_ptr(lse_p, torch.float32, "lse_p"),
        _dev_ptr(lse_q, torch.float32, "lse_q"), _dev_ptr(expected_accept, torch.float32, "expected_accept"),
        _stream_ptr(stream))
    if st != PPOW_OK:
        raise PpowError(st, "ppow_expected_acceptance")


def ppow_reference_logprob(params: ppow_params, ref_target_logits, valid_len, row_logp, ref_logp, stream=None) -> None:
    lib = load_library()
    lt = LOGIT_DTYPES[params.dtype]
    st = lib.ppow_reference_logprob(ctypes.byref(params), _dev_ptr(ref_target_logits, lt, "ref_target_logits"),
                                    _dev_ptr(valid_len, torch.int32, "valid_len"),
                                    _dev_ptr(row_logp, torch.float32, "row_logp"),
                                    _dev_ptr(ref_logp, torch.float32, "ref_logp"), _stream_ptr(stream))
    if st != PPOW_OK:
        raise PpowError(st, "ppow_reference_logprob")


# The calls below take a few microseconds on the device for one window of tokens, so their checks are one chain of cheap
# comparisons per tensor, and pointers go to the library as plain integers.


def _index_of(t: torch.Tensor, name) -> int:
    """Index of the CUDA device that holds ``t``."""
    i = t.get_device()
    if i < 0:
        raise ValueError("%s must live on a CUDA device (no CPU path exists)" % name)
    return i


def _arg(t: Optional[torch.Tensor], dtype, shape, dev: int, name):
    """Address of a contiguous tensor of this type and shape on device ``dev`` (None for None)."""
    if t is None:
        return None
    if t.get_device() != dev or t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
        if not t.is_cuda:
            raise ValueError("%s must live on a CUDA device (no CPU path exists)" % name)
        raise ValueError("%s must be a contiguous %s tensor of shape %s on cuda:%d, got %s, %s, strides %s on %s" % (
            name, dtype, tuple(shape), dev, t.dtype, tuple(t.shape), t.stride(), t.device))
    return t.data_ptr()


def _rows_arg(t: torch.Tensor, dtype, shape, dev: int, name):
    """Address and row stride (elements) of a 2-D tensor whose rows are contiguous."""
    if t.get_device() != dev or t.dtype is not dtype or t.shape != shape or (shape[1] > 1 and t.stride(1) != 1):
        if not t.is_cuda:
            raise ValueError("%s must live on a CUDA device (no CPU path exists)" % name)
        raise ValueError("%s must be a %s tensor of shape %s with contiguous rows on cuda:%d, got %s, %s, strides %s on %s" % (
            name, dtype, tuple(shape), dev, t.dtype, tuple(t.shape), t.stride(), t.device))
    return t.data_ptr(), (t.stride(0) if shape[0] > 1 else shape[1])


def _workspace_arg(t: torch.Tensor, dev: int):
    if t.dim() != 1:
        raise ValueError("workspace must be one-dimensional")
    return _arg(t, torch.uint8, t.shape, dev, "workspace"), t.shape[0]


def _raw_stream(stream, dev: int) -> int:
    """cudaStream_t of ``stream``, or of the stream that is current on device ``dev``."""
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(dev)
    if stream.device_index != dev:
        raise ValueError("stream must belong to cuda:%d" % dev)
    return stream.cuda_stream


def _call(fn, where, dev: int, *args) -> None:
    """Calls the library with device ``dev`` current."""
    if torch._C._cuda_getDevice() == dev:
        st = fn(*args)
    else:
        with torch.cuda.device(dev):
            st = fn(*args)
    if st != PPOW_OK:
        raise PpowError(st, where)


_PLAIN = contextlib.nullcontext()


def _on(stream):
    """Context in which ``stream``, if one is given, is current: what is allocated inside belongs to it, so that the allocator
    hands it on only behind the work enqueued there."""
    return _PLAIN if stream is None else torch.cuda.stream(stream)


def make_head_params(hidden, weight, temperature=1.0) -> ppow_head_params:
    """Sizes, type and row strides of a head call, from its tensors ``hidden`` [T, D] and ``weight`` [V, D]."""
    if hidden.dtype not in (torch.bfloat16, torch.float16):
        raise ValueError("hidden must be bfloat16 or float16, got %s" % hidden.dtype)
    if hidden.dim() != 2 or weight.dim() != 2:
        raise ValueError("hidden and weight must be 2-D")
    (T, D), V = hidden.shape, weight.shape[0]
    return ppow_head_params(T, V, D, DTYPE_CODES[hidden.dtype], hidden.stride(0) if T > 1 else D, weight.stride(0) if V > 1 else D,
                            float(temperature))


def ppow_head_workspace_bytes(params: ppow_head_params, backward: bool) -> int:
    return load_library().ppow_head_workspace_bytes(ctypes.byref(params), 1 if backward else 0)


def ppow_head_plan(params: ppow_head_params, live: int):
    """How the gradient is cut with ``live`` rows that are not masked: [(first, columns)] of the vocabulary's pieces, and the shares
    of each that grad_hidden is added up from.  Host only."""
    lib, first, columns, shares = load_library(), ctypes.c_int32(), ctypes.c_int32(), ctypes.c_int32()
    pieces = []
    for i in range(lib.ppow_head_plan(ctypes.byref(params), live, 0, None, None, None)):
        lib.ppow_head_plan(ctypes.byref(params), live, i, ctypes.byref(first), ctypes.byref(columns), ctypes.byref(shares))
        pieces.append((first.value, columns.value))
    return pieces, shares.value


def ppow_head_logprob(params: ppow_head_params, hidden, weight, tokens, logp, lse, workspace, stream=None) -> None:
    """Enqueue log-probabilities of ``tokens`` [T] from ``hidden`` [T, D] and ``weight`` [V, D] into ``logp`` and ``lse``."""
    T, V, D, dt, dev = params.T, params.V, params.D, LOGIT_DTYPES[params.dtype], _index_of(hidden, "hidden")
    h, params.hidden_stride = _rows_arg(hidden, dt, (T, D), dev, "hidden")
    w, params.weight_stride = _rows_arg(weight, dt, (V, D), dev, "weight")
    _call(load_library().ppow_head_logprob, "ppow_head_logprob", dev, ctypes.byref(params), h, w,
          _arg(tokens, torch.int32, (T,), dev, "tokens"), _arg(logp, torch.float32, (T,), dev, "logp"),
          _arg(lse, torch.float32, (T,), dev, "lse"), *_workspace_arg(workspace, dev), _raw_stream(stream, dev))


def ppow_head_logprob_backward(params: ppow_head_params, hidden, weight, tokens, lse, grad_logp, grad_hidden, grad_weight, workspace,
                               stream=None) -> None:
    """Enqueue the gradient of sum(grad_logp * logp); ``grad_hidden`` or ``grad_weight`` may be None."""
    T, V, D, dt, dev = params.T, params.V, params.D, LOGIT_DTYPES[params.dtype], _index_of(hidden, "hidden")
    h, params.hidden_stride = _rows_arg(hidden, dt, (T, D), dev, "hidden")
    w, params.weight_stride = _rows_arg(weight, dt, (V, D), dev, "weight")
    _call(load_library().ppow_head_logprob_backward, "ppow_head_logprob_backward", dev, ctypes.byref(params), h, w,
          _arg(tokens, torch.int32, (T,), dev, "tokens"), _arg(lse, torch.float32, (T,), dev, "lse"),
          _arg(grad_logp, torch.float32, (T,), dev, "grad_logp"), _arg(grad_hidden, dt, (T, D), dev, "grad_hidden"),
          _arg(grad_weight, dt, (V, D), dev, "grad_weight"), *_workspace_arg(workspace, dev), _raw_stream(stream, dev))


CHECKPOINT_DTYPE = torch.float8_e4m3fn   # codes; scales are uint8, exponent + 127
CHECKPOINT_BLOCK = 128                  # values along a row that share a scale


def make_norm_params(R, D, dtype, param_dtype, eps=1e-5) -> ppow_norm_params:
    if dtype not in DTYPE_CODES or param_dtype not in DTYPE_CODES:
        raise ValueError("types must be float32, bfloat16 or float16, got %s and %s" % (dtype, param_dtype))
    return ppow_norm_params(R, D, DTYPE_CODES[dtype], DTYPE_CODES[param_dtype], eps)


def _packed_args(packed, scale, R, D, dev):
    return (_arg(packed, CHECKPOINT_DTYPE, (R, D), dev, "packed"),
            _arg(scale, torch.uint8, (R, (D + CHECKPOINT_BLOCK - 1) // CHECKPOINT_BLOCK), dev, "scale"))


def ppow_layer_norm(params: ppow_norm_params, x, weight, bias, y, mean, rstd, packed=None, scale=None, stream=None) -> None:
    """Enqueue the forward pass on ``x`` [R, D]; with ``packed`` and ``scale`` it also writes the 8-bit form of ``x``."""
    R, D, dt, pt, dev = params.R, params.D, LOGIT_DTYPES[params.dtype], LOGIT_DTYPES[params.param_dtype], _index_of(x, "x")
    f32 = torch.float32
    _call(load_library().ppow_layer_norm, "ppow_layer_norm", dev, ctypes.byref(params), *_rows_arg(x, dt, (R, D), dev, "x"),
          _arg(weight, pt, (D,), dev, "weight"), _arg(bias, pt, (D,), dev, "bias"), _arg(y, dt, (R, D), dev, "y"),
          _arg(mean, f32, (R,), dev, "mean"), _arg(rstd, f32, (R,), dev, "rstd"), *_packed_args(packed, scale, R, D, dev),
          _raw_stream(stream, dev))


def ppow_layer_norm_workspace_bytes(params: ppow_norm_params) -> int:
    return load_library().ppow_layer_norm_workspace_bytes(ctypes.byref(params))


def ppow_layer_norm_backward(params: ppow_norm_params, grad_y, x, packed, scale, weight, mean, rstd, grad_x, grad_weight, grad_bias,
                             workspace, stream=None) -> None:
    """Enqueue the gradient; the forward pass's input is either ``x`` or, where that is None, ``packed`` and ``scale``."""
    R, D, dt, pt, dev = params.R, params.D, LOGIT_DTYPES[params.dtype], LOGIT_DTYPES[params.param_dtype], _index_of(grad_y, "grad_y")
    f32 = torch.float32
    xp, xs = (None, D) if x is None else _rows_arg(x, dt, (R, D), dev, "x")
    _call(load_library().ppow_layer_norm_backward, "ppow_layer_norm_backward", dev, ctypes.byref(params),
          *_rows_arg(grad_y, dt, (R, D), dev, "grad_y"), xp, xs, *_packed_args(packed, scale, R, D, dev),
          _arg(weight, pt, (D,), dev, "weight"), _arg(mean, f32, (R,), dev, "mean"), _arg(rstd, f32, (R,), dev, "rstd"),
          _arg(grad_x, dt, (R, D), dev, "grad_x"), _arg(grad_weight, pt, (D,), dev, "grad_weight"),
          _arg(grad_bias, pt, (D,), dev, "grad_bias"), *_workspace_arg(workspace, dev), _raw_stream(stream, dev))


def _storage_code(dtype, name) -> int:
    code = DTYPE_CODES.get(dtype)
    if code is None:
        raise ValueError("%s must be float32, bfloat16 or float16, got %s" % (name, dtype))
    return code


def ppow_pack_activation(x, packed, scale, stream=None) -> None:
    """Enqueue the 8-bit form of ``x`` [R, D]: codes into ``packed`` [R, D], exponents into ``scale`` [R, ceil(D/128)]."""
    R, D = x.shape
    code, dev = _storage_code(x.dtype, "x"), _index_of(x, "x")
    _call(load_library().ppow_pack_activation, "ppow_pack_activation", dev, *_rows_arg(x, x.dtype, (R, D), dev, "x"), R, D, code,
          *_packed_args(packed, scale, R, D, dev), _raw_stream(stream, dev))


def ppow_unpack_activation(packed, scale, x, stream=None) -> None:
    """Enqueue the way back: values of the 8-bit form into ``x`` [R, D], rounded to its type."""
    R, D = packed.shape
    code, dev = _storage_code(x.dtype, "x"), _index_of(packed, "packed")
    _call(load_library().ppow_unpack_activation, "ppow_unpack_activation", dev, *_packed_args(packed, scale, R, D, dev), R, D, code,
          _arg(x, x.dtype, (R, D), dev, "x"), _raw_stream(stream, dev))


def _maybe_rows_arg(t: Optional[torch.Tensor], dtype, shape, dev: int, name):
    """_rows_arg, or no address and the plain stride where there is no tensor."""
    return (None, shape[1]) if t is None else _rows_arg(t, dtype, shape, dev, name)


def ppow_rms_norm(params: ppow_norm_params, x, residual, weight, sum, y, rstd, y_packed=None, y_scale=None, packed=None, scale=None,
                  stream=None) -> None:
    """Enqueue the forward pass on ``x`` [R, D], to which ``residual`` is added if it is not None; then ``sum`` receives the sum."""
    R, D, dt, pt, dev = params.R, params.D, LOGIT_DTYPES[params.dtype], LOGIT_DTYPES[params.param_dtype], _index_of(x, "x")
    _call(load_library().ppow_rms_norm, "ppow_rms_norm", dev, ctypes.byref(params), *_rows_arg(x, dt, (R, D), dev, "x"),
          *_maybe_rows_arg(residual, dt, (R, D), dev, "residual"), _arg(weight, pt, (D,), dev, "weight"), _arg(sum, dt, (R, D), dev, "sum"),
          _arg(y, dt, (R, D), dev, "y"), _arg(rstd, torch.float32, (R,), dev, "rstd"), *_packed_args(y_packed, y_scale, R, D, dev),
          *_packed_args(packed, scale, R, D, dev), _raw_stream(stream, dev))


def ppow_rms_norm_workspace_bytes(params: ppow_norm_params) -> int:
    return load_library().ppow_rms_norm_workspace_bytes(ctypes.byref(params))


def ppow_rms_norm_backward(params: ppow_norm_params, grad_y, grad_sum, x, packed, scale, weight, rstd, grad_x, grad_weight, workspace,
                           stream=None) -> None:
    """Enqueue the gradient; what the forward pass normalised is either ``x`` or, where that is None, ``packed`` and ``scale``."""
    R, D, dt, pt, dev = params.R, params.D, LOGIT_DTYPES[params.dtype], LOGIT_DTYPES[params.param_dtype], _index_of(grad_y, "grad_y")
    _call(load_library().ppow_rms_norm_backward, "ppow_rms_norm_backward", dev, ctypes.byref(params),
          *_rows_arg(grad_y, dt, (R, D), dev, "grad_y"), *_maybe_rows_arg(grad_sum, dt, (R, D), dev, "grad_sum"),
          *_maybe_rows_arg(x, dt, (R, D), dev, "x"), *_packed_args(packed, scale, R, D, dev), _arg(weight, pt, (D,), dev, "weight"),
          _arg(rstd, torch.float32, (R,), dev, "rstd"), _arg(grad_x, dt, (R, D), dev, "grad_x"), _arg(grad_weight, pt, (D,), dev, "grad_weight"),
          *_workspace_arg(workspace, dev), _raw_stream(stream, dev))


def ppow_clip_workspace_bytes(n: int) -> int:
    return load_library().ppow_clip_workspace_bytes(n)


def _dense(t: torch.Tensor) -> bool:
    """Whether the elements fill their stretch of memory, in any order of the dimensions."""
    want = 1
    for stride, size in sorted((st, n) for st, n in zip(t.stride(), t.shape) if n != 1):
        if stride != want:
            return t.numel() == 0
        want *= size
    return True


def ppow_clip_gradients(grads, out, max_norm: float, norm, workspace, stream=None) -> None:
    """Enqueue the global norm of ``grads`` (a sequence of tensors) into ``norm`` (one float32) and, unless ``out`` is None, the clipped
    gradients into the tensors of ``out``, which may be ``grads``."""
    dev, n = _index_of(norm, "norm"), len(grads)
    if out is not None and len(out) != n:
        raise ValueError("out must have as many tensors as grads")
    for i, t in enumerate(grads):
        if t.dtype not in DTYPE_CODES or t.get_device() != dev or not _dense(t):
            raise ValueError("grads[%d] must be a dense float32, bfloat16 or float16 tensor on cuda:%d, got %s, %s, strides %s on %s" % (
                i, dev, t.dtype, tuple(t.shape), t.stride(), t.device))
        if out is not None:
            o = out[i]
            if o.dtype is not t.dtype or o.shape != t.shape or o.get_device() != dev or (t.numel() > 1 and any(
                    a != b for a, b, s in zip(o.stride(), t.stride(), t.shape) if s > 1)):
                raise ValueError("out[%d] must be like its gradient: %s, %s, strides %s on cuda:%d" % (i, t.dtype, tuple(t.shape), t.stride(), dev))
    ptrs, i64s, i32s = ctypes.c_void_p * n, ctypes.c_int64 * n, ctypes.c_int32 * n
    _call(load_library().ppow_clip_gradients, "ppow_clip_gradients", dev, n, ptrs(*[t.data_ptr() for t in grads]),
          None if out is None else ptrs(*[t.data_ptr() for t in out]), i64s(*[t.numel() for t in grads]),
          i32s(*[DTYPE_CODES[t.dtype] for t in grads]), float(max_norm), _arg(norm, torch.float32, norm.shape, dev, "norm"),
          *_workspace_arg(workspace, dev), _raw_stream(stream, dev))
    if out is not None:
        torch.autograd.graph.increment_version([t for t in out if not t.is_inference()])


def make_sample_params(logits, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0) -> ppow_sample_params:
    """Sizes, type and row stride of a draw, from its logits [R, V], and the filters."""
    if logits.dim() != 2:
        raise ValueError("logits must be 2-D")
    R, V = logits.shape
    top_k = max(-1, min(int(top_k), 2 ** 31 - 1))            # what is out of range stays so
    return ppow_sample_params(min(R, 2 ** 31 - 1), min(V, 2 ** 31 - 1), _storage_code(logits.dtype, "logits"), top_k, logits.stride(0) if R > 1 else V, float(temperature),
                              float(top_p), float(min_p))


def ppow_sample_tokens(params: ppow_sample_params, logits, uniforms, tokens, logp, kept=None, stream=None) -> None:
    """Enqueue the draw of one token for each row of ``logits`` [R, V]; ``kept`` may be None."""
    R, V, dt, dev = params.R, params.V, LOGIT_DTYPES[params.dtype], _index_of(logits, "logits")
    x, params.logits_stride = _rows_arg(logits, dt, (R, V), dev, "logits")
    _call(load_library().ppow_sample_tokens, "ppow_sample_tokens", dev, ctypes.byref(params), x,
          _arg(uniforms, torch.float32, (R,), dev, "uniforms"), _arg(tokens, torch.int32, (R,), dev, "tokens"),
          _arg(logp, torch.float32, (R,), dev, "logp"), _arg(kept, torch.int32, (R,), dev, "kept"), _raw_stream(stream, dev))


def _host_ptr(t: Optional[torch.Tensor], dtype=None, name="tensor"):
    if t is None:
        return None
    if t.is_cuda or not t.is_contiguous():
        raise ValueError("%s must be a contiguous host tensor" % name)
    if dtype is not None and t.dtype != dtype:
        raise ValueError("%s must have dtype %s, got %s" % (name, dtype, t.dtype))
    return ctypes.c_void_p(t.data_ptr())


def ppow_host_scratch_bytes(params: ppow_params, chunk_windows: int) -> int:
    return int(load_library().ppow_host_scratch_bytes(ctypes.byref(params), int(chunk_windows)))


def ppow_score_and_select_host(params: ppow_params, draft_logits, target_logits, draft_tokens, uniforms, valid_len,
                               ref_logp, outputs_host: dict, n_keep: int, selected_host, mask_host,
                               device_scratch: torch.Tensor, stream=None) -> None:
    """Host-buffer entry point: all tensors except ``device_scratch`` are host tensors (pinned for async copies)."""
    lib = load_library()
    lt = LOGIT_DTYPES[params.dtype]
    o = ppow_outputs()
    for name, _ in ppow_outputs._fields_:
        want = _ALL_OUTPUTS[name]
        p = _host_ptr(outputs_host.get(name), want, name)
        setattr(o, name, p.value if p is not None else None)
    st = lib.ppow_score_and_select_host(
        ctypes.byref(params), _host_ptr(draft_logits, lt, "draft_logits"), _host_ptr(target_logits, lt, "target_logits"),
        _host_ptr(draft_tokens, torch.int32, "draft_tokens"), _host_ptr(uniforms, torch.float32, "uniforms"),
        _host_ptr(valid_len, torch.int32, "valid_len"), _host_ptr(ref_logp, torch.float32, "ref_logp"),
        ctypes.byref(o), int(n_keep), _host_ptr(selected_host, torch.int32, "selected_host"),
        _host_ptr(mask_host, torch.uint8, "mask_host"), _dev_ptr(device_scratch, torch.uint8, "device_scratch"),
        device_scratch.numel(), _stream_ptr(stream))
    if st != PPOW_OK:
        raise PpowError(st, "ppow_score_and_select_host")


# ---- convenience wrappers (allocation + the calls above; no arithmetic) -----------------------


def score_windows(draft_logits, target_logits, draft_tokens, *, mode, c, temperature=1.0, eta=1.0, eps=0.5,
                  uniforms=None, valid_len=None, ref_logp=None, stream=None, train_outputs=False) -> dict:
    """Allocate outputs and workspace, run ppow_score_windows, return the dict of output tensors
    (with ``train_outputs`` also kl_rev, kl_rev_mean, nabla, lse_p, lse_q)."""
    N, K, V = draft_logits.shape
    dt = DTYPE_CODES[draft_logits.dtype]
    params = make_params(N, K, V, dt, mode, c, temperature, eta, eps)
    dev = draft_logits.device
    with torch.cuda.device(dev):
        out = alloc_outputs(N, K, dev)
        if train_outputs:
            out.update(alloc_train_outputs(N, K, dev))
        ws = alloc_workspace(ppow_score_workspace_bytes(params), dev)
        ppow_score_windows(params, draft_logits, target_logits, draft_tokens, uniforms, valid_len, ref_logp, out,
                           ws, stream)
    out["_workspace"] = ws
    return out


def select_windows(score, n_keep: int, want_mask: bool = False, stream=None):
    """Allocate and run ppow_select_windows; returns selected indices (and the mask if asked)."""
    N = int(score.numel())
    dev = score.device
    with torch.cuda.device(dev):
        sel = torch.empty((max(int(n_keep), 0),), dtype=torch.int32, device=dev)
        mask = torch.empty((N,), dtype=torch.uint8, device=dev) if want_mask else None
        ws = alloc_workspace(ppow_select_workspace_bytes(N), dev)
        ppow_select_windows(score, n_keep, sel, mask, ws, stream)
    return (sel, mask) if want_mask else sel


# The wrappers below are plain calls outside autograd: what they return is detached, whatever their inputs require, and each gradient
# has a call of its own.
# They go through the extension module first, which marshals a call in a fifth of the time and answers None where
# something is not as it should be, or where the call is for another stream or device: the rest of the wrapper is for those.
# It hands the addresses of what it has just allocated straight to the library.


def _quick():
    if _calls is None:
        load_library()
    return _calls


def _done(got, where):
    if got[0] != PPOW_OK:
        raise PpowError(got[0], where)
    return got[1:]


def _workspace(nbytes: int, dev) -> torch.Tensor:
    return torch.empty(nbytes or 256, dtype=torch.uint8, device=dev)


def head_logprob(hidden, weight, tokens, *, temperature=1.0, want_workspace=False, stream=None) -> dict:
    """Allocate outputs and workspace, run ppow_head_logprob; returns logp and lse, both [T] float32, outside autograd (the gradient is
    head_logprob_backward's).  With ``want_workspace`` also
    ``_workspace``, whose error word ppow_read_error_flags reads (tokens behind the vocabulary, a device wait that ran out); it is not
    kept otherwise, because it holds 8 bytes for every 128 logits and a copy of the rows."""
    if stream is None:
        got = _quick().head_logprob(hidden, weight, tokens, temperature, want_workspace)
        if got is not None:
            logp, lse, ws = _done(got, "ppow_head_logprob")
            return {"logp": logp, "lse": lse, "_workspace": ws} if want_workspace else {"logp": logp, "lse": lse}
    params, lib, f32 = make_head_params(hidden, weight, temperature), load_library(), torch.float32
    T, V, D, dt, device, dev = params.T, params.V, params.D, hidden.dtype, hidden.device, _index_of(hidden, "hidden")
    h, w = _rows_arg(hidden, dt, (T, D), dev, "hidden")[0], _rows_arg(weight, dt, (V, D), dev, "weight")[0]
    y = _arg(tokens, torch.int32, (T,), dev, "tokens")
    with _on(stream):
        logp, lse = torch.empty(T, dtype=f32, device=device), torch.empty(T, dtype=f32, device=device)
        nbytes = lib.ppow_head_workspace_bytes(ctypes.byref(params), 0)
        ws = _workspace(nbytes, device)
    _call(lib.ppow_head_logprob, "ppow_head_logprob", dev, ctypes.byref(params), h, w, y, logp.data_ptr(), lse.data_ptr(),
          ws.data_ptr(), nbytes, _raw_stream(stream, dev))
    return {"logp": logp, "lse": lse, "_workspace": ws} if want_workspace else {"logp": logp, "lse": lse}


def head_logprob_backward(hidden, weight, tokens, lse, grad_logp, *, temperature=1.0, want_hidden=True, want_weight=True,
                          want_workspace=False, stream=None):
    """Allocate gradients and workspace, run ppow_head_logprob_backward; returns (grad_hidden, grad_weight), None where not wanted.
    With ``want_workspace`` the workspace is returned as a third, for ppow_read_error_flags (it holds up to 512 MiB and more)."""
    if stream is None:
        got = _quick().head_logprob_backward(hidden, weight, tokens, lse, grad_logp, temperature, want_hidden, want_weight, want_workspace)
        if got is not None:
            return _done(got, "ppow_head_logprob_backward")[:3 if want_workspace else 2]
    params, lib, f32 = make_head_params(hidden, weight, temperature), load_library(), torch.float32
    T, V, D, dt, device, dev = params.T, params.V, params.D, hidden.dtype, hidden.device, _index_of(hidden, "hidden")
    h, w = _rows_arg(hidden, dt, (T, D), dev, "hidden")[0], _rows_arg(weight, dt, (V, D), dev, "weight")[0]
    y = _arg(tokens, torch.int32, (T,), dev, "tokens")
    l, g = _arg(lse, f32, (T,), dev, "lse"), _arg(grad_logp, f32, (T,), dev, "grad_logp")
    with _on(stream):
        gh = torch.empty(T, D, dtype=dt, device=device) if want_hidden else None
        gw = torch.empty(V, D, dtype=dt, device=device) if want_weight else None
        nbytes = lib.ppow_head_workspace_bytes(ctypes.byref(params), 1)
        ws = _workspace(nbytes, device)
    _call(lib.ppow_head_logprob_backward, "ppow_head_logprob_backward", dev, ctypes.byref(params), h, w, y, l, g,
          None if gh is None else gh.data_ptr(), None if gw is None else gw.data_ptr(), ws.data_ptr(), nbytes, _raw_stream(stream, dev))
    return (gh, gw, ws) if want_workspace else (gh, gw)


def layer_norm(x, weight, bias=None, *, eps=1e-5, checkpoint=False, stream=None) -> dict:
    """Allocate outputs and run ppow_layer_norm on ``x`` [R, D]; returns y, mean, rstd and, with ``checkpoint``, the 8-bit form of
    ``x`` as packed and scale, all outside autograd (the gradient is layer_norm_backward's)."""
    if stream is None:
        got = _quick().layer_norm(x, weight, bias, eps, checkpoint)
        if got is not None:
            y, mean, rstd, packed, scale = _done(got, "ppow_layer_norm")
            out = {"y": y, "mean": mean, "rstd": rstd}
            if checkpoint:
                out["packed"], out["scale"] = packed, scale
            return out
    R, D = x.shape
    dt, pt, device, dev, f32 = x.dtype, weight.dtype, x.device, _index_of(x, "x"), torch.float32
    params = make_norm_params(R, D, dt, pt, eps)
    xp, xs = _rows_arg(x, dt, (R, D), dev, "x")
    w, b = _arg(weight, pt, (D,), dev, "weight"), _arg(bias, pt, (D,), dev, "bias")
    with _on(stream):
        out = {"y": torch.empty(R, D, dtype=dt, device=device), "mean": torch.empty(R, dtype=f32, device=device),
               "rstd": torch.empty(R, dtype=f32, device=device)}
        if checkpoint:
            out["packed"], out["scale"] = _alloc_packed(R, D, device)
    _call(load_library().ppow_layer_norm, "ppow_layer_norm", dev, ctypes.byref(params), xp, xs, w, b, out["y"].data_ptr(),
          out["mean"].data_ptr(), out["rstd"].data_ptr(), out["packed"].data_ptr() if checkpoint else None,
          out["scale"].data_ptr() if checkpoint else None, _raw_stream(stream, dev))
    return out


def layer_norm_backward(grad_y, x, weight, mean, rstd, *, want_bias=True, stream=None):
    """Allocate gradients and workspace, run ppow_layer_norm_backward; returns (grad_x, grad_weight, grad_bias or None).
    ``x`` is the forward pass's input or the pair (packed, scale) that the forward pass left."""
    if stream is None:
        direct, (packed, scale) = (None, x) if isinstance(x, (tuple, list)) else (x, (None, None))
        got = _quick().layer_norm_backward(grad_y, direct, packed, scale, weight, mean, rstd, want_bias)
        if got is not None:
            return _done(got, "ppow_layer_norm_backward")
    R, D = grad_y.shape
    dt, pt, device, dev, f32 = grad_y.dtype, weight.dtype, grad_y.device, _index_of(grad_y, "grad_y"), torch.float32
    params, lib = make_norm_params(R, D, dt, pt), load_library()
    gp, gs = _rows_arg(grad_y, dt, (R, D), dev, "grad_y")
    if isinstance(x, (tuple, list)):
        (xp, xs), (q, s) = (None, D), _packed_args(*x, R, D, dev)
    else:
        (xp, xs), (q, s) = _rows_arg(x, dt, (R, D), dev, "x"), (None, None)
    w, m, r = _arg(weight, pt, (D,), dev, "weight"), _arg(mean, f32, (R,), dev, "mean"), _arg(rstd, f32, (R,), dev, "rstd")
    with _on(stream):
        gx = torch.empty(R, D, dtype=dt, device=device)
        gw = torch.empty(D, dtype=pt, device=device)
        gb = torch.empty(D, dtype=pt, device=device) if want_bias else None
        nbytes = lib.ppow_layer_norm_workspace_bytes(ctypes.byref(params))
        ws = _workspace(nbytes, device)
    _call(lib.ppow_layer_norm_backward, "ppow_layer_norm_backward", dev, ctypes.byref(params), gp, gs, xp, xs, q, s, w, m, r,
          gx.data_ptr(), gw.data_ptr(), None if gb is None else gb.data_ptr(), ws.data_ptr(), nbytes, _raw_stream(stream, dev))
    return gx, gw, gb


def _alloc_packed(R: int, D: int, device):
    return (torch.empty(R, D, dtype=CHECKPOINT_DTYPE, device=device),
            torch.empty(R, (D + CHECKPOINT_BLOCK - 1) // CHECKPOINT_BLOCK, dtype=torch.uint8, device=device))


def pack_activation(x, stream=None):
    """Allocate and run ppow_pack_activation; returns (packed, scale), outside autograd."""
    if stream is None:
        got = _quick().pack_activation(x)
        if got is not None:
            return _done(got, "ppow_pack_activation")
    R, D = x.shape
    code, dev = _storage_code(x.dtype, "x"), _index_of(x, "x")
    xp, xs = _rows_arg(x, x.dtype, (R, D), dev, "x")
    with _on(stream):
        packed, scale = _alloc_packed(R, D, x.device)
    _call(load_library().ppow_pack_activation, "ppow_pack_activation", dev, xp, xs, R, D, code, packed.data_ptr(), scale.data_ptr(),
          _raw_stream(stream, dev))
    return packed, scale


def unpack_activation(packed, scale, dtype=torch.bfloat16, stream=None):
    """Allocate and run ppow_unpack_activation; returns the restored activation in ``dtype``, outside autograd."""
    if stream is None and dtype in DTYPE_CODES:
        got = _quick().unpack_activation(packed, scale, DTYPE_CODES[dtype])
        if got is not None:
            return _done(got, "ppow_unpack_activation")[0]
    R, D = packed.shape
    code, dev = _storage_code(dtype, "dtype"), _index_of(packed, "packed")
    q, s = _packed_args(packed, scale, R, D, dev)
    with _on(stream):
        x = torch.empty(R, D, dtype=dtype, device=packed.device)
    _call(load_library().ppow_unpack_activation, "ppow_unpack_activation", dev, q, s, R, D, code, x.data_ptr(), _raw_stream(stream, dev))
    return x


def rms_norm(x, weight, residual=None, *, eps=1e-6, checkpoint=False, packed_output=False, stream=None) -> dict:
    """Allocate outputs and run ppow_rms_norm on ``x`` [R, D]; returns y and rstd, with ``residual`` also sum = x + residual (what was
    normalised), with ``checkpoint`` the 8-bit form of that as packed and scale; with ``packed_output`` y_packed and y_scale in the
    place of y.  All outside autograd (the gradient is rms_norm_backward's)."""
    if stream is None:
        got = _quick().rms_norm(x, weight, residual, eps, checkpoint, packed_output)
        if got is not None:
            got = _done(got, "ppow_rms_norm")
            return {k: t for k, t in zip(("sum", "y", "rstd", "y_packed", "y_scale", "packed", "scale"), got) if t is not None}
    R, D = x.shape
    dt, pt, device, dev = x.dtype, weight.dtype, x.device, _index_of(x, "x")
    params = make_norm_params(R, D, dt, pt, eps)
    xp, xs = _rows_arg(x, dt, (R, D), dev, "x")
    rp, rs = _maybe_rows_arg(residual, dt, (R, D), dev, "residual")
    w, out = _arg(weight, pt, (D,), dev, "weight"), {}
    with _on(stream):
        if residual is not None:
            out["sum"] = torch.empty(R, D, dtype=dt, device=device)
        if packed_output:
            out["y_packed"], out["y_scale"] = _alloc_packed(R, D, device)
        else:
            out["y"] = torch.empty(R, D, dtype=dt, device=device)
        out["rstd"] = torch.empty(R, dtype=torch.float32, device=device)
        if checkpoint:
            out["packed"], out["scale"] = _alloc_packed(R, D, device)
    at = {k: t.data_ptr() for k, t in out.items()}
    _call(load_library().ppow_rms_norm, "ppow_rms_norm", dev, ctypes.byref(params), xp, xs, rp, rs, w, at.get("sum"), at.get("y"), at["rstd"],
          at.get("y_packed"), at.get("y_scale"), at.get("packed"), at.get("scale"), _raw_stream(stream, dev))
    return out


def rms_norm_backward(grad_y, x, weight, rstd, *, grad_sum=None, stream=None):
    """Allocate gradients and workspace, run ppow_rms_norm_backward; returns (grad_x, grad_weight).  ``x`` is what the forward pass
    normalised (its sum, where it had a residual) or the pair (packed, scale) that it left; ``grad_sum`` is what reaches that sum past
    the norm.  grad_x is the gradient of the forward pass's x and residual alike."""
    if stream is None:
        direct, (packed, scale) = (None, x) if isinstance(x, (tuple, list)) else (x, (None, None))
        got = _quick().rms_norm_backward(grad_y, direct, packed, scale, weight, rstd, grad_sum)
        if got is not None:
            return _done(got, "ppow_rms_norm_backward")
    R, D = grad_y.shape
    dt, pt, device, dev = grad_y.dtype, weight.dtype, grad_y.device, _index_of(grad_y, "grad_y")
    params, lib = make_norm_params(R, D, dt, pt), load_library()
    gp, gs = _rows_arg(grad_y, dt, (R, D), dev, "grad_y")
    sp, ss = _maybe_rows_arg(grad_sum, dt, (R, D), dev, "grad_sum")
    if isinstance(x, (tuple, list)):
        (xp, xs), (q, s) = (None, D), _packed_args(*x, R, D, dev)
    else:
        (xp, xs), (q, s) = _rows_arg(x, dt, (R, D), dev, "x"), (None, None)
    w, r = _arg(weight, pt, (D,), dev, "weight"), _arg(rstd, torch.float32, (R,), dev, "rstd")
    with _on(stream):
        gx, gw = torch.empty(R, D, dtype=dt, device=device), torch.empty(D, dtype=pt, device=device)
        nbytes = lib.ppow_rms_norm_workspace_bytes(ctypes.byref(params))
        ws = _workspace(nbytes, device)
    _call(lib.ppow_rms_norm_backward, "ppow_rms_norm_backward", dev, ctypes.byref(params), gp, gs, sp, ss, xp, xs, q, s, w, r, gx.data_ptr(),
          gw.data_ptr(), ws.data_ptr(), nbytes, _raw_stream(stream, dev))
    return gx, gw


def clip_gradients(grads, max_norm, *, out=None, stream=None):
    """Scale the gradients ``grads`` (a sequence of CUDA tensors of one device, dense, of any shapes and float types) by
    min(1, max_norm / norm), norm the square root of the sum of all their squares: in place, or into the tensors of ``out``, which have
    the gradients' shapes, types and strides.  Returns norm, a float32 tensor without dimensions; nothing waits for it.  To autograd the
    tensors written are modified in place: a backward pass that saved one raises."""
    return _clip(grads, grads if out is None else out, max_norm, stream)


def gradient_norm(grads, *, stream=None):
    """The norm that clip_gradients goes by, alone."""
    return _clip(grads, None, 0.0, stream)


def _clip(grads, out, max_norm, stream):
    grads = list(grads)
    out = None if out is None else list(out)
    if not grads:
        raise ValueError("grads must hold at least one tensor")
    if stream is None:
        got = _quick().clip_gradients(grads, out, max_norm)
        if got is not None:
            return _done(got, "ppow_clip_gradients")[0]
    device = grads[0].device
    _index_of(grads[0], "grads[0]")
    with _on(stream):
        norm = torch.empty((), dtype=torch.float32, device=device)
        ws = _workspace(ppow_clip_workspace_bytes(len(grads)), device)
    ppow_clip_gradients(grads, out, max_norm, norm, ws, stream)
    return norm


def sample_tokens(logits, uniforms, *, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, stream=None) -> dict:
    """Allocate outputs and run ppow_sample_tokens on ``logits`` [R, V] and ``uniforms`` [R]; returns tokens (int32), logp (of the
    distribution that was drawn from, after temperature and filters) and kept (how many tokens the filters left)."""
    if stream is None:
        got = _quick().sample_tokens(logits, uniforms, temperature, top_k, top_p, min_p)
        if got is not None:
            tokens, logp, kept = _done(got, "ppow_sample_tokens")
            return {"tokens": tokens, "logp": logp, "kept": kept}
    params, device, dev = make_sample_params(logits, temperature, top_k, top_p, min_p), logits.device, _index_of(logits, "logits")
    R, V = logits.shape
    x = _rows_arg(logits, logits.dtype, (R, V), dev, "logits")[0]
    u = _arg(uniforms, torch.float32, (R,), dev, "uniforms")
    with _on(stream):
        out = {"tokens": torch.empty(R, dtype=torch.int32, device=device), "logp": torch.empty(R, dtype=torch.float32, device=device),
               "kept": torch.empty(R, dtype=torch.int32, device=device)}
    _call(load_library().ppow_sample_tokens, "ppow_sample_tokens", dev, ctypes.byref(params), x, u, out["tokens"].data_ptr(),
          out["logp"].data_ptr(), out["kept"].data_ptr(), _raw_stream(stream, dev))
    return out
