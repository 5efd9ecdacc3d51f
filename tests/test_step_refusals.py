"""What the entry points of drawn tokens, the RMS norm and gradient clipping refuse, on the CPU: every refusal comes before anything is
launched, so made-up addresses will do, and the binding refuses tensors that do not live on a device or have another type, shape or order."""
import ctypes
import math

import pytest
import torch

from paper_2605_14978_b200 import binding as B
from paper_2605_14978_b200 import build as build_mod

OK, ARG, UNSUPPORTED, WORKSPACE = B.PPOW_OK, B.PPOW_ERR_INVALID_ARG, B.PPOW_ERR_UNSUPPORTED, B.PPOW_ERR_WORKSPACE
P = 1 << 20          # an aligned address that is never used


@pytest.fixture(scope="module")
def lib():
    build_mod.build()
    return B.load_library()


# ------------------------------------------------------------------ drawn tokens


def sample(lib, R=4, V=100, dtype=B.PPOW_BF16, top_k=0, stride=None, temperature=1.0, top_p=1.0, min_p=0.0, z=P, u=P, t=P, l=P, k=P):
    p = B.ppow_sample_params(R, V, dtype, top_k, V if stride is None else stride, temperature, top_p, min_p)
    return lib.ppow_sample_tokens(ctypes.byref(p), z, u, t, l, k, None)


@pytest.mark.parametrize("bad", [dict(R=-1), dict(R=(1 << 27) + 1), dict(V=0), dict(V=-5), dict(dtype=3), dict(dtype=-1), dict(top_k=-1), dict(stride=99),
                                 dict(stride=0), dict(stride=-100), dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=math.inf),
                                 dict(temperature=math.nan), dict(temperature=1e-31), dict(top_p=0.0), dict(top_p=-0.1), dict(top_p=1.1),
                                 dict(top_p=math.nan), dict(min_p=-0.1), dict(min_p=1.5), dict(min_p=math.nan), dict(z=None), dict(z=P + 1),
                                 dict(u=None), dict(u=P + 2), dict(t=None), dict(t=P + 2), dict(l=None), dict(l=P + 1), dict(k=P + 2)])
def test_sample_arguments(lib, bad):
    assert sample(lib, **bad) == ARG


def test_sample_limits(lib):
    assert sample(lib, V=(1 << 22) + 1) == UNSUPPORTED
    assert sample(lib, R=0, z=None, u=None, t=None, l=None, k=None) == OK
    assert lib.ppow_sample_tokens(None, P, P, P, P, P, None) == ARG


# ------------------------------------------------------------------ RMS norm


def norm(R=4, D=64, dtype=B.PPOW_BF16, params=B.PPOW_F32, eps=1e-6):
    return B.ppow_norm_params(R, D, dtype, params, eps)


def forward(lib, p, x=P, xs=64, r=P, rs=64, w=P, s=P, y=P, rstd=P, yq=None, ys=None, q=None, sc=None):
    return lib.ppow_rms_norm(ctypes.byref(p) if p else None, x, xs, r, rs, w, s, y, rstd, yq, ys, q, sc, None)


def backward(lib, p, gy=P, gys=64, gs=P, gss=64, x=P, xs=64, q=None, sc=None, w=P, rstd=P, gx=P, gw=P, ws=P, n=1 << 40):
    return lib.ppow_rms_norm_backward(ctypes.byref(p) if p else None, gy, gys, gs, gss, x, xs, q, sc, w, rstd, gx, gw, ws, n, None)


@pytest.mark.parametrize("bad", [dict(R=-1), dict(R=(1 << 28) + 1), dict(D=0), dict(D=-4), dict(dtype=3), dict(params=9), dict(params=B.PPOW_F16),
                                 dict(dtype=B.PPOW_F32, params=B.PPOW_BF16), dict(eps=-1e-6), dict(eps=math.nan), dict(eps=math.inf)])
def test_rms_parameters(lib, bad):
    p = norm(**bad)
    assert lib.ppow_rms_norm_workspace_bytes(ctypes.byref(p)) == 0
    assert forward(lib, p) == ARG and backward(lib, p) == ARG


def test_rms_width_strides_pointers_and_workspace(lib):
    wide = norm(D=16385)
    assert lib.ppow_rms_norm_workspace_bytes(ctypes.byref(wide)) == 0
    assert forward(lib, wide, xs=16385, rs=16385) == UNSUPPORTED and backward(lib, wide, gys=16385, gss=16385, xs=16385) == UNSUPPORTED
    p = norm()
    for k in ("x", "w", "rstd"):
        assert forward(lib, p, **{k: None}) == ARG
    for k in ("x", "r", "w", "s", "y", "rstd"):
        assert forward(lib, p, **{k: P + 1}) == ARG
    for bad in (dict(xs=63), dict(rs=63), dict(rs=-64), dict(r=None), dict(s=None), dict(y=None), dict(yq=P), dict(ys=P), dict(q=P), dict(sc=P)):
        assert forward(lib, p, **bad) == ARG, bad
    assert forward(lib, None) == ARG
    for k in ("gy", "w", "rstd", "gx"):
        assert backward(lib, p, **{k: None}) == ARG
    for k in ("gy", "gs", "x", "w", "rstd", "gx", "gw"):
        assert backward(lib, p, **{k: P + 1}) == ARG
    for bad in (dict(gys=63), dict(gss=63), dict(xs=63), dict(x=None), dict(q=P, sc=P), dict(x=None, q=P), dict(x=None, sc=P)):
        assert backward(lib, p, **bad) == ARG, bad
    need = lib.ppow_rms_norm_workspace_bytes(ctypes.byref(p))
    assert need == 4 * 64 * 4
    for bad in (dict(ws=None), dict(ws=P + 128), dict(n=need - 1)):
        assert backward(lib, p, **bad) == WORKSPACE, bad
    assert backward(lib, None) == ARG
    assert forward(lib, norm(R=0), x=None, r=None, s=None, w=None, y=None, rstd=None) == OK
    assert backward(lib, norm(R=0), gw=None, ws=None, n=0) == OK


# ------------------------------------------------------------------ clipping


def clip(lib, grads, out, sizes, dtypes, max_norm=1.0, norm=P, ws=P, n=None, nbytes=1 << 40):
    k = len(sizes)
    ptrs = ctypes.c_void_p * max(k, 1)
    return lib.ppow_clip_gradients(k if n is None else n, ptrs(*grads), None if out is None else ptrs(*out), (ctypes.c_int64 * max(k, 1))(*sizes),
                                   (ctypes.c_int32 * max(k, 1))(*dtypes), max_norm, norm, ws, nbytes, None)


def test_clip_arguments(lib):
    Q, F = P * 8, B.PPOW_F32
    for args in (([P], [P], [-1], [F]), ([P], [P], [(1 << 40) + 1], [F]), ([P], [P], [4], [3]), ([None], [P], [4], [F]), ([P], [None], [4], [F]),
                 ([P + 2], [P], [4], [F]), ([P], [P + 1], [4], [B.PPOW_BF16]), ([P, Q], [P, Q], [1 << 40, 1], [F, F])):
        assert clip(lib, *args) == ARG, args
    good = ([P], [P], [4], [F])
    for bad in (dict(max_norm=-1.0), dict(max_norm=math.nan), dict(max_norm=math.inf), dict(norm=None), dict(norm=P + 2), dict(n=-1), dict(n=65537)):
        assert clip(lib, *good, **bad) == ARG, bad
    assert lib.ppow_clip_gradients(1, None, None, None, None, 1.0, P, P, 1 << 40, None) == ARG
    need = lib.ppow_clip_workspace_bytes(1)
    for bad in (dict(ws=None), dict(ws=P + 16), dict(nbytes=need - 1)):
        assert clip(lib, *good, **bad) == WORKSPACE, bad
    assert lib.ppow_clip_workspace_bytes(-1) == 0 and lib.ppow_clip_workspace_bytes(65537) == 0
    assert 0 < lib.ppow_clip_workspace_bytes(0) <= need <= lib.ppow_clip_workspace_bytes(65536)


def test_clip_overlaps(lib):
    F = B.PPOW_F32
    for grads, out, sizes in (([P, P], [P, P], [4, 4]), ([P, P + 12], [P, P + 12], [4, 4]), ([P, P + 64], [P + 64, P], [4, 4]),
                              ([P, P + 64], [P + 128, P + 132], [4, 4]), ([P], [P + 4], [4]), ([P + 4], [P], [4]),
                              ([P, P + 4096], [P + 8192, P + 8], [4, 4]), ([P + 8, P + 4096], [P + 8192, P], [4, 4]),
                              ([P, P + 4], [P + 64, P + 4], [8, 1])):
        assert clip(lib, grads, out, sizes, [F] * len(sizes)) == ARG, (grads, out)


def test_binding_refuses_tensors_of_the_wrong_kind(lib):
    h, f = torch.zeros((4, 16), dtype=torch.bfloat16), torch.zeros(4)
    with pytest.raises(ValueError, match="CUDA device"):
        B.sample_tokens(h, f)
    with pytest.raises(ValueError, match="2-D"):
        B.sample_tokens(h[0], f)
    with pytest.raises(ValueError, match="float32, bfloat16 or float16"):
        B.sample_tokens(h.double(), f)
    with pytest.raises(ValueError, match="CUDA device"):
        B.rms_norm(h, torch.ones(16))
    with pytest.raises(ValueError, match="CUDA device"):
        B.rms_norm_backward(h, h, torch.ones(16), f)
    with pytest.raises(ValueError, match="types must be"):
        B.rms_norm(h, torch.ones(16, dtype=torch.float64)) if h.is_cuda else B.make_norm_params(4, 16, torch.float64, torch.float32)
    with pytest.raises(ValueError, match="CUDA device"):
        B.clip_gradients([h, f], 1.0)
    with pytest.raises(ValueError, match="CUDA device"):
        B.gradient_norm([h])
    for empty in ([], ()):
        with pytest.raises(ValueError, match="at least one"):
            B.clip_gradients(empty, 1.0)


def test_a_large_top_k_stays_large(lib):
    z = torch.zeros((2, 8), dtype=torch.bfloat16)
    assert B.make_sample_params(z, top_k=1 << 32).top_k == 2 ** 31 - 1 and B.make_sample_params(z, top_k=-(1 << 32)).top_k == -1


def test_struct_layout(lib):
    assert ctypes.sizeof(B.ppow_sample_params) == 4 * 4 + 8 + 3 * 8 and B.ppow_sample_params.temperature.offset == 24
