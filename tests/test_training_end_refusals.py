"""What the training-end entry points refuse, on the CPU: every refusal comes before anything is launched, so made-up addresses
will do, and the binding refuses tensors that do not live on a device or have another type, shape or order."""
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


def head(T=8, V=1000, D=64, dtype=B.PPOW_BF16, hs=None, ws=None, temperature=1.0):
    return B.ppow_head_params(T, V, D, dtype, D if hs is None else hs, D if ws is None else ws, temperature)


BAD_HEAD = [dict(T=-1), dict(T=(1 << 20) + 1), dict(V=1), dict(V=(1 << 22) + 1), dict(D=0), dict(D=12), dict(D=65544), dict(dtype=B.PPOW_F32),
            dict(dtype=7), dict(hs=63), dict(ws=56), dict(ws=68), dict(ws=-64), dict(temperature=0.0), dict(temperature=-1.0),
            dict(temperature=math.inf), dict(temperature=math.nan)]


@pytest.mark.parametrize("bad", BAD_HEAD)
def test_head_parameters(lib, bad):
    p = ctypes.byref(head(**bad))
    assert lib.ppow_head_workspace_bytes(p, 0) == 0 and lib.ppow_head_workspace_bytes(p, 1) == 0
    assert lib.ppow_head_logprob(p, P, P, P, P, P, P, 1 << 40, None) == ARG
    assert lib.ppow_head_logprob_backward(p, P, P, P, P, P, P, P, P, 1 << 40, None) == ARG


def test_head_pointers_and_workspaces(lib):
    p = head()
    q = ctypes.byref(p)
    need, need_back = lib.ppow_head_workspace_bytes(q, 0), lib.ppow_head_workspace_bytes(q, 1)
    assert need > 8 * 64 * 2 and need_back > 8 * 1000 * 2
    assert lib.ppow_head_logprob(None, P, P, P, P, P, P, need, None) == ARG
    args = [P] * 5
    for i in range(5):
        for wrong in ([None] if i == 0 else [None, P + 2]):       # hidden rows may start anywhere
            bad = list(args)
            bad[i] = wrong
            assert lib.ppow_head_logprob(q, *bad, P, need, None) == ARG
    assert lib.ppow_head_logprob(q, P + 1, P, P, P, P, P, need, None) == ARG
    for ws, n in ((None, need), (P + 16, need), (P, need - 1), (P, 0)):
        assert lib.ppow_head_logprob(q, *args, ws, n, None) == WORKSPACE
    args = [P] * 7
    for i in range(5):
        for wrong in ([None] if i == 0 else [None, P + 2]):
            bad = list(args)
            bad[i] = wrong
            assert lib.ppow_head_logprob_backward(q, *bad, P, need_back, None) == ARG
    for gh, gw in ((None, None), (P + 8, P), (P, P + 8), (P + 2, None)):
        assert lib.ppow_head_logprob_backward(q, *args[:5], gh, gw, P, need_back, None) == ARG
    for ws, n in ((None, need_back), (P + 16, need_back), (P, need_back - 1)):
        assert lib.ppow_head_logprob_backward(q, *args, ws, n, None) == WORKSPACE
    empty = ctypes.byref(head(T=0))
    assert lib.ppow_head_logprob(empty, None, None, None, None, None, None, 0, None) == OK
    assert lib.ppow_head_logprob_backward(empty, None, None, None, None, None, P, None, None, 0, None) == OK


def test_head_workspace_is_bounded(lib):
    # one piece of dz is at most 512 MiB; the rest grows with the tokens, not with tokens times vocabulary
    for T in (1, 100, 129, 4096, 65536):
        for V in (2, 1000, 128256, 1 << 22):
            for D in (8, 4096):
                rows = max(16, T + 255)
                n = lib.ppow_head_workspace_bytes(ctypes.byref(head(T=T, V=V, D=D)), 1)
                assert 0 < n < (512 << 20) + rows * (512 + 40 + 6 * D) + 600 * 256 * (D + 256) * 4 + 65536, (T, V, D, n)


def norm(R=4, D=64, dtype=B.PPOW_BF16, params=B.PPOW_F32, eps=1e-5):
    return B.ppow_norm_params(R, D, dtype, params, eps)


def forward(lib, p, x=P, stride=64, w=P, b=P, y=P, m=P, r=P, q=None, s=None):
    return lib.ppow_layer_norm(ctypes.byref(p) if p else None, x, stride, w, b, y, m, r, q, s, None)


def backward(lib, p, gy=P, gs=64, x=P, xs=64, q=None, s=None, w=P, m=P, r=P, gx=P, gw=P, gb=P, ws=P, n=1 << 40):
    return lib.ppow_layer_norm_backward(ctypes.byref(p) if p else None, gy, gs, x, xs, q, s, w, m, r, gx, gw, gb, ws, n, None)


@pytest.mark.parametrize("bad", [dict(R=-1), dict(R=(1 << 28) + 1), dict(D=0), dict(D=-4), dict(dtype=3), dict(params=9), dict(params=B.PPOW_F16),
                                 dict(dtype=B.PPOW_F32, params=B.PPOW_BF16), dict(eps=-1e-6), dict(eps=math.nan), dict(eps=math.inf)])
def test_norm_parameters(lib, bad):
    p = norm(**bad)
    assert lib.ppow_layer_norm_workspace_bytes(ctypes.byref(p)) == 0
    assert forward(lib, p) == ARG and backward(lib, p) == ARG


def test_norm_width_strides_pointers_and_workspace(lib):
    wide = norm(D=16385)
    assert lib.ppow_layer_norm_workspace_bytes(ctypes.byref(wide)) == 0
    assert forward(lib, wide, stride=16385) == UNSUPPORTED and backward(lib, wide, gs=16385, xs=16385) == UNSUPPORTED
    p = norm()
    for k in ("x", "w", "y", "m", "r"):
        assert forward(lib, p, **{k: None}) == ARG
        assert forward(lib, p, **{k: P + 1}) == ARG
    assert forward(lib, p, b=P + 2) == ARG and forward(lib, p, stride=63) == ARG and forward(lib, p, stride=-64) == ARG
    assert forward(lib, p, q=P) == ARG and forward(lib, p, s=P) == ARG and forward(lib, None) == ARG
    for k in ("gy", "w", "m", "r", "gx"):
        assert backward(lib, p, **{k: None}) == ARG
        assert backward(lib, p, **{k: P + 1}) == ARG
    for bad in (dict(gs=63), dict(xs=63), dict(x=None), dict(q=P, s=P), dict(x=None, q=P), dict(x=None, s=P), dict(x=P + 1), dict(gw=P + 2),
                dict(gb=P + 2)):
        assert backward(lib, p, **bad) == ARG, bad
    need = lib.ppow_layer_norm_workspace_bytes(ctypes.byref(p))
    assert need == 4 * 2 * 64 * 4
    for bad in (dict(ws=None), dict(ws=P + 128), dict(n=need - 1)):
        assert backward(lib, p, **bad) == WORKSPACE, bad
    assert backward(lib, None) == ARG
    assert forward(lib, norm(R=0), x=None, w=None, y=None, m=None, r=None) == OK
    assert backward(lib, norm(R=0), gw=None, gb=None, ws=None, n=0) == OK


def test_checkpoint_arguments(lib):
    def pack(x=P, stride=64, R=2, D=64, dtype=B.PPOW_F16, q=P, s=P):
        return lib.ppow_pack_activation(x, stride, R, D, dtype, q, s, None)

    def unpack(q=P, s=P, R=2, D=64, dtype=B.PPOW_F16, x=P):
        return lib.ppow_unpack_activation(q, s, R, D, dtype, x, None)

    for bad in (dict(R=-1), dict(D=0), dict(D=(1 << 20) + 1), dict(dtype=4), dict(x=None), dict(x=P + 1), dict(q=None), dict(s=None)):
        assert pack(**bad) == ARG and unpack(**bad) == ARG, bad
    assert pack(stride=63) == ARG
    assert pack(R=0, x=None, q=None, s=None) == OK and unpack(R=0, x=None, q=None, s=None) == OK


def test_binding_refuses_tensors_of_the_wrong_kind(lib):
    h, w = torch.zeros((4, 16), dtype=torch.bfloat16), torch.zeros((10, 16), dtype=torch.bfloat16)
    tok, f = torch.zeros(4, dtype=torch.int32), torch.zeros(4)
    with pytest.raises(ValueError, match="CUDA device"):
        B.head_logprob(h, w, tok)
    with pytest.raises(ValueError, match="CUDA device"):
        B.head_logprob_backward(h, w, tok, f, f)
    with pytest.raises(ValueError, match="bfloat16 or float16"):
        B.head_logprob(h.float(), w.float(), tok)
    with pytest.raises(ValueError, match="2-D"):
        B.head_logprob(h[0], w, tok)
    with pytest.raises(ValueError, match="CUDA device"):
        B.layer_norm(h, torch.ones(16))
    with pytest.raises(ValueError, match="CUDA device"):
        B.layer_norm_backward(h, h, torch.ones(16), f, f)
    with pytest.raises(ValueError, match="CUDA device"):
        B.pack_activation(h)
    with pytest.raises(ValueError, match="float32, bfloat16 or float16"):
        B.pack_activation(tok[:, None])
    with pytest.raises(ValueError, match="float32, bfloat16 or float16"):
        B.unpack_activation(torch.zeros((4, 16), dtype=torch.float8_e4m3fn), torch.zeros((4, 1), dtype=torch.uint8), torch.float64)
    with pytest.raises(ValueError, match="CUDA device"):
        B.unpack_activation(torch.zeros((4, 16), dtype=torch.float8_e4m3fn), torch.zeros((4, 1), dtype=torch.uint8))
    with pytest.raises(ValueError, match="types must be"):
        B.make_norm_params(4, 16, torch.float64, torch.float32)


def test_struct_layouts(lib):
    assert ctypes.sizeof(B.ppow_head_params) == 4 * 4 + 2 * 8 + 8 and B.ppow_head_params.temperature.offset == 32
    assert ctypes.sizeof(B.ppow_norm_params) == 5 * 4
