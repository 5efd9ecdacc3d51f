"""Log-probability of given tokens straight from hidden states and the head's weight, and its gradient, against the
definition in float64.

Tolerances are bounds, element by element.  u = half a step of the storage type (2^-8 bf16, 2^-11 f16, relative).
  logits   products of 16-bit values are exact in float32; a sum of D of them takes at most D/16 accumulations of 16
           products, each off by at most two steps 2^-23 of the running magnitude, which is at most A = |h| |w|^T.  One
           rounding of the scale and one of the scaled value (2^-24 of A each) and one of the exponential follow.
  lse      moves by at most as much as the logits; the exponentials and sums of a tile add at most 2^-20 relative.
  dz       rounded once (u), its softmax off by the errors of the logits and of the float32 lse that is passed in.
  dh, dW   the errors of dz carried through |W| or |h|, the accumulation of the product, one rounding (u) at the end; in
           f16 also the smallest steps of dz, of the rows brought down by a power of two, and of the result.
"""
import numpy as np
import pytest
import torch

from paper_2605_14978_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def make(T, V, D, dtype, seed=0, masked=0.2):
    g = torch.Generator(device=DEV).manual_seed(seed * 7919 + T * 31 + V * 7 + D)
    w = (torch.randn((V, D), generator=g, device=DEV) * (2.5 / D ** 0.5)).to(dtype)
    tok = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    h = (torch.randn((T, D), generator=g, device=DEV) + 1.2 * w[tok.long()].float()).to(dtype)
    tok[torch.rand(T, generator=g, device=DEV) < masked] = -1
    grad = torch.randn(T, generator=g, device=DEV) / max(T, 1)
    return h, w, tok, grad


def accumulation(n):
    return (2 * (n / 16 + 1)) * 2.0 ** -23


def logits(h, w, temperature):
    """z in float64 and the bound of the error of the float32 logits."""
    h, w = h.double(), w.double()
    z = h @ w.t() / temperature
    a = h.abs() @ w.abs().t() / temperature
    return z, a * (accumulation(h.shape[1]) + 3 * 2.0 ** -24)


def check_forward(h, w, tok, temperature, out):
    live = (tok >= 0).cpu()
    z, dz = logits(h[tok >= 0], w, temperature)
    y = tok[tok >= 0].long()
    lse = torch.logsumexp(z, 1)
    err = dz.amax(1) + 2.0 ** -20 + lse.abs() * 2.0 ** -22
    inside = y < w.shape[0]
    logp = z.gather(1, y.clamp(max=w.shape[0] - 1)[:, None])[:, 0] - lse
    got_lse, got = out["lse"][tok >= 0].double(), out["logp"][tok >= 0].double()
    assert torch.all((got_lse - lse).abs() <= err), float(((got_lse - lse).abs() / err).max())
    e2 = 2 * err + logp.abs() * 2.0 ** -22
    assert torch.all((got - logp)[inside].abs() <= e2[inside])
    assert torch.all(got[~inside] == -float("inf"))
    for k in ("logp", "lse"):
        assert torch.all(out[k].cpu()[~live] == 0.0), k
    if len(lse):
        # far below the worst case, the errors of many rows average out
        assert float((got_lse - lse).norm() / lse.norm()) < 1e-5


def gradient(h, w, tok, lse, grad, temperature):
    """(dh, dW) in float64 and their bounds."""
    dtype, u = h.dtype, U[h.dtype]
    V, D = w.shape
    live = (tok >= 0) & (tok < V) & (grad != 0)
    dh = torch.zeros(h.shape, dtype=torch.float64, device=DEV)
    th = torch.zeros_like(dh)
    hl, wl = h[live], w.double()
    z, ez = logits(hl, w, temperature)
    hl = hl.double()
    n = hl.shape[0]
    g = (grad[live].double() / temperature)[:, None]
    p = torch.exp(z - lse[live].double()[:, None])
    hot = torch.zeros_like(p)
    hot[torch.arange(n, device=DEV), tok[live].long()] = 1.0
    dz = g * (hot - p)
    e = torch.expm1(ez + 2.0 ** -22 + 2.0 ** -22 * lse[live].double().abs()[:, None])
    dz_err = dz.abs() * (u + 2.0 ** -22) + g.abs() * p * e * (1 + u) + g.abs() * 2.0 ** -23
    if dtype == torch.float16 and n:
        _, ex = torch.frexp(g[:, 0])
        up = torch.exp2(ex.double() - 15)                       # what brings a row back
        dz_err = dz_err + 2.0 ** -25 * up[:, None]
    dh[live] = dz @ wl
    th[live] = dz_err @ wl.abs() + (dz.abs() @ wl.abs()) * accumulation(V)
    dw = dz.t() @ hl
    tw = dz_err.t() @ hl.abs() + (dz.abs().t() @ hl.abs()) * accumulation(n)
    if dtype == torch.float16 and n:
        top = torch.exp2(ex.double().max() - 15)
        down = torch.exp2(ex.double() - ex.double().max())
        tw = tw + (dz.abs() / up[:, None]).t() @ (torch.full_like(hl, 2.0 ** -25)) * top
        tw = tw + (dz.abs().t() @ (hl.abs() * 2.0 ** -11)) * (down.min() < 2.0 ** -14)
    tiny = 2.0 ** -25 if dtype == torch.float16 else 0.0
    return dh, th * (1 + u) + dh.abs() * u + tiny, dw, tw * (1 + u) + dw.abs() * u + tiny


def check_backward(h, w, tok, lse, grad, temperature, gh, gw):
    dh, th, dw, tw = gradient(h, w, tok, lse, grad, temperature)
    u = U[h.dtype]
    for name, got, want, tol in (("grad_hidden", gh, dh, th), ("grad_weight", gw, dw, tw)):
        if got is None:
            continue
        bad = ~((got.double() - want).abs() <= tol)
        assert not bad.any(), (name, int(bad.sum()), got[bad][:4], want[bad][:4], tol[bad][:4])
        if float(want.norm()) > 1e-3 * h.dtype.is_floating_point and want.numel() > 4096:
            assert float((got.double() - want).norm() / want.norm()) < 2 * u, name
    masked = (tok < 0) | (grad == 0)
    if gh is not None:
        assert torch.all(gh[masked] == 0)


def run(h, w, tok, grad, temperature=1.0):
    out = B.head_logprob(h, w, tok, temperature=temperature)
    gh, gw = B.head_logprob_backward(h, w, tok, out["lse"], grad, temperature=temperature)
    torch.cuda.synchronize()
    return out, gh, gw


SHAPES = [(1, 2, 8), (1, 1000, 64), (7, 257, 72), (129, 256, 64), (255, 1001, 520), (256, 512, 64), (257, 300, 256),
          (300, 4097, 136), (513, 1500, 1000), (31, 32000, 256), (16, 777, 96), (17, 1001, 264), (64, 4099, 128), (65, 900, 1032),
          (128, 2500, 328)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,V,D", SHAPES)
def test_forward_matches_the_definition(T, V, D, dtype):
    h, w, tok, _ = make(T, V, D, dtype)
    for temperature in (1.0, 0.7):
        out = B.head_logprob(h, w, tok, temperature=temperature)
        torch.cuda.synchronize()
        check_forward(h, w, tok, temperature, out)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,V,D", SHAPES)
def test_gradient_matches_the_definition(T, V, D, dtype):
    h, w, tok, grad = make(T, V, D, dtype, seed=1)
    out, gh, gw = run(h, w, tok, grad, 0.7)
    check_forward(h, w, tok, 0.7, out)
    check_backward(h, w, tok, out["lse"], grad, 0.7, gh, gw)
