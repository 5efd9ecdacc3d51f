"""Layer norm with its gradient, and the 8-bit form of activations, against their definitions in float64.

Tolerances are bounds, element by element; e = 2^-24 is half a step of float32, u half a step of the storage type.
  sums      a thread adds at most 32 values in turn, 5 steps join a warp, at most 32 warps follow: 80 e of the sum of
            magnitudes covers them
  mean      dm = 80 e max|x|
  variance  128 e of itself, and what an inexact mean adds: 4 dm sigma + 4 dm^2
  8 bits    no tolerance: the format is defined value by value
"""
import pytest
import torch

from paper_2605_14978_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
E = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TYPES = [torch.bfloat16, torch.float16, torch.float32]


def make(R, D, dtype, seed=0, offset=0.3):
    g = torch.Generator(device=DEV).manual_seed(seed * 104729 + R * 131 + D)
    gain = torch.exp(torch.randn(D, generator=g, device=DEV))
    x = (torch.randn((R, D), generator=g, device=DEV) * gain + offset).to(dtype)
    w = 1.0 + 0.3 * torch.randn(D, generator=g, device=DEV)
    b = 0.2 * torch.randn(D, generator=g, device=DEV)
    gy = (0.1 * torch.randn((R, D), generator=g, device=DEV)).to(dtype)
    return x, w, b, gy


def tiny(dtype):
    return 2.0 ** -25 if dtype == torch.float16 else 2.0 ** -133      # half the smallest step


def check_forward(x, w, b, eps, out):
    u = HALF[x.dtype]
    xd, wd = x.double(), w.double()
    bd = torch.zeros_like(wd) if b is None else b.double()
    mean = xd.mean(1)
    var = (xd - mean[:, None]).square().mean(1)
    dm = 80 * E * xd.abs().amax(1)
    assert torch.all((out["mean"].double() - mean).abs() <= dm + E * mean.abs())
    dv = 128 * E * var + 4 * dm * var.sqrt() + 4 * dm ** 2
    rstd = 1.0 / torch.sqrt(var + eps)
    # 1/sqrt over the interval of variances that rounding allows
    lo = 1.0 / torch.sqrt(var + dv + eps) * (1 - 4 * E)
    hi = 1.0 / torch.sqrt((var - dv).clamp(min=0) + eps) * (1 + 4 * E)
    got = out["rstd"].double()
    assert torch.all((got >= lo) & (got <= hi))
    dr = torch.maximum(hi - rstd, rstd - lo)[:, None]
    xc = (xd - mean[:, None]).abs()
    y = (xd - mean[:, None]) * rstd[:, None] * wd + bd
    err = ((xc + dm[:, None]) * dr + (xc * 3 * E + dm[:, None]) * rstd[:, None]) * wd.abs() + 2 * E * (y.abs() + bd.abs())
    tol = err * (1 + u) + u * y.abs() + tiny(x.dtype)
    bad = ~((out["y"].double() - y).abs() <= tol)
    assert not bad.any(), (int(bad.sum()), out["y"][bad][:4], y[bad][:4], tol[bad][:4])


def reference_pack(x):
    """Codes (as values) and exponents, value by value in float64 from the definition."""
    R, D = x.shape
    n = -(-D // 128)
    v = torch.zeros((R, n * 128), dtype=torch.float64, device=x.device)
    v[:, :D] = x.double()
    v = v.view(R, n, 128)
    top = torch.where(v.isfinite(), v.abs(), torch.zeros_like(v)).amax(2)
    e = torch.full_like(top, -126.0)
    for k in range(-126, 121):                                # the smallest exponent that holds the block
        e = torch.where(top > 448.0 * 2.0 ** (k), torch.full_like(e, k + 1.0), e)
    u = v / torch.exp2(e)[..., None]
    _, ex = torch.frexp(u)
    step = torch.exp2((ex - 1).clamp(min=-6).double() - 3.0)
    q = torch.round(u / step) * step
    q = torch.where(v.isfinite(), q, torch.full_like(q, float("nan")))
    return q.view(R, -1)[:, :D], e, (q * torch.exp2(e)[..., None]).view(R, -1)[:, :D]


def check_packed(x, packed, scale):
    q, e, _ = reference_pack(x)
    assert torch.equal(scale.double() - 127.0, e)
    torch.testing.assert_close(packed.double(), q, rtol=0, atol=0, equal_nan=True)


def check_backward(gy, xv, w, mean, rstd, got, n_params):
    """xv: the input in float64, from the tensor itself or from the 8-bit form."""
    gx, gw, gb = got
    u = HALF[gy.dtype]
    g, wd, m, r = gy.double(), w.double(), mean.double()[:, None], rstd.double()[:, None]
    xh = (xv - m) * r
    a = g * wd
    c1, c2 = a.mean(1, keepdim=True), (a * xh).mean(1, keepdim=True)
    want = r * (a - c1 - xh * c2)
    d1, d2 = 82 * E * a.abs().mean(1, keepdim=True), 88 * E * (a * xh).abs().mean(1, keepdim=True)
    err = r * (a.abs() * 3 * E + d1 + xh.abs() * d2 + 6 * E * (xh * c2).abs() + 4 * E * (a.abs() + c1.abs() + (xh * c2).abs()))
    tol = err * (1 + u) + u * want.abs() + tiny(gy.dtype)
    bad = ~((gx.double() - want).abs() <= tol)
    assert not bad.any(), (int(bad.sum()), gx[bad][:4], want[bad][:4], tol[bad][:4])
    R = g.shape[0]
    for name, s, terms in (("grad_weight", gw, g * xh), ("grad_bias", gb, g)):
        if s is None:
            continue
        up = HALF[s.dtype]
        total = terms.sum(0)
        tol = (R + 20) * E * terms.abs().sum(0) * (1 + up) + up * total.abs() + tiny(s.dtype)
        bad = ~((s.double() - total).abs() <= tol)
        assert not bad.any(), (name, int(bad.sum()), s[bad][:4], total[bad][:4])


SIZES = [(1, 1), (3, 2), (5, 7), (2, 64), (9, 127), (4, 128), (6, 129), (700, 72), (33, 1000), (17, 1024), (1003, 1027), (5, 1531),
         (650, 4096), (3, 4099), (301, 8192), (7, 8200), (4, 16383), (190, 16384)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("R,D", SIZES)
def test_forward_and_checkpoint(R, D, dtype):
    x, w, b, _ = make(R, D, dtype)
    for params, bias, ckpt in ((torch.float32, True, True), (dtype, False, False)):
        wt, bt = w.to(params), b.to(params) if bias else None
        out = B.layer_norm(x, wt, bt, eps=1e-5, checkpoint=ckpt)
        torch.cuda.synchronize()
        check_forward(x, wt, bt, 1e-5, out)
        if ckpt:
            check_packed(x, out["packed"], out["scale"])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("R,D", SIZES)
def test_gradient_from_the_input_and_from_the_checkpoint(R, D, dtype):
    x, w, b, gy = make(R, D, dtype, seed=1)
    for params in (torch.float32, dtype):
        wt = w.to(params)
        out = B.layer_norm(x, wt, b.to(params), checkpoint=True)
        got = B.layer_norm_backward(gy, x, wt, out["mean"], out["rstd"], want_bias=params == dtype)
        packed = B.layer_norm_backward(gy, (out["packed"], out["scale"]), wt, out["mean"], out["rstd"])
        torch.cuda.synchronize()
        assert got[2] is not None or params != dtype
        check_backward(gy, x.double(), wt, out["mean"], out["rstd"], got, params)
        check_backward(gy, reference_pack(x)[2], wt, out["mean"], out["rstd"], packed, params)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("R,D", SIZES)
def test_pack_and_unpack(R, D, dtype):
    x = make(R, D, dtype, seed=2)[0]
    x[0, 0] = 0.0
    q, s = B.pack_activation(x)
    backs = {t: B.unpack_activation(q, s, t) for t in TYPES}
    torch.cuda.synchronize()
    check_packed(x, q, s)
    value = reference_pack(x)[2]
    for t, back in backs.items():
        assert torch.equal(back, value.to(t)), t
