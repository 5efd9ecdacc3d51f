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


# ------------------------------------------------------------------ odd inputs, strides, streams


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [64, 1000, 1531, 4096])
def test_constant_rows_large_offsets_and_zero_gradient(D, dtype):
    x, w, b, gy = make(40, D, dtype, seed=3)
    x[0], x[1], x[2] = 0.0, 3.0, -0.5
    x[3:10] += 500.0                                          # a mean far above the spread
    gy[5] = 0.0
    out = B.layer_norm(x, w, b, eps=1e-5, checkpoint=True)
    got = B.layer_norm_backward(gy, x, w, out["mean"], out["rstd"])
    packed = B.layer_norm_backward(gy, (out["packed"], out["scale"]), w, out["mean"], out["rstd"])
    torch.cuda.synchronize()
    check_forward(x, w, b, 1e-5, out)
    check_packed(x, out["packed"], out["scale"])
    check_backward(gy, x.double(), w, out["mean"], out["rstd"], got, torch.float32)
    check_backward(gy, reference_pack(x)[2], w, out["mean"], out["rstd"], packed, torch.float32)
    assert not got[0][5].any() and torch.all(out["y"][0] == b.to(dtype))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [64, 777, 4096, 8200])
def test_rows_that_are_not_finite_stay_among_themselves(D, dtype):
    x, w, b, gy = make(9, D, dtype, seed=4)
    clean = B.layer_norm(x, w, b, checkpoint=True)
    x[2, D // 2], x[5, 0], x[7, D - 1] = float("nan"), float("inf"), -float("inf")
    out = B.layer_norm(x, w, b, checkpoint=True)
    torch.cuda.synchronize()
    bad = torch.tensor([2, 5, 7], device=DEV)
    good = torch.tensor([0, 1, 3, 4, 6, 8], device=DEV)
    for k in ("y", "mean", "rstd", "scale"):
        assert torch.equal(out[k][good], clean[k][good]), k
    assert torch.equal(out["packed"].view(torch.uint8)[good], clean["packed"].view(torch.uint8)[good])
    assert out["y"][bad].isnan().any(1).all()
    check_packed(x, out["packed"], out["scale"])             # the scale goes by the finite values, what is not finite is NaN
    q, s = B.pack_activation(x)
    torch.cuda.synchronize()
    assert torch.equal(q.view(torch.uint8), out["packed"].view(torch.uint8)) and torch.equal(s, out["scale"])
    gx, _, _ = B.layer_norm_backward(gy, x, w, out["mean"], out["rstd"])
    want, _, _ = B.layer_norm_backward(gy, torch.where(x.isfinite(), x, 0), w, clean["mean"], clean["rstd"])
    torch.cuda.synchronize()
    assert torch.equal(gx[good], want[good])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [128, 131, 640])
def test_edges_of_the_8_bit_format(D, dtype):
    top = torch.finfo(dtype).max
    rows = []
    for k in (0, 1, 5, -3, 8):                               # borders of the scale: 448 * 2^k and its neighbours
        for f in (1.0, 1.0 + torch.finfo(dtype).eps, 1.0 - torch.finfo(dtype).eps / 2, 0.5, 448.5 / 448):
            rows.append(448.0 * 2.0 ** k * f)
    rows += [top, torch.finfo(dtype).tiny, torch.finfo(dtype).smallest_normal / 4, 0.0, 2.0 ** -9, 1.0]
    x = torch.zeros((len(rows), D), dtype=torch.float64, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(D)
    ramp = 2.0 ** -torch.randint(0, 20, (len(rows), D), generator=g, device=DEV).double()
    ramp *= 1 + torch.randint(0, 64, (len(rows), D), generator=g, device=DEV) / 64            # ties of the rounding among them
    x = (ramp * torch.tensor(rows, dtype=torch.float64, device=DEV)[:, None] / 2).to(dtype)
    x[:, D // 3] = torch.tensor(rows, dtype=torch.float64, device=DEV).to(dtype)
    x[::2] = -x[::2]
    q, s = B.pack_activation(x)
    back = {t: B.unpack_activation(q, s, t) for t in TYPES}
    torch.cuda.synchronize()
    check_packed(x, q, s)
    value = reference_pack(x)[2]
    for t in TYPES:                                          # 448 * 2^8 is an infinity in float16 and comes back as NaN
        torch.testing.assert_close(back[t], value.to(t), rtol=0, atol=0, equal_nan=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("R,D,offset,pad", [(30, 512, 1, 0), (30, 512, 16, 16), (5, 4096, 3, 2), (17, 1531, 0, 5), (3, 8192, 8, 8)])
def test_rows_of_other_strides_and_alignments(R, D, offset, pad, dtype):
    x, w, b, gy = make(R, D, dtype, seed=5)

    def view(t):
        wide = torch.full((R, D + offset + pad), float("nan"), dtype=dtype, device=DEV)
        wide[:, offset:offset + D] = t
        return wide[:, offset:offset + D]
    a = B.layer_norm(x, w, b, checkpoint=True)
    v = B.layer_norm(view(x), w, b, checkpoint=True)
    q, s = B.pack_activation(view(x))
    ga = B.layer_norm_backward(gy, x, w, a["mean"], a["rstd"])
    gv = B.layer_norm_backward(view(gy), view(x), w, a["mean"], a["rstd"])
    gp = B.layer_norm_backward(view(gy), (a["packed"], a["scale"]), w, a["mean"], a["rstd"])
    torch.cuda.synchronize()
    check_forward(x, w, b, 1e-5, v)
    assert torch.equal(a["packed"].view(torch.uint8), v["packed"].view(torch.uint8)) and torch.equal(a["scale"], v["scale"])
    assert torch.equal(q.view(torch.uint8), a["packed"].view(torch.uint8)) and torch.equal(s, a["scale"])
    check_backward(gy, x.double(), w, a["mean"], a["rstd"], ga, torch.float32)
    check_backward(gy, x.double(), w, a["mean"], a["rstd"], gv, torch.float32)
    check_backward(gy, reference_pack(x)[2], w, a["mean"], a["rstd"], gp, torch.float32)


@pytest.mark.parametrize("offset", [1, 2, 3, 5])
def test_parameters_and_packed_bytes_at_odd_addresses(offset):
    R, D = 6, 256
    x, w, b, gy = make(R, D, torch.bfloat16, seed=6)
    par = torch.zeros(2 * D + 16, device=DEV)
    wv, bv = par[offset:offset + D], par[D + offset:2 * D + offset]
    wv.copy_(w), bv.copy_(b)
    buf = torch.zeros(R * D + 16, dtype=torch.uint8, device=DEV)
    sc = torch.zeros(R * 2 + 16, dtype=torch.uint8, device=DEV)
    qv, sv = buf[offset:offset + R * D].view(R, D).view(torch.float8_e4m3fn), sc[offset:offset + 2 * R].view(R, 2)
    want = B.layer_norm(x, w, b, checkpoint=True)
    out = {k: torch.empty_like(v) for k, v in want.items()}
    p = B.make_norm_params(R, D, x.dtype, torch.float32)
    B.ppow_layer_norm(p, x, wv, bv, out["y"], out["mean"], out["rstd"], qv, sv)
    g1 = B.layer_norm_backward(gy, (qv, sv), wv, want["mean"], want["rstd"])
    g2 = B.layer_norm_backward(gy, (want["packed"], want["scale"]), w, want["mean"], want["rstd"])
    torch.cuda.synchronize()
    check_forward(x, w, b, 1e-5, out)
    check_packed(x, qv, sv)
    for g in (g1, g2):
        check_backward(gy, reference_pack(x)[2], w, want["mean"], want["rstd"], g, torch.float32)
    assert not buf[:offset].any() and not buf[offset + R * D:].any() and not sc[:offset].any() and not sc[offset + 2 * R:].any()


@pytest.mark.parametrize("R,D,dtype", [(700, 4096, torch.bfloat16), (4000, 72, torch.float16), (50, 1531, torch.float32)])
def test_same_results_every_time_and_nothing_behind_them_is_touched(R, D, dtype):
    x, w, b, gy = make(R, D, dtype, seed=7)
    p = B.make_norm_params(R, D, dtype, torch.float32)
    first = None
    for fill in (0, 255):
        o = {"y": torch.full((R + 1, D), 7.0, device=DEV, dtype=dtype), "m": torch.full((R + 4,), 7.0, device=DEV),
             "r": torch.full((R + 4,), 7.0, device=DEV), "gx": torch.full((R + 1, D), 7.0, device=DEV, dtype=dtype),
             "gw": torch.full((D + 4,), 7.0, device=DEV), "gb": torch.full((D + 4,), 7.0, device=DEV)}
        ws = torch.full((B.ppow_layer_norm_workspace_bytes(p),), fill, dtype=torch.uint8, device=DEV)
        B.ppow_layer_norm(p, x, w, b, o["y"][:R], o["m"][:R], o["r"][:R])
        B.ppow_layer_norm_backward(p, gy, x, None, None, w, o["m"][:R], o["r"][:R], o["gx"][:R], o["gw"][:D], o["gb"][:D], ws)
        torch.cuda.synchronize()
        for k, n in (("y", R), ("m", R), ("r", R), ("gx", R), ("gw", D), ("gb", D)):
            assert torch.all(o[k][n:] == 7), k
        assert first is None or all(torch.equal(first[k], o[k]) for k in o)
        first = o


def test_no_rows():
    x, w, b, gy = make(3, 200, torch.bfloat16)
    out = B.layer_norm(x[:0], w, b, checkpoint=True)
    assert out["y"].shape == (0, 200) and out["packed"].shape == (0, 200) and out["scale"].shape == (0, 2)
    gx, gw, gb = B.layer_norm_backward(gy[:0], x[:0], w, out["mean"], out["rstd"])
    torch.cuda.synchronize()
    assert gx.shape == (0, 200) and not gw.any() and not gb.any()
    q, s = B.pack_activation(x[:0])
    assert B.unpack_activation(q, s).shape == (0, 200)


def test_wider_than_supported():
    x = torch.zeros((2, 16385), device=DEV, dtype=torch.bfloat16)
    w = torch.zeros(16385, device=DEV)
    with pytest.raises(B.PpowError) as e:
        B.layer_norm(x, w)
    assert e.value.status == B.PPOW_ERR_UNSUPPORTED
    q, s = B.pack_activation(x)                              # a checkpoint may be wider
    assert torch.equal(B.unpack_activation(q, s), x)


def test_streams_and_replays():
    x, w, b, gy = make(900, 1000, torch.bfloat16, seed=8)
    x2, _, _, gy2 = make(900, 1000, torch.bfloat16, seed=9)

    def step(x, gy, **k):
        out = B.layer_norm(x, w, b, checkpoint=True, **k)
        q, s = B.pack_activation(gy, **k)
        return (out["y"], *B.layer_norm_backward(gy, (out["packed"], out["scale"]), w, out["mean"], out["rstd"], **k),
                B.unpack_activation(q, s, **k))
    want, want2 = step(x, gy), step(x2, gy2)
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        a, c = step(x, gy, stream=s1), step(x2, gy2, stream=s2)
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(a, want)) and all(torch.equal(p, q) for p, q in zip(c, want2))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(x, gy)
    x.copy_(x2), gy.copy_(gy2)
    for _ in range(2):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want2))


@pytest.mark.parametrize("R,D", [(5, 96), (3, 1531)])
def test_gradient_against_differences_of_the_forward_pass(R, D):
    # float32: along a unit direction d of the row's space the loss is smooth; its third derivative times h^2/6 and the forward
    # pass's rounding over h bound the difference.  Along x + h d, y = w (x - mean) rstd + b with sigma about 1: derivatives of
    # 1/sigma up to order three stay below 15 for |d| = 1 and sigma >= 1/2, hence below 15 max|gy w| sqrt(D) in all.
    x, w, b, gy = make(R, D, torch.float32, seed=10, offset=0.0)
    x = torch.randn((R, D), device=DEV, generator=torch.Generator(device=DEV).manual_seed(1))
    g = torch.Generator(device=DEV).manual_seed(11)
    d = torch.randn((R, D), generator=g, device=DEV)
    d = d / d.norm(dim=1, keepdim=True)
    h = 2.0 ** -5
    at = [x + s * h * d for s in (1, -1)]
    step = (at[0].double() - at[1].double())                 # what was added after rounding
    loss = [(B.layer_norm(t, w, b)["y"].double() * gy.double()).sum(1) for t in at]
    out = B.layer_norm(x, w, b)
    gx, _, _ = B.layer_norm_backward(gy, x, w, out["mean"], out["rstd"])
    got, want = (gx.double() * step).sum(1), loss[0] - loss[1]
    a = (gy * w).double().abs()
    smooth = 2 * h ** 3 / 6 * 15 * a.amax(1) * D ** 0.5
    y = out["y"].double().abs()
    rounding = 2 * (gy.double().abs() * (256 * E * (y + b.double().abs()) + 160 * E * x.double().abs().amax(1, keepdim=True) * w.double().abs())).sum(1)
    back = (step.abs() * (256 * E * (a + a.mean(1, keepdim=True)) * 2)).sum(1)
    assert torch.all((got - want).abs() <= smooth + rounding + back)
    # and not by being loose: without the two mean terms the difference is far outside
    naive = ((gy * w).double() * out["rstd"].double()[:, None] * step).sum(1)
    assert float((naive - want).abs().max()) > 4 * float((got - want).abs().max())


@pytest.mark.parametrize("R,D,dtype", [(1 << 20, 3, torch.float16), (1 << 20, 64, torch.bfloat16), (70000, 136, torch.float32)])
def test_many_short_rows(R, D, dtype):
    x, w, b, gy = make(R, D, dtype, seed=12)
    out = B.layer_norm(x, w, b, checkpoint=True)
    got = B.layer_norm_backward(gy, (out["packed"], out["scale"]), w, out["mean"], out["rstd"])
    back = B.unpack_activation(out["packed"], out["scale"], dtype)
    torch.cuda.synchronize()
    check_forward(x, w, b, 1e-5, out)
    check_packed(x, out["packed"], out["scale"])
    value = reference_pack(x)[2]
    assert torch.equal(back, value.to(dtype))
    check_backward(gy, value, w, out["mean"], out["rstd"], got, torch.float32)


def test_a_checkpoint_of_more_than_two_to_the_31_values():
    R, D = 40000, 54000                                      # 2.16e9 values: offsets pass 32 bits
    x = torch.zeros((R, D), dtype=torch.bfloat16, device=DEV)
    probe = [0, 1, R // 2, R - 2, R - 1]
    g = torch.Generator(device=DEV).manual_seed(0)
    x[probe] = torch.randn((len(probe), D), generator=g, device=DEV).bfloat16()
    q, s = B.pack_activation(x)
    back = B.unpack_activation(q, s)
    torch.cuda.synchronize()
    check_packed(x[probe], q[probe], s[probe])
    assert torch.equal(back[probe].double(), reference_pack(x[probe])[2])
    assert not back[2].any() and int((s != 1).any(1).sum()) == len(probe)
