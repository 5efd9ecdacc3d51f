"""RMS norm with the residual's addition, its gradient and its 8-bit outputs, against the definitions in float64.

Tolerances are bounds, element by element; E = 2^-24 is half a step of float32, u half a step of the storage type.
  sums      a thread adds at most 32 values, 5 steps join a warp, at most 32 warps follow: 80 E of the sum of magnitudes
  rstd      the interval of 1/sqrt over the mean squares that this allows, and 4 E
  y         two products of float32: 3 E with the conversion of 1/sqrt's interval apart
  8 bits    of s: none, the format is defined value by value; of y: 2^-4 of the value and half the smallest step 2^(e-10)
"""
import pytest
import torch

from paper_2605_14978_b200 import binding as B

import test_gpu_norm as norm

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
E, HALF, TYPES, SIZES = norm.E, norm.HALF, norm.TYPES, norm.SIZES


def make(R, D, dtype, seed=0):
    x, w, _, gy = norm.make(R, D, dtype, seed, offset=0.0)
    g = torch.Generator(device=DEV).manual_seed(seed * 7919 + R + D)
    r = (2.0 * torch.randn((R, D), generator=g, device=DEV)).to(dtype)
    gs = (0.1 * torch.randn((R, D), generator=g, device=DEV)).to(dtype)
    return x, r, w, gy, gs


def added(x, r):
    return x if r is None else (x.float() + r.float()).to(x.dtype)      # one rounding in float32 at most, one to the type


def y_of(s, w, eps):
    """y in float64, and how far its float32 value may be off."""
    sd, wd = s.double(), w.double()
    ms = sd.square().mean(1)
    rstd = 1.0 / torch.sqrt(ms + eps)
    lo, hi = (1.0 / torch.sqrt((ms * (1 + k * 82 * E) + eps) * (1 + k * 2 * E)) * (1 - k * 4 * E) for k in (1, -1))
    dr = torch.maximum(hi - rstd, rstd - lo)
    y = sd * rstd[:, None] * wd
    return y, (sd * wd).abs() * dr[:, None] + 3 * E * y.abs(), lo, hi


def check_forward(x, r, w, eps, out):
    s = added(x, r)
    assert ("sum" in out) == (r is not None)
    if r is not None:
        assert torch.equal(out["sum"], s)
    y, err, lo, hi = y_of(s, w, eps)
    got = out["rstd"].double()
    assert torch.all((got >= lo) & (got <= hi))
    if "y" in out:
        u = HALF[x.dtype]
        tol = err * (1 + u) + u * y.abs() + norm.tiny(x.dtype)
        bad = ~((out["y"].double() - y).abs() <= tol)
        assert not bad.any(), (int(bad.sum()), out["y"][bad][:4], y[bad][:4], tol[bad][:4])
    if "y_packed" in out:
        e = out["y_scale"].double() - 127.0
        R, D = y.shape
        pad = torch.zeros((R, e.shape[1] * 128), dtype=torch.float64, device=DEV)
        for sign, compare in ((1, torch.le), (-1, torch.ge)):    # the least exponent that holds the block, up to the error
            pad[:, :D] = (y.abs() + sign * err).clamp(min=0)
            top = pad.view(R, -1, 128).amax(2)
            least = torch.full_like(top, -126.0)
            for k in range(-126, 121):
                least = torch.where(top > 448.0 * 2.0 ** k, torch.full_like(top, k + 1.0), least)
            assert compare(e, least).all()
        step = torch.exp2(e).repeat_interleave(128, 1)[:, :D]
        value = out["y_packed"].double() * step
        tol = err * (1 + 2.0 ** -4) + 2.0 ** -4 * y.abs() + step * 2.0 ** -10
        assert torch.all((value - y).abs() <= tol)
    if "packed" in out:
        norm.check_packed(s, out["packed"], out["scale"])


def check_backward(gy, sv, w, rstd, gs, got):
    """sv: what was normalised, in float64, from the tensor itself or from the 8-bit form."""
    gx, gw = got
    u = HALF[gy.dtype]
    g, wd, r = gy.double(), w.double(), rstd.double()[:, None]
    more = torch.zeros_like(g) if gs is None else gs.double()
    xh, a = sv * r, g * wd
    c2, d2 = (a * xh).mean(1, keepdim=True), 88 * E * (a * xh).abs().mean(1, keepdim=True)
    want = r * (a - xh * c2) + more
    err = r * (xh.abs() * d2 + 6 * E * (xh * c2).abs() + 4 * E * (a.abs() + (xh * c2).abs())) + 2 * E * (want.abs() + more.abs())
    tol = err * (1 + u) + u * want.abs() + norm.tiny(gy.dtype)
    bad = ~((gx.double() - want).abs() <= tol)
    assert not bad.any(), (int(bad.sum()), gx[bad][:4], want[bad][:4], tol[bad][:4])
    up, terms = HALF[gw.dtype], g * xh
    total = terms.sum(0)
    tol = (g.shape[0] + 20) * E * terms.abs().sum(0) * (1 + up) + up * total.abs() + norm.tiny(gw.dtype)
    bad = ~((gw.double() - total).abs() <= tol)
    assert not bad.any(), (int(bad.sum()), gw[bad][:4], total[bad][:4])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("R,D", SIZES)
def test_forward(R, D, dtype):
    x, r, w, _, _ = make(R, D, dtype)
    for params, res, ckpt, packed in ((torch.float32, r, True, True), (dtype, r, False, False), (dtype, None, True, False),
                                      (torch.float32, None, False, True)):
        wt = w.to(params)
        out = B.rms_norm(x, wt, res, eps=1e-6, checkpoint=ckpt, packed_output=packed)
        torch.cuda.synchronize()
        assert set(out) == {"rstd"} | ({"sum"} if res is not None else set()) | ({"packed", "scale"} if ckpt else set()) | (
            {"y_packed", "y_scale"} if packed else {"y"})
        check_forward(x, res, wt, 1e-6, out)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("R,D", SIZES)
def test_gradient(R, D, dtype):
    x, r, w, gy, gs = make(R, D, dtype, seed=1)
    for params, more in ((torch.float32, gs), (dtype, None)):
        wt = w.to(params)
        out = B.rms_norm(x, wt, r, checkpoint=True)
        got = B.rms_norm_backward(gy, out["sum"], wt, out["rstd"], grad_sum=more)
        packed = B.rms_norm_backward(gy, (out["packed"], out["scale"]), wt, out["rstd"], grad_sum=more)
        torch.cuda.synchronize()
        check_backward(gy, out["sum"].double(), wt, out["rstd"], more, got)
        check_backward(gy, norm.reference_pack(out["sum"])[2], wt, out["rstd"], more, packed)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [64, 777, 4096, 8200])
def test_rows_that_are_zero_or_not_finite_stay_among_themselves(D, dtype):
    x, r, w, gy, gs = make(9, D, dtype, seed=4)
    x[3], r[3] = 0.0, 0.0
    clean = B.rms_norm(x, w, r, checkpoint=True)
    assert torch.all(clean["y"][3] == 0) and abs(float(clean["rstd"][3]) - 1000.0) < 1e-3
    x[2, D // 2], x[5, 0], r[7, D - 1] = float("nan"), float("inf"), -float("inf")
    out = B.rms_norm(x, w, r, checkpoint=True)
    both = B.rms_norm(x, w, r, packed_output=True)
    torch.cuda.synchronize()
    good = torch.tensor([0, 1, 3, 4, 6, 8], device=DEV)
    for k in ("y", "rstd", "sum", "scale"):
        assert torch.equal(out[k][good], clean[k][good]), k
    check_forward(x[good], r[good], w, 1e-6, {k: v[good] for k, v in both.items()})
    assert out["y"][[2, 5, 7]].isnan().any(1).all() and both["y_packed"][[2, 5, 7]].float().isnan().any(1).all()
    norm.check_packed(out["sum"], out["packed"], out["scale"])
    gx, _ = B.rms_norm_backward(gy, out["sum"], w, out["rstd"], grad_sum=gs)
    want, _ = B.rms_norm_backward(gy, clean["sum"], w, clean["rstd"], grad_sum=gs)
    torch.cuda.synchronize()
    assert torch.equal(gx[good], want[good])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("R,D,offset,pad", [(30, 512, 1, 0), (30, 512, 16, 16), (5, 4096, 3, 2), (17, 1531, 0, 5), (3, 8192, 8, 8), (1, 640, 1, 0)])
def test_rows_of_other_strides_and_alignments(R, D, offset, pad, dtype):
    x, r, w, gy, gs = make(R, D, dtype, seed=5)

    def view(t):
        wide = torch.full((R, D + offset + pad), float("nan"), dtype=dtype, device=DEV)
        wide[:, offset:offset + D] = t
        return wide[:, offset:offset + D]
    for a, b in ((view(x), view(r)), (x, view(r)), (view(x), r), (view(x), None)):
        out = B.rms_norm(a, w, b, checkpoint=True)
        two = B.rms_norm(a, w, b, packed_output=True)
        torch.cuda.synchronize()
        check_forward(x, None if b is None else r, w, 1e-6, out)
        check_forward(x, None if b is None else r, w, 1e-6, two)
    s = added(x, r)
    rstd = B.rms_norm(s, w)["rstd"]
    q, sc = B.pack_activation(s)
    for g, t, m in ((view(gy), view(s), view(gs)), (gy, s, view(gs)), (view(gy), s, None)):
        got = B.rms_norm_backward(g, t, w, rstd, grad_sum=m)
        packed = B.rms_norm_backward(g, (q, sc), w, rstd, grad_sum=m)
        torch.cuda.synchronize()
        check_backward(gy, s.double(), w, rstd, None if m is None else gs, got)
        check_backward(gy, norm.reference_pack(s)[2], w, rstd, None if m is None else gs, packed)


@pytest.mark.parametrize("D", [96, 1531, 4096])
@pytest.mark.parametrize("into", ["x", "residual"])
def test_the_sum_may_take_an_input_s_place(D, into):
    x, r, w, _, _ = make(700, D, torch.bfloat16, seed=6)
    want = B.rms_norm(x, w, r)
    xa, ra = x.clone(), r.clone()
    y, rstd = torch.empty_like(x), torch.empty(700, device=DEV)
    B.ppow_rms_norm(B.make_norm_params(700, D, x.dtype, w.dtype, 1e-6), xa, ra, w, xa if into == "x" else ra, y, rstd)
    torch.cuda.synchronize()
    assert torch.equal(xa if into == "x" else ra, want["sum"]) and torch.equal(y, want["y"]) and torch.equal(rstd, want["rstd"])


@pytest.mark.parametrize("offset", [1, 2, 3, 5])
def test_parameters_and_packed_bytes_at_odd_addresses(offset):
    R, D = 6, 256
    x, r, w, gy, gs = make(R, D, torch.bfloat16, seed=7)
    par = torch.zeros(D + 16, device=DEV)
    wv = par[offset:offset + D]
    wv.copy_(w)
    bufs = [torch.zeros(R * D + 16, dtype=torch.uint8, device=DEV) for _ in range(2)]
    scs = [torch.zeros(R * 2 + 16, dtype=torch.uint8, device=DEV) for _ in range(2)]
    q = [b[offset:offset + R * D].view(R, D).view(torch.float8_e4m3fn) for b in bufs]
    s = [b[offset:offset + 2 * R].view(R, 2) for b in scs]
    out = {"sum": torch.empty_like(x), "y": torch.empty_like(x), "rstd": torch.empty(R, device=DEV)}
    B.ppow_rms_norm(B.make_norm_params(R, D, x.dtype, w.dtype, 1e-6), x, r, wv, out["sum"], out["y"], out["rstd"], q[0], s[0], q[1], s[1])
    got = B.rms_norm_backward(gy, (q[1], s[1]), wv, out["rstd"], grad_sum=gs)
    torch.cuda.synchronize()
    check_forward(x, r, w, 1e-6, dict(out, y_packed=q[0], y_scale=s[0], packed=q[1], scale=s[1]))
    check_backward(gy, norm.reference_pack(out["sum"])[2], w, out["rstd"], gs, got)
    for b, n in ((bufs, R * D), (scs, 2 * R)):
        assert all(not t[:offset].any() and not t[offset + n:].any() for t in b)


@pytest.mark.parametrize("R,D,dtype", [(900, 4096, torch.bfloat16), (5000, 72, torch.float16), (50, 1531, torch.float32)])
def test_same_results_every_time_and_nothing_behind_them_is_touched(R, D, dtype):
    x, r, w, gy, gs = make(R, D, dtype, seed=8)
    p = B.make_norm_params(R, D, dtype, torch.float32, 1e-6)
    first = None
    for fill in (0, 255):
        o = {"s": torch.full((R + 1, D), 7.0, device=DEV, dtype=dtype), "y": torch.full((R + 1, D), 7.0, device=DEV, dtype=dtype),
             "r": torch.full((R + 4,), 7.0, device=DEV), "gx": torch.full((R + 1, D), 7.0, device=DEV, dtype=dtype),
             "gw": torch.full((D + 4,), 7.0, device=DEV)}
        ws = torch.full((B.ppow_rms_norm_workspace_bytes(p),), fill, dtype=torch.uint8, device=DEV)
        B.ppow_rms_norm(p, x, r, w, o["s"][:R], o["y"][:R], o["r"][:R])
        B.ppow_rms_norm_backward(p, gy, gs, o["s"][:R], None, None, w, o["r"][:R], o["gx"][:R], o["gw"][:D], ws)
        torch.cuda.synchronize()
        for k, n in (("s", R), ("y", R), ("r", R), ("gx", R), ("gw", D)):
            assert torch.all(o[k][n:] == 7), k
        assert first is None or all(torch.equal(first[k], o[k]) for k in o)
        first = o


def test_no_rows_and_too_wide():
    x, r, w, gy, gs = make(3, 200, torch.bfloat16)
    out = B.rms_norm(x[:0], w, r[:0], checkpoint=True, packed_output=True)
    assert out["sum"].shape == (0, 200) and out["y_packed"].shape == (0, 200) and out["scale"].shape == (0, 2)
    gx, gw = B.rms_norm_backward(gy[:0], x[:0], w, out["rstd"], grad_sum=gs[:0])
    torch.cuda.synchronize()
    assert gx.shape == (0, 200) and not gw.any()
    with pytest.raises(B.PpowError) as e:
        B.rms_norm(torch.zeros((2, 16385), device=DEV), torch.zeros(16385, device=DEV))
    assert e.value.status == B.PPOW_ERR_UNSUPPORTED


def test_streams_and_replays():
    x, r, w, gy, gs = make(900, 1000, torch.bfloat16, seed=9)
    other = make(900, 1000, torch.bfloat16, seed=10)

    def step(x, r, gy, gs, **k):
        out = B.rms_norm(x, w, r, checkpoint=True, **k)
        return (*out.values(), *B.rms_norm_backward(gy, (out["packed"], out["scale"]), w, out["rstd"], grad_sum=gs, **k))

    def same(a, b):
        return all(torch.equal(p.view(torch.uint8), q.view(torch.uint8)) for p, q in zip(a, b))
    x2, r2, _, gy2, gs2 = other
    want, want2 = step(x, r, gy, gs), step(x2, r2, gy2, gs2)
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        a, c = step(x, r, gy, gs, stream=s1), step(x2, r2, gy2, gs2, stream=s2)
        torch.cuda.synchronize()
        assert same(a, want) and same(c, want2)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(x, r, gy, gs)
    for t, t2 in ((x, x2), (r, r2), (gy, gy2), (gs, gs2)):
        t.copy_(t2)
    for _ in range(2):
        graph.replay()
        torch.cuda.synchronize()
        assert same(got, want2)


@pytest.mark.parametrize("R,D", [(5, 96), (3, 1531)])
def test_gradient_against_differences_of_the_forward_pass(R, D):
    # float32, along a unit direction d of the row's space: the third derivative of y = w s / sqrt(mean s^2 + eps) times h^2/6 and
    # the forward pass's rounding over h bound the difference.  With t = |s| / sqrt(D) >= 1/2, derivatives of 1/t along d up to order three
    # stay below 15 (1/sqrt(D))^k times powers of 2, hence those of the loss below 15 max|gy w| sqrt(D) in all.
    _, _, w, gy, gs = make(R, D, torch.float32, seed=11)
    g = torch.Generator(device=DEV).manual_seed(12)
    s, r = torch.randn((R, D), generator=g, device=DEV), torch.randn((R, D), generator=g, device=DEV) * 2.0 ** -20
    d = torch.randn((R, D), generator=g, device=DEV)
    d = d / d.norm(dim=1, keepdim=True)
    h = 2.0 ** -5
    at = [s + k * h * d for k in (1, -1)]
    outs = [B.rms_norm(t, w, r) for t in at]
    step = outs[0]["sum"].double() - outs[1]["sum"].double()
    loss = [((o["y"].double() * gy.double()) + o["sum"].double() * gs.double()).sum(1) for o in outs]
    out = B.rms_norm(s, w, r)
    gx, _ = B.rms_norm_backward(gy, out["sum"], w, out["rstd"], grad_sum=gs)
    got, want = (gx.double() * step).sum(1), loss[0] - loss[1]
    a = (gy * w).double().abs()
    smooth = 2 * h ** 3 / 6 * 15 * a.amax(1) * D ** 0.5
    rounding = 2 * (gy.double().abs() * 256 * E * out["y"].double().abs()).sum(1)
    back = (step.abs() * 512 * E * (a + a.mean(1, keepdim=True) + gs.double().abs())).sum(1)
    assert torch.all((got - want).abs() <= smooth + rounding + back)
    # and not by being loose: without the mean, or without what passes the norm, the difference is far outside
    naive = (((gy * w).double() * out["rstd"].double()[:, None] + gs.double()) * step).sum(1)
    assert float((naive - want).abs().max()) > 4 * float((got - want).abs().max())


@pytest.mark.parametrize("R,D,dtype", [(1 << 20, 3, torch.float16), (1 << 20, 64, torch.bfloat16), (300000, 8192, torch.bfloat16)])
def test_many_rows(R, D, dtype):
    if R * D < 1 << 31:
        x, r, w, gy, gs = make(R, D, dtype, seed=13)
        out = B.rms_norm(x, w, r, checkpoint=True)
        got = B.rms_norm_backward(gy, (out["packed"], out["scale"]), w, out["rstd"], grad_sum=gs)
        torch.cuda.synchronize()
        check_forward(x, r, w, 1e-6, out)
        check_backward(gy, norm.reference_pack(out["sum"])[2], w, out["rstd"], gs, got)
        return
    # offsets pass 32 bits: a few rows are looked at, the others are zeros and leave the sums alone
    probe = [0, 1, R // 2, 262143, 262144, R - 1]
    xs, rs, w, gys, gss = make(len(probe), D, dtype, seed=14)
    x, r, gy = (torch.zeros((R, D), dtype=dtype, device=DEV) for _ in range(3))
    x[probe], r[probe], gy[probe] = xs, rs, gys
    out = B.rms_norm(x, w, r)
    gx, gw = B.rms_norm_backward(gy, out["sum"], w, out["rstd"])
    torch.cuda.synchronize()
    check_forward(xs, rs, w, 1e-6, {k: v[probe] for k, v in out.items()})
    check_backward(gys, out["sum"][probe].double(), w, out["rstd"][probe], None, (gx[probe], gw))
    assert not gx[2].any() and not out["y"][R - 2].any()
