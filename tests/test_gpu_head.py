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


# ------------------------------------------------------------------ masks, strides, ends of the ranges


def test_masked_rows_may_hold_anything_and_get_zeros():
    h, w, tok, grad = make(300, 1500, 200, torch.bfloat16, seed=2, masked=0.0)
    clean = h.clone()
    dead = torch.zeros(300, dtype=torch.bool, device=DEV)
    dead[::3] = True
    dead[256:290] = True
    tok[dead] = torch.where(torch.arange(int(dead.sum()), device=DEV) % 2 == 0, -1, -2 ** 31).int()
    h[dead] = torch.tensor([float("nan"), float("inf"), -float("inf")], device=DEV).repeat(67).to(h.dtype)[:200]
    grad[dead] = float("nan")
    clean[dead] = 0
    out, gh, gw = run(h, w, tok, grad)
    check_forward(clean, w, tok, 1.0, out)
    grad[dead] = 1.0
    check_backward(clean, w, tok, out["lse"], grad, 1.0, gh, gw)


def test_rows_without_gradient_are_masked_in_the_backward_pass():
    h, w, tok, grad = make(70, 900, 72, torch.float16, seed=3, masked=0.0)
    out = B.head_logprob(h, w, tok)
    grad[5:40] = 0.0
    grad[41] = -0.0
    clean = h.clone()
    h[5:40] = float("nan")
    gh, gw = B.head_logprob_backward(h, w, tok, out["lse"], grad)
    torch.cuda.synchronize()
    check_backward(clean, w, tok, out["lse"], grad, 1.0, gh, gw)


@pytest.mark.parametrize("T", [1, 16, 100, 300, 1000])
def test_all_rows_masked(T):
    h, w, tok, grad = make(T, 600, 64, torch.bfloat16, masked=0.0)
    tok.fill_(-1)
    h.fill_(float("nan"))
    out, gh, gw = run(h, w, tok, grad)
    assert not out["logp"].any() and not out["lse"].any() and not gh.any() and not gw.any()


def test_no_tokens():
    h, w, tok, grad = make(4, 600, 64, torch.bfloat16)
    out, gh, gw = run(h[:0], w, tok[:0], grad[:0])
    assert out["logp"].shape == (0,) and gh.shape == (0, 64) and not gw.any()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T", [40, 400])
@pytest.mark.parametrize("offset,pad", [(1, 3), (8, 8), (0, 1)])
def test_rows_of_other_strides_and_alignments(T, offset, pad, dtype):
    h, w, tok, grad = make(T, 1000, 136, dtype, seed=4)
    wide = torch.full((T, 136 + offset + pad), float("nan"), dtype=dtype, device=DEV)
    hv = wide[:, offset:offset + 136]
    hv.copy_(h)
    ww = torch.full((1000, 136 + 24), float("nan"), dtype=dtype, device=DEV)
    wv = ww[:, 8:144]
    wv.copy_(w)
    a, b = run(h, w, tok, grad), run(hv, wv, tok, grad)
    assert torch.equal(a[0]["logp"], b[0]["logp"]) and torch.equal(a[0]["lse"], b[0]["lse"])
    assert torch.equal(a[1], b[1]) and torch.equal(a[2], b[2])


@pytest.mark.parametrize("T", [20, 500])
def test_tokens_behind_the_vocabulary_are_reported(T):
    h, w, tok, grad = make(T, 777, 64, torch.bfloat16, seed=5, masked=0.0)
    tok[3], tok[11] = 777, 2 ** 31 - 1
    p = B.make_head_params(h, w)
    for backward in (False, True):
        ws = B.alloc_workspace(B.ppow_head_workspace_bytes(p, backward), DEV)
        if not backward:
            logp, lse = torch.empty(T, device=DEV), torch.empty(T, device=DEV)
            B.ppow_head_logprob(p, h, w, tok, logp, lse, ws)
        else:
            gh, gw = torch.empty_like(h), torch.empty_like(w)
            B.ppow_head_logprob_backward(p, h, w, tok, lse, grad, gh, gw, ws)
        assert B.ppow_read_error_flags(ws) == B.PPOW_FLAG_TOKEN_RANGE
    check_forward(h, w, tok, 1.0, {"logp": logp, "lse": lse})
    assert not gh[3].any() and not gh[11].any()
    check_backward(h, w, tok, lse, grad, 1.0, gh, gw)
    tok[3] = tok[11] = 0
    ws.fill_(255)                                             # whatever the workspace held before
    B.ppow_head_logprob_backward(p, h, w, tok, lse, grad, gh, gw, ws)
    assert B.ppow_read_error_flags(ws) == 0


@pytest.mark.parametrize("T", [90, 300])
def test_either_gradient_alone(T):
    h, w, tok, grad = make(T, 1100, 264, torch.bfloat16, seed=6)
    out, gh, gw = run(h, w, tok, grad)
    only_h = B.head_logprob_backward(h, w, tok, out["lse"], grad, want_weight=False)
    only_w = B.head_logprob_backward(h, w, tok, out["lse"], grad, want_hidden=False)
    torch.cuda.synchronize()
    assert only_h[1] is None and only_w[0] is None
    assert torch.equal(only_h[0], gh) and torch.equal(only_w[1], gw)


def test_gradients_of_very_different_rows_in_half_precision():
    h, w, tok, grad = make(200, 1000, 64, torch.float16, seed=7, masked=0.0)
    grad *= torch.logspace(-9, 3, 200, device=DEV)
    out, gh, gw = run(h, w, tok, grad)
    check_backward(h, w, tok, out["lse"], grad, 1.0, gh, gw)


def test_several_pieces_of_the_vocabulary():
    # 2304 rows of dz over 128256 entries are 591 MB: two pieces, the second shorter, sums of grad_hidden carried over
    h, w, tok, grad = make(2304, 128256, 64, torch.bfloat16, seed=8)
    out, gh, gw = run(h, w, tok, grad)
    check_forward(h, w, tok, 1.0, out)
    check_backward(h, w, tok, out["lse"], grad, 1.0, gh, gw)


def test_results_do_not_depend_on_the_run_and_nothing_behind_them_is_touched():
    for T, dtype in ((50, torch.float16), (700, torch.bfloat16)):
        h, w, tok, grad = make(T, 2000, 328, dtype, seed=9)
        p = B.make_head_params(h, w, 0.9)
        first = None
        for fill in (0.0, float("nan")):
            bufs = {"logp": torch.full((T + 8,), 7.0, device=DEV), "lse": torch.full((T + 8,), 7.0, device=DEV),
                    "gh": torch.full((T + 2, 328), 7.0, device=DEV, dtype=dtype), "gw": torch.full((2002, 328), 7.0, device=DEV, dtype=dtype)}
            ws = [B.alloc_workspace(B.ppow_head_workspace_bytes(p, b), DEV) for b in (False, True)]
            for x in ws:
                x.view(torch.float32)[:].fill_(fill) if x.numel() % 4 == 0 else x.fill_(255)
            B.ppow_head_logprob(p, h, w, tok, bufs["logp"][:T], bufs["lse"][:T], ws[0])
            B.ppow_head_logprob_backward(p, h, w, tok, bufs["lse"][:T], grad, bufs["gh"][:T], bufs["gw"][:2000], ws[1])
            torch.cuda.synchronize()
            assert torch.all(bufs["logp"][T:] == 7) and torch.all(bufs["lse"][T:] == 7)
            assert torch.all(bufs["gh"][T:] == 7) and torch.all(bufs["gw"][2000:] == 7)
            if first is not None:
                assert all(torch.equal(first[k], bufs[k]) for k in bufs)
            first = bufs


def test_two_streams_at_once_and_a_stream_that_is_not_current():
    cases = [make(T, 3001, 256, torch.bfloat16, seed=10 + T) for T in (33, 600)]
    want = [run(*c) for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(3):
        got = []
        for (h, w, tok, grad), s in zip(cases, streams):
            out = B.head_logprob(h, w, tok, stream=s)
            got.append((out, *B.head_logprob_backward(h, w, tok, out["lse"], grad, stream=s)))
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert torch.equal(a[0]["logp"], b[0]["logp"]) and torch.equal(a[1], b[1]) and torch.equal(a[2], b[2])


@pytest.mark.parametrize("T", [60, 700])
def test_captured_and_replayed_on_new_inputs(T):
    h, w, tok, grad = make(T, 2500, 136, torch.bfloat16, seed=11)
    h2, w2, tok2, grad2 = make(T, 2500, 136, torch.bfloat16, seed=12, masked=0.6)
    want = run(h2, w2, tok2, grad2)
    run(h, w, tok, grad)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = B.head_logprob(h, w, tok)
        gh, gw = B.head_logprob_backward(h, w, tok, out["lse"], grad)
    for a, b in ((h, h2), (w, w2), (tok, tok2), (grad, grad2)):
        a.copy_(b)
    for _ in range(2):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out["logp"], want[0]["logp"]) and torch.equal(gh, want[1]) and torch.equal(gw, want[2])


@pytest.mark.parametrize("T", [12, 300])
def test_gradient_against_differences_of_the_forward_pass(T):
    # hidden states on a grid of 2^-6, moved by one step along u in {-1, 1}^D: exact in float16.  Along u the logits are linear,
    # with slopes a = W u; the third derivative of lse is their third cumulant, at most (max a - min a)^3 in magnitude.
    g = torch.Generator(device=DEV).manual_seed(13)
    V, D, step = 300, 64, 2.0 ** -6
    h = (torch.randint(-64, 65, (T, D), generator=g, device=DEV) * step).half()
    w = (torch.randn((V, D), generator=g, device=DEV) * 0.1).half()
    tok = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    grad = torch.randn(T, generator=g, device=DEV)
    u = (torch.randint(0, 2, (T, D), generator=g, device=DEV) * 2 - 1).half()
    logp = [B.head_logprob(h + s * step * u, w, tok)["logp"].double() for s in (1, -1)]
    out, gh, _ = run(h, w, tok, grad)
    got = (gh.double() * u.double()).sum(1)
    want = grad.double() * (logp[0] - logp[1]) / (2 * step)
    a = u.double() @ w.double().t()
    spread = a.amax(1) - a.amin(1)
    err = logits(h, w, 1.0)[1].amax(1) * 2 + 2.0 ** -19 + out["lse"].double().abs() * 2.0 ** -21
    tol = grad.double().abs() * (step ** 2 / 6 * spread ** 3 + err / step)
    dh, th, _, _ = gradient(h, w, tok, out["lse"], grad, 1.0)
    assert torch.all((got - want).abs() <= tol + th.sum(1))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T", [1, 2, 5, 22, 32])
def test_few_tokens_lose_no_more_than_the_rounding_of_the_results(T, dtype):
    # One rounding of values v is off by at most half a step; uniform within it, the error's root mean square is a step / sqrt(12)
    # = 2u / sqrt(12) = 0.577 u of the power of two below v, so of v at most.  dz is rounded too, but its largest terms are made
    # good and the others average out: 0.62 u.  With dz rounded and left at that a call of one token is off by up to u.
    u = U[dtype]
    for seed in range(6):
        h, w, tok, grad = make(T, 4001, 200, dtype, seed=30 + seed, masked=0.0)
        out, gh, gw = run(h, w, tok, grad)
        dh, _, dw, _ = gradient(h, w, tok, out["lse"], grad, 1.0)
        assert float((gh.double() - dh).norm() / dh.norm()) < 0.62 * u
        assert float((gw.double() - dw).norm() / dw.norm()) < 0.62 * u


def test_a_single_confident_token_keeps_its_log_probability():
    # logp close to 0 is a difference of two numbers near 20: what the sums cut off would show
    for seed in range(8):
        h, w, tok, _ = make(1, 1000, 4096, torch.bfloat16, seed=60 + seed, masked=0.0)
        out = B.head_logprob(h, w, tok, temperature=0.7)
        z = h.double() @ w.double().t() / 0.7
        lse = torch.logsumexp(z, 1)
        # 16 partial sums of 16 additions of 16 products, each off by at most a step 2^-23 of |z| <= 64, and their sum
        assert float((out["lse"].double() - lse).abs()) < (16 + 16) * 2.0 ** -23 * 64
        want = z[0, int(tok[0])] - lse[0]
        assert float((out["logp"][0].double() - want).abs()) < 2 * (16 + 16) * 2.0 ** -23 * 64


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T", [2, 16, 31, 64, 100, 128])
def test_few_tokens_where_they_lie_and_gathered(T, dtype):
    # on 16-byte boundaries the forward pass reads a few rows in place, masked ones among them, whatever they hold; off them it
    # gathers the live ones: the same numbers either way
    h, w, tok, grad = make(T, 5000, 264, dtype, seed=90 + T, masked=0.0)
    tok[::2] = -1
    tok[1] = 5000 if T > 2 else tok[1]
    clean = h.clone()
    clean[::2] = 0
    junk = torch.tensor([float("nan"), float("inf"), -float("inf"), 3e4], device=DEV).to(dtype)
    h[::2] = junk.repeat(66)
    p = B.make_head_params(h, w)
    got = []
    for hidden in (h, torch.nn.functional.pad(h, (1, 1))[:, 1:265]):
        ws = B.alloc_workspace(B.ppow_head_workspace_bytes(p, False), DEV)
        ws.fill_(255)
        logp, lse = torch.full((T + 4,), 7.0, device=DEV), torch.full((T + 4,), 7.0, device=DEV)
        B.ppow_head_logprob(p, hidden, w, tok, logp[:T], lse[:T], ws)
        assert B.ppow_read_error_flags(ws) == (B.PPOW_FLAG_TOKEN_RANGE if T > 2 else 0)
        check_forward(clean, w, tok, 1.0, {"logp": logp[:T], "lse": lse[:T]})
        assert torch.all(logp[T:] == 7) and torch.all(lse[T:] == 7)
        got.append((logp, lse))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])


@pytest.mark.parametrize("T,V,D", [(1, 1 << 22, 8), (70000, 300, 8), (1 << 20, 2, 8), (5, 300, 1 << 16), (300, 290, 1 << 16), (140, 70000, 16)])
def test_ends_of_the_ranges(T, V, D):
    h, w, tok, grad = make(T, V, D, torch.bfloat16, seed=40, masked=0.1 if T > 5 else 0.0)
    out, gh, gw = run(h, w, tok, grad)
    check_forward(h, w, tok, 1.0, out)
    check_backward(h, w, tok, out["lse"], grad, 1.0, gh, gw)
    torch.cuda.empty_cache()
