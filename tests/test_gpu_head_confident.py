"""Gradients at tokens that the drafter is nearly sure of: dz = g/T (1 - p) is a small difference, and an error d of the token's
logarithm of p appears in it as d / (1 - p).

The error of a row of grad_hidden has three parts that have nothing to do with one another:
  r   the rounding of the result, known exactly from the reference;
  o   the roundings of dz at the other entries: u |dz| / sqrt(3) in the root mean square, each times |w_v|;
  z   the error d of the token's product, times g p |w_y|.  The product of hidden state and weight is summed in float32 over the 8
      products of a 16-byte unit and in float64 from there on.  Up to 8 roundings of at most 2^-24 s, s the sum of the unit's
      magnitudes, uniform within that: sqrt(8/3) 2^-24 s, and d = sqrt(8/3) 2^-24 sqrt(sum of s^2 over the units) / T.
      Temperature and difference are float64; the result is rounded to float32, 2^-24 of itself.
Over the rows of a band of p their root mean square is held to the sum of squares, with 10 % for the scatter of a hundred rows and more.
A product summed in the tensor cores over 4096 of width is off by 3e-6 or so: 3 % of the gradient where p is 0.9999."""
import numpy as np
import pytest
import torch

from paper_2605_14978_b200 import binding as B

import test_gpu_head as head

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("temperature", [1.0, 0.7])
@pytest.mark.parametrize("T,V,D", [(512, 1000, 4096), (128, 1000, 4096), (300, 2000, 2056)])
def test_gradient_of_confident_tokens(T, V, D, temperature, dtype):
    temperature = float(np.float32(temperature))              # the type that the call takes: 0.7 itself is 2e-8 of z away
    sums = {}
    for seed in range(3 if T >= 300 else 8):
        g = torch.Generator(device=DEV).manual_seed(900 + seed)
        w = (torch.randn((V, D), generator=g, device=DEV) * (2.5 / D ** 0.5)).to(dtype)
        tok = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
        lift = (1.6 + 1.2 * torch.rand((T, 1), generator=g, device=DEV)) * temperature
        h = (0.2 * torch.randn((T, D), generator=g, device=DEV) + lift * w[tok.long()].float()).to(dtype)
        grad = torch.randn(T, generator=g, device=DEV)
        lse = B.head_logprob(h, w, tok, temperature=temperature)["lse"]
        gh, _ = B.head_logprob_backward(h, w, tok, lse, grad, temperature=temperature, want_weight=False)
        x, wd, y = h.double(), w.double(), tok.long()
        q = torch.exp(x @ wd.t() / temperature - lse.double()[:, None])
        p = q.gather(1, y[:, None])[:, 0]
        dz = -q
        dz.scatter_(1, y[:, None], -torch.expm1((x * wd[y]).sum(1) / temperature - lse.double())[:, None])
        k = grad.double()[:, None] / temperature
        want = k * (dz @ wd)
        r = (want.to(dtype).double() - want).square().sum(1)
        others = dz.scatter(1, y[:, None], 0.0)
        o = head.U[dtype] ** 2 / 3 * (k * others).square() @ wd.square().sum(1)
        s = torch.nn.functional.pad((x * wd[y]).abs(), (0, -D % 8)).view(T, -1, 8).sum(2)
        d = (8 / 3) ** 0.5 * 2.0 ** -24 * s.square().sum(1).sqrt() / temperature
        z = (k[:, 0] * p * d).square() * wd[y].square().sum(1)
        size = want.square().sum(1)
        off = (gh.double() - want).square().sum(1)
        for lo, hi in ((0.9, 0.99), (0.99, 0.999), (0.999, 0.9999), (0.9999, 0.999999)):
            m = (p >= lo) & (p < hi)
            a = sums.setdefault(lo, [0, 0.0, 0.0])
            a[0] += int(m.sum())
            a[1] += float((off / size)[m].sum())
            a[2] += float(((r + o + z) / size)[m].sum())
    assert sum(a[0] >= 100 for a in sums.values()) >= 3, sums
    for lo, (n, got, bound) in sums.items():
        if n >= 100:
            assert got <= 1.1 ** 2 * bound, (lo, n, (got / n) ** 0.5, (bound / n) ** 0.5)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("temperature", [1.0, 0.7])
@pytest.mark.parametrize("T", [512, 128, 8])
def test_normaliser_and_log_probability_of_confident_tokens(T, temperature, dtype):
    temperature = float(np.float32(temperature))
    # Where p >= 0.9999 the normaliser is the token's logit but for 1e-4 and less: its error is d as above, the rounding to float32
    # (at most 2^-24 of itself, uniform), and 1e-4 of the others' error, at most the bound of test_gpu_head: 1e-4 * 6e-3.  The
    # logarithm of p is the others' share, right to their relative error, and d / (1 - p): all in all within 1 % of itself.
    V, D, n, got, bound, worst = 1000, 4096, 0, 0.0, 0.0, 0.0
    for seed in range(2048 // T if T < 512 else 3):
        g = torch.Generator(device=DEV).manual_seed(950 + seed)
        w = (torch.randn((V, D), generator=g, device=DEV) * (2.5 / D ** 0.5)).to(dtype)
        tok = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
        lift = (2.5 + 0.8 * torch.rand((T, 1), generator=g, device=DEV)) * temperature
        h = (0.2 * torch.randn((T, D), generator=g, device=DEV) + lift * w[tok.long()].float()).to(dtype)
        out = B.head_logprob(h, w, tok, temperature=temperature)
        x, wd, y = h.double(), w.double(), tok.long()
        z = x @ wd.t() / temperature
        lse = torch.logsumexp(z, 1)
        others = torch.logsumexp(z.scatter(1, y[:, None], -float("inf")), 1)
        want = -torch.log1p(torch.exp(others - (x * wd[y]).sum(1) / temperature))
        m = want > -1e-4
        s = (x * wd[y]).abs().view(T, -1, 8).sum(2)
        d = (8 / 3) ** 0.5 * 2.0 ** -24 * s.square().sum(1).sqrt() / temperature
        n += int(m.sum())
        got += float((out["lse"].double() - lse)[m].square().sum())
        bound += float((d.square() + (2.0 ** -24 * lse).square() / 3 + 6e-7 ** 2)[m].sum())
        worst = max([worst] + ((out["logp"].double() - want).abs() / want.abs())[m].tolist())
    assert n >= 100 and got <= 1.1 ** 2 * bound, (n, (got / n) ** 0.5, (bound / n) ** 0.5)
    assert worst < 0.01
