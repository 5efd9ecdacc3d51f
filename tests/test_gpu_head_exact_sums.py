"""The sums behind the normaliser where every product is exact: rows of +-1 against entries that are multiples of 2^-8 of them, so that
logits near 60 are multiples of 1/4 and nothing is lost in the tensor cores.  The token shares the softmax with one other entry, and
the logarithm of its p is -log(1 + others / token): what rounding the others' large logits (in units of log 2, times log2(e) / T) would
do shows in it undamped.
  others   one exponential of a small difference (ex2.approx: 2^-22 relative), sums and products of a few roundings (4 * 2^-24):
           at most e = 2^-22 + 2^-22 of themselves; log p is off by (1 - p) e, and its own rounding is 2^-24 of it."""
import numpy as np
import pytest
import torch

from paper_2605_14978_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("temperature", [1.0, 0.7])
@pytest.mark.parametrize("T", [1, 8, 16, 31, 64, 128, 300])
def test_log_probability_between_two_large_logits(T, temperature, dtype):
    temperature, V, D = float(np.float32(temperature)), 1000, 64
    for seed in range(1 + 128 // T):
        g = torch.Generator(device=DEV).manual_seed(seed)
        h = (torch.randint(0, 2, (T, D), generator=g, device=DEV) * 2 - 1).to(dtype)
        w = torch.zeros((V, D), dtype=dtype, device=DEV)
        place = torch.randperm(V, generator=g, device=DEV)[:2 * T].view(2, T)
        q = torch.randint(200, 250, (T,), generator=g, device=DEV)
        near = torch.randint(-3, 4, (T,), generator=g, device=DEV)
        w[place[0]] = h * (q / 256)[:, None].to(dtype)
        w[place[1]] = h * ((q + near) / 256)[:, None].to(dtype)
        out = B.head_logprob(h, w, place[1].int().contiguous(), temperature=temperature)
        z = h.double() @ w.double().t() / temperature
        want = torch.log_softmax(z, 1).gather(1, place[1][:, None])[:, 0]
        tol = (1 - want.exp()) * 2.0 ** -21 + want.abs() * 2.0 ** -24
        off = (out["logp"].double() - want).abs()
        assert torch.all(off <= tol), float((off / tol).max())
