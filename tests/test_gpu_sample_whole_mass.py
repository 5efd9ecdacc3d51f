"""Filters that leave all of the mass but a rounding of it: top_p next below 1, where the border lies behind the last element that counts."""
import numpy as np
import pytest
import torch

from paper_2605_14978_b200 import binding as B

from test_gpu_sample import TYPES

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NEXT_TO_1 = [1.0 - k * 2.0 ** -53 for k in (1, 2, 3, 6, 40)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("R,V", [(900, 100), (900, 3000), (300, 20000), (4, 70001)])       # sorted, counted or searched; the last one shared
def test_top_p_next_below_one(R, V, dtype):
    g = torch.Generator(device=DEV).manual_seed(V)
    spread = torch.tensor([0.25, 1.0, 3.0, 12.0], device=DEV).repeat(R // 4)[:, None]
    z = (torch.randn((R, V), generator=g, device=DEV) * spread).to(dtype)
    z[2::8, V // 3:] = -float("inf")
    z[5::8, 1::2] = torch.finfo(dtype).min                   # elements without mass behind the last one with some
    u = torch.rand(R, generator=g, device=DEV)
    full = B.sample_tokens(z, u)
    w = np.exp(z.double().cpu().numpy() - z.double().max(1, keepdim=True).values.cpu().numpy())
    tail = np.cumsum(np.sort(w, 1), 1)                       # the mass of so many of the smallest
    for p in NEXT_TO_1:
        got = B.sample_tokens(z, u, top_p=p)
        torch.cuda.synchronize()
        # what is left out is 1e-13 of the mass at most, and a draw (u <= 1 - 2^-24) is not among it
        assert torch.equal(got["tokens"], full["tokens"]), p
        assert torch.all((got["logp"] - full["logp"]).abs() <= 2.0 ** -23 * full["logp"].abs() + 1e-12), p
        kept, n = got["kept"].cpu().numpy(), full["kept"].cpu().numpy()
        assert np.all((kept >= 1) & (kept <= n))
        out = V - kept                                       # left out, with the -inf
        gone = np.where(out > 0, np.take_along_axis(tail, np.maximum(out - 1, 0)[:, None], 1)[:, 0], 0.0)
        assert np.all(gone <= 1e-13 * tail[:, -1]), p
    assert int(full["tokens"].min()) >= 0
