"""Drawn tokens of 16-bit rows with logits at the limits of the range that is counted, beside every kind of neighbour, in either half of a word:
against the definition in float64, as in test_gpu_sample.py."""
import math

import pytest
import torch

from paper_2605_14978_b200 import binding as B

from test_gpu_sample import check

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
INF = math.inf
UNWRITTEN = 0x7a7a7a7a

# the limits, and the numbers next to them on either side
LIMITS = {torch.bfloat16: [8128.0, 8160.0, 8192.0, 8256.0, 2.0 ** -51 * (1 + 2.0 ** -7), 2.0 ** -51, 2.0 ** -51 * (1 - 2.0 ** -8), 2.0 ** -52],
          torch.float16: [2046.0, 2047.0, 2048.0, 2050.0, 2.0 ** -24]}
BESIDE = {torch.bfloat16: [0.0, -0.0, 2.0 ** -133, -2.0 ** -52, 2.0 ** -51, -8192.0, 1.0, -INF],
          torch.float16: [0.0, -0.0, 2.0 ** -24, -2.0 ** -14, -2048.0, 1.0, -INF]}


def draw(z, u, **k):
    R = u.numel()
    t = torch.full((R + 2,), UNWRITTEN, dtype=torch.int32, device=DEV)
    l, n = torch.full((R + 2,), 7.0, device=DEV), torch.full((R + 2,), UNWRITTEN, dtype=torch.int32, device=DEV)
    B.ppow_sample_tokens(B.make_sample_params(z, **k), z, u, t[1:-1], l[1:-1], n[1:-1])
    torch.cuda.synchronize()
    assert all(int(a[i]) == UNWRITTEN for a in (t, n) for i in (0, -1))
    return {"tokens": t[1:-1], "logp": l[1:-1], "kept": n[1:-1]}


def rows_of(V, dtype):
    """A row for each limit, sign, neighbour and half: the number with that neighbour on both sides, in the middle and near the end."""
    pairs = [(sign * a, b) for a in LIMITS[dtype] for sign in (1.0, -1.0) for b in BESIDE[dtype]]
    z = (-3.0 - (torch.arange(V, device=DEV) % 5).double()).repeat(2 * len(pairs), 1)
    for i, (a, b) in enumerate(pairs):
        for half in (0, 1):
            for at in (V // 4 * 2 + half, V // 4 * 4 - 6 + half):
                z[2 * i + half, at - 1:at + 2] = torch.tensor([b, a, b], dtype=torch.float64, device=DEV)
    return z.to(dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("V", [61, 70001])                   # one CTA to a row, and (28 rows at a time) eight
def test_limits_of_the_counted_range_beside_every_neighbour(V, offset, dtype):
    z = rows_of(V, dtype)
    R = z.shape[0]
    wide = torch.full((R, V + 3), INF, dtype=dtype, device=DEV)
    wide[:, offset:offset + V] = z
    g = torch.Generator(device=DEV).manual_seed(V + offset)
    u = torch.rand(R, generator=g, device=DEV)
    step = R if V < 1000 else 28
    for k in (dict(), dict(temperature=3000.0, top_p=0.9), dict(min_p=0.04, top_k=V // 2)) if V < 1000 else (dict(temperature=2.0, top_p=0.95),):
        for at in (u, torch.zeros_like(u), torch.full_like(u, 1.0 - 2.0 ** -24)) if V < 1000 else (u,):
            for i in range(0, R, step):
                rows = slice(i, i + step)
                check(z[rows], at[rows], draw(wide[rows, offset:offset + V], at[rows], **k), **k)


def test_forbidden_tokens_of_minus_8192_beside_zeros():
    # every other token forbidden by the lowest number outside the range: half of the row was given the weight of a zero
    z = torch.zeros((64, 1000), dtype=torch.bfloat16, device=DEV)
    z[:, 1::2] = -8192.0
    u = torch.linspace(0.0, 1.0 - 2.0 ** -24, 64, device=DEV)
    for k in (dict(), dict(top_p=0.5), dict(top_k=700), dict(min_p=0.5)):
        got = draw(z, u, **k)
        check(z, u, got, **k)
        assert not (got["tokens"] % 2).any()
