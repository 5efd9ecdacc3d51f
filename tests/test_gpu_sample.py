"""Tokens drawn with given uniforms, against the definition in float64: tokens and counts are equal, log-probabilities right to half a
step of float32 and 1e-12 (the error of the masses, 1e-13, and of the definition's own sums)."""
import math

import numpy as np
import pytest
import torch

from paper_2605_14978_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.bfloat16, torch.float16, torch.float32]
INF = math.inf


def reference(logits, uniforms, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """Row by row on the CPU, in numpy's float64."""
    tokens, logps, kept = [], [], []
    for z, u in zip(logits.cpu().double().numpy(), uniforms.cpu().numpy().astype(np.float64)):
        if np.isnan(z).any() or (z == INF).any() or (z == -INF).all():
            tokens.append(-1), logps.append(-INF if (z == -INF).all() else math.nan), kept.append(0)
            continue
        order = np.argsort(-z, kind="stable")
        order = order[z[order] > -INF]
        w = np.exp((z[order] - z[order[0]]) / temperature)
        n = min(top_k, len(order)) if top_k else len(order)
        C = np.cumsum(w)
        if top_p < 1.0:
            n = min(n, int(np.searchsorted(C[:n], top_p * C[n - 1], side="left")) + 1)
        if min_p > 0.0:
            n = min(n, int((w >= min_p).sum()))
        at = 0.0 if math.isnan(u) else min(max(u, 0.0), 1.0 - 2.0 ** -24)
        j = min(int(np.searchsorted(C[:n], at * C[n - 1], side="right")), n - 1)
        tokens.append(order[j]), kept.append(n)
        logps.append((z[order[j]] - z[order[0]]) / temperature - math.log(C[n - 1]))
    return np.array(tokens), np.array(logps), np.array(kept)


def check(logits, uniforms, got, **k):
    torch.cuda.synchronize()
    tokens, logps, kept = reference(logits, uniforms, **k)
    assert got["tokens"].dtype == got["kept"].dtype == torch.int32
    np.testing.assert_array_equal(got["kept"].cpu().numpy(), kept)
    np.testing.assert_array_equal(got["tokens"].cpu().numpy(), tokens)
    lp, ok = got["logp"].cpu().double().numpy(), np.isfinite(logps)
    np.testing.assert_array_equal(lp[~ok], logps[~ok])
    assert np.all(np.abs(lp[ok] - logps[ok]) <= 2.0 ** -24 * np.abs(logps[ok]) + 1e-12)


def make(R, V, dtype, seed=0, spread=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed * 7 + R * 31 + V)
    z = -torch.log(1.0 + torch.rand((R, V), generator=g, device=DEV) * (V - 1)) + torch.randn((R, V), generator=g, device=DEV) * spread
    return z.to(dtype), torch.rand(R, generator=g, device=DEV)


FILTERS = [dict(), dict(temperature=0.7, top_k=50), dict(top_p=0.9), dict(temperature=1.3, min_p=0.02), dict(top_k=1),
           dict(temperature=0.6, top_k=40, top_p=0.8, min_p=0.05), dict(top_k=1 << 22, top_p=0.999), dict(temperature=30.0, top_p=0.5),
           dict(temperature=0.01), dict(min_p=1.0), dict(top_p=1e-9), dict(top_k=3, top_p=0.99, min_p=1e-6)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("R,V", [(1, 1), (3, 2), (5, 7), (2, 129), (40, 1000), (9, 4099), (1, 8192), (7, 32000), (3, 128256), (1, 300001)])
def test_draws(R, V, dtype):
    z, u = make(R, V, dtype)
    for k in FILTERS:
        check(z, u, B.sample_tokens(z, u, **k), **k)


@pytest.mark.parametrize("dtype", TYPES)
def test_many_rows_and_a_row_alone(dtype):
    z, u = make(700, 5003, dtype, seed=1)
    for k in (dict(), dict(top_p=0.95), dict(temperature=0.7, top_k=20, min_p=0.01)):
        got = B.sample_tokens(z, u, **k)
        check(z, u, got, **k)
        for rows in ([0], [699], list(range(100, 110))):     # shared by up to eight CTAs: the same to the last bit
            few = B.sample_tokens(z[rows].contiguous(), u[rows].contiguous(), **k)
            assert all(torch.equal(few[n], got[n][rows]) for n in few)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [64, 5003, 70000])
def test_ties_go_to_the_lowest_index(V, dtype):
    g = torch.Generator(device=DEV).manual_seed(V)
    z = torch.randint(-3, 3, (24, V), generator=g, device=DEV).to(dtype)
    z[3], z[4] = 1.5, 0.0
    z[5] = torch.where(torch.rand(V, generator=g, device=DEV) < 0.5, 0.0, -0.0).to(dtype)       # one number
    z[6] = z[5]
    z[6, V // 2] = 1.0
    z[7] = -z[5] - 2 * (torch.arange(V, device=DEV) % 2).to(dtype)
    u = torch.rand(24, generator=g, device=DEV)
    u[3], u[4] = 0.5, 1.0 - 2.0 ** -24
    for k in (dict(), dict(top_k=V // 3 + 1), dict(top_p=0.75), dict(top_k=10, top_p=0.5), dict(top_p=0.25, temperature=2.0)):
        check(z, u, B.sample_tokens(z, u, **k), **k)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [9, 1000, 33001])
def test_masks_and_rows_without_a_distribution(V, dtype):
    z, u = make(16, V, dtype, seed=2)
    low = torch.finfo(dtype).min
    z[0] = -INF
    z[1, 1:] = -INF
    z[2, :-1] = -INF
    z[3, ::2] = -INF
    z[4, 1:] = low
    z[5, ::2] = low
    z[6] = low
    z[7, V // 2] = math.nan
    z[8, V - 1] = INF
    z[9, 0], z[9, 1] = math.nan, INF
    z[10] = -INF
    z[10, 3] = math.nan
    z[11, 2:] = -10000.0
    z[12] = -10000.0
    z[13, 1:] = -INF
    z[13, 0] = low
    z[14] = -INF
    z[14, V - 1], z[14, 4] = low, low / 2
    for k in (dict(), dict(top_k=5), dict(top_p=0.9), dict(min_p=0.1, temperature=0.5), dict(top_k=V, min_p=1e-30), dict(temperature=1000.0)):
        check(z, u, B.sample_tokens(z, u, **k), **k)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("R", [2, 12, 360])                  # several CTAs to a row, and one
def test_rows_that_counting_does_not_fit(R, dtype):
    # large logits, more than 65535 equal ones, few beside many, and ordinary rows among them
    V = 140001
    z, u = make(min(R, 12), V, dtype, seed=3)
    g = torch.Generator(device=DEV).manual_seed(4)
    z[0] = 0.25
    z[1] = z[1] + 5000.0
    if R > 2:
        z[5, :70000] = -1.0
        z[6] = torch.where(torch.rand(V, generator=g, device=DEV) < 0.9, -2.0, 3.0).to(dtype)
        z[7, 100] = 30000.0
        z[8] = z[8] * 4000.0
        z[9] = z[9].abs() * 1e-3 + 2050.0
        z[10, 1:] = -30000.0
        z[11] = (torch.rand(V, generator=g, device=DEV) * 1e-6).to(dtype)
    for k in (dict(), dict(top_k=69000, top_p=0.9), dict(temperature=500.0, top_p=0.7), dict(top_k=66000, min_p=1e-4)):
        if R <= 12:
            check(z, u, B.sample_tokens(z, u, **k), **k)
            continue
        got = B.sample_tokens(z.repeat(R // 12, 1), u.repeat(R // 12), **k)
        check(z, u, {n: t[:12] for n, t in got.items()}, **k)
        assert all(torch.equal(t.view(torch.int32).view(-1, 12), t[:12].view(torch.int32).expand(R // 12, 12)) for t in got.values())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tiny", [2.0 ** -50, 2.0 ** -51, 2.0 ** -52, 1e-17, 2.0 ** -63, 2.0 ** -64, 1e-30, 1e-39, 2.0 ** -24])
def test_logits_next_to_zero(tiny, dtype):
    # few logits near zero decide a row of otherwise deep ones, and order among themselves by sign and magnitude
    z, u = make(8, 3000, dtype, seed=13)
    z = (z - 30.0).to(dtype)
    for i in range(8):
        near = torch.tensor([tiny, -tiny, 0.0, -0.0, 2 * tiny, -3 * tiny, -0.5, 0.25][: i + 1], dtype=torch.float64, device=DEV)
        z[i, 17 * (i + 1):17 * (i + 1) + 7 * near.numel():7] = near.to(dtype)
    for k in (dict(), dict(top_k=3), dict(top_p=0.6), dict(min_p=0.9), dict(temperature=0.1, top_p=0.9)):
        check(z, u, B.sample_tokens(z, u, **k), **k)


@pytest.mark.parametrize("dtype", TYPES)
def test_uniforms_at_the_ends_and_outside(dtype):
    z, _ = make(12, 3001, dtype, seed=5)
    u = torch.tensor([0.0, 1.0 - 2.0 ** -24, 2.0 ** -149, 0.5, 1.0, 2.0, -1.0, math.nan, INF, -INF, -0.0, 2.0 ** -30], device=DEV)
    for k in (dict(), dict(top_k=7), dict(top_p=0.5), dict(min_p=0.2)):
        check(z, u, B.sample_tokens(z, u, **k), **k)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("offset,pad", [(1, 0), (3, 2), (8, 8), (0, 5), (5, 0)])
def test_rows_of_other_strides_and_alignments(offset, pad, dtype):
    R, V = 11, 4097
    z, u = make(R, V, dtype, seed=6)
    wide = torch.full((R, V + offset + pad), INF, dtype=dtype, device=DEV)       # what lies around the rows would show
    wide[:, offset:offset + V] = z
    for rows in (slice(None), slice(0, 1), slice(0, None, 3)):
        for k in (dict(), dict(top_p=0.8, top_k=900)):
            check(z[rows], u[rows].contiguous(), B.sample_tokens(wide[rows, offset:offset + V], u[rows].contiguous(), **k), **k)


def test_offsets_past_31_bits():
    R, V = 18000, 128256                                     # 2.3e9 logits
    z = torch.full((R, V), -INF, dtype=torch.bfloat16, device=DEV)
    probe = [0, 1, 16742, 16743, 16744, R - 1]
    few, _ = make(len(probe), V, torch.bfloat16, seed=7)
    z[probe] = few
    u = torch.rand(R, device=DEV, generator=torch.Generator(device=DEV).manual_seed(1))
    got = B.sample_tokens(z, u, top_p=0.9)
    torch.cuda.synchronize()
    check(few, u[probe], {k: v[probe] for k, v in got.items()}, top_p=0.9)
    rest = torch.ones(R, dtype=torch.bool, device=DEV)
    rest[probe] = False
    assert torch.all(got["tokens"][rest] == -1) and torch.all(got["logp"][rest] == -INF) and torch.all(got["kept"][rest] == 0)


@pytest.mark.parametrize("dtype", TYPES)
def test_outputs_are_left_alone_around_the_rows_and_kept_may_be_absent(dtype):
    z, u = make(5, 999, dtype, seed=8)
    t, l, k = torch.full((9,), 77, dtype=torch.int32, device=DEV), torch.full((9,), 77.0, device=DEV), torch.full((9,), 77, dtype=torch.int32, device=DEV)
    p = B.make_sample_params(z, top_p=0.9)
    B.ppow_sample_tokens(p, z, u, t[2:7], l[2:7], k[2:7])
    check(z, u, {"tokens": t[2:7], "logp": l[2:7], "kept": k[2:7]}, top_p=0.9)
    assert all(torch.all(a[[0, 1, 7, 8]] == 77) for a in (t, l, k))
    t2 = torch.zeros(5, dtype=torch.int32, device=DEV)
    B.ppow_sample_tokens(p, z, u, t2, l[2:7])
    torch.cuda.synchronize()
    assert torch.equal(t2, t[2:7])
    none = B.sample_tokens(z[:0], u[:0])
    assert none["tokens"].shape == (0,)
    with pytest.raises(B.PpowError) as e:
        B.sample_tokens(torch.zeros((1, (1 << 22) + 1), dtype=dtype, device=DEV), u[:1])
    assert e.value.status == B.PPOW_ERR_UNSUPPORTED


def test_the_largest_vocabulary():
    for dtype in (torch.float16, torch.float32):
        z, u = make(2, 1 << 22, dtype, seed=9)
        for k in (dict(), dict(top_k=100000, top_p=0.9)):
            check(z, u, B.sample_tokens(z, u, **k), **k)


@pytest.mark.parametrize("dtype", TYPES)
def test_streams_and_replays(dtype):
    z, u = make(6, 40000, dtype, seed=10)
    z2, u2 = make(6, 40000, dtype, seed=11)
    k = dict(temperature=0.8, top_p=0.95)
    want, want2 = B.sample_tokens(z, u, **k), B.sample_tokens(z2, u2, **k)
    check(z, u, want, **k)
    check(z2, u2, want2, **k)
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        a, b = B.sample_tokens(z, u, stream=s1, **k), B.sample_tokens(z2, u2, stream=s2, **k)
        torch.cuda.synchronize()
        assert all(torch.equal(a[n], want[n]) and torch.equal(b[n], want2[n]) for n in want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = B.sample_tokens(z, u, **k)
    z.copy_(z2), u.copy_(u2)
    for _ in range(2):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(got[n], want2[n]) for n in got)


def test_draws_follow_the_distribution():
    # 200000 uniforms at equal steps: each token's share is its probability to a step
    z, _ = make(1, 50, torch.bfloat16, seed=12)
    n = 200000
    u = (torch.arange(n, device=DEV).double() / n).float()
    got = B.sample_tokens(z.repeat(n, 1), u, temperature=0.9)
    torch.cuda.synchronize()
    p = torch.softmax(z[0].double() / 0.9, 0)
    share = torch.bincount(got["tokens"].long(), minlength=50).double() / n
    assert float((share - p).abs().max()) <= 1.5 / n
    assert torch.all((got["logp"].double() - p.log()[got["tokens"].long()]).abs() < 1e-6)
