"""The global norm of gradients and clipping, against the definition in float64.

E = 2^-24, half a step of float32.  A square is rounded once, at most 32 additions follow in float32 (then float64): the sum of
squares is off by 36 E at most, its root by 18 E, the returned norm by 19 E.  The factor adds its own rounding and the product one
more: 22 E, then half a step of the type.
"""
import pytest
import torch

from paper_2605_14978_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
E = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -149}
TYPES = [torch.bfloat16, torch.float16, torch.float32]


def make(shapes, dtypes, scale=0.01, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return [(scale * torch.randn(s, generator=g, device=DEV)).to(dtypes[i % len(dtypes)]) for i, s in enumerate(shapes)]


def exact_norm(grads):
    return torch.stack([t.double().square().sum() for t in grads]).sum().sqrt()


def check(grads, max_norm, norm, out):
    want = exact_norm(grads)
    assert norm.shape == () and abs(float(norm) - float(want)) <= 19 * E * float(want) + 2.0 ** -150
    factor = min(1.0, max_norm / float(want)) if float(want) > 0 else 1.0
    for g, o in zip(grads, out):
        if float(want) <= max_norm * (1 - 20 * E):
            assert torch.equal(g, o)
            continue
        y = g.double() * factor
        assert torch.all((o.double() - y).abs() <= (22 * E * (1 + HALF[g.dtype]) + HALF[g.dtype]) * y.abs() + TINY[g.dtype])


SHAPES = [[(1,)], [(3,)], [(7, 5)], [(4096,)], [(1000003,)], [(64, 64), (64,), (300, 64)], [(2048, 1024)] * 4 + [(1024,)] * 9,
          [(i % 37 + 1, 129) for i in range(49)], [(i % 5 * 17,) for i in range(1500)], [(3, 0), (), (8, 2, 5)], [(0,)]]


@pytest.mark.parametrize("dtypes", [[t] for t in TYPES] + [TYPES])
@pytest.mark.parametrize("shapes", SHAPES)
def test_clipped_and_kept(shapes, dtypes):
    grads = make(shapes, dtypes, seed=len(shapes))
    norm = float(exact_norm(grads))
    for max_norm in (0.3 * norm, 1.5 * norm, 0.0):
        out = [torch.full_like(t, 7.0) for t in grads]
        got = B.clip_gradients(grads, max_norm, out=out)
        placed = [t.clone() for t in grads]
        again = B.clip_gradients(placed, max_norm)
        alone = B.gradient_norm(grads)
        torch.cuda.synchronize()
        check(grads, max_norm, got, out)
        assert torch.equal(got, again) and torch.equal(got, alone) and all(torch.equal(a, b) for a, b in zip(out, placed))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("start", [0, 1, 2, 3, 7])
def test_tensors_at_any_address_leave_their_neighbours_alone(start, dtype):
    sizes = [1, 2, 5, 17, 4095, 8, 33000, 3, 16384]
    flat = make([(sum(sizes) + 16,)], [dtype], seed=start)[0]
    grads, at = [], start
    for n in sizes:
        grads.append(flat[at:at + n])
        at += n
    for shift in (0, 1):                                     # outputs aligned as the gradients are, and otherwise
        buf = torch.full((flat.numel() + 1,), 7.0, dtype=dtype, device=DEV)
        out = [buf[g.storage_offset() + shift:g.storage_offset() + shift + g.numel()] for g in grads]
        norm = B.clip_gradients(grads, 0.5, out=out)
        torch.cuda.synchronize()
        check(grads, 0.5, norm, out)
        assert torch.all(buf[:start + shift] == 7) and torch.all(buf[at + shift:] == 7)
    before = flat.clone()
    mid = grads[3:6]
    B.clip_gradients(mid, 1e-3)
    torch.cuda.synchronize()
    lo, hi = mid[0].storage_offset(), mid[-1].storage_offset() + mid[-1].numel()
    assert torch.equal(flat[:lo], before[:lo]) and torch.equal(flat[hi:], before[hi:]) and not torch.equal(flat[lo:hi], before[lo:hi])


def test_dense_tensors_of_any_order():
    g = torch.Generator(device=DEV).manual_seed(3)
    a, b, c = (torch.randn(s, generator=g, device=DEV) for s in ((40, 60), (4, 5, 6), (2, 3, 4, 5)))
    grads = [a.t(), b.permute(2, 0, 1), c.contiguous(memory_format=torch.channels_last), torch.randn((7, 1, 3), generator=g, device=DEV)[:, :1]]
    out = [torch.empty_like(t) for t in grads]
    norm = B.clip_gradients(grads, 1.0, out=out)
    torch.cuda.synchronize()
    check(grads, 1.0, norm, out)
    for wrong in (a[:, ::2], a[:, :30], a[:1].expand(40, 60), a.double()):
        with pytest.raises(ValueError, match="dense"):
            B.clip_gradients([b, wrong], 1.0)
    for o in (a, a.t().contiguous(), a.t().half(), a.t()[:, :20]):
        with pytest.raises(ValueError, match="like its gradient"):
            B.clip_gradients([a.t()], 1.0, out=[o])


@pytest.mark.parametrize("dtype,scale", [(torch.float32, 1e-30), (torch.float32, 1e-42), (torch.float32, 1e25), (torch.bfloat16, 1e-33),
                                         (torch.bfloat16, 1e30), (torch.float16, 1e-7), (torch.float16, 3e4)])
def test_magnitudes_whose_squares_float32_does_not_hold(dtype, scale):
    g = torch.Generator(device=DEV).manual_seed(5)
    grads = [(torch.rand((n,), generator=g, device=DEV).double() * scale).to(dtype) for n in (5, 70000, 999)]
    grads.append(torch.zeros(100000, dtype=dtype, device=DEV))
    norm = float(exact_norm(grads))
    out = [torch.empty_like(t) for t in grads]
    got = B.clip_gradients(grads, 0.01 * norm, out=out)
    torch.cuda.synchronize()
    check(grads, 0.01 * norm, got, out)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("max_norm", [1e-5, 1e-20, 1e-30, 1e-37, 1e-42])
def test_factors_that_float32_does_not_hold(max_norm, dtype):
    # the factor lies far below 2^-126, the clipped gradients are ordinary numbers (of the last two, small ones)
    g = torch.Generator(device=DEV).manual_seed(8)
    grads = [(torch.randn((n,), generator=g, device=DEV).double() * 1e35).to(dtype) for n in (5, 70000, 999)]
    grads.append((torch.randn((5000,), generator=g, device=DEV).double() * 1e-3).to(dtype))          # nothing is left of these
    out = [torch.empty_like(t) for t in grads]
    got = B.clip_gradients(grads, max_norm, out=out)
    torch.cuda.synchronize()
    check(grads, max_norm, got, out)


def test_zeros_infinities_and_nan():
    grads = [torch.zeros(1000, device=DEV, dtype=torch.bfloat16), torch.zeros(3, device=DEV)]
    assert float(B.clip_gradients(grads, 0.0)) == 0.0 and not grads[0].any()
    grads = make([(100,), (5000,)], [torch.float32])
    grads[1][77] = float("inf")
    norm = B.clip_gradients(grads, 1.0)
    torch.cuda.synchronize()
    assert float(norm) == float("inf") and not grads[0].any() and grads[1][77].isnan() and not grads[1][:77].any()
    grads = make([(100,), (5000,)], [torch.float16])
    grads[0][5] = float("nan")
    norm = B.clip_gradients(grads, 1.0)
    torch.cuda.synchronize()
    assert norm.isnan() and all(t.isnan().all() for t in grads)


def test_overlaps_are_refused_and_repeats_count():
    flat = make([(10000,)], [torch.float32])[0]
    a, b, c = flat[:4000], flat[4000:8000], flat[3999:5000]
    for grads, out in (([a, a], None), ([a, c], None), ([a, b], [a, a]), ([a, b], [b, a]), ([a, b], [flat[1:4001], flat[6000:]]), ([a, c], [a, c])):
        with pytest.raises(B.PpowError) as e:
            B.clip_gradients(grads, 1.0, out=out)
        assert e.value.status == B.PPOW_ERR_INVALID_ARG
    out = [torch.empty_like(a), torch.empty_like(a), torch.empty_like(c)]
    norm = B.clip_gradients([a, a, c], 0.1, out=out)         # read more than once, into places of their own
    torch.cuda.synchronize()
    check([a, a, c], 0.1, norm, out)
    keep = flat.clone()
    norm = B.clip_gradients([a, b], 0.1, out=[a, torch.empty_like(b)])
    torch.cuda.synchronize()
    assert torch.equal(flat[4000:], keep[4000:]) and not torch.equal(flat[:4000], keep[:4000])


def test_streams_replays_and_order():
    grads = make([(513, 700), (31,), (1 << 20,), (9, 9)], TYPES, seed=6)
    other = make([(513, 700), (31,), (1 << 20,), (9, 9)], TYPES, seed=7)
    outs = [[torch.empty_like(t) for t in grads] for _ in range(4)]
    want = [B.clip_gradients(g, 1.0, out=o) for g, o in ((grads, outs[0]), (other, outs[1]))]
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        got = [B.clip_gradients(g, 1.0, out=o, stream=s) for g, o, s in ((grads, outs[2], s1), (other, outs[3], s2))]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert all(torch.equal(a, b) for k in (0, 1) for a, b in zip(outs[k], outs[k + 2]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        norm = B.clip_gradients(grads, 1.0)
    for t, o in zip(grads, other):
        t.copy_(o)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(norm, want[1]) and all(torch.equal(a, b) for a, b in zip(grads, outs[1]))


def test_more_than_two_to_the_31_elements():
    n = (1 << 31) + 12345
    big = torch.zeros(n, dtype=torch.bfloat16, device=DEV)
    probe = torch.tensor([0, 5, (1 << 31) - 1, 1 << 31, n - 1], device=DEV)
    big[probe] = torch.tensor([3.0, -1.0, 2.0, 4.0, -6.0], dtype=torch.bfloat16, device=DEV)
    small = torch.full((10,), 0.5, device=DEV)
    norm = B.clip_gradients([small, big], 1.0)
    torch.cuda.synchronize()
    want = (66.0 + 2.5) ** 0.5
    assert abs(float(norm) - want) <= 19 * E * want
    got = torch.tensor([3.0, -1.0, 2.0, 4.0, -6.0], dtype=torch.float64, device=DEV) / want
    assert torch.all((big[probe].double() - got).abs() <= 2.0 ** -8 * 1.001 * got.abs()) and int((big != 0).sum()) == 5
