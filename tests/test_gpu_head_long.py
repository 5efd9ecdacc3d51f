"""Gradients of long batches: many pieces of the vocabulary, the last one short, most rows masked or none, against the definition in
float64 with the bounds of test_gpu_head; and the error word of each call."""
import pytest
import torch

from paper_2605_14978_b200 import binding as B

import test_gpu_head as head

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def backward(h, w, tok, lse, grad):
    p = B.make_head_params(h, w)
    ws = B.alloc_workspace(B.ppow_head_workspace_bytes(p, True), DEV)
    gh, gw = torch.empty_like(h), torch.empty_like(w)
    B.ppow_head_logprob_backward(p, h, w, tok, lse, grad, gh, gw, ws)
    assert B.ppow_read_error_flags(ws) == 0
    return gh, gw


def check(h, w, tok, lse, grad, gh, gw):
    """Element by element within the bounds of head.gradient; and all in all: two half steps u of each value, and in float16, whose
    steps below 2^-14 are 2^-24 whatever the value, half of such a step each, 2^-25 sqrt(count) in the norm.  (Gradients over a
    batch of T are of the order of 1/T: with T = 262144 nearly all of them lie there.)"""
    dh, th, dw, tw = head.gradient(h, w, tok, lse, grad, 1.0)
    for got, want, tol in ((gh, dh, th), (gw, dw, tw)):
        off = got.double() - want
        assert torch.all(off.abs() <= tol)
        least = 2.0 ** -25 * want.numel() ** 0.5 if h.dtype == torch.float16 else 0.0
        assert float(off.norm()) < 2 * head.U[h.dtype] * float(want.norm()) + least


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,V,D,live", [(262144, 3129, 768, 6700), (51896, 128256, 1024, 3483), (49152, 129280, 2048, 2000), (65536, 65537, 256, 300)])
def test_many_pieces_most_rows_masked(T, V, D, live, dtype):
    g = torch.Generator(device=DEV).manual_seed(T + live)
    h, w, tok, grad = head.make(T, V, D, dtype, seed=50, masked=0.0)
    keep = torch.zeros(T, dtype=torch.bool, device=DEV)
    keep[torch.randperm(T, generator=g, device=DEV)[:live]] = True
    tok[~keep] = -1
    assert len(B.ppow_head_plan(B.make_head_params(h, w), live)[0]) > 2
    lse = B.head_logprob(h, w, tok)["lse"]
    gh, gw = backward(h, w, tok, lse, grad)
    assert not gh[~keep].any()
    check(h[keep], w, tok[keep], lse[keep], grad[keep], gh[keep], gw)
    torch.cuda.empty_cache()


def test_many_pieces_no_row_masked():
    T, V, D, rows = 65536, 65537, 256, 8192
    h, w, tok, grad = head.make(T, V, D, torch.bfloat16, seed=51, masked=0.0)
    lse = B.head_logprob(h, w, tok)["lse"]
    gh, gw = backward(h, w, tok, lse, grad)
    dw = torch.zeros((V, D), dtype=torch.float64, device=DEV)
    for i in range(0, T, rows):
        s = slice(i, i + rows)
        dh, th, part, _ = head.gradient(h[s], w, tok[s], lse[s], grad[s], 1.0)
        dw += part
        assert torch.all((gh[s].double() - dh).abs() <= th), i
    assert float((gw.double() - dw).norm() / dw.norm()) < 2 * head.U[torch.bfloat16]
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T", [8192, 8193, 65536, 262144])
def test_sums_over_many_tokens_whose_terms_have_one_sign(T, dtype):
    # Hidden states with a mean of 1, a loss of equal weights: every entry's softmax pulls its row of dW the same way.  Besides the
    # roundings of the result and of dz (see test_gpu_head_rounding) the tensor cores cut off what does not fit: in a sum of 8192 tokens
    # 513 times, at most two steps 2^-23 of its magnitude each, 1.3e-4 of sum |dz| |h|.
    V, D, rows = 300, 64, 8192
    g = torch.Generator(device=DEV).manual_seed(T)
    w = (torch.randn((V, D), generator=g, device=DEV) * 0.1).to(dtype)
    h = (1 + 0.2 * torch.randn((T, D), generator=g, device=DEV)).to(dtype)
    tok = torch.randint(0, V // 2, (T,), generator=g, device=DEV, dtype=torch.int32)
    grad = torch.full((T,), -1.0 / 64, device=DEV)
    lse = B.head_logprob(h, w, tok)["lse"]
    _, gw = backward(h, w, tok, lse, grad)
    want, size, others = torch.zeros((3, V, D), dtype=torch.float64, device=DEV)
    for i in range(0, T, rows):
        x, y = h[i:i + rows].double(), tok[i:i + rows].long()[:, None]
        q = torch.exp(x @ w.double().t() - lse[i:i + rows].double()[:, None])
        dz = (q - torch.zeros_like(q).scatter(1, y, 1.0)) / 64
        want += dz.t() @ x
        size += dz.abs().t() @ x.abs()
        others += dz.scatter(1, y, 0.0).square().t() @ x.square()
    own = (want.to(dtype).double() - want).square().sum()
    most = 1.05 * (own + head.U[dtype] ** 2 / 3 * others.sum()).sqrt() + 1.3e-4 * size.norm()
    assert float((gw.double() - want).norm()) <= float(most)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,V", [(6000, 3000), (9000, 40)])
def test_rows_ordered_by_lists_give_the_same_every_time(T, V, dtype):
    # above 4096 tokens the rows' order comes from lists that threads fill in any order: either gradient alone, eager and captured,
    # on two streams at once, always the same bits
    h, w, tok, grad = head.make(T, V, 136, dtype, seed=52, masked=0.3)
    lse = B.head_logprob(h, w, tok)["lse"]
    gh, gw = backward(h, w, tok, lse, grad)
    check(h, w, tok, lse, grad, gh, gw)
    assert torch.equal(B.head_logprob_backward(h, w, tok, lse, grad, want_weight=False)[0], gh)
    assert torch.equal(B.head_logprob_backward(h, w, tok, lse, grad, want_hidden=False)[1], gw)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [B.head_logprob_backward(h, w, tok, lse, grad, stream=streams[i % 2]) for i in range(4)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, gh) and torch.equal(b, gw) for a, b in got)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a, b = B.head_logprob_backward(h, w, tok, lse, grad)
    other = head.make(T, V, 136, dtype, seed=53, masked=0.6)
    want = B.head_logprob_backward(other[0], other[1], other[2], lse, other[3])
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(a, gh) and torch.equal(b, gw)
    for x, y in zip((h, w, tok, grad), other):
        x.copy_(y)
    graph.replay()
    torch.cuda.synchronize()
    # bit by bit: lse is the first inputs', and a p far above 1 is infinite in float16
    assert torch.equal(a.view(torch.int16), want[0].view(torch.int16)) and torch.equal(b.view(torch.int16), want[1].view(torch.int16))
