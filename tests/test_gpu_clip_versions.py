"""Clipping counts as a modification in place to autograd, by either way of marshalling: a backward pass that saved what is written raises."""
import pytest
import torch

from paper_2605_14978_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(params=["module", "python"], autouse=True)
def marshalling(request, monkeypatch):
    monkeypatch.setattr(B, "_calls", B._quick() if request.param == "module" else B._NoCalls())


def test_versions_of_what_is_written():
    grads = [torch.ones(5, device=DEV), torch.ones((3, 4), device=DEV).half(), torch.ones(0, device=DEV)]
    out = [torch.empty_like(t) for t in grads]
    v, w = [t._version for t in grads], [t._version for t in out]
    B.gradient_norm(grads)
    assert [t._version for t in grads] == v
    B.clip_gradients(grads, 1.0, out=out)
    assert [t._version for t in grads] == v and [t._version for t in out] == [n + 1 for n in w]
    B.clip_gradients(tuple(grads), 1.0)
    assert [t._version for t in grads] == [n + 1 for n in v]
    v = [t._version for t in grads]
    with pytest.raises(B.PpowError):
        B.clip_gradients(grads, -1.0)
    assert [t._version for t in grads] == v
    torch.cuda.synchronize()


def test_a_gradient_kept_for_a_second_backward_pass():
    x = torch.full((7,), 2.0, device=DEV, requires_grad=True)
    (g,) = torch.autograd.grad((x ** 3).sum(), x, create_graph=True)
    loss = (g * g).sum()                                     # its gradient needs g
    B.clip_gradients([g.detach()], 1.0)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    torch.cuda.synchronize()


def test_tensors_without_versions():
    with torch.inference_mode():
        t = torch.ones(6, device=DEV)
        u = torch.ones(6, device=DEV)
        B.clip_gradients([u], 1.0)
    norm = B.clip_gradients([t], 1.0)
    torch.cuda.synchronize()
    assert torch.equal(t, u) and float(t.sum()) < 6.0 and abs(float(norm) - 6.0 ** 0.5) < 1e-6
