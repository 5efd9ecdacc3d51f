"""Refusals of the RMS norm and of clipping that need tensors on a device, by either way of marshalling."""
import pytest
import torch

from paper_2605_14978_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(params=["module", "python"], autouse=True)
def marshalling(request, monkeypatch):
    monkeypatch.setattr(B, "_calls", B._quick() if request.param == "module" else B._NoCalls())


def test_types_of_the_rms_norm():
    x, r = torch.zeros((4, 16), dtype=torch.bfloat16, device=DEV), torch.ones(4, device=DEV)
    gain = torch.ones(16, device=DEV)
    for w in (gain.double(), gain.int()):
        with pytest.raises(ValueError, match="types must be"):
            B.rms_norm(x, w)
        with pytest.raises(ValueError, match="types must be"):
            B.rms_norm_backward(x, x, w, r)
    with pytest.raises(ValueError, match="types must be"):
        B.rms_norm(x.double(), gain)
    with pytest.raises(ValueError, match="types must be"):
        B.rms_norm_backward(x.double(), x.double(), gain, r)
    for w in (gain.half(), gain[:8], gain[None], gain.cpu()):        # another 16-bit type than the rows', other shapes, another device
        with pytest.raises((ValueError, B.PpowError)):
            B.rms_norm(x, w)
        with pytest.raises((ValueError, B.PpowError)):
            B.rms_norm_backward(x, x, w, r)
    with pytest.raises(ValueError, match="rstd"):
        B.rms_norm_backward(x, x, gain, r.double())
    with pytest.raises(ValueError, match="residual"):
        B.rms_norm(x, gain, x.half())


def test_outputs_of_a_clipping_that_are_not_like_their_gradients():
    g = torch.ones((4, 6), device=DEV)
    for out in (g.half(), g.cpu(), g[:2], g.t(), torch.ones((6, 4), device=DEV).t(), g.double()):
        with pytest.raises(ValueError, match="like its gradient"):
            B.clip_gradients([g], 1.0, out=[out])
    with pytest.raises(ValueError, match="as many"):
        B.clip_gradients([g, g], 1.0, out=[torch.empty_like(g)])
    assert torch.all(g == 1)
