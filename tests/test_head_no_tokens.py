"""A batch without tokens: allowed in every form of the gradient, the one for a frozen head too, whose only output is empty and may
have no address."""
import ctypes

import pytest
import torch

from paper_2605_14978_b200 import binding as B
from paper_2605_14978_b200 import build as build_mod

P = 1 << 20          # an aligned address that is never used


def test_a_frozen_head_without_tokens_is_accepted():
    build_mod.build()
    lib = B.load_library()
    none = B.ppow_head_params(0, 1000, 64, B.PPOW_BF16, 64, 64, 1.0)
    for gh in (None, P):
        assert lib.ppow_head_logprob_backward(ctypes.byref(none), None, None, None, None, None, gh, None, None, 0, None) == B.PPOW_OK
    one = B.ppow_head_params(1, 1000, 64, B.PPOW_BF16, 64, 64, 1.0)
    assert lib.ppow_head_logprob_backward(ctypes.byref(one), P, P, P, P, P, None, None, P, 1 << 40, None) == B.PPOW_ERR_INVALID_ARG


@pytest.mark.gpu
@pytest.mark.parametrize("stream", [False, True])
def test_every_form_of_the_gradient_without_tokens(stream):
    dev = "cuda:0"
    s = torch.cuda.Stream() if stream else None
    h, w = torch.empty((0, 64), dtype=torch.bfloat16, device=dev), torch.randn((600, 64), device=dev).bfloat16()
    tok, f = torch.empty(0, dtype=torch.int32, device=dev), torch.empty(0, device=dev)
    torch.cuda.synchronize()
    for want_hidden, want_weight in ((True, True), (True, False), (False, True)):
        gh, gw = B.head_logprob_backward(h, w, tok, f, f, want_hidden=want_hidden, want_weight=want_weight, stream=s)
        torch.cuda.synchronize()
        assert gh.shape == (0, 64) if want_hidden else gh is None
        assert gw.shape == (600, 64) and not gw.any() if want_weight else gw is None
