"""The error word of the head's allocating wrappers: whoever wants to know gets the workspace, on every path of a call."""
import pytest
import torch

from paper_2605_14978_b200 import binding as B

import test_gpu_head as head

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("own_stream", [False, True])
@pytest.mark.parametrize("T", [20, 500])
def test_the_wrappers_hand_the_workspace_back(T, own_stream):
    h, w, tok, grad = head.make(T, 777, 64, torch.bfloat16, seed=5, masked=0.1)
    stream = torch.cuda.Stream() if own_stream else None
    for behind, flags in ((False, 0), (True, B.PPOW_FLAG_TOKEN_RANGE)):
        if behind:
            tok[3] = 777
        torch.cuda.synchronize()
        out = B.head_logprob(h, w, tok, want_workspace=True, stream=stream)
        assert B.ppow_read_error_flags(out["_workspace"], stream) == flags
        plain = B.head_logprob(h, w, tok, stream=stream)
        back = B.head_logprob_backward(h, w, tok, out["lse"], grad, want_workspace=True, stream=stream)
        assert B.ppow_read_error_flags(back[2], stream) == flags
        gh, gw = B.head_logprob_backward(h, w, tok, out["lse"], grad, stream=stream)
        torch.cuda.synchronize()
        assert set(plain) == {"logp", "lse"} and torch.equal(plain["logp"], out["logp"])
        assert torch.equal(gh, back[0]) and torch.equal(gw, back[1]) and bool(gh.isfinite().all())


def test_without_tokens_too():
    h, w, tok, grad = head.make(4, 600, 64, torch.bfloat16)
    junk = [torch.full((1 << 20,), 255, dtype=torch.uint8, device=h.device) for _ in range(8)]    # what the allocator may hand out
    del junk
    out = B.head_logprob(h[:0], w, tok[:0], want_workspace=True)
    assert B.ppow_read_error_flags(out["_workspace"]) == 0
    assert B.ppow_read_error_flags(B.head_logprob_backward(h[:0], w, tok[:0], out["lse"], grad[:0], want_workspace=True)[2]) == 0
