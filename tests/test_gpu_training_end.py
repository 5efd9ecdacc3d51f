"""The end of a training step as it is used: windows are scored, their rewards become advantages, and the log-probabilities of the
drafted tokens take their gradient through the head, the norm in front of it and the norm's 8-bit input.  Every stage is held
to its definition in float64 on the inputs that it received from the stage before."""
import numpy as np
import pytest
import torch

from paper_2605_14978_b200 import binding as B
from paper_2605_14978_b200 import workloads as W

import test_gpu_head as head
import test_gpu_norm as norm

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_scored_windows_to_gradients(dtype):
    w = W.scaled(W.WORKLOADS[3], 48)                         # ragged windows of up to ten positions
    N, K, V, D, G = w.N, w.K, 4000, 320, 8
    g = torch.Generator(device=DEV).manual_seed(5)
    x = {"draft": torch.randn((N, K, V), generator=g, device=DEV), "u": torch.rand((N, K), generator=g, device=DEV),
         "tok": torch.randint(0, V, (N, K), generator=g, device=DEV, dtype=torch.int32),
         "len": torch.randint(0, K + 1, (N,), generator=g, device=DEV, dtype=torch.int32)}
    target = (x["draft"] + 0.5 * torch.randn((N, K, V), generator=g, device=DEV)).bfloat16()
    scored = B.score_windows(x["draft"].bfloat16(), target, x["tok"], mode=B.PPOW_STOCHASTIC, c=w.c, uniforms=x["u"], valid_len=x["len"])
    adv = torch.empty_like(scored["reward"])
    B.ppow_group_advantage(scored["reward"], G, 1e-4, adv)

    # the drafter's last hidden states, its final norm and head
    states, gain, shift, gy = norm.make(N * K, D, dtype, seed=6, offset=0.0)
    del gy
    weight = (torch.randn((V, D), generator=g, device=DEV) * 0.1).to(dtype)
    tokens = torch.where(torch.arange(K, device=DEV)[None] < x["len"][:, None], x["tok"], -1).reshape(-1).contiguous()
    n = B.layer_norm(states, gain, shift, checkpoint=True)
    out = B.head_logprob(n["y"], weight, tokens)
    # minus the advantage of the token's window over the valid tokens
    grad_logp = (-adv[:, None].expand(N, K) / max(1, int(x["len"].sum()))).reshape(-1).contiguous()
    gh, gw = B.head_logprob_backward(n["y"], weight, tokens, out["lse"], grad_logp)
    grads = B.layer_norm_backward(gh, (n["packed"], n["scale"]), gain, n["mean"], n["rstd"])
    torch.cuda.synchronize()

    norm.check_forward(states, gain, shift, 1e-5, n)
    norm.check_packed(states, n["packed"], n["scale"])
    head.check_forward(n["y"], weight, tokens, 1.0, out)
    head.check_backward(n["y"], weight, tokens, out["lse"], grad_logp, 1.0, gh, gw)
    norm.check_backward(gh, norm.reference_pack(states)[2], gain, n["mean"], n["rstd"], grads, torch.float32)
    live = (tokens >= 0) & (grad_logp != 0)
    assert 0 < int(live.sum()) < N * K and not grads[0][~live].any() and grads[0][live].any()
    # the same log-probabilities as the scoring pass takes from logits, where those are written out (rounded to 16 bits)
    logits = (n["y"].float() @ weight.float().t()).view(N, K, V)
    again = B.score_windows(logits.contiguous(), logits.contiguous(), x["tok"], mode=B.PPOW_GREEDY, c=w.c, valid_len=x["len"],
                            train_outputs=True)
    torch.cuda.synchronize()
    np.testing.assert_allclose(again["lse_p"].reshape(-1)[tokens >= 0].cpu().numpy(), out["lse"][tokens >= 0].cpu().numpy(), rtol=2e-5, atol=1e-4)
    np.testing.assert_allclose(again["logp_tok"].reshape(-1)[tokens >= 0].cpu().numpy(), out["logp"][tokens >= 0].cpu().numpy(), rtol=2e-5, atol=1e-4)


def test_gradients_add_up_over_micro_batches():
    # the same tokens in one call and in two: grad_hidden row by row, grad_weight as the sum (two roundings instead of one)
    h, w, tok, grad = head.make(600, 1200, 128, torch.bfloat16, seed=20)
    lse = B.head_logprob(h, w, tok)["lse"]
    gh, gw = B.head_logprob_backward(h, w, tok, lse, grad)
    a = B.head_logprob_backward(h[:250], w, tok[:250], lse[:250], grad[:250])
    b = B.head_logprob_backward(h[250:], w, tok[250:], lse[250:], grad[250:])
    torch.cuda.synchronize()
    want, tol = head.gradient(h, w, tok, lse, grad, 1.0)[2:]
    assert torch.all((gw.double() - want).abs() <= tol)
    parts = [head.gradient(h[s], w, tok[s], lse[s], grad[s], 1.0)[3] for s in (slice(0, 250), slice(250, 600))]
    assert torch.all((a[1].double() + b[1].double() - want).abs() <= parts[0] + parts[1])
    dh, th = head.gradient(h, w, tok, lse, grad, 1.0)[:2]
    assert torch.all((torch.cat([a[0], b[0]]).double() - dh).abs() <= th) and torch.all((gh.double() - dh).abs() <= th)
