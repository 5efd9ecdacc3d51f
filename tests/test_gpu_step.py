"""A training step from the drafter's hidden states to clipped gradients, as it is used: the block's output joins the residual stream under an
RMS norm, tokens are drawn from the head's logits, windows are scored, and the log-probabilities of the drawn tokens take their gradient
through the head and the norm to gradients that are clipped together.  Every stage is held to its definition in float64 on the inputs
that it received from the stage before.  And: both ways of marshalling a call give the same."""
import numpy as np
import pytest
import torch

from paper_2605_14978_b200 import binding as B
from paper_2605_14978_b200 import workloads as W

import test_gpu_clip as clip
import test_gpu_head as head
import test_gpu_norm as norm
import test_gpu_rms as rms
import test_gpu_sample as sample

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def inputs(dtype, seed=3):
    w = W.scaled(W.WORKLOADS[3], 48)
    N, K, V, D = w.N, w.K, 4000, 320
    g = torch.Generator(device=DEV).manual_seed(seed)
    x, res, gain, _, _ = rms.make(N * K, D, dtype, seed=seed)
    return dict(w=w, N=N, K=K, V=V, D=D, x=x, res=res, gain=gain, weight=(torch.randn((V, D), generator=g, device=DEV) * 0.15).to(dtype),
                u_draw=torch.rand(N * K, generator=g, device=DEV), u=torch.rand((N, K), generator=g, device=DEV),
                noise=0.5 * torch.randn((N, K, V), generator=g, device=DEV))


def step(s, **k):
    """All calls of a step; ``k`` may name a stream."""
    N, K, V = s["N"], s["K"], s["V"]
    n = B.rms_norm(s["x"], s["gain"], s["res"], checkpoint=True, **k)
    logits = torch.mm(n["y"], s["weight"].t())               # 16-bit logits, as a drafter's head leaves them
    drawn = B.sample_tokens(logits, s["u_draw"], temperature=0.8, top_k=500, top_p=0.95, min_p=0.001, **k)
    target = (logits.float().view(N, K, V) + s["noise"]).to(logits.dtype)
    scored = B.score_windows(logits.view(N, K, V), target, drawn["tokens"].view(N, K), mode=B.PPOW_STOCHASTIC, c=s["w"].c, uniforms=s["u"],
                             temperature=0.8)
    adv = torch.empty_like(scored["reward"])
    B.ppow_group_advantage(scored["reward"], 8, 1e-4, adv)
    out = B.head_logprob(n["y"], s["weight"], drawn["tokens"], temperature=0.8, **k)
    grad_logp = (-adv[:, None].expand(N, K) / (N * K)).reshape(-1).contiguous()
    gh, gw = B.head_logprob_backward(n["y"], s["weight"], drawn["tokens"], out["lse"], grad_logp, temperature=0.8, **k)
    gx, ggain = B.rms_norm_backward(gh, (n["packed"], n["scale"]), s["gain"], n["rstd"], **k)
    grads = [gw, ggain, gx]
    clipped = [torch.empty_like(t) for t in grads]
    total = B.clip_gradients(grads, 0.01, out=clipped, **k)
    return dict(n=n, logits=logits, drawn=drawn, scored=scored, adv=adv, out=out, grad_logp=grad_logp, gh=gh, gw=gw, gx=gx, ggain=ggain, grads=grads,
                clipped=clipped, total=total)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_hidden_states_to_clipped_gradients(dtype):
    s = inputs(dtype)
    r = step(s)
    torch.cuda.synchronize()
    rms.check_forward(s["x"], s["res"], s["gain"], 1e-6, r["n"])
    sample.check(r["logits"], s["u_draw"], r["drawn"], temperature=0.8, top_k=500, top_p=0.95, min_p=0.001)
    tokens = r["drawn"]["tokens"]
    assert int(tokens.min()) >= 0 and int(tokens.max()) < s["V"] and int(r["drawn"]["kept"].max()) <= 500
    head.check_forward(r["n"]["y"], s["weight"], tokens, 0.8, r["out"])
    head.check_backward(r["n"]["y"], s["weight"], tokens, r["out"]["lse"], r["grad_logp"], 0.8, r["gh"], r["gw"])
    rms.check_backward(r["gh"], norm.reference_pack(r["n"]["sum"])[2], s["gain"], r["n"]["rstd"], None, (r["gx"], r["ggain"]))
    clip.check(r["grads"], 0.01, r["total"], r["clipped"])
    # without filters the draw's log-probability is the scoring pass's
    plain = B.sample_tokens(r["logits"], s["u_draw"], temperature=0.8)
    z = r["logits"].view(s["N"], s["K"], s["V"])
    again = B.score_windows(z, z, plain["tokens"].view(s["N"], s["K"]), mode=B.PPOW_GREEDY, c=s["w"].c, temperature=0.8)
    torch.cuda.synchronize()
    np.testing.assert_allclose(again["logq_tok"].reshape(-1).cpu().numpy(), plain["logp"].cpu().numpy(), rtol=1e-4, atol=1e-6)
    # and top_k = 1 is the greedy token
    greedy = B.sample_tokens(r["logits"], s["u_draw"], top_k=1)
    torch.cuda.synchronize()
    assert torch.equal(greedy["tokens"], again["target_argmax"].reshape(-1)) and not greedy["logp"].any()


def test_a_step_repeats_on_another_stream_and_from_a_graph():
    s = inputs(torch.bfloat16)
    want = step(s)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = step(s)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        held = step(s)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    for r in (other, held):
        assert torch.equal(r["drawn"]["tokens"], want["drawn"]["tokens"]) and torch.equal(r["drawn"]["logp"], want["drawn"]["logp"])
        assert torch.equal(r["total"], want["total"]) and all(torch.equal(a, b) for a, b in zip(r["clipped"], want["clipped"]))


def variants():
    """(wrapper, arguments, keywords): calls that are right in every layout that the documentation allows, and calls that are not."""
    bf, f32 = torch.bfloat16, torch.float32
    h = torch.randn((40, 64), device=DEV).to(bf)
    wide = torch.randn((40, 200), device=DEV).to(bf)
    u = torch.rand(40, device=DEV)
    rows = (h, wide[:, 8:72], wide[:, 3:67], h[:1], h[:0], h[::2], wide[:1, 3:67], h.t().contiguous().t(), h[0].expand(40, 64), h.float(), h.half(), h[0],
            h.cpu(), h[:, :63], h[None], h.double())
    for x in rows:
        n, d = (x.shape[0], x.shape[1]) if x.dim() == 2 else (40, 64)
        for v in (u[:n], u[:n].double(), torch.stack([u, u], 1)[:n, 0], u[:n].cpu(), u):
            yield "sample_tokens", (x, v), dict(top_p=0.9)
        for k in (dict(top_k=-1), dict(top_k=1 << 40), dict(temperature=0.0), dict(top_p=0.0), dict(min_p=2.0), dict(top_k=3, min_p=0.5)):
            yield "sample_tokens", (x, u[:n]), k
        like = torch.randn((n, d), device=DEV).to(x.dtype)
        for gain in (torch.ones(d, device=DEV), torch.ones(d, device=DEV, dtype=bf), torch.ones(d + 1, device=DEV), torch.ones(d)):
            for res in (None, like, like[:, :1], like.half(), wide[:n, 5:5 + d]):
                yield "rms_norm", (x, gain, res), dict(checkpoint=True)
                yield "rms_norm", (x, gain, res), dict(packed_output=True)
            for more in (None, like, like.cpu(), wide[:n, :d]):
                yield "rms_norm_backward", (like, x, gain, u[:n]), dict(grad_sum=more)
                yield "rms_norm_backward", (x, like, gain, u[:n]), dict(grad_sum=more)
    q, s = B.pack_activation(h)
    for pair in ((q, s), (q[:, :32], s), (q.cpu(), s), (q[:0], s[:0]), (q, s.int())):
        yield "rms_norm_backward", (h[:pair[0].shape[0]], pair, torch.ones(64, device=DEV), u[:pair[0].shape[0]]), {}
    a, b = torch.randn((30, 20), device=DEV), torch.randn(7, device=DEV).half()
    for grads in ([a, b], (a, b), [a.t(), b], [a[:, ::2]], [a, b.cpu()], [a.double()], [a, a], [a[0], b[:0]], [a[0, 0]], [a, 3], [wide[:, 1:]], []):
        yield "clip_gradients", (grads, 1.0), dict(out="empty")
        yield "clip_gradients", (grads, 1.0), dict(out="one short")
        yield "gradient_norm", (grads,), {}
    yield "clip_gradients", ([a, b], -1.0), dict(out="empty")
    yield "clip_gradients", ([a, b], 1.0), dict(out=[a.t().contiguous().t(), b.clone()])


def call(name, args, keys):
    try:
        keys = dict(keys)
        if isinstance(keys.get("out"), str):
            kind = keys["out"]
            keys["out"] = [torch.zeros_like(t) for t in args[0]][:None if kind == "empty" else -1]
        out = getattr(B, name)(*args, **keys)
        got = [out[k] for k in sorted(out)] if isinstance(out, dict) else list(out) if isinstance(out, tuple) else [out]
        return [t.float().nan_to_num() for t in got + list(keys.get("out") or [])]
    except (ValueError, B.PpowError, AttributeError, TypeError) as e:
        return type(e)


def test_both_ways_of_marshalling_accept_refuse_and_return_the_same(monkeypatch):
    quick, slow, tried, ran = B._quick(), B._NoCalls(), 0, 0
    for name, args, keys in variants():
        monkeypatch.setattr(B, "_calls", quick)
        a = call(name, args, keys)
        monkeypatch.setattr(B, "_calls", slow)
        b = call(name, args, keys)
        tried += 1
        what = (name, [getattr(t, "shape", t) for t in args], keys, a, b)
        if isinstance(a, type) or isinstance(b, type):
            assert a is b, what
            continue
        ran += 1
        assert len(a) == len(b) and all(torch.equal(x, y) for x, y in zip(a, b)), what
    torch.cuda.synchronize()
    assert tried > 300 and ran > 80
