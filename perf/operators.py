"""Cases and plain forms of the training-end operators: the log-probability of given tokens straight from hidden
states and the head's weight (and its gradient), layer normalisation (and its gradient), and 8-bit checkpoints of
activations, alone and as the saved input of the layer norm.

``own`` selects between the plain form (elementary torch operations in float32) and the library's calls.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
DEV = "cuda"
MOST_LOGITS = 4096 * 128256 * 4096          # tokens x vocabulary x width of the largest listed head case
MOST_ELEMENTS = 16384 * 8192                # rows x width of the largest listed activation


def listed():
    return [
        # one window of eight drafted tokens against a large vocabulary: the weight's bytes are everything
        dict(name="head_one_window", op="head", tokens=8, width=4096, vocab=128256, dtype="bf16", temperature=1.0, masked=0.0),
        # the smallest problem of the workload list, an odd vocabulary, some positions masked
        dict(name="head_tiny", op="head", tokens=77, width=520, vocab=1001, dtype="f16", temperature=0.7, masked=0.3),
        # a training batch: 512 windows of eight tokens
        dict(name="head_batch", op="head", tokens=4096, width=4096, vocab=128256, dtype="bf16", temperature=1.0, masked=0.0),
        # the gradient of a few windows, in half precision, at a sampling temperature
        dict(name="head_grad_small", op="head_grad", tokens=157, width=1024, vocab=32000, dtype="f16", temperature=0.7,
             masked=0.2, frozen=False),
        # ragged windows (lengths 4 to 10 of 10), the head frozen (shared with the target model): only the hidden gradient
        dict(name="head_grad_frozen_ragged", op="head_grad", tokens=2560, width=2048, vocab=151936, dtype="bf16",
             temperature=0.7, masked=0.3, frozen=True),
        # the gradient of a training batch, of hidden states and weight
        dict(name="head_grad_batch", op="head_grad", tokens=4096, width=4096, vocab=128256, dtype="bf16", temperature=1.0,
             masked=0.0, frozen=False),
        # the final norm of one window
        dict(name="norm_one_window", op="norm", rows=8, width=4096, dtype="f16", params="f16", bias=True, checkpoint=False),
        # the norm of a long batch that keeps its input in 8 bits for the backward pass
        dict(name="norm_checkpoint", op="norm", rows=16384, width=4096, dtype="bf16", params="f32", bias=True, checkpoint=True),
        # odd sizes in full precision
        dict(name="norm_grad_odd", op="norm_grad", rows=1003, width=1531, dtype="f32", params="f32", bias=True, checkpoint=False),
        # the backward pass of a long batch, its input read from the 8-bit checkpoint
        dict(name="norm_grad_checkpoint", op="norm_grad", rows=16384, width=4096, dtype="bf16", params="f32", bias=True,
             checkpoint=True),
        # packing and restoring one layer's activations
        dict(name="checkpoint_layer", op="checkpoint", rows=16384, width=8192, dtype="bf16"),
        dict(name="checkpoint_odd", op="checkpoint", rows=77, width=1000, dtype="f32"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["head", "head_grad", "head_grad", "norm", "norm_grad", "checkpoint"])
    if op.startswith("head"):
        while True:
            t, d, v = _log_uniform(rng, 1, 4096), 8 * _log_uniform(rng, 8, 512), _log_uniform(rng, 1000, 152064)
            if t * d * v <= MOST_LOGITS:
                break
        c = dict(op=op, tokens=t, width=d, vocab=v, dtype=rng.choice(["bf16", "f16"]),
                 temperature=rng.choice([0.7, 1.0, 1.3]), masked=rng.choice([0.0, 0.2, 0.5]))
        if op == "head_grad":
            c["frozen"] = rng.choice([False, False, True])
        return c
    while True:
        r, d = _log_uniform(rng, 1, 16384), _log_uniform(rng, 64, 8192)
        if rng.random() < 0.5:
            d = max(64, d // 64 * 64)
        if r * d <= MOST_ELEMENTS // 2:
            break
    c = dict(op=op, rows=r, width=d, dtype=rng.choice(["bf16", "f16", "f32"]))
    if op != "checkpoint":
        c["params"] = rng.choice(["f32", c["dtype"]])
        c["bias"] = rng.choice([True, True, False])
        c["checkpoint"] = rng.choice([False, True])
    return c


def _activations(r, d, g):
    """A residual stream: unit noise, a few channels much larger than the others, a small offset."""
    x = torch.randn((r, d), generator=g, device=DEV)
    gain = torch.exp(0.5 * torch.randn(d, generator=g, device=DEV))
    gain[torch.randint(0, d, (max(1, d // 256),), generator=g, device=DEV)] *= 20.0
    return x * gain + 0.1 * torch.randn(d, generator=g, device=DEV)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    if case["op"].startswith("head"):
        t, d, v = case["tokens"], case["width"], case["vocab"]
        weight = torch.empty((v, d), dtype=dt, device=DEV).normal_(0.0, 2.5 / math.sqrt(d), generator=g)
        tokens = torch.randint(0, v, (t,), generator=g, device=DEV, dtype=torch.int32)
        # a trained drafter: the drafted token's logit stands well above the others
        hidden = torch.randn((t, d), generator=g, device=DEV) + 1.6 * weight[tokens.long()].float()
        tokens[torch.rand(t, generator=g, device=DEV) < case["masked"]] = -1
        s = dict(case=case, hidden=hidden.to(dt), weight=weight, tokens=tokens)
        if case["op"] == "head_grad":
            # policy gradient: minus the advantage of the token's window over the number of tokens
            s["grad_logp"] = torch.randn(t, generator=g, device=DEV) / -t
            s["lse"] = _lse(s["hidden"], weight, case["temperature"])
        return s
    r, d = case["rows"], case["width"]
    s = dict(case=case, x=_activations(r, d, g).to(dt))
    if case["op"] != "checkpoint":
        pt = DTYPES[case["params"]]
        s["weight"] = (1.0 + 0.2 * torch.randn(d, generator=g, device=DEV)).to(pt)
        s["bias"] = (0.1 * torch.randn(d, generator=g, device=DEV)).to(pt) if case["bias"] else None
    if case["op"] == "norm_grad":
        x = s["x"].double()
        mean = x.mean(-1)
        s["mean"] = mean.float()
        s["rstd"] = torch.rsqrt((x - mean[:, None]).square().mean(-1) + EPS).float()
        s["grad_y"] = (torch.randn((r, d), generator=g, device=DEV) * 0.1).to(dt)
        if case["checkpoint"]:
            s["packed"], s["scale"] = _pack(s.pop("x"))
    return s


EPS = 1e-5
BLOCK = 128


def _lse(hidden, weight, temperature):
    """What the forward pass left: the normaliser of each row, to float32 accuracy, over pieces of the vocabulary."""
    h = hidden.float()
    pieces = [torch.logsumexp(h @ weight[i:i + 16384].float().t() / temperature, -1) for i in range(0, weight.shape[0], 16384)]
    return torch.logsumexp(torch.stack(pieces), 0)


def _pack(x):
    """8-bit form: blocks of 128 along a row share 2^e, the smallest power of two that brings the block's largest
    finite magnitude to 448 or less; values are rounded to nearest even in e4m3."""
    r, d = x.shape
    n = (d + BLOCK - 1) // BLOCK
    f = torch.zeros((r, n * BLOCK), dtype=torch.float32, device=x.device)
    f[:, :d] = x.float()
    f = f.view(r, n, BLOCK)
    top = f.abs().amax(-1)
    m, ex = torch.frexp(top)
    e = (ex - 9 + (m > 0.875).int()).clamp(min=-126)
    e = torch.where(top == 0, torch.full_like(e, -126), e)
    q = torch.ldexp(f, -e[..., None]).view(r, n * BLOCK)[:, :d].to(torch.float8_e4m3fn)
    return q.contiguous(), (e + 127).to(torch.uint8)


def _unpack(q, scale):
    r, d = q.shape
    e = scale.int() - 127
    return torch.ldexp(q.float(), e.repeat_interleave(BLOCK, 1)[:, :d])


def _plain(s):
    c = s["case"]
    op = c["op"]
    dt = DTYPES[c["dtype"]]
    if op.startswith("head"):
        h, w, y = s["hidden"].float(), s["weight"].float(), s["tokens"].long()
        live = y >= 0
        z = (h @ w.t()) / c["temperature"]
        if op == "head":
            top = z.amax(-1, keepdim=True)
            lse = (torch.exp(z - top).sum(-1).log() + top[:, 0])
            logp = z.gather(1, y.clamp(min=0)[:, None])[:, 0] - lse
            return {"logp": torch.where(live, logp, 0.0), "lse": torch.where(live, lse, 0.0)}
        dz = torch.exp(z - s["lse"][:, None]).neg_()
        del z
        dz.scatter_add_(1, y.clamp(min=0)[:, None], torch.ones_like(dz[:, :1]))
        dz *= (torch.where(live, s["grad_logp"], 0.0) / c["temperature"])[:, None]
        out = {"grad_hidden": (dz @ w).to(dt)}
        if not c["frozen"]:
            out["grad_weight"] = (dz.t() @ h).to(dt)
        return out
    if op == "checkpoint":
        q, scale = _pack(s["x"])
        return {"packed": q, "scale": scale, "restored": _unpack(q, scale).to(dt)}
    w = s["weight"].float()
    if op == "norm":
        x = s["x"].float()
        mean = x.mean(-1)
        xc = x - mean[:, None]
        rstd = torch.rsqrt((xc * xc).mean(-1) + EPS)
        y = xc * rstd[:, None] * w
        if s["bias"] is not None:
            y = y + s["bias"].float()
        out = {"y": y.to(dt), "mean": mean, "rstd": rstd}
        if c["checkpoint"]:
            out["packed"], out["scale"] = _pack(s["x"])
        return out
    x = _unpack(s["packed"], s["scale"]) if c["checkpoint"] else s["x"].float()
    gy = s["grad_y"].float()
    xhat = (x - s["mean"][:, None]) * s["rstd"][:, None]
    gx = gy * w
    gx = (gx - gx.mean(-1, keepdim=True) - xhat * (gx * xhat).mean(-1, keepdim=True)) * s["rstd"][:, None]
    out = {"grad_x": gx.to(dt), "grad_weight": (gy * xhat).sum(0).to(s["weight"].dtype)}
    if c["bias"]:
        out["grad_bias"] = gy.sum(0).to(s["weight"].dtype)
    return out


def run(state):
    if not own:
        return _plain(state)
    from paper_2605_14978_b200 import binding as B
    c = state["case"]
    op = c["op"]
    if op == "head":
        return B.head_logprob(state["hidden"], state["weight"], state["tokens"], temperature=c["temperature"])
    if op == "head_grad":
        gh, gw = B.head_logprob_backward(state["hidden"], state["weight"], state["tokens"], state["lse"], state["grad_logp"],
                                         temperature=c["temperature"], want_weight=not c["frozen"])
        return {"grad_hidden": gh} if c["frozen"] else {"grad_hidden": gh, "grad_weight": gw}
    if op == "norm":
        return B.layer_norm(state["x"], state["weight"], state["bias"], eps=EPS, checkpoint=c["checkpoint"])
    if op == "norm_grad":
        x = (state["packed"], state["scale"]) if c["checkpoint"] else state["x"]
        gx, gw, gb = B.layer_norm_backward(state["grad_y"], x, state["weight"], state["mean"], state["rstd"],
                                           want_bias=c["bias"])
        out = {"grad_x": gx, "grad_weight": gw}
        if c["bias"]:
            out["grad_bias"] = gb
        return out
    q, scale = B.pack_activation(state["x"])
    return {"packed": q, "scale": scale, "restored": B.unpack_activation(q, scale, state["x"].dtype)}


def work(case):
    es = 4 if case["dtype"] == "f32" else 2
    if case["op"].startswith("head"):
        t, d, v = case["tokens"], case["width"], case["vocab"]
        flops = 2.0 * t * (1.0 - case["masked"]) * d * v
        bytes_ = v * d * es + t * d * es + 4 * t + 8 * t
        if case["op"] == "head":
            return {"bytes": bytes_, "flops": flops}
        products = 2 if case["frozen"] else 3
        return {"bytes": bytes_ + t * d * es + (0 if case["frozen"] else v * d * es), "flops": products * flops}
    r, d = case["rows"], case["width"]
    q = r * d + r * ((d + BLOCK - 1) // BLOCK)
    if case["op"] == "checkpoint":
        return {"bytes": 2 * r * d * es + 2 * q, "flops": 4.0 * r * d}
    ps = 4 if case["params"] == "f32" else 2
    if case["op"] == "norm":
        return {"bytes": 2 * r * d * es + 8 * r + 2 * d * ps + (q if case["checkpoint"] else 0), "flops": 8.0 * r * d}
    saved = q if case["checkpoint"] else r * d * es
    return {"bytes": 2 * r * d * es + saved + 8 * r + 3 * d * ps, "flops": 14.0 * r * d}


def _exact_pack(x):
    """The same format from its definition, in float64: returns values before scaling, and the exponents."""
    r, d = x.shape
    v = x.double()
    blocks = [v[:, i:i + BLOCK] for i in range(0, d, BLOCK)]
    top = torch.stack([b.abs().max(1).values for b in blocks], 1)
    e = torch.ceil(torch.log2(top / 448.0))
    e = torch.where(top / torch.exp2(e - 1) <= 448.0, e - 1, e)          # the logarithm may be off by one at a border
    e = torch.where(top / torch.exp2(e) > 448.0, e + 1, e)
    e = torch.where(top > 0, e.clamp(min=-126.0), torch.full_like(e, -126.0))
    u = torch.cat([b / torch.exp2(e[:, i:i + 1]) for i, b in enumerate(blocks)], 1)
    _, ex = torch.frexp(u)
    step = torch.exp2((ex - 1).clamp(min=-6).double() - 3.0)              # spacing of e4m3 around u
    return torch.round(u / step) * step, e


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"].startswith("head"):
        t, d, v = case["tokens"], case["width"], case["vocab"]
        w = s["weight"].double()
        inv = 1.0 / case["temperature"]
        rows = max(1, min(t, (1 << 28) // v))
        live = [i for i, y in enumerate(s["tokens"].tolist()) if y >= 0]
        logp = torch.zeros(t, dtype=torch.float64, device=DEV)
        lse = torch.zeros(t, dtype=torch.float64, device=DEV)
        grad_h = torch.zeros((t, d), dtype=torch.float64, device=DEV)
        grad_w = None if case.get("frozen", True) else torch.zeros((v, d), dtype=torch.float64, device=DEV)
        for a in range(0, len(live), rows):
            at = torch.tensor(live[a:a + rows], device=DEV)
            h = s["hidden"][at].double()
            y = s["tokens"][at].long()
            z = torch.mm(h, w.t()).mul_(inv)
            if case["op"] == "head":
                lse[at] = torch.logsumexp(z, 1)
                logp[at] = z[torch.arange(len(at), device=DEV), y] - lse[at]
                continue
            # d logp / d z = onehot - softmax, times the incoming gradient
            p = torch.exp(z.sub_(s["lse"][at].double()[:, None]))
            p[torch.arange(len(at), device=DEV), y] -= 1.0
            p.mul_(-inv * s["grad_logp"][at].double()[:, None])
            grad_h[at] = torch.mm(p, w)
            if grad_w is not None:
                grad_w.addmm_(p.t(), h)
        if case["op"] == "head":
            return {"logp": logp, "lse": lse}
        return {"grad_hidden": grad_h} if grad_w is None else {"grad_hidden": grad_h, "grad_weight": grad_w}
    if case["op"] == "checkpoint":
        q, e = _exact_pack(s["x"])
        back = torch.cat([q[:, i * BLOCK:(i + 1) * BLOCK] * torch.exp2(e[:, i:i + 1]) for i in range(e.shape[1])], 1)
        return {"packed": q, "scale": (e + 127).to(torch.int64), "restored": back}
    w = s["weight"].double()
    if case["op"] == "norm":
        var, mean = torch.var_mean(s["x"].double(), dim=1, correction=0)
        rstd = 1.0 / torch.sqrt(var + EPS)
        y = (s["x"].double() - mean[:, None]) * rstd[:, None] * w[None, :]
        if s["bias"] is not None:
            y += s["bias"].double()[None, :]
        out = {"y": y, "mean": mean, "rstd": rstd}
        if case["checkpoint"]:
            q, e = _exact_pack(s["x"])
            out["packed"], out["scale"] = q, (e + 127).to(torch.int64)
        return out
    if case["checkpoint"]:
        q, e = s["packed"].double(), s["scale"].double() - 127.0
        x = torch.cat([q[:, i * BLOCK:(i + 1) * BLOCK] * torch.exp2(e[:, i:i + 1]) for i in range(e.shape[1])], 1)
    else:
        x = s["x"].double()
    gy = s["grad_y"].double()
    rstd = s["rstd"].double()[:, None]
    xhat = (x - s["mean"].double()[:, None]) * rstd
    a = gy * w[None, :]
    d = x.shape[1]
    gx = rstd / d * (d * a - a.sum(1, keepdim=True) - xhat * (a * xhat).sum(1, keepdim=True))
    out = {"grad_x": gx, "grad_weight": (gy * xhat).sum(0)}
    if case["bias"]:
        out["grad_bias"] = gy.sum(0)
    return out
