"""Cases and plain forms of operators around a drafter's training step: tokens drawn from logits with given uniforms
(temperature, top-k, top-p, min-p), root-mean-square norm with the residual's addition (and its gradient, with 8-bit
outputs and checkpoints), and the global norm of many gradients with clipping.

``own`` selects between the plain form (elementary torch operations) and the library's calls.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
DEV = "cuda"
EPS = 1e-6
BLOCK = 128
MOST_LOGITS = 4096 * 128256                  # rows x vocabulary of the largest listed draw, 16 bits each
MOST_ELEMENTS = 16384 * 4096                 # rows x width of the largest listed activation
MOST_GRADIENTS = 743 * 10 ** 6               # elements of the largest listed set of gradients


def listed():
    return [
        # the next token of eight sequences, nucleus sampling: latency
        dict(name="sample_next_token", op="sample", rows=8, vocab=128256, dtype="bf16", temperature=1.0, top_k=0, top_p=0.95, min_p=0.0,
             masked=0.0),
        # the smallest workload's windows, in full precision
        dict(name="sample_tiny", op="sample", rows=256, vocab=1000, dtype="f32", temperature=1.0, top_k=50, top_p=1.0, min_p=0.0, masked=0.1),
        # one position of 80 groups of eight rollouts, all filters, some tokens forbidden
        dict(name="sample_rollouts", op="sample", rows=640, vocab=151936, dtype="bf16", temperature=0.7, top_k=1000, top_p=0.9, min_p=0.01,
             masked=0.2),
        # 512 windows of eight positions drawn from the whole distribution, as rejection sampling wants it
        dict(name="sample_windows", op="sample", rows=4096, vocab=128256, dtype="bf16", temperature=1.0, top_k=0, top_p=1.0, min_p=0.0,
             masked=0.0),
        # logits kept in full precision
        dict(name="sample_full_precision", op="sample", rows=512, vocab=152064, dtype="f32", temperature=1.3, top_k=0, top_p=0.9, min_p=0.0,
             masked=0.0),
        # the last norm of one window, the block's output added to the residual stream
        dict(name="rms_one_window", op="rms", rows=8, width=4096, dtype="f16", params="f16", residual=True, checkpoint=False, packed=False),
        # a long batch whose norm feeds an 8-bit product
        dict(name="rms_packed", op="rms", rows=16384, width=4096, dtype="bf16", params="bf16", residual=True, checkpoint=False, packed=True),
        # odd sizes in full precision, without a residual
        dict(name="rms_grad_odd", op="rms_grad", rows=1003, width=1531, dtype="f32", params="f32", residual=False, checkpoint=False),
        # the gradient of a long batch, the norm's input kept in 8 bits, joined by the residual stream's gradient
        dict(name="rms_grad_checkpoint", op="rms_grad", rows=16384, width=4096, dtype="bf16", params="f32", residual=True, checkpoint=True),
        # a drafter of one layer with its head: few large tensors and the norms' vectors
        dict(name="clip_drafter", op="clip", layers=1, width=4096, inner=12288, vocab=128256, dtype="bf16", tight=False),
        # a deep, narrow model: 217 small tensors
        dict(name="clip_many_small", op="clip", layers=24, width=128, inner=512, vocab=1000, dtype="f32", tight=False),
        # odd widths, tensors one behind the other without padding
        dict(name="clip_odd", op="clip", layers=3, width=1531, inner=4099, vocab=0, dtype="f16", tight=True),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["sample", "sample", "rms", "rms_grad", "clip"])
    if op == "sample":
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        while True:
            r, v = _log_uniform(rng, 1, 4096), _log_uniform(rng, 1000, 152064)
            if rng.random() < 0.5:
                v = v // 64 * 64
            if r * v * (2 if dtype == "f32" else 1) <= MOST_LOGITS:
                break
        return dict(op=op, rows=r, vocab=v, dtype=dtype, temperature=rng.choice([0.6, 0.7, 1.0, 1.3]),
                    top_k=rng.choice([0, 0, 1, 20, 50, 1000]), top_p=rng.choice([1.0, 1.0, 0.95, 0.9, 0.5]),
                    min_p=rng.choice([0.0, 0.0, 0.01, 0.1]), masked=rng.choice([0.0, 0.0, 0.3, 0.95]))
    if op == "clip":
        while True:
            c = dict(op=op, layers=_log_uniform(rng, 1, 32), width=_log_uniform(rng, 64, 4096), inner=0,
                     vocab=rng.choice([0, _log_uniform(rng, 1000, 152064)]), dtype=rng.choice(["bf16", "f16", "f32"]),
                     tight=rng.choice([False, False, True]))
            c["inner"] = int(c["width"] * rng.uniform(2.0, 4.0))
            n = sum(math.prod(s) for s in _gradient_shapes(c)[0])
            if n * (2 if c["dtype"] == "f32" else 1) <= MOST_GRADIENTS:
                return c
    while True:
        r, d = _log_uniform(rng, 1, 32768), _log_uniform(rng, 64, 8192)
        if rng.random() < 0.6:
            d = max(64, d // 64 * 64)
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        if r * d * (2 if dtype == "f32" else 1) <= MOST_ELEMENTS:
            break
    c = dict(op=op, rows=r, width=d, dtype=dtype, params=rng.choice(["f32", dtype]), residual=rng.choice([True, True, False]),
             checkpoint=rng.choice([False, True]))
    if op == "rms":
        c["packed"] = rng.choice([False, True])
    return c


def _gradient_shapes(case):
    """Shapes of a model's weights (in the case's type) and of its norms' vectors (float32)."""
    d, f, n = case["width"], case["inner"], case["layers"]
    big = ([(d, d)] * 4 + [(f, d)] * 2 + [(d, f)]) * n + ([(case["vocab"], d)] if case["vocab"] else [])
    return big, [(d,)] * (2 * n)


def _views(flat, shapes, pad):
    out, at = [], 0
    for s in shapes:
        n = math.prod(s)
        out.append(flat[at:at + n].view(s))
        at += -(-n // pad) * pad
    return out


def _flat(shapes, pad, dtype):
    return torch.zeros(max(1, sum(-(-math.prod(s) // pad) * pad for s in shapes)), dtype=dtype, device=DEV)


def _activations(r, d, g):
    """A residual stream: unit noise, a few channels much larger than the others."""
    gain = torch.exp(0.5 * torch.randn(d, generator=g, device=DEV))
    gain[torch.randint(0, d, (max(1, d // 256),), generator=g, device=DEV)] *= 20.0
    return torch.randn((r, d), generator=g, device=DEV) * gain


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    s = dict(case=case)
    if case["op"] == "sample":
        r, v = case["rows"], case["vocab"]
        logits = torch.empty((r, v), dtype=dt, device=DEV)
        for i in range(0, r, 256):                          # -ln(rank) with noise, as a language model's logits fall off
            n = min(256, r - i)
            z = torch.rand((n, v), generator=g, device=DEV).mul_(v - 1).add_(1.0).log_().neg_()
            z.add_(torch.randn((n, v), generator=g, device=DEV))
            if case["masked"] > 0:
                z[:, torch.rand(v, generator=g, device=DEV) < case["masked"]] = -math.inf
                z[:, 0] = z[:, 0].clamp(min=-20.0)          # something stays allowed
            logits[i:i + n] = z
        s["logits"] = logits
        s["uniforms"] = torch.rand(r, generator=g, device=DEV)
        return s
    if case["op"] == "clip":
        pad = 1 if case["tight"] else 64
        big, small = _gradient_shapes(case)
        s["flat"] = [_flat(big, pad, dt), _flat(small, pad, torch.float32)]
        s["grads"] = _views(s["flat"][0], big, pad) + _views(s["flat"][1], small, pad)
        for t in s["grads"]:
            t.copy_(torch.randn(t.shape, generator=g, device=DEV, dtype=torch.float32 if dt is torch.float32 else dt).mul_(3e-3))
        s["out_flat"] = [torch.zeros_like(f) for f in s["flat"]]
        s["out"] = _views(s["out_flat"][0], big, pad) + _views(s["out_flat"][1], small, pad)
        return s
    r, d = case["rows"], case["width"]
    x = _activations(r, d, g)
    s["weight"] = (1.0 + 0.2 * torch.randn(d, generator=g, device=DEV)).to(DTYPES[case["params"]])
    if case["op"] == "rms":
        s["x"] = x.to(dt)
        s["residual"] = (2.0 * torch.randn((r, d), generator=g, device=DEV)).to(dt) if case["residual"] else None
        return s
    x = x.to(dt)
    s["rstd"] = torch.rsqrt(x.double().square().mean(1) + EPS).float()
    s["grad_y"] = (0.1 * torch.randn((r, d), generator=g, device=DEV)).to(dt)
    s["grad_sum"] = (0.1 * torch.randn((r, d), generator=g, device=DEV)).to(dt) if case["residual"] else None
    if case["checkpoint"]:
        s["packed"], s["scale"] = _pack(x)
    else:
        s["x"] = x
    return s


def _pack(x):
    """8-bit form: blocks of 128 along a row share 2^e, the smallest power of two that brings the block's largest
    magnitude to 448 or less; values are rounded to nearest even in e4m3."""
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
    e = scale.int() - 127
    return torch.ldexp(q.float(), e.repeat_interleave(BLOCK, 1)[:, :q.shape[1]])


def _plain_sample(s):
    c = s["case"]
    z, at = torch.sort(s["logits"].float(), dim=1, descending=True, stable=True)
    finite = (z > -math.inf).sum(1)
    top = z[:, :1].double()
    w = torch.exp((z.double() - top) / c["temperature"])     # 64 bits: a draw lies next to one of many borders
    total = torch.cumsum(w, 1)
    n = finite.clamp(max=c["top_k"]) if c["top_k"] else finite
    mass = total.gather(1, n[:, None] - 1)
    if c["top_p"] < 1.0:
        n = torch.minimum((total < c["top_p"] * mass).sum(1) + 1, n)
    if c["min_p"] > 0.0:
        n = torch.minimum((w >= c["min_p"]).sum(1), n)
    mass = total.gather(1, n[:, None] - 1)
    j = torch.minimum((total <= s["uniforms"].double()[:, None] * mass).sum(1), n - 1)[:, None]
    logp = (z.gather(1, j).double() - top) / c["temperature"] - mass.log()
    return {"tokens": at.gather(1, j)[:, 0].int(), "logp": logp[:, 0].float(), "kept": n.int()}


def _plain_clip(s):
    total = sum(f.float().square().sum(dtype=torch.float64) for f in s["flat"])
    norm = total.sqrt()
    factor = torch.clamp(1.0 / norm, max=1.0).float()
    return {"norm": norm.float(), "out": [(f.float() * factor).to(f.dtype) for f in s["flat"]]}


def _plain(s):
    c = s["case"]
    if c["op"] == "sample":
        return _plain_sample(s)
    if c["op"] == "clip":
        return _plain_clip(s)
    dt, w = DTYPES[c["dtype"]], s["weight"].float()
    if c["op"] == "rms":
        out = {}
        x = s["x"]
        if s["residual"] is not None:
            out["sum"] = x = (x.float() + s["residual"].float()).to(dt)
        f = x.float()
        out["rstd"] = torch.rsqrt(f.square().mean(1) + EPS)
        y = f * out["rstd"][:, None] * w
        if c["packed"]:
            out["y"] = _unpack(*_pack(y)).to(dt)             # as the values that the 8 bits stand for
        else:
            out["y"] = y.to(dt)
        if c["checkpoint"]:
            out["packed"], out["scale"] = _pack(x)
        return out
    x = _unpack(s["packed"], s["scale"]) if c["checkpoint"] else s["x"].float()
    gy = s["grad_y"].float()
    xh = x * s["rstd"][:, None]
    a = gy * w
    gx = (a - xh * (a * xh).mean(1, keepdim=True)) * s["rstd"][:, None]
    if s["grad_sum"] is not None:
        gx = gx + s["grad_sum"].float()
    return {"grad_x": gx.to(dt), "grad_weight": (gy * xh).sum(0).to(s["weight"].dtype)}


def run(state):
    if not own:
        return _plain(state)
    from paper_2605_14978_b200 import binding as B
    c = state["case"]
    if c["op"] == "sample":
        return B.sample_tokens(state["logits"], state["uniforms"], temperature=c["temperature"], top_k=c["top_k"], top_p=c["top_p"],
                               min_p=c["min_p"])
    if c["op"] == "clip":
        return {"norm": B.clip_gradients(state["grads"], 1.0, out=state["out"]), "out": state["out_flat"]}
    if c["op"] == "rms":
        out = B.rms_norm(state["x"], state["weight"], state["residual"], eps=EPS, checkpoint=c["checkpoint"], packed_output=c["packed"])
        if c["packed"]:
            out["y"] = B.unpack_activation(out.pop("y_packed"), out.pop("y_scale"), state["x"].dtype)
        return out
    x = (state["packed"], state["scale"]) if c["checkpoint"] else state["x"]
    gx, gw = B.rms_norm_backward(state["grad_y"], x, state["weight"], state["rstd"], grad_sum=state["grad_sum"])
    return {"grad_x": gx, "grad_weight": gw}


def work(case):
    es = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "sample":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * es + 16 * case["rows"], "flops": 4.0 * n}
    if case["op"] == "clip":
        big, small = (sum(math.prod(s) for s in part) for part in _gradient_shapes(case))
        return {"bytes": 2 * (big * es + small * 4), "flops": 3.0 * (big + small)}
    r, d = case["rows"], case["width"]
    ps = 4 if case["params"] == "f32" else 2
    q = r * d + r * ((d + BLOCK - 1) // BLOCK)
    if case["op"] == "rms":
        rows = (3 if case["residual"] else 1) * r * d * es + (2 * q if case["packed"] else 0) + r * d * es + (q if case["checkpoint"] else 0)
        return {"bytes": rows + 4 * r + d * ps, "flops": 5.0 * r * d}
    saved = q if case["checkpoint"] else r * d * es
    return {"bytes": (3 if case["residual"] else 2) * r * d * es + saved + 4 * r + 2 * d * ps, "flops": 10.0 * r * d}


def _exact_pack(v):
    """The 8-bit format from its definition, in float64: values before scaling, and the exponents."""
    blocks = [v[:, i:i + BLOCK] for i in range(0, v.shape[1], BLOCK)]
    top = torch.stack([b.abs().max(1).values for b in blocks], 1)
    e = torch.ceil(torch.log2(top / 448.0))
    e = torch.where(top / torch.exp2(e - 1) <= 448.0, e - 1, e)          # the logarithm may be off by one at a border
    e = torch.where(top / torch.exp2(e) > 448.0, e + 1, e)
    e = torch.where(top > 0, e.clamp(min=-126.0), torch.full_like(e, -126.0))
    u = torch.cat([b / torch.exp2(e[:, i:i + 1]) for i, b in enumerate(blocks)], 1)
    _, ex = torch.frexp(u)
    step = torch.exp2((ex - 1).clamp(min=-6).double() - 3.0)              # spacing of e4m3 around u
    return torch.round(u / step) * step, e


def _exact_values(q, e):
    return torch.cat([q[:, i * BLOCK:(i + 1) * BLOCK] * torch.exp2(e[:, i:i + 1]) for i in range(e.shape[1])], 1)


def _exact_sample(case, s):
    tokens, logps, kept = [], [], []
    step = max(1, (1 << 27) // case["vocab"])
    for i in range(0, case["rows"], step):
        z = s["logits"][i:i + step].double() / case["temperature"]
        order = torch.argsort(-z, dim=1, stable=True)
        p = torch.softmax(z, 1).gather(1, order)
        rank = torch.arange(case["vocab"], device=DEV)[None]
        keep = torch.isfinite(z).gather(1, order)
        if case["top_k"]:
            keep &= rank < case["top_k"]
        p = torch.where(keep, p, 0.0)
        p /= p.sum(1, keepdim=True)
        if case["top_p"] < 1.0:
            keep &= (p.cumsum(1) - p) < case["top_p"]         # what comes before has not reached it yet
        if case["min_p"] > 0.0:
            keep &= p >= case["min_p"] * p[:, :1] * (1 - 1e-15)
        p = torch.where(keep, p, 0.0)
        p /= p.sum(1, keepdim=True)
        n = keep.sum(1)
        j = torch.minimum((p.cumsum(1) <= s["uniforms"][i:i + step].double()[:, None]).sum(1), n - 1)[:, None]
        tokens.append(order.gather(1, j)[:, 0])
        logps.append(p.gather(1, j)[:, 0].log())
        kept.append(n)
    return {"tokens": torch.cat(tokens).int(), "logp": torch.cat(logps), "kept": torch.cat(kept).int()}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "sample":
        return _exact_sample(case, s)
    if case["op"] == "clip":
        norm = torch.stack([torch.linalg.vector_norm(t, dtype=torch.float64) for t in s["grads"]]).norm()
        return {"norm": norm, "out": [f.double() * min(1.0, 1.0 / float(norm)) for f in s["flat"]]}
    w = s["weight"].double()[None, :]
    if case["op"] == "rms":
        out = {}
        x = s["x"].double()
        if s["residual"] is not None:
            x = (x + s["residual"].double()).to(DTYPES[case["dtype"]]).double()      # the norm reads what is stored
            out["sum"] = x
        rstd = 1.0 / torch.sqrt((x * x).sum(1) / x.shape[1] + EPS)
        out["rstd"] = rstd
        y = x * rstd[:, None] * w
        out["y"] = _exact_values(*_exact_pack(y)) if case["packed"] else y
        if case["checkpoint"]:
            q, e = _exact_pack(x)
            out["packed"], out["scale"] = q, (e + 127).to(torch.int64)
        return out
    x = _exact_values(s["packed"].double(), s["scale"].double() - 127.0) if case["checkpoint"] else s["x"].double()
    gy, rstd, d = s["grad_y"].double(), s["rstd"].double()[:, None], x.shape[1]
    a = gy * w
    gx = rstd * a - x * rstd ** 3 * ((a * x).sum(1, keepdim=True) / d)
    if s["grad_sum"] is not None:
        gx += s["grad_sum"].double()
    return {"grad_x": gx, "grad_weight": (gy * x * rstd).sum(0)}
