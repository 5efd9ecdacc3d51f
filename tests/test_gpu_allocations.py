"""What the wrappers allocate is seen by dispatch modes and the profiler, and filled where deterministic algorithms ask for it, as the tensors of
torch's own functions are."""
import pytest
import torch
from torch.utils._python_dispatch import TorchDispatchMode

from paper_2605_14978_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


class Allocations(TorchDispatchMode):
    def __init__(self):
        super().__init__()
        self.made = []

    def __torch_dispatch__(self, func, types, args=(), kwargs=None):
        out = func(*args, **(kwargs or {}))
        if func is torch.ops.aten.empty.memory_format:
            self.made.append(out.data_ptr())
        return out


def calls():
    """Name, call, how many tensors it allocates: outputs, and a workspace where there is one."""
    x, gain, h = torch.randn((6, 64), device=DEV).bfloat16(), torch.ones(64, device=DEV), torch.randn((300, 64), device=DEV).bfloat16()
    y, u, g = torch.zeros(6, dtype=torch.int32, device=DEV), torch.rand(6, device=DEV), torch.randn(6, device=DEV)
    n, r, lse = B.layer_norm(x, gain, gain), B.rms_norm(x, gain), B.head_logprob(x, h, y)["lse"]
    packed = B.pack_activation(x)
    yield "layer_norm", lambda: B.layer_norm(x, gain, gain, checkpoint=True), 5
    yield "layer_norm_backward", lambda: B.layer_norm_backward(x, x, gain, n["mean"], n["rstd"]), 4
    yield "pack_activation", lambda: B.pack_activation(x), 2
    yield "unpack_activation", lambda: B.unpack_activation(*packed), 1
    yield "head_logprob", lambda: B.head_logprob(x, h, y), 3
    yield "head_logprob_backward", lambda: B.head_logprob_backward(x, h, y, lse, g), 3
    yield "rms_norm", lambda: B.rms_norm(x, gain, x, checkpoint=True), 5
    yield "rms_norm_backward", lambda: B.rms_norm_backward(x, x, gain, r["rstd"]), 3
    yield "gradient_norm", lambda: B.gradient_norm([x, gain]), 2
    yield "sample_tokens", lambda: B.sample_tokens(x, u), 3


def tensors(out):
    return [t for t in (out.values() if isinstance(out, dict) else out if isinstance(out, tuple) else [out]) if t is not None]


def test_dispatch_modes_see_what_is_allocated():
    for name, call, many in calls():
        with Allocations() as seen:
            out = call()
        assert len(seen.made) == many, (name, seen.made)
        assert all(t.data_ptr() in seen.made for t in tensors(out)), name
    torch.cuda.synchronize()


def test_the_profiler_sees_what_is_allocated():
    for name, call, many in calls():
        with torch.profiler.profile(activities=[torch.profiler.ProfilerActivity.CPU]) as p:
            call()
        assert sum(e.count for e in p.key_averages() if e.key == "aten::empty") == many, name
    torch.cuda.synchronize()


def test_deterministic_algorithms_fill_what_is_allocated():
    hidden, weight = torch.zeros((0, 64), dtype=torch.bfloat16, device=DEV), torch.zeros((300, 64), dtype=torch.bfloat16, device=DEV)
    tokens = torch.zeros(0, dtype=torch.int32, device=DEV)
    torch.use_deterministic_algorithms(True)
    try:
        got = B.head_logprob(hidden, weight, tokens, want_workspace=True)["_workspace"].clone()
    finally:
        torch.use_deterministic_algorithms(False)
    torch.cuda.synchronize()
    assert got.numel() > 1024 and torch.all(got[1024:] == 255)          # without tokens only the header is written
