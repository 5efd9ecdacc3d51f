"""The extension module that marshals the training-end calls is an addition: without it, or with one built against another torch, the
library loads, everything else is as it was, and the wrappers go their Python way."""
import sys

import pytest
import torch

import paper_2605_14978_b200 as package
from paper_2605_14978_b200 import binding as B
from paper_2605_14978_b200 import build as build_mod

NAMES = ("head_logprob", "head_logprob_backward", "layer_norm", "layer_norm_backward", "pack_activation", "unpack_activation")


@pytest.fixture(autouse=True)
def built():
    build_mod.build()
    B.load_library()


def fresh(monkeypatch):
    monkeypatch.setattr(B, "_lib", None)
    monkeypatch.setattr(B, "_calls", None)


def test_the_module_is_bound(monkeypatch):
    fresh(monkeypatch)
    B.load_library()
    assert B._calls.torch_version == torch.__version__ and all(hasattr(B._calls, n) for n in NAMES)


def test_a_missing_module_closes_nothing(monkeypatch):
    fresh(monkeypatch)
    monkeypatch.delattr(package, "_calls", raising=False)
    monkeypatch.setitem(sys.modules, package.__name__ + "._calls", None)          # its import fails
    with pytest.warns(RuntimeWarning, match="_calls.so does not load"):
        B.load_library()
    assert B.ppow_version() >= 100 and B.ppow_score_workspace_bytes(B.make_params(4, 8, 1000, B.PPOW_BF16, 0, 0.04)) > 0
    assert all(getattr(B._quick(), n)(1, 2, 3) is None for n in NAMES)
    h = torch.zeros((4, 16), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="CUDA device"):
        B.head_logprob(h, h, torch.zeros(4, dtype=torch.int32))
    with pytest.raises(ValueError, match="CUDA device"):
        B.pack_activation(h)


def test_a_module_of_another_torch_is_not_used_and_built_again(monkeypatch):
    fresh(monkeypatch)
    assert not build_mod.calls_are_stale()
    monkeypatch.setattr(torch, "__version__", "1.0.0")
    assert build_mod.calls_are_stale()
    with pytest.warns(RuntimeWarning, match="built against torch"):
        B.load_library()
    assert B._quick().pack_activation(None) is None


def test_the_library_is_built_before_the_module(monkeypatch, tmp_path):
    # what stops the module from building does not stop the library
    done = []
    monkeypatch.setattr(build_mod, "is_stale", lambda lib: True)
    monkeypatch.setattr(build_mod, "_build_library", lambda *a: done.append(a[0]))

    def fails(force):
        raise RuntimeError("no headers")
    monkeypatch.setattr(build_mod, "build_calls", fails)
    with pytest.raises(RuntimeError, match="no headers"):
        build_mod.build()
    assert done == [build_mod.LIB]


def variants():
    """(name, arguments): calls that are right in every layout that the documentation allows, and calls that are not."""
    dev, bf, f32 = "cuda:0", torch.bfloat16, torch.float32
    h, w = torch.randn((40, 64), device=dev).to(bf), torch.randn((300, 64), device=dev).to(bf)
    tok, f = torch.randint(0, 300, (40,), device=dev, dtype=torch.int32), torch.randn(40, device=dev)
    wide = torch.randn((40, 200), device=dev).to(bf)
    for x in (h, wide[:, 8:72], wide[:, 3:67], h[:1], h[:0], h[::2], wide[:1, 3:67], h.t().contiguous().t(), h[0].expand(40, 64), h.float(), h.half(), h[0],
              h.cpu(), h[:, :63], h[:, :8], h[None]):
        n = x.shape[0] if x.dim() == 2 else 40
        for weight in (w, torch.randn((300, 80), device=dev).to(bf)[:, 8:72], w[:1], w[:, 4:], w.float(), w.cpu(), w[:, :8]):
            yield "head_logprob", (x, weight, tok[:n], 1.0, False)
        for y in (tok[:n].long(), tok[:n - 1], torch.stack([tok, tok], 1)[:n, 0], tok[:n].cpu()):
            yield "head_logprob", (x, w, y, 1.0, False)
        for lse, g in ((f[:n], f[:n]), (f[:n].half(), f[:n]), (f[:n], torch.stack([f, f], 1)[:n, 0]), (f[:n].cpu(), f[:n])):
            yield "head_logprob_backward", (x, w, tok[:n], lse, g, 1.0, True, True, False)
        d = x.shape[-1]
        for gain in (torch.ones(d, device=dev), torch.ones(d, device=dev, dtype=bf), torch.ones(d, device=dev).half(), torch.ones(d + 1, device=dev),
                     torch.ones(d), torch.ones((1, d), device=dev)):
            yield "layer_norm", (x, gain, None, 1e-5, True)
            yield "layer_norm", (x, gain, gain, 1e-5, False)
            yield "layer_norm", (x, gain, torch.ones(d, device=dev, dtype=torch.float64), 1e-5, False)
            yield "layer_norm_backward", (h[:n, :d] if d <= 64 else h, x, None, None, gain, f[:n], f[:n], True)
        yield "pack_activation", (x,)
    q, s = B.pack_activation(h)
    for a, b in ((q, s), (q[:, :32], s), (q, s[:, :0]), (q.view(torch.uint8), s), (q[::2], s[::2]), (q, s.int()), (q.cpu(), s), (q[:0], s[:0])):
        yield "unpack_activation", (a, b, B.PPOW_BF16)
        yield "layer_norm_backward", (h[:a.shape[0]], None, a, b, torch.ones(64, device=dev), f[:a.shape[0]], f[:a.shape[0]], False)
    yield "layer_norm_backward", (h, None, None, None, torch.ones(64, device=dev), f, f, False)


def call(name, a):
    """The wrapper's call with these arguments: its outputs, or the exception's type."""
    try:
        if name == "head_logprob":
            out = list(B.head_logprob(a[0], a[1], a[2]).values())
        elif name == "head_logprob_backward":
            out = B.head_logprob_backward(*a[:5])
        elif name == "layer_norm":
            out = list(B.layer_norm(a[0], a[1], a[2], checkpoint=a[4]).values())
        elif name == "layer_norm_backward":
            out = B.layer_norm_backward(a[0], a[1] if a[2] is None else (a[2], a[3]), a[4], a[5], a[6], want_bias=a[7])
        elif name == "pack_activation":
            out = B.pack_activation(a[0])
        else:
            out = [B.unpack_activation(a[0], a[1])]
        return [None if t is None else t.float().nan_to_num() for t in out]
    except (ValueError, B.PpowError, AttributeError, TypeError) as e:
        return type(e)


@pytest.mark.gpu
def test_both_ways_accept_refuse_and_return_the_same(monkeypatch):
    quick, slow, tried, taken = B._quick(), B._NoCalls(), 0, 0
    for name, args in variants():
        monkeypatch.setattr(B, "_calls", quick)
        a = call(name, args)
        monkeypatch.setattr(B, "_calls", slow)
        b = call(name, args)
        tried += 1
        if isinstance(a, type) or isinstance(b, type):
            assert a is b, (name, a, b, [getattr(t, "shape", t) for t in args])
            continue
        assert len(a) == len(b) and all((x is None and y is None) or torch.equal(x, y) for x, y in zip(a, b)), name
        # what the Python way accepts on the current device and stream is not turned away by the module
        try:
            got = getattr(quick, name)(*args)
        except TypeError:
            got = None
        taken += got is not None
        assert got is not None and got[0] == B.PPOW_OK, (name, [getattr(t, "shape", t) for t in args])
    torch.cuda.synchronize()
    assert tried > 300 and taken > 60
