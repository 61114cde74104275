"""The Python binding of the packed-sequence operators against a library that only records its calls: no GPU."""
import ctypes
import weakref

import pytest
import torch

import paper_2606_27748_amd as F
from paper_2606_27748_amd import _lib
from tests.seq_util import BF16, offsets


class Recorder:
    """Stands for the library: sizing calls answer 4096 bytes, the others call `entered` with their name."""
    flex_status_string = staticmethod(lambda status: b"refused")

    def __init__(self, entered):
        self.entered = entered

    def __getattr__(self, name):
        if name.endswith("_size"):
            def size(desc, *args):
                ctypes.cast(args[-1], ctypes.POINTER(ctypes.c_size_t))[0] = 4096
                return F.FLEX_OK
            return size

        def call(*args):
            self.entered(name, args)
            return F.FLEX_OK
        return call


@pytest.fixture
def calls(monkeypatch):
    """Calls run on tensors of the CPU up to the library's door; what they allocate is in `made` (weak references)."""
    made, seen = [], []
    empty = torch.empty

    def counted(*a, **k):
        t = empty(*a, **k)
        if k.get("dtype") is torch.uint8:
            made.append(weakref.ref(t))
        return t

    def entered(name, args):
        seen.append((name, args, [r() is not None for r in made]))

    monkeypatch.setattr(_lib, "load", lambda: Recorder(entered))
    monkeypatch.setattr(torch, "empty", counted)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: None)   # the index of a CPU tensor's device
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: 0, raising=False)
    check = _lib._expect

    class OnGpu:
        type = "cuda"

        def __eq__(self, other):
            return True

    monkeypatch.setattr(_lib, "_expect", lambda what, dev, *a, **k: check(what, OnGpu(), *a, **k))
    return made, seen


def _attn():
    desc = F.make_attn_desc(1, 2, 1, 32, 5, 5)
    q, k, off = torch.zeros(5, 2, 32, dtype=BF16), torch.zeros(5, 1, 32, dtype=BF16), offsets([5])
    return desc, q, k, off


def _delta():
    desc = F.make_delta_desc(1, 1, 2, 64, 5)
    q, v, off = torch.zeros(5, 1, 64, dtype=BF16), torch.zeros(5, 2, 64, dtype=BF16), offsets([5])
    g = torch.zeros(5, 2)
    return desc, (q, q, v, g, g, off), v, torch.zeros(4096, dtype=torch.uint8)


def _run(name, ws):
    if name.startswith("flex_attn"):
        desc, q, k, off = _attn()
        if name == "flex_attn_fwd":
            return F.flex_attn_fwd(desc, q, k, k, off, off, ws=ws)
        return F.flex_attn_bwd(desc, q, k, k, off, off, q, torch.zeros(5, 2), q, ws=ws)
    desc, rows, dO, saved = _delta()
    return F.flex_delta_fwd(desc, *rows, ws=ws) if name == "flex_delta_fwd" else F.flex_delta_bwd(desc, *rows, dO, saved, ws=ws)


@pytest.mark.parametrize("small", [False, True])
@pytest.mark.parametrize("name", ["flex_attn_fwd", "flex_attn_bwd", "flex_delta_fwd", "flex_delta_bwd"])
def test_workspace_lives_until_the_call_returns(calls, name, small):
    """A workspace that the binding allocates is still held when the library queues its kernels: freed before, another
    thread could be given its memory."""
    made, seen = calls
    _run(name, torch.zeros(16, dtype=torch.uint8) if small else None)
    assert len(seen) == 1 and seen[0][0] == name and len(made) == 1
    assert seen[0][2] == [True]
    assert made[0]() is None   # and no longer


@pytest.mark.parametrize("name", ["flex_attn_fwd", "flex_attn_bwd", "flex_delta_fwd", "flex_delta_bwd"])
def test_workspace_of_the_caller(calls, name):
    made, seen = calls
    ws = torch.zeros(5000, dtype=torch.uint8)
    _run(name, ws)
    assert made == [] and seen[0][1][-3:-1] == (ws.data_ptr(), 5000)


def _refused(f, status=F.FLEX_ERR_INVALID_ARG):
    with pytest.raises(F.FlexError) as e:
        f()
    assert e.value.status == status


def test_missing_tensors_are_refused(calls):
    """A required tensor that is None is the binding's own error, and nothing is called."""
    _, seen = calls
    desc, q, k, off = _attn()
    lse = torch.zeros(5, 2)
    for entry, ok in ((F.flex_attn_fwd, [q, k, k, off, off]), (F.flex_attn_bwd, [q, k, k, off, off, q, lse, q])):
        for i in range(len(ok)):
            _refused(lambda: entry(desc, *ok[:i], None, *ok[i + 1:]))
    desc, rows, dO, saved = _delta()
    state = torch.zeros(1, 2, 64, 64)
    one = [x[:1].contiguous() for x in rows[:5]]
    for entry, d, ok in ((F.flex_delta_fwd, desc, [*rows]), (F.flex_delta_bwd, desc, [*rows, dO]),
                         (F.flex_delta_step, F.make_delta_desc(1, 1, 2, 64, 1), [*one, state])):
        more = [saved] if entry is F.flex_delta_bwd else []
        for i in range(len(ok)):
            _refused(lambda: entry(d, *ok[:i], None, *ok[i + 1:], *more))
    _refused(lambda: F.flex_delta_bwd(desc, *rows, dO, None), F.FLEX_ERR_WORKSPACE)
    assert seen == []
    F.flex_delta_step(F.make_delta_desc(1, 1, 2, 64, 1), *one, state)   # what may be left out
    assert [n for n, _, _ in seen] == ["flex_delta_step"]
