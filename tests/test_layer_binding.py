"""The Python binding of the operators of selective state-space layers against a library that only records its calls:
no GPU."""
import pytest
import torch

import paper_2606_27748_amd as F
from tests.seq_util import BF16, F32, offsets
from tests.test_seq_binding import _refused, calls  # noqa: F401

T, D, K, H, N, P = 5, 16, 4, 2, 64, 64


def io(*shape):
    return torch.zeros(*shape, dtype=BF16)


def f32(*shape):
    return torch.zeros(*shape)


def _rows():
    return [io(T, H, P), io(T, 1, N), io(T, 1, N), f32(T, H), f32(T, H), f32(H)]


def _entries():
    """(entry, descriptor, needed arguments by position, which of them may be None)"""
    off, saved = offsets([T]), torch.zeros(4096, dtype=torch.uint8)
    conv, scan, norm = F.make_conv_desc(1, T, D, K), F.make_scan_desc(1, 1, H, N, P, T), F.make_norm_desc(T, D, D)
    step = [x[:1].contiguous() for x in _rows()[:5]] + [f32(H)]
    return [
        (F.flex_conv_fwd, conv, [io(T, D), f32(D, K), f32(D), off], {2}),
        (F.flex_conv_bwd, conv, [io(T, D), f32(D, K), f32(D), off, io(T, D)], {2}),
        (F.flex_conv_step, F.make_conv_desc(1, 1, D, K), [io(1, D), f32(D, K), f32(D), io(1, K - 1, D)], {2}),
        (F.flex_scan_fwd, scan, [*_rows(), off], {5}),
        (F.flex_scan_bwd, scan, [*_rows(), off, io(T, H, P), saved], {5}),
        (F.flex_scan_step, F.make_scan_desc(1, 1, H, N, P, 1), [*step, f32(1, H, N, P)], {5}),
        (F.flex_norm_fwd, norm, [io(T, D), io(T, D), f32(D)], set()),
        (F.flex_norm_bwd, norm, [io(T, D), io(T, D), f32(D), io(T, D)], set()),
    ]


@pytest.mark.parametrize("i", range(8))
def test_missing_and_other_tensors_are_refused(calls, i):  # noqa: F811
    """A needed tensor that is None, of another type, another shape or with gaps is the binding's own error, and
    nothing is called."""
    _, seen = calls
    entry, desc, ok, free = _entries()[i]
    for k, x in enumerate(ok):
        is_saved = x.dtype is torch.uint8
        status = F.FLEX_ERR_WORKSPACE if is_saved else F.FLEX_ERR_INVALID_ARG
        wrong = [x[:-1]] if is_saved else [x.double(), torch.cat([x, x])]
        if not is_saved and x.dim() > 1:
            wrong.append(torch.cat([x, x], -1)[..., :x.shape[-1]] if x.shape[0] > 1 else torch.cat([x, x], -1))
        for y in wrong + ([] if k in free else [None]):
            _refused(lambda: entry(desc, *ok[:k], y, *ok[k + 1:]), status)
    assert seen == []
    entry(desc, *ok)
    for k in free:
        entry(desc, *ok[:k], None, *ok[k + 1:])
    assert [n for n, _, _ in seen] == [entry.__name__] * (1 + len(free))


@pytest.mark.parametrize("small", [False, True])
@pytest.mark.parametrize("i", [1, 3, 4, 7])
def test_workspace_lives_until_the_call_returns(calls, i, small):  # noqa: F811
    made, seen = calls
    entry, desc, ok, _ = _entries()[i]
    entry(desc, *ok, ws=torch.zeros(16, dtype=torch.uint8) if small else None)
    assert len(seen) == 1 and len(made) == 1 and seen[0][2] == [True]
    assert made[0]() is None   # and no longer


@pytest.mark.parametrize("i", [1, 3, 4, 7])
def test_workspace_of_the_caller(calls, i):  # noqa: F811
    made, seen = calls
    entry, desc, ok, _ = _entries()[i]
    ws = torch.zeros(5000, dtype=torch.uint8)
    entry(desc, *ok, ws=ws)
    assert made == [] and seen[0][1][-3:-1] == (ws.data_ptr(), 5000)


def test_strided_gradients(calls):  # noqa: F811
    """Gradients of slices: given ones must have the descriptor's strides, new ones get them."""
    _, _ = calls
    entry, desc, ok, _ = _entries()[4]
    desc.dx_stride, desc.db_stride = H * P + 8, N + 8
    got = entry(desc, *ok)
    assert got["dX"].stride() == (H * P + 8, P, 1) and got["dB"].stride() == (N + 8, N, 1) and got["dC"].is_contiguous()
    assert got["dX"].shape == (T, H, P) and got["dX"].dtype is BF16 and got["dD"].dtype is F32
    wide = io(T, H * P + 8)[:, :H * P].unflatten(1, (H, P))
    assert entry(desc, *ok, dX=wide)["dX"] is wide
    _refused(lambda: entry(desc, *ok, dX=io(T, H, P)))


def test_what_is_not_asked_for(calls):  # noqa: F811
    _, seen = calls
    entry, desc, ok, _ = _entries()[1]
    assert entry(desc, *ok[:2], None, *ok[3:])["dbias"] is None
    entry, desc, ok, _ = _entries()[4]
    assert entry(desc, *ok[:5], None, *ok[6:])["dD"] is None
    none = F.make_norm_desc(T, D, D, gate="none")
    x, w = io(T, D), f32(D)
    assert F.flex_norm_bwd(none, x, None, w, x)["dZ"] is None
    n = len(seen)
    _refused(lambda: F.flex_norm_fwd(none, x, x, w))
    _refused(lambda: F.flex_norm_bwd(none, x, None, w, x, dZ=x))
    assert len(seen) == n
