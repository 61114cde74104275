"""Selective scan where sequences go in segments of several chunks, whose loops have one chunk's rows on their way while another is
worked on: every value against float64 (tests.scan_chunks), and against the recurrence; calls of millions of values; values
that are not finite."""
import pytest
import torch

from tests import scan_chunks
from tests.layer_util import SCAN_ROWS, near, scan_desc, scan_oracle
from tests.seq_util import BF16, F32

pytestmark = pytest.mark.gpu
IDS = [f"{n}x{p}-{g}-{h}" for n, p, g, h, _ in scan_chunks.MANY_CHUNKS]
GRADS = ("dX", "dB", "dC", "ddt", "dg", "dD")


@pytest.fixture(scope="module")
def F():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2606_27748_amd as F
    F.load()
    return F


def run(F, x, dtype, start, backward=True, in_place=False):
    desc = scan_desc(F, x, dtype)
    args = [desc, *(x[n] for n in SCAN_ROWS), x["off"]]
    s0 = x["state0"].clone() if start else None
    saved = torch.empty(F.scan_saved_size(desc), dtype=torch.uint8, device="cuda") if backward else None
    Y, state = F.flex_scan_fwd(*args, state0=s0, state=s0 if in_place else None, saved=saved, want_state=True)
    out = {"Y": Y, "state": state}
    return {**out, **F.flex_scan_bwd(*args, x["dY"], saved)} if backward else out


def check(F, x, dtype, start):
    ref, mag = scan_chunks.results(x, start)
    bound = scan_chunks.bounds(x, ref, mag, dtype, start)
    got = run(F, x, dtype, start)
    for n in ("Y", "state", "dX", "dB", "dC", "dD"):
        scan_chunks.hold(n, got[n], ref[n], bound[n])
    # not held to bounds of their own: the 2-norms of the small tests
    near("ddt", got["ddt"], ref["ddt"].cpu(), 1e-2 if dtype == BF16 else 1.2e-5)
    return got


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,P,G,H,lengths", scan_chunks.MANY_CHUNKS, ids=IDS)
@pytest.mark.parametrize("start", [False, True])
def test_every_value(F, start, N, P, G, H, lengths, dtype):
    assert scan_chunks.tokens_of_a_segment(F, len(lengths), sum(lengths), G, H, N, P) >= 128
    x = scan_chunks.inputs(lengths, G, H, N, P, dtype, N + H, "cuda")
    got = check(F, x, dtype, start)
    # without what a backward needs, and in place: the same bits; and once more
    alone = run(F, x, dtype, start, backward=False, in_place=start)
    assert torch.equal(alone["Y"], got["Y"]) and torch.equal(alone["state"], got["state"])
    again = run(F, x, dtype, start)
    assert all(torch.equal(again[n], v) for n, v in got.items())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("which", [0, 3])
def test_the_recurrence(F, which, dtype):
    """All gradients, against the recurrence token by token."""
    N, P, G, H, lengths = scan_chunks.MANY_CHUNKS[which]
    x = scan_chunks.inputs(lengths, G, H, N, P, dtype, 5 + which, "cuda")
    with torch.device("cuda"):
        ref = {k: v.cpu() for k, v in scan_oracle(x, True, grads=True).items()}
    got = run(F, x, dtype, True)
    near("Y", got["Y"], ref["Y"], 3.4e-3 if dtype == BF16 else 2.4e-6)
    near("state", got["state"], ref["state"], 2.4e-6)
    for n in GRADS:
        near(n, got[n], ref[n], 1e-2 if dtype == BF16 and n != "dD" else 1.2e-5)


@pytest.mark.parametrize("N,P,G,H,dtype,lengths", [
    (128, 64, 1, 64, BF16, [8000, 1, 5300, 3083]), (128, 128, 2, 16, BF16, [20000, 77, 4500]),
    (64, 64, 4, 32, BF16, [8192, 8192]), (64, 64, 1, 24, F32, [9000, 63, 300]), (128, 128, 2, 8, F32, [8192])])
def test_every_value_of_a_large_call(F, N, P, G, H, dtype, lengths):
    """Tens of millions of values, of which one that a store left wrong would be off by about its own size: bounds are
    two hundredths of it, of dB and dC up to a tenth.  Three times over, the same bits."""
    x = scan_chunks.inputs(lengths, G, H, N, P, dtype, 3, "cuda")
    got = check(F, x, dtype, False)
    for _ in range(2):
        again = run(F, x, dtype, False)
        assert all(torch.equal(again[n], v) for n, v in got.items())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("which", [0, 1, 2])
@pytest.mark.parametrize("name", ["X", "Bt", "Ct", "dt", "g"])
def test_rows_that_are_not_finite_reach_no_earlier_token(F, name, which, dtype):
    """In the first chunk of a segment, in a later one, in a later segment."""
    N, P, G, H, lengths = scan_chunks.MANY_CHUNKS[which]
    x = scan_chunks.inputs(lengths, G, H, N, P, dtype, 7, "cuda")
    clean = run(F, x, dtype, False, backward=False)
    end, r = lengths[0], H // G
    for row, value in ((20, float("nan")), (100, float("inf")), (end - 300, float("nan"))):
        h, c = H // 2, 37
        at = {"X": (row, h, c), "Bt": (row, h // r, 5), "Ct": (row, h // r, 5)}.get(name, (row, h))
        y = dict(x, **{name: x[name].clone()})
        y[name][at] = value
        got = run(F, y, dtype, False, backward=False)
        heads = slice(h // r * r, h // r * r + r) if name in ("Bt", "Ct") else slice(h, h + 1)
        hit = torch.zeros_like(got["Y"], dtype=torch.bool)
        hit[row:row + 1 if name == "Ct" else end, heads, slice(c, c + 1) if name == "X" else slice(None)] = True
        assert torch.equal(got["Y"][~hit], clean["Y"][~hit]) and not torch.isfinite(got["Y"][hit]).any()
        hit = torch.zeros_like(got["state"], dtype=torch.bool)
        if name != "Ct":
            hit[0, heads, :, slice(c, c + 1) if name == "X" else slice(None)] = True
        assert torch.equal(got["state"][~hit], clean["state"][~hit])
        if name in ("X", "dt", "g"):
            assert not torch.isfinite(got["state"][hit]).any()
