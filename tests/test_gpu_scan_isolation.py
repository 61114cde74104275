"""Selective scan, backward: what is not finite in a row of one sequence reaches no gradient of another one."""
import pytest
import torch

from tests import scan_chunks
from tests.layer_util import SCAN_ROWS, scan_desc
from tests.seq_util import BF16, F32

pytestmark = pytest.mark.gpu
# one part of a group's heads and several, one chunk a segment and several, states through LDS at once and one by one
CASES = [(64, 64, 4, 4, [60, 140, 50]), (64, 64, 1, 4, [60, 140, 50]), (128, 128, 1, 4, [1, 190, 64]), (128, 64, 3, 9, [64, 64, 64]),
         (64, 128, 2, 2, [0, 130, 3]), (64, 64, 16, 16, [700, 900, 500])]


@pytest.fixture(scope="module")
def F():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2606_27748_amd as F
    F.load()
    return F


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,P,G,H,lengths", CASES)
@pytest.mark.parametrize("start", [False, True])
def test_other_sequences_keep_their_gradients(F, start, N, P, G, H, lengths, dtype):
    x = scan_chunks.inputs(lengths, G, H, N, P, dtype, 4, "cuda")
    desc = scan_desc(F, x, dtype)
    # one workspace for all calls, as a program has it: what a call leaves there reaches no later one
    ws = torch.empty(max(F.scan_workspace_size(desc, p) for p in (F.FLEX_PASS_FWD, F.FLEX_PASS_BWD)), dtype=torch.uint8, device="cuda")
    saved = torch.empty(F.scan_saved_size(desc), dtype=torch.uint8, device="cuda")

    def grads(x):
        args = [desc, *(x[n] for n in SCAN_ROWS), x["off"]]
        F.flex_scan_fwd(*args, state0=x["state0"] if start else None, saved=saved, ws=ws)
        return F.flex_scan_bwd(*args, x["dY"], saved, ws=ws)

    clean = grads(x)
    a, b = lengths[0], lengths[0] + lengths[1]
    rows = torch.ones(sum(lengths), dtype=torch.bool)
    rows[a:b] = False
    for name in ("X", "Bt", "Ct", "dt", "g", "dY"):
        for row, value in ((a, float("nan")), (b - 1, float("inf")), ((a + b) // 2, float("nan"))):
            y = dict(x, **{name: x[name].clone()})
            y[name][row, -1] = value
            got = grads(y)
            for n in ("dX", "dB", "dC", "ddt", "dg"):
                assert torch.equal(got[n][rows], clean[n][rows]), (name, row, n)
    if start:
        y = dict(x, state0=x["state0"].clone())
        y["state0"][1] = float("nan")
        got = grads(y)
        for n in ("dX", "dB", "dC", "ddt", "dg"):
            assert torch.equal(got[n][rows], clean[n][rows]), ("state0", n)
    again = grads(x)
    assert all(torch.equal(again[n], clean[n]) for n in clean)
