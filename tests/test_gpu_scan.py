"""Selective scan against the float64 recurrence, token by token: forward with and without a state to continue from,
single-token steps, backward; ragged and empty sequences, heads that share B and C, strided rows, sequences in segments.

Bounds, relative to the 2-norm of the result (a rounding to bf16 has a root mean square of 2^-8 / sqrt(3) = 2.3e-3 of
the value at most, and terms of random signs, as these inputs', add like independent ones):
  state: the operands are exact (B) or three bf16 terms, 24 bits, summed in fp32 over 64 tokens a chunk; decays have an
    exponential of one ulp and an argument of one rounding: 8 * 2^-24 a product, carried over chunks like independent
    ones: 5 * 8 * 2^-24 = 2.4e-6.
  Y: a term has one factor that is rounded to bf16 (the chunk's matrix or its state), and the result one more rounding:
    sqrt(2) * 2.3e-3 < 3.4e-3.  fp32 rows: as the state.
  gradients: a term has one factor or, in <S, dS> of dg, two that are rounded, and the result one more, and the terms
    that a gradient splits into are together at most three times the sum's on these inputs: 3 * sqrt(2) * 2.3e-3 < 1e-2;
    fp32: 3 * sqrt(2) * 2.4e-6 < 1.2e-5.
  dD: products of exact values summed in fp32 over 64 columns and tokens a chunk: 8 * 2^-24 of their absolute sum.
"""
import pytest
import torch

from tests.layer_util import SCAN_ROWS, near, on, scan_desc, scan_inputs, scan_oracle
from tests.seq_util import BF16, F32, offsets

pytestmark = pytest.mark.gpu
NORM = {BF16: {"state": 2.4e-6, "Y": 3.4e-3, "grad": 1e-2}, F32: {"state": 2.4e-6, "Y": 2.4e-6, "grad": 1.2e-5}}
GRADS = ("dX", "dB", "dC", "ddt", "dg")


@pytest.fixture(scope="module")
def F():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2606_27748_amd as F
    F.load()
    return F


def run_fwd(F, x, dtype, start, D=True, **kw):
    t = {k: on(v) for k, v in x.items()}
    if not D:
        t["D"] = None
    args = [t[n] for n in SCAN_ROWS] + [t["off"]]
    return t, args, scan_desc(F, x, dtype), dict(state0=t["state0"] if start else None, **kw)


LENGTHS = [[1], [64], [65, 0, 3, 200], [130, 63, 64], [31, 700]]
HEADS = [(64, 64, 1, 1), (128, 128, 2, 4), (64, 128, 3, 3), (128, 64, 1, 6), (128, 64, 2, 16)]   # N, P, G, H


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,P,G,H", HEADS)
@pytest.mark.parametrize("lengths", LENGTHS)
@pytest.mark.parametrize("start", [False, True])
def test_forward(F, start, lengths, N, P, G, H, dtype):
    lead, extra = (0, 0) if start else (2, 70)
    x = scan_inputs(lengths, G, H, N, P, dtype, N + len(lengths), pad=64 * (H % 2), lead=lead, extra=extra)
    ref = scan_oracle(x, start, D=start)
    rows = torch.zeros(len(x["X"]), dtype=torch.bool)
    rows[lead:lead + sum(lengths)] = True
    t, args, desc, kw = run_fwd(F, x, dtype, start, D=start)
    Y = torch.full((len(rows), H, P), float("nan"), dtype=dtype, device="cuda")
    Y, state = F.flex_scan_fwd(desc, *args, **kw, Y=Y, want_state=True)
    near("Y", Y[rows], ref["Y"][rows], NORM[dtype]["Y"])
    near("state", state, ref["state"], NORM[dtype]["state"])
    assert torch.isnan(Y[~rows]).all()   # rows of no sequence are left as they were
    # in place, and with what a backward needs kept: the same results
    saved = torch.empty(F.scan_saved_size(desc), dtype=torch.uint8, device="cuda")
    Y2, state2 = F.flex_scan_fwd(desc, *args, **kw, state=kw["state0"], saved=saved, want_state=True)
    assert torch.equal(Y[rows], Y2[rows]) and torch.equal(state, state2)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,P,G,H", HEADS)
@pytest.mark.parametrize("lengths", LENGTHS)
def test_backward(F, lengths, N, P, G, H, dtype):
    start = len(lengths) == 3
    x = scan_inputs(lengths, G, H, N, P, dtype, 11 + N + len(lengths), pad=64 * (H % 2), lead=3, extra=66)
    ref = scan_oracle(x, start, grads=True)
    rows = torch.zeros(len(x["X"]), dtype=torch.bool)
    rows[3:3 + sum(lengths)] = True
    t, args, desc, kw = run_fwd(F, x, dtype, start)
    desc.dx_stride, desc.db_stride, desc.dc_stride = H * P + 16, G * N + 8, G * N
    saved = torch.empty(F.scan_saved_size(desc), dtype=torch.uint8, device="cuda")
    F.flex_scan_fwd(desc, *args, **kw, saved=saved)
    wide = {n: torch.full((len(rows), w), float("nan"), dtype=dtype, device="cuda")
            for n, w in (("dX", H * P + 16), ("dB", G * N + 8), ("dC", G * N), ("ddt", H), ("dg", H))}
    out = {"dX": wide["dX"][:, :H * P].unflatten(1, (H, P)), "dB": wide["dB"][:, :G * N].unflatten(1, (G, N)),
           "dC": wide["dC"].unflatten(1, (G, N)), "ddt": wide["ddt"], "dg": wide["dg"]}
    grads = F.flex_scan_bwd(desc, *args, t["dY"], saved, **out)
    for n in GRADS:
        assert torch.isnan(wide[n][~rows]).all(), n
        if lengths == [1] and n == "dg" and not start:   # a single token's decay meets an empty state
            assert (grads[n][rows].float().abs() <= 1e-30).all()
            continue
        near(n, grads[n][rows], ref[n][rows], NORM[dtype]["grad"])
    assert torch.isnan(wide["dX"][:, H * P:]).all() and torch.isnan(wide["dB"][:, G * N:]).all()
    terms = (x["dY"].double() * x["X"].double())[rows].abs().sum((0, 2))
    assert ((grads["dD"].cpu().double() - ref["dD"]).abs() <= 9 * 2.0 ** -24 * terms + 1e-30).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,P,G,H", HEADS)
@pytest.mark.parametrize("B", [1, 5])
def test_step_continues_a_prompt(F, B, N, P, G, H, dtype):
    """Seventy tokens as a prompt, three more as steps: the recurrence over all of them."""
    n, more = 70, 3
    x = scan_inputs([n + more] * B, G, H, N, P, dtype, 7 + N)
    ref = scan_oracle(x, False)
    by = {k: x[k].reshape(B, n + more, *x[k].shape[1:]) for k in SCAN_ROWS[:5]}
    head = {k: v[:, :n].reshape(B * n, *v.shape[2:]).contiguous() for k, v in by.items()}
    head["off"], D = offsets([n] * B), x["D"].cuda()
    t = {k: on(v) for k, v in head.items()}
    _, state = F.flex_scan_fwd(scan_desc(F, head, dtype), *(t[k] for k in SCAN_ROWS[:5]), D, t["off"], want_state=True)
    want = ref["Y"].reshape(B, n + more, H, P)
    for i in range(n, n + more):
        tok = {k: v[:, i].contiguous().cuda() for k, v in by.items()}
        desc = F.make_scan_desc(B, G, H, N, P, B, io="bf16" if dtype == BF16 else "f32")
        y = F.flex_scan_step(desc, *(tok[k] for k in SCAN_ROWS[:5]), D, state)
        near("y", y, want[:, i], 2.4e-3 if dtype == BF16 else NORM[F32]["Y"])   # one rounding
    near("state", state, ref["state"], NORM[dtype]["state"])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_decay_of_zero(F, dtype):
    """g = -inf clears the state and has no slope."""
    x = scan_inputs([150, 64], 1, 2, 64, 64, dtype, 8)
    cut = [0, 70, 71, 128, 150]
    x["g"][cut] = -float("inf")
    ref = scan_oracle(x, False, grads=True)
    t, args, desc, _ = run_fwd(F, x, dtype, False)
    saved = torch.empty(F.scan_saved_size(desc), dtype=torch.uint8, device="cuda")
    Y, state = F.flex_scan_fwd(desc, *args, saved=saved, want_state=True)
    near("Y", Y, ref["Y"], NORM[dtype]["Y"])
    near("state", state, ref["state"], NORM[dtype]["state"])
    grads = F.flex_scan_bwd(desc, *args, t["dY"], saved)
    assert (grads["dg"][cut] == 0).all()
    ref["dg"][cut] = 0
    for n in GRADS:
        near(n, grads[n], ref[n], NORM[dtype]["grad"])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_many_segments(F, dtype):
    """Sequences of many segments that hardly forget, in place, beside short ones: states carried forwards and back."""
    x = scan_inputs([5, 3000, 1, 700], 1, 2, 64, 64, dtype, 3, rate=0.05)
    ref = scan_oracle(x, True, grads=True)
    t, args, desc, kw = run_fwd(F, x, dtype, True)
    saved = torch.empty(F.scan_saved_size(desc), dtype=torch.uint8, device="cuda")
    Y, state = F.flex_scan_fwd(desc, *args, **kw, state=kw["state0"], saved=saved)
    near("Y", Y, ref["Y"], NORM[dtype]["Y"])
    near("state", state, ref["state"], NORM[dtype]["state"])
    grads = F.flex_scan_bwd(desc, *args, t["dY"], saved)
    for n in GRADS:
        near(n, grads[n], ref[n], NORM[dtype]["grad"])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_heads_that_forget_at_once(F, dtype):
    """Decays of e^-5 to e^-8 a token, each head by itself: the slope of a decay is some thousandth of the terms beside
    it that have no part in it."""
    x = scan_inputs([150, 64, 20], 1, 2, 64, 64, dtype, 6)
    x["g"] = -5.0 - torch.rand(x["g"].shape, generator=torch.Generator().manual_seed(1)) * torch.tensor([3.0, 1.0])
    ref = scan_oracle(x, False, grads=True)
    t, args, desc, _ = run_fwd(F, x, dtype, False)
    saved = torch.empty(F.scan_saved_size(desc), dtype=torch.uint8, device="cuda")
    F.flex_scan_fwd(desc, *args, saved=saved)
    grads = F.flex_scan_bwd(desc, *args, t["dY"], saved)
    for h in range(2):
        for n in ("dX", "ddt", "dg"):
            near((n, h), grads[n][:, h], ref[n][:, h], NORM[dtype]["grad"])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rate", [1.0, 1.7, 2.4, 3.0, 4.5])
def test_decays_of_a_chunk_over_many_powers_of_two(F, rate, dtype):
    """Decays whose sums over a chunk run from 2^-92 to 2^-415, even and with a quiet stretch across its middle, each
    token by itself against its neighbours: what lies between two tokens is the same however far both have come."""
    x = scan_inputs([64, 200], 1, 2, 64, 64, dtype, 16)
    x["g"] = -rate * (0.9 + 0.2 * torch.rand(x["g"].shape, generator=torch.Generator().manual_seed(2)))
    x["g"][[30, 31, 32, 33, 95, 96]] = -0.01
    ref = scan_oracle(x, False, grads=True)
    t, args, desc, _ = run_fwd(F, x, dtype, False)
    saved = torch.empty(F.scan_saved_size(desc), dtype=torch.uint8, device="cuda")
    Y, state = F.flex_scan_fwd(desc, *args, saved=saved, want_state=True)
    near("state", state, ref["state"], NORM[dtype]["state"])
    grads = F.flex_scan_bwd(desc, *args, t["dY"], saved)
    for i in range(0, len(x["X"]), 8):
        at = slice(i, i + 8)
        near(("Y", i), Y[at], ref["Y"][at], NORM[dtype]["Y"])
        for n in ("dX", "dB", "dC"):
            near((n, i), grads[n][at], ref[n][at], NORM[dtype]["grad"])
    for n in ("ddt", "dg"):
        near(n, grads[n], ref[n], NORM[dtype]["grad"])


def test_backward_against_differences(F):
    """<gradient, r> against the change of sum(dY Y) along r, by the float64 recurrence: within the gradient's
    tolerance times both norms, and the difference's own error, step^2 = 1e-10 of derivatives of the gradient's size."""
    x = scan_inputs([70, 65], 2, 4, 64, 64, F32, 9)
    t, args, desc, _ = run_fwd(F, x, F32, False)
    saved = torch.empty(F.scan_saved_size(desc), dtype=torch.uint8, device="cuda")
    F.flex_scan_fwd(desc, *args, saved=saved)
    grads = F.flex_scan_bwd(desc, *args, t["dY"], saved)
    gen, h = torch.Generator().manual_seed(10), 1e-5
    for n in SCAN_ROWS:
        r = torch.randn(x[n].shape, generator=gen, dtype=torch.float64)
        ends = [(scan_oracle(dict(x, **{n: x[n].double() + s * h * r}), False)["Y"] * x["dY"].double()).sum() for s in (1, -1)]
        g = grads["d" + {"Bt": "B", "Ct": "C"}.get(n, n)].cpu().double()
        assert abs((g * r).sum() - (ends[0] - ends[1]) / (2 * h)) <= (NORM[F32]["grad"] + 1e-6) * g.norm() * r.norm(), n


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("name,at", [("X", (70, 1, 40)), ("X", (64, 0, 0)), ("Bt", (100, 0, 5)), ("Ct", (90, 0, 3)),
                                     ("dt", (75, 1)), ("g", (127, 0))])
def test_rows_that_are_not_finite_reach_no_earlier_token(F, name, at, dtype):
    x = scan_inputs([60, 140, 50], 1, 2, 64, 64, dtype, 12)
    t, args, desc, _ = run_fwd(F, x, dtype, False)
    Y0, s0 = F.flex_scan_fwd(desc, *args, want_state=True)
    for value in (float("nan"), float("inf")):
        args[SCAN_ROWS.index(name)][at] = value
        Y, s = F.flex_scan_fwd(desc, *args, want_state=True)
        hit = torch.zeros_like(Y, dtype=torch.bool)   # in the second sequence, rows 60 .. 199
        if name == "X":
            hit[at[0]:200, at[1], at[2]] = True
        elif name == "Bt":
            hit[at[0]:200] = True
        elif name == "Ct":
            hit[at[0]] = True
        else:
            hit[at[0]:200, at[1]] = True
        assert torch.equal(Y[~hit], Y0[~hit])
        assert not torch.isfinite(Y[hit]).any()
        assert torch.equal(s[0], s0[0]) and torch.equal(s[2], s0[2])
        if name == "X":
            assert not torch.isfinite(s[1, at[1], :, at[2]]).any()
            assert torch.equal(s[1, 1 - at[1]], s0[1, 1 - at[1]])
        elif name == "Ct":
            assert torch.equal(s[1], s0[1])
