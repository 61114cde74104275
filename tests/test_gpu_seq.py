"""The packed-sequence operators as they are used: a recurrent and an attention layer one after the
other, trained and served; captured and replayed; on a stream of the caller's; hidden rows that
hold anything; and the binding's refusals."""
import math

import pytest
import torch

from tests.seq_util import BF16, F32, attn_oracle, check, delta_oracle, offsets, rows, to_dev
from tests.test_gpu_delta import NORM, desc_of, dev, make, near

pytestmark = pytest.mark.gpu
NAMES = ("Q", "K", "V", "g", "beta", "off")


@pytest.fixture(scope="module")
def F():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2606_27748_amd as F
    F.load()
    return F


def _step(F, x, t, ddesc, adesc, saved, keep=None):
    """The delta rule's output is the attention's V: forward, then backward of both."""
    k = keep or {}
    O, _ = F.flex_delta_fwd(ddesc, *(t[n] for n in NAMES), saved=saved, O=k.get("O"))
    Y, lse = F.flex_attn_fwd(adesc, t["Q2"], t["K2"], O, t["off"], t["off"], O=k.get("Y"), lse=k.get("lse"))
    ga = F.flex_attn_bwd(adesc, t["Q2"], t["K2"], O, t["off"], t["off"], Y, lse, t["dY"], dQ=k.get("dQ2"), dK=k.get("dK2"),
                         dV=k.get("dO"), ws=k.get("wsa"))
    gd = F.flex_delta_bwd(ddesc, *(t[n] for n in NAMES), ga["dV"], saved, ws=k.get("wsd"),
                          **{n: k.get(n) for n in ("dQ", "dK", "dV", "dg", "dbeta")})
    return {"O": O, "Y": Y, "lse": lse, "dQ2": ga["dQ"], "dK2": ga["dK"], "dO": ga["dV"], **gd}


def _layers(F, dtype, lengths, seed):
    x = make(lengths, 2, 4, 64, 64, dtype, seed)
    gen = torch.Generator().manual_seed(seed + 1)
    T = sum(lengths)
    x["Q2"], x["K2"], x["dY"] = rows(gen, T, 8, 64, dtype), rows(gen, T, 4, 64, dtype), rows(gen, T, 8, 64, dtype)
    adesc = F.make_attn_desc(len(lengths), 8, 4, 64, T, T, io="bf16" if dtype == BF16 else "f32")
    return x, dev(x), desc_of(F, x, dtype), adesc


def test_two_layers_trained(F):
    """fp32: the chain of both against the chain of the oracles.  An output of the first enters the second with its
    own error, and so on down the chain: the sum of the stages' tolerances."""
    x, t, ddesc, adesc = _layers(F, F32, [70, 1, 0, 131], 21)
    saved = torch.empty(F.delta_saved_size(ddesc), dtype=torch.uint8, device="cuda")
    got = _step(F, x, t, ddesc, adesc, saved)
    fwd = delta_oracle(*(x[n] for n in NAMES))
    att, _ = attn_oracle(x["Q2"], x["K2"], fwd["O"], x["off"], x["off"], dO=x["dY"])
    bwd = delta_oracle(*(x[n] for n in NAMES), dO=att["dV"])
    near("Y", got["Y"], att["O"], 1e-5)
    for n, r in (("dQ2", att["dQ"]), ("dK2", att["dK"]), *((n, bwd[n]) for n in ("dQ", "dK", "dV", "dg", "dbeta"))):
        near(n, got[n], r, 2 * NORM[F32]["grad"])


def test_two_layers_served(F):
    """Prompts through both layers, then tokens one at a time (a step of the state, the attention against a cache
    with a slot per sequence): the rows of the whole sequences' forward."""
    n, more, B, cap = 90, 4, 3, 128
    x, t, _, _ = _layers(F, BF16, [n + more] * B, 31)
    fwd = delta_oracle(*(x[k] for k in NAMES))
    by = {k: v.reshape(B, n + more, *v.shape[1:]) for k, v in t.items() if k not in ("off", "state0")}
    head = {k: v[:, :n].reshape(B * n, *v.shape[2:]).contiguous() for k, v in by.items()}
    off = offsets([n] * B, "cuda")
    ddesc = F.make_delta_desc(B, 2, 4, 64, B * n)
    O, state = F.flex_delta_fwd(ddesc, *(head[k] for k in NAMES[:5]), off, want_state=True)
    Kc = torch.full((B, cap, 4, 64), float("nan"), dtype=BF16, device="cuda")
    Vc = Kc.clone()
    Kc[:, :n], Vc[:, :n] = by["K2"][:, :n], O.reshape(B, n, 4, 64)
    slots = offsets([cap] * B, "cuda")
    sdesc = F.make_delta_desc(B, 2, 4, 64, B)
    adesc = F.make_attn_desc(B, 8, 4, 64, B, B * cap)
    for i in range(n, n + more):
        tok = {k: v[:, i].contiguous() for k, v in by.items()}
        o = F.flex_delta_step(sdesc, *(tok[k] for k in NAMES[:5]), state)
        Kc[:, i], Vc[:, i] = tok["K2"], o
        y, _ = F.flex_attn_fwd(adesc, tok["Q2"], Kc.view(B * cap, 4, 64), Vc.view(B * cap, 4, 64),
                               offsets([1] * B, "cuda"), slots, k_len=torch.full((B,), i + 1, dtype=torch.int32, device="cuda"))
        near("o", o, fwd["O"].reshape(B, n + more, 4, 64)[:, i], NORM[BF16]["O"])
        ref, mag = attn_oracle(tok["Q2"].cpu(), Kc.cpu().reshape(-1, 4, 64)[:, :], Vc.cpu().reshape(-1, 4, 64),
                               offsets([1] * B), slots.cpu(), k_len=torch.full((B,), i + 1))
        check("y", y, ref["O"], mag["O"], 1.1, BF16)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_graph_replays_on_a_side_stream(F, dtype):
    """The training step of both layers captured on a stream of the caller's and replayed between eager work: bit for
    bit the eager step's results, every time."""
    x, t, ddesc, adesc = _layers(F, dtype, [130, 0, 67], 41)
    size = lambda n: torch.empty(max(n, 256), dtype=torch.uint8, device="cuda")  # noqa: E731
    saved = size(F.delta_saved_size(ddesc))
    ref = {k: v.clone() for k, v in _step(F, x, t, ddesc, adesc, saved).items()}
    keep = {k: torch.empty_like(v) for k, v in ref.items()}
    keep["wsa"] = size(F.attn_workspace_size(adesc, F.FLEX_PASS_BWD))
    keep["wsd"] = size(F.delta_workspace_size(ddesc, F.FLEX_PASS_BWD))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _step(F, x, t, ddesc, adesc, saved, keep)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _step(F, x, t, ddesc, adesc, saved, keep)
    other = size(F.delta_saved_size(ddesc))
    for rep in range(4):
        for k in ref:
            keep[k].fill_(float("nan"))
        _step(F, x, t, ddesc, adesc, other)   # eager work in between
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for k, v in ref.items():
            assert torch.equal(keep[k], v), (rep, k)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("nq,nk", [([100], [100]), ([5], [300]), ([200, 40], [200, 40])])
def test_hidden_rows_hold_anything(F, nq, nk, dtype):
    """NaN and infinities in K and V rows that only later queries see: the earlier ones' results are those without."""
    g = torch.Generator().manual_seed(5)
    Q, K, V = rows(g, sum(nq), 4, 64, dtype), rows(g, sum(nk), 2, 64, dtype), rows(g, sum(nk), 2, 64, dtype)
    qo, ko = offsets(nq), offsets(nk)
    out, mag = attn_oracle(Q, K, V, qo, ko)
    seen = torch.ones(sum(nq), dtype=torch.bool)
    for b in range(len(nq)):   # the last two keys of each sequence: hidden from all but its last two queries
        K[int(ko[b + 1]) - 2] = float("nan")
        V[int(ko[b + 1]) - 2] = float("nan")
        V[int(ko[b + 1]) - 1, 0] = float("inf")
        seen[int(qo[b + 1]) - 2:int(qo[b + 1])] = False
    desc = F.make_attn_desc(len(nq), 4, 2, 64, sum(nq), sum(nk), io="bf16" if dtype == BF16 else "f32")
    O, lse = F.flex_attn_fwd(desc, *(x.cuda() for x in (Q, K, V, qo, ko)))
    # summed again one key at a time: a term's fp32 rounding per key, under the bounds of the other tests
    check("O", O.cpu()[seen], out["O"][seen], mag["O"][seen], {BF16: 1.1, F32: 64.0}[dtype], dtype)
    assert (lse.cpu().double() - out["lse"])[seen].abs().max() <= 64 * 2.0 ** -24 * 16
    assert not torch.isfinite(O.cpu()[~seen].float()).all()


def test_same_results_every_time(F):
    x, t, ddesc, adesc = _layers(F, BF16, [300, 17, 129], 51)
    saved = torch.empty(F.delta_saved_size(ddesc), dtype=torch.uint8, device="cuda")
    a, b = ({k: v.clone() for k, v in _step(F, x, t, ddesc, adesc, saved).items()} for _ in range(2))
    assert all(torch.equal(a[k], b[k]) for k in a)


def test_binding_refuses(F):
    d = F.make_attn_desc(1, 2, 1, 32, 5, 5)
    q, k = torch.zeros(5, 2, 32, dtype=BF16, device="cuda"), torch.zeros(5, 1, 32, dtype=BF16, device="cuda")
    off = offsets([5], "cuda")
    wide = torch.zeros(5, 4, 32, dtype=BF16, device="cuda")
    bad = ((q.float(), k, k, off, off), (q[:4], k, k, off, off), (q, k, k, off.long(), off), (wide[:, :2], k, k, off, off),
           (q.transpose(0, 1).contiguous().transpose(0, 1), k, k, off, off), (q, k, k, off.cpu(), off))
    for args in bad:
        with pytest.raises(F.FlexError) as e:
            F.flex_attn_fwd(d, *args)
        assert e.value.status == F.FLEX_ERR_INVALID_ARG
    x = make([5], 1, 1, 64, 64, BF16, 1)
    t = dev(x)
    desc = desc_of(F, x, BF16)
    args = [t[n] for n in NAMES]
    with pytest.raises(F.FlexError) as e:   # too small a buffer for a backward
        F.flex_delta_fwd(desc, *args, saved=torch.empty(100, dtype=torch.uint8, device="cuda"))
    assert e.value.status == F.FLEX_ERR_WORKSPACE
    with pytest.raises(F.FlexError) as e:   # a state of another shape
        F.flex_delta_fwd(desc, *args, state0=torch.zeros(1, 1, 64, 32, device="cuda"))
    assert e.value.status == F.FLEX_ERR_INVALID_ARG


@pytest.mark.parametrize("B", [64, 65, 129, 4096, 4100])
def test_many_short_sequences(F, B):
    """As many sequences as the search of a tile's takes one round for, or two, or three, of 0 to 5 tokens; every
    fiftieth has 70 (further blocks, further tiles)."""
    g = torch.Generator().manual_seed(B)
    lengths = [70 if b % 50 == 7 else int(torch.randint(0, 6, (1,), generator=g)) for b in range(B - 1)] + [3]
    x, t, ddesc, adesc = _layers(F, F32, lengths, 61)
    saved = torch.empty(F.delta_saved_size(ddesc), dtype=torch.uint8, device="cuda")
    got = _step(F, x, t, ddesc, adesc, saved)
    pick = sorted({0, 1, 7, B // 2, B - 2, B - 1} | {b for b in range(0, B, 501)})   # the oracle's share
    part = {n: torch.cat([x[n][int(x["off"][b]):int(x["off"][b + 1])] for b in pick]) for n in (*NAMES[:5], "dO", "Q2", "K2", "dY")}
    off = offsets([lengths[b] for b in pick])
    take = lambda y: torch.cat([y.cpu()[int(x["off"][b]):int(x["off"][b + 1])] for b in pick])  # noqa: E731
    fwd = delta_oracle(*(part[n] for n in NAMES[:5]), off)
    att, _ = attn_oracle(part["Q2"], part["K2"], fwd["O"], off, off, dO=part["dY"])
    bwd = delta_oracle(*(part[n] for n in NAMES[:5]), off, dO=att["dV"])
    near("O", take(got["O"]), fwd["O"], NORM[F32]["O"])
    near("Y", take(got["Y"]), att["O"], 1e-5)
    for n, r in (("dQ2", att["dQ"]), ("dK2", att["dK"]), *((n, bwd[n]) for n in ("dQ", "dK", "dV", "dg", "dbeta"))):
        near(n, take(got[n]), r, 2 * NORM[F32]["grad"])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_before_the_first_sequence(F, dtype):
    """Offsets from 37 on: the results of the same rows on their own, and what lies before them left."""
    lengths, skip = [70, 0, 131], 37
    x, t, ddesc, adesc = _layers(F, dtype, lengths, 71)
    saved = torch.empty(F.delta_saved_size(ddesc), dtype=torch.uint8, device="cuda")
    ref = _step(F, x, t, ddesc, adesc, saved)
    T = sum(lengths) + skip
    late = {n: torch.cat([torch.full((skip, *v.shape[1:]), float("nan"), dtype=v.dtype, device="cuda"), v])
            for n, v in t.items() if n not in ("off", "state0")}
    late["off"] = t["off"] + skip
    io = "bf16" if dtype == BF16 else "f32"
    ddesc, adesc = F.make_delta_desc(3, 2, 4, 64, T, io=io), F.make_attn_desc(3, 8, 4, 64, T, T, io=io)
    keep = {n: torch.full((T, *v.shape[1:]), 7.0, dtype=v.dtype, device="cuda") for n, v in ref.items()}
    got = _step(F, late, late, ddesc, adesc, torch.empty(F.delta_saved_size(ddesc), dtype=torch.uint8, device="cuda"), keep)
    for n, v in ref.items():
        assert torch.equal(got[n][skip:], v), n
        assert (got[n][:skip] == 7.0).all(), n


def test_offsets_that_fall(F):
    """Wrong offsets give wrong results, but no access outside the tensors: the rows around them are left."""
    x, t, _, _ = _layers(F, BF16, [73], 81)
    t["off"] = torch.tensor([0, 900, 30, -5, 70, 10000], dtype=torch.int32, device="cuda")
    ddesc, adesc = F.make_delta_desc(5, 2, 4, 64, 73), F.make_attn_desc(5, 8, 4, 64, 73, 73)
    shapes = {"O": (4, 64), "Y": (8, 64), "lse": (8,), "dQ2": (8, 64), "dK2": (4, 64), "dO": (4, 64), "dQ": (2, 64),
              "dK": (2, 64), "dV": (4, 64), "dg": (4,), "dbeta": (4,)}
    wide = {n: torch.full((16 + 73 + 16, *s), 7.0, dtype=F32 if n == "lse" else BF16, device="cuda") for n, s in shapes.items()}
    saved = torch.zeros(F.delta_saved_size(ddesc), dtype=torch.uint8, device="cuda")
    _step(F, x, t, ddesc, adesc, saved, {n: v[16:16 + 73] for n, v in wide.items()})
    torch.cuda.synchronize()
    for n, v in wide.items():
        assert (v[:16] == 7.0).all() and (v[-16:] == 7.0).all(), n
