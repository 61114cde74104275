"""Packed-sequence operators and rows that a query does not see: NaN and infinities in them change nothing."""
import pytest
import torch

from tests.seq_util import BF16, F32, attn_oracle, check, offsets, rows
from tests.test_gpu_attn import TERMS
from tests.test_gpu_delta import desc_of, dev
from tests.test_gpu_delta_heads import inputs

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def F():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2606_27748_amd as F
    F.load()
    return F


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d,dv", [(64, 64), (128, 128), (128, 64)])
@pytest.mark.parametrize("save", [False, True])
def test_delta_rule_looks_at_no_later_row(F, save, d, dv, dtype):
    """What is not finite in a token's row of K, V, g or beta: the tokens before it in the sequence (of the same chunk
    too), other sequences and, for V, the other columns have the bits that they have without it; from the token on
    the results are not finite.  In Q: the token's own row alone."""
    x = inputs([70, 130, 20], 1, 2, d, dv, dtype, 41, (0.0, [0.05, 0.5]))
    desc = desc_of(F, x, dtype)

    def forward(y):
        t = dev(y)
        saved = torch.empty(F.delta_saved_size(desc), dtype=torch.uint8, device="cuda") if save else None
        O, state = F.flex_delta_fwd(desc, *(t[n] for n in ("Q", "K", "V", "g", "beta", "off")), saved=saved, want_state=True)
        return O.cpu(), state.cpu()

    clean, clean_state = forward(x)
    assert torch.isfinite(clean).all() and torch.isfinite(clean_state).all()
    for name, at, value in (("V", (5, 0, 3), NAN), ("V", (63, 1, dv - 1), INF), ("V", (64 + 16, 1, 17), -INF),
                            ("K", (0, 0, 9), NAN), ("K", (31, 0, d - 1), INF), ("K", (40, 0, 0), NAN), ("K", (110, 0, 1), NAN),
                            ("g", (17, 1), NAN), ("g", (50, 0), INF), ("beta", (48, 0), NAN), ("beta", (2, 1), -INF),
                            ("Q", (33, 0, 5), NAN)):
        y = {n: v.clone() for n, v in x.items()}
        tok, where = 70 + at[0], at[1:]
        y[name][(tok, *where)] = value
        O, state = forward(y)
        heads = slice(None) if name in ("K", "Q") else where[0]
        cols = where[1] if name == "V" else slice(None)
        hit = torch.zeros(clean.shape, dtype=torch.bool)
        hit[tok:tok + 1 if name == "Q" else 200, heads, cols] = True
        same = (O == clean) | hit
        assert same.all(), (name, at, value, (~same).nonzero()[:4].tolist())
        assert not torch.isfinite(O[hit]).any(), (name, at, value)
        kept = torch.ones(clean_state.shape, dtype=torch.bool)
        if name != "Q":
            kept[1, heads, :, cols] = False
        assert torch.equal(state[kept], clean_state[kept]) and not torch.isfinite(state[~kept]).any(), (name, at, value)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_delta_gradients_of_other_sequences(F, dtype):
    """What is not finite in one sequence: the gradients of the others have the bits that they have without it."""
    x = inputs([70, 130, 20], 1, 2, 64, 64, dtype, 42, (0.0, [0.05, 0.5]))
    desc, names = desc_of(F, x, dtype), ("Q", "K", "V", "g", "beta", "off")

    def backward(y):
        t = dev(y)
        saved = torch.empty(F.delta_saved_size(desc), dtype=torch.uint8, device="cuda")
        F.flex_delta_fwd(desc, *(t[n] for n in names), saved=saved)
        return {n: v.cpu() for n, v in F.flex_delta_bwd(desc, *(t[n] for n in names), t["dO"], saved).items()}

    clean = backward(x)
    for name in ("Q", "K", "V", "g", "beta", "dO"):
        y = {n: v.clone() for n, v in x.items()}
        y[name][100] = NAN
        got = backward(y)
        for n, v in got.items():   # a gradient may not depend on the row at all, as dV on V
            assert torch.equal(v[:70], clean[n][:70]) and torch.equal(v[200:], clean[n][200:]), (name, n)
        assert any(not torch.isfinite(v[70:200].float()).all() for v in got.values()), name


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d,Hq,Hkv", [(32, 2, 2), (64, 4, 2), (128, 8, 2)])
@pytest.mark.parametrize("nq,nk", [([330], [330]), ([5], [700]), ([40, 200], [300, 200])])
def test_attention_forward_looks_at_no_hidden_row(F, nq, nk, d, Hq, Hkv, dtype):
    """V with a NaN in one column of one row and an infinity in another's, K with a NaN row: a query that sees one
    has its results not finite there, and every other value is what it is without them, within the bounds of the
    other tests (a sum formed again rounds its products once more in fp32, far below a rounding of bf16)."""
    g = torch.Generator().manual_seed(d + len(nq))
    Q, K, V = rows(g, sum(nq), Hq, d, dtype), rows(g, sum(nk), Hkv, d, dtype), rows(g, sum(nk), Hkv, d, dtype)
    qo, ko = offsets(nq), offsets(nk)
    out, mag = attn_oracle(Q, K, V, qo, ko)
    hit = torch.zeros(out["O"].shape, dtype=torch.bool)
    grp = Hq // Hkv
    for b in range(len(nq)):
        first = lambda key: max(key - (nk[b] - nq[b]), 0) + int(qo[b])  # noqa: E731  the first query that sees it
        end, k0 = int(qo[b + 1]), int(ko[b])
        for key, head, col, value in ((nk[b] // 3, 0, 3, NAN), (nk[b] - 4, Hkv - 1, d - 1, INF), (nk[b] - 90, 0, 9, -INF)):
            V[k0 + key, head, col] = value
            hit[first(key):end, head * grp:(head + 1) * grp, col] = True
        K[k0 + nk[b] - 2, 0] = NAN
        hit[first(nk[b] - 2):end, :grp] = True
    desc = F.make_attn_desc(len(nq), Hq, Hkv, d, sum(nq), sum(nk), io="bf16" if dtype == BF16 else "f32")
    O, lse = F.flex_attn_fwd(desc, *(x.cuda() for x in (Q, K, V, qo, ko)))
    O, lse = O.cpu(), lse.cpu().double()
    check("O", O[~hit], out["O"][~hit], mag["O"][~hit], TERMS[dtype]["O"], dtype)
    assert not torch.isfinite(O[hit]).any()
    rest = ~hit.all(-1)
    assert (lse - out["lse"])[rest].abs().max() <= 64 * 2.0 ** -24 * 16


def test_a_visible_nan_costs_a_few_times_the_call(F):
    """A NaN in the first row of V, which every query sees: its sums are formed again as products.  Three times
    the call's time; one key at a time it was thirty times, so ten tells them apart."""
    T, H, d = 8192, 8, 64
    g = torch.Generator().manual_seed(3)
    Q, K, V = (rows(g, T, H, d, BF16).cuda() for _ in range(3))
    off, desc = offsets([T], "cuda"), F.make_attn_desc(1, H, H, d, T, T)

    def us():
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        best = 1e9
        for _ in range(5):
            a.record()
            F.flex_attn_fwd(desc, Q, K, V, off, off)
            b.record()
            b.synchronize()
            best = min(best, a.elapsed_time(b) * 1e3)
        return best

    clean = us()
    V[0, :, 0] = NAN
    bad = us()
    print(f"{clean:.0f} us, with a NaN {bad:.0f} us")
    assert bad <= 10 * clean


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d,Hq,Hkv", [(32, 2, 2), (64, 4, 2), (128, 8, 2)])
@pytest.mark.parametrize("nq,nk", [([330], [330]), ([40, 200], [301, 200]), ([150, 70], [100, 1100])])
def test_attention_backward_looks_at_no_hidden_row(F, nq, nk, d, Hq, Hkv, dtype):
    """A NaN row of Q, K, V or dO in the last sequence: the gradients that it has a part in are not finite (of a row of
    K, those of each query that sees it and, through those, of every key), all others are what they are without it.
    Rows of Q and dO take no part in the gradients of keys that they do not see, rows of K and V none in those of
    queries that do not see them."""
    g = torch.Generator().manual_seed(d + sum(nk))
    Q, K, V = rows(g, sum(nq), Hq, d, dtype), rows(g, sum(nk), Hkv, d, dtype), rows(g, sum(nk), Hkv, d, dtype)
    dO, qo, ko, grp = rows(g, sum(nq), Hq, d, dtype), offsets(nq), offsets(nk), Hq // Hkv
    out, mag = attn_oracle(Q, K, V, qo, ko, dO=dO)
    desc = F.make_attn_desc(len(nq), Hq, Hkv, d, sum(nq), sum(nk), io="bf16" if dtype == BF16 else "f32")
    (q0, q1), (k0, k1), shift = qo[-2:].tolist(), ko[-2:].tolist(), nk[-1] - nq[-1]
    for name, row in (("Q", nq[-1] - 37), ("Q", 11), ("dO", nq[-1] - 64), ("K", nk[-1] - 5), ("K", nk[-1] // 2 + 3),
                      ("V", nk[-1] - 41)):
        x = {"Q": Q, "K": K, "V": V, "dO": dO}
        x[name] = x[name].clone()
        x[name][(q0 if name in ("Q", "dO") else k0) + row, 0] = NAN   # head 0
        t = [x[n].cuda() for n in ("Q", "K", "V")] + [qo.cuda(), ko.cuda()]
        O, lse = F.flex_attn_fwd(desc, *t)
        got = {n: v.cpu() for n, v in F.flex_attn_bwd(desc, *t, O, lse, x["dO"].cuda()).items()}
        hit = {n: torch.zeros(out[n].shape, dtype=torch.bool) for n in got}
        if name in ("Q", "dO"):
            seen = min(max(row + shift + 1, 0), nk[-1])   # keys
            if seen:
                hit["dQ"][q0 + row, 0] = hit["dK"][k0:k0 + seen, 0] = hit["dV"][k0:k0 + seen, 0] = True
        else:
            first = max(row - shift, 0)   # query
            hit["dQ"][q0 + first:q1, :grp] = hit["dK"][k0:k1, 0] = True
            if name == "K":
                hit["dV"][k0:k1, 0] = True
        for n, v in got.items():
            rest = ~hit[n]
            check(f"{n} with {name} {row}", v[rest], out[n][rest], mag[n][rest], TERMS[dtype][n], dtype)
            assert not torch.isfinite(v[hit[n]]).any(), (n, name, row)
