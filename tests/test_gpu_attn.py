"""Exact attention over packed sequences against the float64 oracle: forward, single tokens
against a cache, backward; ragged and empty sequences, grouped heads, strided rows.

Bounds (see seq_util.check), in roundings u of the io type of the sum of absolute terms:
  O: bf16 rounds each probability once (1 u); its fp32 exponent is off by 2^-23 of a logit in units of
     log2 that stays under 2^5 here, far below u, and fp32 sums add (number of terms) 2^-24.  fp32: the
     probability's exponent, exp2 and the sums each contribute a few 2^-24 of logits up to 2^5: 64 u.
  dV: as O.  dQ, dK: dS = P (dP - delta) is rounded once, delta comes from O rounded once: 2 u, and
     the second-order terms: 3 u.  fp32: the products' own sums over d and the logits: 128 u.
A sum of n terms in fp32 adds n 2^-24: n is at most 2100 here, 2^-13 = u / 32 for bf16.
"""
import math

import pytest
import torch

from tests.seq_util import BF16, F32, attn_oracle, check, offsets, rows, to_dev

pytestmark = pytest.mark.gpu
TERMS = {BF16: {"O": 1.1, "dV": 1.1, "dQ": 3.0, "dK": 3.0}, F32: {"O": 64.0, "dV": 64.0, "dQ": 128.0, "dK": 128.0}}


@pytest.fixture(scope="module")
def F():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2606_27748_amd as F
    F.load()
    return F


def _io(dtype):
    return "bf16" if dtype == BF16 else "f32"


def _inputs(nq, nk, Hq, Hkv, d, dtype, seed=0, pad=0, extra=0):
    g = torch.Generator().manual_seed(seed)
    Tq, Tk = sum(nq) + extra, sum(nk) + extra
    return (rows(g, Tq, Hq, d, dtype, pad, 1.4), rows(g, Tk, Hkv, d, dtype, pad, 1.4), rows(g, Tk, Hkv, d, dtype, pad),
            rows(g, Tq, Hq, d, dtype), offsets(nq), offsets(nk))


def _desc(F, Q, K, V, B, causal, dtype, **kw):
    return F.make_attn_desc(B, Q.shape[1], K.shape[1], Q.shape[2], len(Q), len(K), causal=causal, io=_io(dtype),
                            q_stride=Q.stride(0) if len(Q) > 1 else 0, k_stride=K.stride(0) if len(K) > 1 else 0,
                            v_stride=V.stride(0) if len(V) > 1 else 0, **kw)


def _check_fwd(out, mag, O, lse, dtype):
    check("O", O, out["O"], mag["O"], TERMS[dtype]["O"], dtype)
    got, ref = lse.cpu().double(), out["lse"]
    assert torch.equal(torch.isinf(got), torch.isinf(ref))
    fin = torch.isfinite(ref)
    assert (got - ref)[fin].abs().max() <= 64 * 2.0 ** -24 * 16 if fin.any() else True


SHAPES = [([1], [1]), ([64], [64]), ([33, 0, 1, 200], [33, 0, 1, 200]), ([130, 5, 257], [130, 5, 257]),
          ([7, 100, 3, 64], [7, 612, 0, 65]), ([90, 40], [30, 40])]   # the last: queries that see no key


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d,Hq,Hkv", [(32, 3, 1), (64, 4, 2), (128, 8, 2)])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("nq,nk", SHAPES)
def test_forward_backward(F, nq, nk, causal, d, Hq, Hkv, dtype):
    Q, K, V, dO, qo, ko = _inputs(nq, nk, Hq, Hkv, d, dtype, seed=len(nq) + d, pad=Hq % 3)
    out, mag = attn_oracle(Q, K, V, qo, ko, causal=causal, dO=dO)
    desc = _desc(F, Q, K, V, len(nq), causal, dtype)
    q, k, v, g, a, b = (to_dev(x) for x in (Q, K, V, dO, qo, ko))
    O, lse = F.flex_attn_fwd(desc, q, k, v, a, b)
    grads = F.flex_attn_bwd(desc, q, k, v, a, b, O, lse, g)
    torch.cuda.synchronize()
    _check_fwd(out, mag, O, lse, dtype)
    for n in ("dQ", "dK", "dV"):
        check(n, grads[n], out[n], mag[n], TERMS[dtype][n], dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d,Hq,Hkv", [(32, 2, 2), (64, 12, 4), (128, 16, 2), (128, 40, 1)])
def test_single_tokens_against_a_cache(F, d, Hq, Hkv, dtype):
    """One token of each sequence (and three of one) against slots of 1300 rows, used lengths from 0 to all."""
    cap, nk = 1300, [0, 1, 31, 32, 129, 1300, 777, 1024]
    nq = [1, 1, 1, 1, 3, 1, 0, 1]
    Q, K, V, _, qo, _ = _inputs(nq, [cap] * len(nk), Hq, Hkv, d, dtype, seed=d + Hq)
    ko = offsets([cap] * len(nk))
    kl = torch.tensor(nk, dtype=torch.int32)
    for b, n in enumerate(nk):   # rows behind the used length hold anything
        K[b * cap + n:(b + 1) * cap] = float("nan")
        V[b * cap + n:(b + 1) * cap] = float("inf")
    out, mag = attn_oracle(Q, K, V, qo, ko, k_len=kl)
    desc = _desc(F, Q, K, V, len(nq), True, dtype)
    assert F.attn_workspace_size(desc, F.FLEX_PASS_FWD) > 0   # the keys are split
    O, lse = F.flex_attn_fwd(desc, *(to_dev(x) for x in (Q, K, V, qo, ko)), k_len=kl.cuda())
    torch.cuda.synchronize()
    _check_fwd(out, mag, O, lse, dtype)


@pytest.mark.parametrize("causal", [True, False])
def test_long_sequence(F, causal):
    nq = [2100]
    Q, K, V, dO, qo, ko = _inputs(nq, nq, 2, 1, 128, BF16, seed=3)
    out, mag = attn_oracle(Q, K, V, qo, ko, causal=causal, dO=dO)
    desc = _desc(F, Q, K, V, 1, causal, BF16)
    q, k, v, g, a, b = (to_dev(x) for x in (Q, K, V, dO, qo, ko))
    O, lse = F.flex_attn_fwd(desc, q, k, v, a, b)
    grads = F.flex_attn_bwd(desc, q, k, v, a, b, O, lse, g)
    _check_fwd(out, mag, O, lse, BF16)
    for n in ("dQ", "dK", "dV"):
        check(n, grads[n], out[n], mag[n], TERMS[BF16][n], BF16)


def test_rows_behind_the_last_sequence_are_left(F):
    nq = [70, 3]
    Q, K, V, dO, qo, ko = _inputs(nq, nq, 4, 2, 64, BF16, seed=4, extra=9)
    desc = _desc(F, Q, K, V, 2, True, BF16)
    q, k, v, g, a, b = (to_dev(x) for x in (Q, K, V, dO, qo, ko))
    mark = lambda *s, dt=BF16: torch.full(s, 7.0, dtype=dt, device="cuda")  # noqa: E731
    O, lse = F.flex_attn_fwd(desc, q, k, v, a, b, O=mark(82, 4, 64), lse=mark(82, 4, dt=F32))
    gr = F.flex_attn_bwd(desc, q, k, v, a, b, O, lse, g, dQ=mark(82, 4, 64), dK=mark(82, 2, 64), dV=mark(82, 2, 64))
    for x in (O, lse, *gr.values()):
        assert (x[73:] == 7.0).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d,Hq,Hkv,prompt", [(64, 2, 2, 333), (128, 8, 2, 100), (32, 6, 2, 65)])
@pytest.mark.parametrize("causal", [True, False])
def test_prompt_among_single_tokens(F, causal, d, Hq, Hkv, prompt, dtype):
    """One prompt and single tokens in a call, few rows on average: every block of 32 rows has workgroups of its own."""
    nq = [1, 1, prompt, 0, 1, 2] + [1] * 6
    nk = [900, 1, prompt + 70, 50, 0, 400] + [64, 65, 31, 32, 700, 5]
    Q, K, V, _, qo, ko = _inputs(nq, nk, Hq, Hkv, d, dtype, seed=prompt, pad=1)
    out, mag = attn_oracle(Q, K, V, qo, ko, causal=causal)
    desc = _desc(F, Q, K, V, len(nq), causal, dtype)
    assert sum(nq) * (Hq // Hkv) <= 64 * len(nq)
    O, lse = F.flex_attn_fwd(desc, *(to_dev(x) for x in (Q, K, V, qo, ko)))
    _check_fwd(out, mag, O, lse, dtype)


@pytest.mark.parametrize("rows_,empty", [(2058, 511), (4200, 40)])
def test_rows_far_apart(F, rows_, empty):
    """Rows 2 MB apart, a sequence of over 4 GB: the bytes between its first and last row pass 32 bits."""
    gen = torch.Generator().manual_seed(rows_)
    Q, K, V = (rows(gen, n, 1, 32, BF16) for n in (1, rows_, rows_))
    qo, ko = offsets([0, 1] + [0] * empty), offsets([0, rows_] + [0] * empty)
    out, mag = attn_oracle(Q, K, V, qo, ko)
    far = 1 << 20
    desc = F.make_attn_desc(len(qo) - 1, 1, 1, 32, 1, rows_, k_stride=far, v_stride=far)

    def apart(x):
        y = torch.empty(rows_ * far, dtype=BF16, device="cuda").as_strided((rows_, 1, 32), (far, 32, 1))
        return y.copy_(x)

    O, lse = F.flex_attn_fwd(desc, Q.cuda(), apart(K), apart(V), qo.cuda(), ko.cuda())
    _check_fwd(out, mag, O, lse, BF16)


def test_backward_against_differences(F):
    """<gradient, r> against the change of sum(dO O) along r, by the float64 definition: within 128 roundings of the
    sums of absolute terms times r's, and the difference's own error, step^2 = 1e-10 of the like."""
    nq, nk = [70, 5], [70, 40]
    Q, K, V, dO, qo, ko = _inputs(nq, nk, 4, 2, 64, F32, seed=12)
    _, mag = attn_oracle(Q, K, V, qo, ko, dO=dO)
    t = [x.cuda() for x in (Q, K, V, qo, ko)]
    desc = _desc(F, Q, K, V, 2, True, F32)
    O, lse = F.flex_attn_fwd(desc, *t)
    grads = F.flex_attn_bwd(desc, *t, O, lse, dO.cuda())
    gen, h = torch.Generator().manual_seed(13), 1e-5
    for i, n in enumerate("QKV"):
        r = torch.randn((Q, K, V)[i].shape, generator=gen, dtype=torch.float64)
        ends = []
        for s in (1, -1):
            x = [y.double() for y in (Q, K, V)]
            x[i] = x[i] + s * h * r
            ends.append((attn_oracle(*x, qo, ko)[0]["O"] * dO.double()).sum())
        g = grads["d" + n].cpu().double()
        bound = ((128 * 2.0 ** -24 + 1e-8) * mag["d" + n] * r.abs()).sum()
        assert abs((g * r).sum() - (ends[0] - ends[1]) / (2 * h)) <= bound, n
