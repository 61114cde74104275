"""Gated delta rule against the float64 recurrence, token by token: forward with and without a
state to continue from, single-token steps, backward; ragged and empty sequences, value heads
that share keys, strided rows.

Bounds.  With unit keys, beta <= 1 and decays <= 1 the recurrence neither amplifies a state nor an
error in it (each step's transition has norm <= 1), so an error of a chunk's new terms stays
of its relative size in the state and in what is read from it.  They are checked against the root
mean square of the result's head: the relative 2-norm of the difference, and its largest element.
  state and O before its own rounding: the operands are two bf16 terms, 2^-17 each; a state passes
    through at most five products of a chunk, and an error made in one chunk adds to those of the
    others like independent ones: 5 * 2^-17 = 4e-5 at most, 2e-5 for the 2-norm.
  O: one rounding, of root mean square 2^-8 / sqrt(3) = 2.3e-3 of the value at most.
  fp32 rows: products of exact operands summed in fp32 over 64 to 128 terms a chunk, 2^-24 a term
    and product: 5 * 8 * 2^-24 = 2.4e-6 for the 2-norm.
  gradients: a term passes one rounding to bf16 of an operand and one of its own, 2.3e-3 each, and dK,
    dg and dbeta are sums of up to six such terms that partly cancel (their 2-norms together at most
    three times the sum's on these inputs): 3 * sqrt(2) * 2.3e-3 < 1e-2.  fp32: 3 * sqrt(2) * 2.4e-6 < 1.2e-5.
"""
import pytest
import torch

from tests.seq_util import BF16, F32, delta_oracle, offsets, rows, to_dev

pytestmark = pytest.mark.gpu
NORM = {BF16: {"state": 2e-5, "O": 2.4e-3, "grad": 1e-2}, F32: {"state": 2.4e-6, "O": 2.4e-6, "grad": 1.2e-5}}


@pytest.fixture(scope="module")
def F():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2606_27748_amd as F
    F.load()
    return F


def near(name, got, ref, tol):
    """2-norm of the difference within tol of the result's, and no element further off than 40 tol of
    the larger of itself and the root mean square (the tolerance of a 2-norm is a root mean square)."""
    got, ref = got.detach().cpu().double(), ref
    assert torch.isfinite(got).all(), name
    if ref.numel() == 0:
        return
    norm, rms = ref.norm(), ref.square().mean().sqrt()
    assert (got - ref).norm() <= tol * norm, (name, float((got - ref).norm() / norm))
    assert ((got - ref).abs() <= 40 * tol * torch.maximum(ref.abs(), rms)).all(), name


def make(lengths, Hk, H, d, dv, dtype, seed, pad=0, extra=0):
    gen = torch.Generator().manual_seed(seed)
    T = sum(lengths) + extra
    x = {}
    for n in ("Q", "K"):
        x[n] = rows(gen, T, Hk, d, dtype, pad)
        v = x[n].double() + 0.3
        x[n].copy_(v / v.norm(dim=-1, keepdim=True))
    x["V"] = rows(gen, T, H, dv, dtype, pad)
    x["beta"] = torch.rand(T, H, generator=gen)
    x["g"] = -torch.rand(T, H, generator=gen) * torch.logspace(-2.5, 0, H)[None]
    x["off"] = offsets(lengths)
    x["dO"] = rows(gen, T, H, dv, dtype)
    x["state0"] = torch.randn(len(lengths), H, d, dv, generator=gen) * 0.3
    return x


def desc_of(F, x, dtype, **kw):
    Q, V = x["Q"], x["V"]
    one = len(Q) > 1
    return F.make_delta_desc(len(x["off"]) - 1, Q.shape[1], V.shape[1], Q.shape[2], len(Q), dv=V.shape[2],
                             io="bf16" if dtype == BF16 else "f32", q_stride=Q.stride(0) if one else 0,
                             k_stride=x["K"].stride(0) if one else 0, v_stride=V.stride(0) if one else 0, **kw)


def dev(x):
    return {k: to_dev(v) for k, v in x.items()}


LENGTHS = [[1], [64], [65, 0, 3, 200], [130, 63, 64]]
HEADS = [(64, 64, 1, 1), (128, 128, 2, 4), (64, 128, 3, 3), (128, 64, 1, 2)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d,dv,Hk,H", HEADS)
@pytest.mark.parametrize("lengths", LENGTHS)
@pytest.mark.parametrize("start", [False, True])
def test_forward(F, start, lengths, d, dv, Hk, H, dtype):
    x = make(lengths, Hk, H, d, dv, dtype, seed=d + len(lengths), pad=H % 2)
    ref = delta_oracle(*(x[n] for n in ("Q", "K", "V", "g", "beta", "off")), state0=x["state0"] if start else None)
    t, desc = dev(x), desc_of(F, x, dtype)
    args = [t[n] for n in ("Q", "K", "V", "g", "beta", "off")]
    s0 = t["state0"] if start else None
    O, state = F.flex_delta_fwd(desc, *args, state0=s0, want_state=True)
    near("O", O, ref["O"], NORM[dtype]["O"])
    near("state", state, ref["state"], NORM[dtype]["state"])
    # in place, and with what a backward needs kept: the same results
    saved = torch.empty(F.delta_saved_size(desc), dtype=torch.uint8, device="cuda")
    O2, state2 = F.flex_delta_fwd(desc, *args, state0=s0, state=s0, saved=saved, want_state=True)
    assert torch.equal(O, O2) and torch.equal(state, state2)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d,dv,Hk,H", HEADS)
@pytest.mark.parametrize("B", [1, 5])
def test_step_continues_a_prompt(F, B, d, dv, Hk, H, dtype):
    """Seventy tokens as a prompt, three more as steps: the recurrence over all of them."""
    n, more = 70, 3
    x = make([n + more] * B, Hk, H, d, dv, dtype, seed=7 + d)
    ref = delta_oracle(*(x[k] for k in ("Q", "K", "V", "g", "beta", "off")))
    by = {k: x[k].reshape(B, n + more, *x[k].shape[1:]) for k in ("Q", "K", "V", "g", "beta")}
    head = {k: v[:, :n].reshape(B * n, *v.shape[2:]).contiguous() for k, v in by.items()}
    head["off"] = offsets([n] * B)
    t = dev(head)
    desc = desc_of(F, head, dtype)
    _, state = F.flex_delta_fwd(desc, *(t[k] for k in ("Q", "K", "V", "g", "beta", "off")), want_state=True)
    want = ref["O"].reshape(B, n + more, H, dv)
    for i in range(n, n + more):
        tok = {k: v[:, i].contiguous().cuda() for k, v in by.items()}
        o = F.flex_delta_step(F.make_delta_desc(B, Hk, H, d, B, dv=dv, io="bf16" if dtype == BF16 else "f32"), tok["Q"],
                              tok["K"], tok["V"], tok["g"], tok["beta"], state)
        near("o", o, want[:, i], NORM[dtype]["O"])
    near("state", state, ref["state"], NORM[dtype]["state"])


def test_decay_of_zero_clears_the_state(F):
    x = make([150], 1, 2, 64, 64, F32, seed=2)
    x["g"][[0, 70, 71, 128]] = -float("inf")
    ref = delta_oracle(*(x[k] for k in ("Q", "K", "V", "g", "beta", "off")))
    t = dev(x)
    O, state = F.flex_delta_fwd(desc_of(F, x, F32), *(t[k] for k in ("Q", "K", "V", "g", "beta", "off")), want_state=True)
    near("O", O, ref["O"], NORM[F32]["O"])
    near("state", state, ref["state"], NORM[F32]["state"])


def test_long_slow_decay(F):
    """Sixty chunks that hardly forget: errors of the carried state add up like independent ones."""
    x = make([3840], 1, 1, 128, 128, BF16, seed=3)
    x["g"] *= 0.1
    ref = delta_oracle(*(x[k] for k in ("Q", "K", "V", "g", "beta", "off")))
    t = dev(x)
    O, state = F.flex_delta_fwd(desc_of(F, x, BF16), *(t[k] for k in ("Q", "K", "V", "g", "beta", "off")), want_state=True)
    near("O", O, ref["O"], NORM[BF16]["O"])
    near("state", state, ref["state"], NORM[BF16]["state"])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d,dv,Hk,H", HEADS)
@pytest.mark.parametrize("lengths", LENGTHS)
def test_backward(F, lengths, d, dv, Hk, H, dtype):
    x = make(lengths, Hk, H, d, dv, dtype, seed=11 + d + len(lengths), pad=H % 2)
    names = ("Q", "K", "V", "g", "beta", "off")
    ref = delta_oracle(*(x[n] for n in names), dO=x["dO"])
    t, desc = dev(x), desc_of(F, x, dtype)
    args = [t[n] for n in names]
    saved = torch.empty(F.delta_saved_size(desc), dtype=torch.uint8, device="cuda")
    F.flex_delta_fwd(desc, *args, saved=saved)
    grads = F.flex_delta_bwd(desc, *args, t["dO"], saved)
    for n in ("dQ", "dK", "dV", "dg", "dbeta"):
        if lengths == [1] and n == "dg":   # a single token's decay meets an empty state
            assert (grads[n].float().abs() <= 1e-30).all()
            continue
        near(n, grads[n], ref[n], NORM[dtype]["grad"])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_backward_over_a_decay_of_zero(F, dtype):
    """g = -inf: what came before has no influence, and the decay itself no slope."""
    x = make([150, 64], 1, 2, 64, 64, dtype, seed=8)
    cut = [0, 70, 71, 128, 150]
    x["g"][cut] = -float("inf")
    names = ("Q", "K", "V", "g", "beta", "off")
    ref = delta_oracle(*(x[n] for n in names), dO=x["dO"])
    t, desc = dev(x), desc_of(F, x, dtype)
    saved = torch.empty(F.delta_saved_size(desc), dtype=torch.uint8, device="cuda")
    F.flex_delta_fwd(desc, *(t[n] for n in names), saved=saved)
    grads = F.flex_delta_bwd(desc, *(t[n] for n in names), t["dO"], saved)
    assert (grads["dg"][cut] == 0).all()
    for n in ("dQ", "dK", "dV", "dg", "dbeta"):
        near(n, grads[n], ref[n], NORM[dtype]["grad"])


def test_backward_against_differences(F):
    """<gradient, r> against the change of sum(dO O) along r, by the float64 recurrence: within the gradient's
    tolerance times both norms, and the difference's own error, step^2 = 1e-10 of derivatives that are of the
    gradient's size here."""
    x = make([70, 65], 2, 4, 64, 64, F32, seed=9)
    names = ("Q", "K", "V", "g", "beta", "off")
    t, desc = dev(x), desc_of(F, x, F32)
    saved = torch.empty(F.delta_saved_size(desc), dtype=torch.uint8, device="cuda")
    F.flex_delta_fwd(desc, *(t[n] for n in names), saved=saved)
    grads = F.flex_delta_bwd(desc, *(t[n] for n in names), t["dO"], saved)
    gen, h = torch.Generator().manual_seed(10), 1e-5
    for n in names[:5]:
        r = torch.randn(x[n].shape, generator=gen, dtype=torch.float64)
        ends = [(delta_oracle(*(x[m].double() + s * h * r if m == n else x[m] for m in names))["O"] * x["dO"].double()).sum()
                for s in (1, -1)]
        g = grads["d" + n].cpu().double()
        assert abs((g * r).sum() - (ends[0] - ends[1]) / (2 * h)) <= (NORM[F32]["grad"] + 1e-6) * g.norm() * r.norm(), n
