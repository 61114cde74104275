"""Gated delta rule, each head of each sequence by itself: heads that forget at once beside heads that hardly
forget, a short sequence beside a long one, gradient states carried over many chunks, a first state.

Bounds, relative to the 2-norm of a head's result and of its terms (tests.delta_terms; a gradient whose terms
cancel is off by roundings of the terms):
  O: one rounding, root mean square 2^-8 / sqrt(3) = 2.3e-3 at most, held to 2.4e-3; fp32 2.4e-6: operands are exact
    and 64 to 128 terms a chunk and product are summed in fp32, 5 products of 8 * 2^-24.
  gradients: a term is the product of two factors that are each rounded to bf16 once, 2.3e-3 each, and the terms
    that a head's state splits into (what the chunk began with, what it wrote, what it corrected) are together
    at most three times the state's: 3 * sqrt(2) * 2.3e-3 < 1e-2; fp32: 3 * sqrt(2) * 2.4e-6 < 1.2e-5.
"""
import pytest
import torch

from tests.delta_terms import delta_terms, near_by_head
from tests.seq_util import BF16, F32, offsets, rows
from tests.test_gpu_delta import HEADS, NORM, desc_of, dev

pytestmark = pytest.mark.gpu
NAMES = ("Q", "K", "V", "g", "beta", "off")


@pytest.fixture(scope="module")
def F():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2606_27748_amd as F
    F.load()
    return F


def inputs(lengths, Hk, H, d, dv, dtype, seed, rates):
    """Unit keys, beta 0 .. 1, g of head h between -rates[0][h] and -rates[1][h]."""
    gen, T = torch.Generator().manual_seed(seed), sum(lengths)
    x = {}
    for n in ("Q", "K"):
        v = rows(gen, T, Hk, d, F32).double() + 0.3
        x[n] = (v / v.norm(dim=-1, keepdim=True)).to(dtype)
    x["V"], x["dO"] = rows(gen, T, H, dv, dtype), rows(gen, T, H, dv, dtype)
    x["beta"] = torch.rand(T, H, generator=gen)
    lo, hi = (torch.as_tensor(r, dtype=torch.float32).expand(H) for r in rates)
    x["g"] = -(lo + (hi - lo) * torch.rand(T, H, generator=gen))
    x["off"] = offsets(lengths)
    x["state0"] = torch.randn(len(lengths), H, d, dv, generator=gen) * 0.3
    return x


def run_and_check(F, x, dtype, start=False):
    ref, quad = delta_terms(*(x[n] for n in NAMES), x["dO"], state0=x["state0"] if start else None)
    t, desc = dev(x), desc_of(F, x, dtype)
    saved = torch.empty(F.delta_saved_size(desc), dtype=torch.uint8, device="cuda")
    args = [t[n] for n in NAMES]
    O, _ = F.flex_delta_fwd(desc, *args, state0=t["state0"] if start else None, saved=saved)
    grads = F.flex_delta_bwd(desc, *args, t["dO"], saved)
    off, Hk = x["off"], x["Q"].shape[1]
    near_by_head("O", O, ref["O"], quad["O"] * 0, off, NORM[dtype]["O"])
    for n in ("dQ", "dK"):   # a key head's: the sum over its group
        ref[n] = ref[n].reshape(len(ref[n]), Hk, -1, ref[n].shape[-1]).sum(2)
        quad[n] = quad[n].reshape(len(ref[n]), Hk, -1, ref[n].shape[-1]).square().sum(2).sqrt()
    for n in ("dQ", "dK", "dV", "dg", "dbeta"):
        near_by_head(n, grads[n], ref[n], quad[n], off, NORM[dtype]["grad"])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d,dv,Hk,H", HEADS)
@pytest.mark.parametrize("lengths", [[64], [3, 0, 65, 200], [20, 63, 130]])
def test_every_head(F, lengths, d, dv, Hk, H, dtype):
    """Decays over two and a half powers of ten between the heads; the longest sequence last."""
    run_and_check(F, inputs(lengths, Hk, H, d, dv, dtype, 31 + d + len(lengths), (0.0, torch.logspace(-2.5, 0, H))), dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d,dv", [(64, 64), (128, 128)])
def test_many_chunks_of_slow_decay(F, d, dv, dtype):
    """Thirty-five chunks whose states, forward and reverse, hardly forget, behind a short sequence."""
    run_and_check(F, inputs([5, 2200], 1, 2, d, dv, dtype, 5, (0.0, [0.003, 0.03])), dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_heads_that_forget_at_once(F, dtype):
    """Decays of e^-5 to e^-8 a token: the slope of a decay is some thousandth of the terms beside it that have no
    part in it."""
    run_and_check(F, inputs([150, 64, 20], 1, 2, 64, 64, dtype, 6, (5.0, [8.0, 6.0])), dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_backward_behind_a_first_state(F, dtype):
    """A forward from state0 that keeps what a backward needs: the gradients with state0 held constant."""
    run_and_check(F, inputs([70, 1, 130], 1, 2, 64, 128, dtype, 7, (0.0, [0.05, 0.5])), dtype, start=True)
