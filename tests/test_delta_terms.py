"""The delta rule's formulas of tests.delta_terms against automatic differentiation of the recurrence.  No GPU."""
import pytest
import torch

from tests.delta_terms import delta_terms
from tests.seq_util import F32, delta_oracle, offsets, rows


@pytest.mark.parametrize("start", [False, True])
def test_formulas_are_the_recurrences(start):
    gen, lengths, Hk, H = torch.Generator().manual_seed(1), [5, 0, 1, 9], 2, 4
    T = sum(lengths)
    Q, K, V, dO = (rows(gen, T, h, n, F32) for h, n in ((Hk, 16), (Hk, 16), (H, 8), (H, 8)))
    K = K / K.norm(dim=-1, keepdim=True)
    g, beta = -torch.rand(T, H, generator=gen), torch.rand(T, H, generator=gen)
    s0 = torch.randn(len(lengths), H, 16, 8, generator=gen) if start else None
    ref = delta_oracle(Q, K, V, g, beta, offsets(lengths), state0=s0, dO=dO)
    out, quad = delta_terms(Q, K, V, g, beta, offsets(lengths), dO, state0=s0)
    for n, x in out.items():
        if n in ("dQ", "dK"):
            x = x.reshape(T, Hk, H // Hk, -1).sum(2)
        assert (x - ref[n]).abs().max() <= 1e-12 * max(1.0, float(ref[n].abs().max())), n
    assert all((quad[n] >= 0).all() for n in quad)
