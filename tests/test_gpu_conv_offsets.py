"""Short convolution where the offsets fall: rows that no sequence holds are left alone, and no row before a sequence's first is
looked for anywhere but among its own first states."""
import pytest
import torch

from tests.layer_util import io_of
from tests.seq_util import BF16, F32

pytestmark = pytest.mark.gpu
T, K = 230, 4


@pytest.fixture(scope="module")
def F():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2606_27748_amd as F
    F.load()
    return F


FALLING = [[0, 200, 220, 60, 230], [10, 120, 200, 30, 40, 210], [230, 220, 60, 0, 230], [0, 64, 230, 100, 101, 99, 230],
           [-7, 500, 300, 20, 1000], [0, 50] + [220 - i for i in range(70)] + [230]]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [64, 1032])
@pytest.mark.parametrize("off", FALLING, ids=range(len(FALLING)))
def test_first_states_are_a_sequences_own(F, off, D, dtype):
    B, gen = len(off) - 1, torch.Generator(device="cuda").manual_seed(D)
    normal = lambda *n: torch.randn(*n, generator=gen, device="cuda")  # noqa: E731
    # finite first states between states of other sequences that are not
    around = torch.full((B + 2 * T, K - 1, D), float("nan"), dtype=dtype, device="cuda")
    state0 = around[T:T + B]
    state0.copy_(normal(B, K - 1, D))
    X, dY, W, bias = normal(T, D).to(dtype), normal(T, D).to(dtype), normal(D, K), normal(D)
    desc = F.make_conv_desc(B, T, D, K, io=io_of(dtype))
    o = torch.tensor(off, dtype=torch.int32, device="cuda")
    Y = torch.full((T, D), 1000.0, dtype=dtype, device="cuda")   # what the results do not reach
    dX = Y.clone()
    F.flex_conv_fwd(desc, X, W, bias, o, state0=state0, Y=Y)
    got = F.flex_conv_bwd(desc, X, W, bias, o, dY, state0=state0, dX=dX)
    for n, x in dict(got, Y=Y).items():
        assert torch.isfinite(x).all(), n
    ends = [min(max(e, 0), T) for e in off]
    none = torch.ones(T, dtype=torch.bool)
    for a, b in zip(ends, ends[1:]):
        none[a:b] = False
    assert (Y[none] == 1000).all() and (dX[none] == 1000).all()
    # the first sequence is whole where all others start behind it
    n = ends[1]
    if ends[0] == 0 and 0 < n <= min(ends[1:]):
        one = F.make_conv_desc(1, n, D, K, io=io_of(dtype))
        o1 = torch.tensor([0, n], dtype=torch.int32, device="cuda")
        want, _ = F.flex_conv_fwd(one, X[:n], W, bias, o1, state0=state0[:1])
        assert torch.equal(Y[:n], want)
        assert torch.equal(dX[:n], F.flex_conv_bwd(one, X[:n], W, bias, o1, dY[:n], state0=state0[:1])["dX"])
