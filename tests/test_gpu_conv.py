"""Short causal convolution against its definition in float64: packed sequences from one row to many, empty ones, rows of
none, first states, strided rows, single tokens.  Every value is held to the bound of its roundings
(tests.layer_util.conv_oracle) and one of its own to the io type."""
import pytest
import torch

from tests.layer_util import conv_inputs, conv_oracle, io_of, on, stride, within
from tests.seq_util import BF16, F32, STEP

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def F():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2606_27748_amd as F
    F.load()
    return F


def desc_of(F, x, dtype, act, **kw):
    return F.make_conv_desc(len(x["off"]) - 1, len(x["X"]), x["X"].shape[1], x["W"].shape[1], act="silu" if act else "none",
                            io=io_of(dtype), x_stride=stride(x["X"]), **kw)


LENGTHS = [[1], [2, 1, 3], [64], [33, 0, 5, 300], [0, 0], [255, 257, 1]]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D,K", [(8, 4), (520, 3), (1032, 4), (64, 2)])
@pytest.mark.parametrize("lengths", LENGTHS)
def test_forward(F, lengths, D, K, dtype):
    for start, act, pad, lead, extra in ((False, True, 0, 0, 0), (True, False, 16, 3, 40)):
        x = conv_inputs(lengths, D, K, dtype, D + K, pad, lead, extra)
        ref, err = conv_oracle(x, act, start, bias=act)
        t = {k: on(v) for k, v in x.items()}
        rows = torch.zeros(len(x["X"]), dtype=torch.bool)
        rows[lead:lead + sum(lengths)] = True
        Y = torch.full((len(rows), D), float("nan"), dtype=dtype, device="cuda")
        s0 = t["state0"] if start else None
        args = (desc_of(F, x, dtype, act), t["X"], t["W"], t["bias"] if act else None, t["off"])
        Y, state = F.flex_conv_fwd(*args, state0=s0, Y=Y, want_state=True)
        within("Y", Y[rows], ref["Y"][rows], err["Y"][rows] + STEP[dtype] * ref["Y"][rows].abs())
        assert torch.isnan(Y[~rows]).all()   # rows of no sequence are left as they were
        assert torch.equal(state.cpu(), ref["state"].to(dtype))
        if start:   # in place
            Y2, state2 = F.flex_conv_fwd(*args, state0=s0, state=s0)
            assert torch.equal(Y2[rows], Y[rows]) and torch.equal(state2, state) and state2 is s0


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D,K", [(8, 4), (520, 3), (1032, 4), (64, 2)])
@pytest.mark.parametrize("lengths", LENGTHS)
def test_backward(F, lengths, D, K, dtype):
    for start, act, pad, lead, extra in ((False, True, 0, 0, 0), (True, False, 16, 3, 40), (True, True, 0, 0, 1)):
        x = conv_inputs(lengths, D, K, dtype, D + K + 1, pad, lead, extra)
        ref, err = conv_oracle(x, act, start, grads=True, bias=act)
        t = {k: on(v) for k, v in x.items()}
        rows = torch.zeros(len(x["X"]), dtype=torch.bool)
        rows[lead:lead + sum(lengths)] = True
        desc = desc_of(F, x, dtype, act, dx_stride=D + pad)
        full = torch.full((len(rows), D + pad), float("nan"), dtype=dtype, device="cuda")
        got = F.flex_conv_bwd(desc, t["X"], t["W"], t["bias"] if act else None, t["off"], t["dY"],
                              state0=t["state0"] if start else None, dX=full[:, :D])
        within("dX", got["dX"][rows], ref["dX"][rows], err["dX"][rows] + STEP[dtype] * ref["dX"][rows].abs())
        assert torch.isnan(full[~rows]).all() and torch.isnan(full[:, D:]).all()
        within("dW", got["dW"], ref["dW"], err["dW"] + STEP[F32] * ref["dW"].abs())
        if act:
            within("dbias", got["dbias"], ref["dbias"], err["dbias"] + STEP[F32] * ref["dbias"].abs())
        else:
            assert got["dbias"] is None


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("K", [2, 4])
def test_every_value_of_a_large_call(F, K, dtype):
    """Small whole numbers and quarters, whose products and sums every type here holds: millions of values without one off.
    |x|, |dy| <= 8, |w| <= 1/2 and |bias| <= 2 in quarters: |z|, |dx| <= 18, 72 quarters; dW and dbias below 64 T = 2^20."""
    T, D = 16384, 1032
    gen = torch.Generator().manual_seed(K)
    whole = lambda n, *shape: torch.randint(-n, n + 1, shape, generator=gen).float()
    X, dY, W, bias = on(whole(8, T, D)), on(whole(8, T, D)), on(whole(2, D, K) / 4), on(whole(8, D) / 4)
    ends = [0, 5000, 5001, 16384]
    off = on(torch.tensor(ends, dtype=torch.int32))
    Y, dX, dW = bias.expand(T, D).clone(), torch.zeros_like(X), torch.zeros_like(W)
    for a, b in zip(ends, ends[1:]):
        for k in range(K):
            back = K - 1 - k
            if b - a > back:
                Y[a + back:b] += W[:, k] * X[a:b - back]
                dX[a:b - back] += W[:, k] * dY[a + back:b]
                dW[:, k] += (dY[a + back:b] * X[a:b - back]).sum(0)
    desc = F.make_conv_desc(3, T, D, K, act="none", io=io_of(dtype))
    args = (desc, X.to(dtype), W, bias, off)
    assert torch.equal(F.flex_conv_fwd(*args)[0].float(), Y)
    got = F.flex_conv_bwd(*args, dY.to(dtype))
    assert torch.equal(got["dX"].float(), dX) and torch.equal(got["dW"], dW) and torch.equal(got["dbias"], dY.sum(0))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D,K,B", [(8, 4, 1), (520, 3, 5), (1032, 4, 33), (64, 2, 2)])
def test_step_continues_a_prompt(F, D, K, B, dtype):
    """Prompts of n tokens, then steps: the same rows as longer prompts give."""
    n, more = 5, 4
    x = conv_inputs([n + more] * B, D, K, dtype, 3)
    ref, err = conv_oracle(x, True, False)
    X = x["X"].view(B, n + more, D)
    off = (torch.arange(B + 1) * n).int().cuda()
    W, bias = x["W"].cuda(), x["bias"].cuda()
    head = X[:, :n].reshape(B * n, D).cuda()
    _, state = F.flex_conv_fwd(F.make_conv_desc(B, B * n, D, K, io=io_of(dtype)), head, W, bias, off, want_state=True)
    full = torch.full((B, D + 64), float("nan"), dtype=dtype, device="cuda")
    desc = F.make_conv_desc(B, B, D, K, io=io_of(dtype), x_stride=D + 64 if B > 1 else 0)
    for i in range(n, n + more):
        full[:, :D] = X[:, i].cuda()
        y = F.flex_conv_step(desc, full[:, :D], W, bias, state)
        r, e = (v["Y"].view(B, n + more, D)[:, i] for v in (ref, err))
        within("y", y, r, e + STEP[dtype] * r.abs())
    assert torch.equal(state.cpu(), ref["state"].to(dtype))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_values_that_are_not_finite_stay_near(F, dtype):
    """A row with NaN reaches itself and the K-1 rows behind it in its sequence, and of the gradients that row's
    channel."""
    x = conv_inputs([40, 30], 16, 4, dtype, 5)
    clean = {k: on(v) for k, v in x.items()}
    args = lambda t: (desc_of(F, x, dtype, True), t["X"], t["W"], t["bias"], t["off"])  # noqa: E731
    Y0, _ = F.flex_conv_fwd(*args(clean))
    g0 = F.flex_conv_bwd(*args(clean), clean["dY"])
    t = dict(clean, X=clean["X"].clone(), dY=clean["dY"].clone())
    t["X"][38, 3] = float("nan")
    t["dY"][50, 5] = float("inf")
    Y, _ = F.flex_conv_fwd(*args(t))
    hit = torch.zeros_like(Y, dtype=torch.bool)
    hit[38:40, 3] = True
    assert torch.isnan(Y[hit]).all() and torch.equal(Y[~hit], Y0[~hit])
    g = F.flex_conv_bwd(*args(t), t["dY"])
    hit[:] = False
    hit[35:40, 3] = True    # dz of rows 38 and 39
    hit[47:51, 5] = True
    assert not torch.isfinite(g["dX"][hit]).any() and torch.equal(g["dX"][~hit], g0["dX"][~hit])
    cols = [c for c in range(16) if c not in (3, 5)]
    assert torch.equal(g["dW"][cols], g0["dW"][cols]) and not torch.isfinite(g["dW"][[3, 5]]).any()
