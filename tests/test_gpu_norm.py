"""Gated norm of rows against its definition in float64: groups from 8 channels to 8192 and odd ones, each gate, strided
rows, one row and many.  Every value is held to the bound of its roundings (tests.layer_util.norm_oracle) and one of its
own to the io type."""
import pytest
import torch

from tests.layer_util import io_of, norm_oracle, on, stride, wide, within
from tests.seq_util import BF16, F32, STEP

pytestmark = pytest.mark.gpu
GROUPS = [(8, 8), (24, 24), (128, 1024), (64, 64), (200, 1000), (520, 1040), (1048, 1048), (2048, 4096), (2056, 2056),
          (4096, 4096), (4104, 8208), (8192, 8192)]


@pytest.fixture(scope="module")
def F():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2606_27748_amd as F
    F.load()
    return F


def make(T, D, dtype, seed, pad=0):
    gen = torch.Generator().manual_seed(seed)
    x = {k: wide(gen, T, D, dtype, pad) for k in ("X", "Z")}
    return {**x, "dY": wide(gen, T, D, dtype), "W": torch.randn(D, generator=gen)}


def desc_of(F, x, group, gate, dtype, eps=1e-5, **kw):
    T, D = x["X"].shape
    return F.make_norm_desc(T, D, group, gate=gate, io=io_of(dtype), eps=eps, x_stride=stride(x["X"]),
                            z_stride=stride(x["Z"]) if gate != "none" else 0, **kw)


@pytest.mark.parametrize("gate", ["none", "first", "last"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("group,D", GROUPS)
def test_forward_and_backward(F, group, D, dtype, gate):
    for T, pad, eps in ((1, 0, 1e-5), (7, 16, 0.1), (300 if D < 2000 else 40, 8, 1e-5)):
        x = make(T, D, dtype, D + T, pad)
        ref, err = norm_oracle(x, group, gate, eps)
        t = {k: on(v) for k, v in x.items()}
        strides = dict(dx_stride=D + pad, dz_stride=0 if gate == "none" else D + pad) if T > 1 else {}
        desc = desc_of(F, x, group, gate, dtype, eps, **strides)
        Z = None if gate == "none" else t["Z"]
        Y = F.flex_norm_fwd(desc, t["X"], Z, t["W"])
        within("Y", Y, ref["Y"], err["Y"] + STEP[dtype] * ref["Y"].abs())
        got = F.flex_norm_bwd(desc, t["X"], Z, t["W"], t["dY"])
        for n in ("dX", "dZ", "dW"):
            if n == "dZ" and gate == "none":
                assert got[n] is None
                continue
            within(n, got[n], ref[n], err[n] + STEP[F32 if n == "dW" else dtype] * ref[n].abs())


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_many_rows(F, dtype):
    """More rows than are walked at once: every row once, dW over all of them."""
    x = make(9001, 136, dtype, 4)
    ref, err = norm_oracle(x, 136, "first", 1e-5)
    t, desc = {k: on(v) for k, v in x.items()}, desc_of(F, x, 136, "first", dtype)
    Y = F.flex_norm_fwd(desc, t["X"], t["Z"], t["W"])
    within("Y", Y, ref["Y"], err["Y"] + STEP[dtype] * ref["Y"].abs())
    got = F.flex_norm_bwd(desc, t["X"], t["Z"], t["W"], t["dY"])
    for n in ("dX", "dZ", "dW"):
        within(n, got[n], ref[n], err[n] + STEP[F32 if n == "dW" else dtype] * ref[n].abs())
    again = F.flex_norm_bwd(desc, t["X"], t["Z"], t["W"], t["dY"])
    assert all(torch.equal(got[n], again[n]) for n in got)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,group,D", [(70001, 8, 8), (40003, 24, 72), (50000, 64, 64), (20000, 56, 504), (9000, 512, 512), (12000, 40, 360)])
def test_many_narrow_rows(F, T, group, D, dtype):
    """Rows of which a workgroup has several, more of them than are walked at once."""
    x = make(T, D, dtype, 5, 8)
    t, desc = {k: on(v) for k, v in x.items()}, desc_of(F, x, group, "last", dtype)
    ref, err = norm_oracle(x, group, "last", 1e-5)
    Y = F.flex_norm_fwd(desc, t["X"], t["Z"], t["W"])
    within("Y", Y, ref["Y"], err["Y"] + STEP[dtype] * ref["Y"].abs())
    got = F.flex_norm_bwd(desc, t["X"], t["Z"], t["W"], t["dY"])
    for n in ("dX", "dZ", "dW"):
        within(n, got[n], ref[n], err[n] + STEP[F32 if n == "dW" else dtype] * ref[n].abs())


def test_rows_are_for_themselves(F):
    """A row of NaN or zeros changes no other row's results."""
    x = make(33, 256, BF16, 6)
    t, desc = {k: on(v) for k, v in x.items()}, desc_of(F, x, 64, "last", BF16)
    Y0 = F.flex_norm_fwd(desc, t["X"], t["Z"], t["W"])
    g0 = F.flex_norm_bwd(desc, t["X"], t["Z"], t["W"], t["dY"])
    t["X"][5, 70] = float("nan")
    t["X"][9] = 0
    Y = F.flex_norm_fwd(desc, t["X"], t["Z"], t["W"])
    g = F.flex_norm_bwd(desc, t["X"], t["Z"], t["W"], t["dY"])
    rest = [i for i in range(33) if i not in (5, 9)]
    assert torch.equal(Y[rest], Y0[rest]) and torch.isnan(Y[5, 64:128]).all() and (Y[9] == 0).all()
    assert torch.equal(Y[5, 128:], Y0[5, 128:])
    for n in ("dX", "dZ"):
        assert torch.equal(g[n][rest], g0[n][rest]) and torch.isfinite(g[n][9]).all()


@pytest.mark.parametrize("gate", ["none", "first", "last"])
def test_backward_against_differences(F, gate):
    """<gradient, r> against the change of sum(dY Y) along r in float64: within the gradients' bounds and the
    difference's own error, step^2 of third derivatives that are of the gradient's size here."""
    x = make(6, 48, F32, 8)
    t, desc = {k: on(v) for k, v in x.items()}, desc_of(F, x, 24, gate, F32)
    got = F.flex_norm_bwd(desc, t["X"], None if gate == "none" else t["Z"], t["W"], t["dY"])
    _, err = norm_oracle(x, 24, gate, 1e-5)
    gen, h = torch.Generator().manual_seed(9), 1e-5
    for n in ("X", "Z", "W"):
        if n == "Z" and gate == "none":
            continue
        r = torch.randn(x[n].shape, generator=gen, dtype=torch.float64)
        ends = [(norm_oracle(dict(x, **{n: x[n].double() + s * h * r}), 24, gate, 1e-5)[0]["Y"] * x["dY"].double()).sum()
                for s in (1, -1)]
        g = got["d" + n].cpu().double()
        slack = (err["d" + n] * r.abs()).sum() + 2.0 ** -24 * (g * r).abs().sum() + 1e-6 * g.norm() * r.norm()
        assert abs((g * r).sum() - (ends[0] - ends[1]) / (2 * h)) <= slack, n
