"""Gated norm of rows whose mean square is below or above what fp32 holds, with an eps that counts for nothing: r is defined, and
so are the results, of the sizes of W and dY."""
import math

import pytest
import torch

from tests.layer_util import io_of, norm_oracle, on, wide, within
from tests.seq_util import BF16, F32, STEP

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def F():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2606_27748_amd as F
    F.load()
    return F


# a lane's pieces, a wave's, a workgroup's; several rows a workgroup and one
@pytest.mark.parametrize("gate", ["none", "first", "last"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("group,D", [(8, 8), (24, 72), (256, 512), (1048, 1048), (2056, 2056), (8192, 8192)])
def test_rows_of_any_size(F, group, D, dtype, gate):
    """Rows of 1e-38 to 1e37 beside ordinary ones, each held to the bounds of its roundings; dY so that no gradient leaves
    fp32's range either.  eps is zero, or a subnormal that is nothing beside the mean squares; the smallest rows' own bits are
    the io type's subnormal ones."""
    sizes = [1.0, 1e-19, 1e-20, 3e-15, 1e-25, 1.0, 1e-38, 1e18, 1e20, 1e37, 1.0, 1e-30]
    gen = torch.Generator().manual_seed(D)
    size = torch.tensor(sizes, dtype=torch.float64)[:, None]
    unit = torch.rand(len(sizes), D, generator=gen, dtype=torch.float64) + 0.5   # none far below its row's others
    x = {"X": (unit * torch.sign(torch.randn(unit.shape, generator=gen)) * size).to(dtype), "Z": wide(gen, len(sizes), D, dtype),
         "dY": (torch.randn(len(sizes), D, generator=gen, dtype=torch.float64) * size.sqrt()).to(dtype),
         "W": torch.rand(D, generator=gen) + 0.5}
    if gate == "first":
        x["Z"] = (x["Z"].abs() + 0.25).to(dtype)   # so that u is of the row's size throughout
    t = {k: on(v) for k, v in x.items()}
    Z = None if gate == "none" else t["Z"]
    for eps in (0.0, 1e-41) if dtype == F32 else (0.0,):
        rows = [i for i, s in enumerate(sizes) if eps == 0 or s > 1e-19]
        ref, err = norm_oracle({k: v if k == "W" else v[rows] for k, v in x.items()}, group, gate, eps)
        desc = F.make_norm_desc(len(sizes), D, group, gate=gate, io=io_of(dtype), eps=eps)
        Y = F.flex_norm_fwd(desc, t["X"], Z, t["W"])
        within("Y", Y[rows], ref["Y"], err["Y"] + STEP[dtype] * ref["Y"].abs())
        got = F.flex_norm_bwd(desc, t["X"], Z, t["W"], t["dY"])
        for n in ("dX", "dZ"):
            if n in ref:
                within(n, got[n][rows], ref[n], err[n] + STEP[dtype] * ref[n].abs())
        if len(rows) == len(sizes):
            within("dW", got["dW"], ref["dW"], err["dW"] + STEP[F32] * ref["dW"].abs())


@pytest.mark.parametrize("gate", ["none", "first", "last"])
@pytest.mark.parametrize("group,D", [(24, 72), (256, 512), (8192, 8192)])
def test_ordinary_rows_beside_them(F, group, D, gate):
    """A row of one team's changes no other's results."""
    gen = torch.Generator().manual_seed(1)
    x = {k: on(wide(gen, 33, D, BF16)) for k in ("X", "Z", "dY")}
    W, Z = torch.ones(D, device="cuda"), None if gate == "none" else x["Z"]
    desc = F.make_norm_desc(33, D, group, gate=gate, eps=0.0)
    Y0, g0 = F.flex_norm_fwd(desc, x["X"], Z, W), F.flex_norm_bwd(desc, x["X"], Z, W, x["dY"])
    X = x["X"].clone()
    odd = [0, 5, 6, 32]
    X[odd] *= torch.tensor([1e-20, 1e30, 0.0, math.inf], device="cuda")[:, None].to(BF16)
    Y, g = F.flex_norm_fwd(desc, X, Z, W), F.flex_norm_bwd(desc, X, Z, W, x["dY"])
    rest = [i for i in range(33) if i not in odd]
    for got, want in ((Y, Y0), (g["dX"], g0["dX"]), (g["dZ"], g0["dZ"])):
        if got is not None:
            assert torch.equal(got[rest], want[rest])
    assert torch.isnan(Y[6]).all()   # 0 / 0, as the formula has it
