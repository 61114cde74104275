"""Packed-sequence operators where sizes and streams could trip them: rows whose bytes lie behind 4 GB, and two
calls at once on two streams.  Each against the same rows on their own: bit for bit."""
import pytest
import torch

from tests.seq_util import BF16, offsets
from tests.test_gpu_delta import dev
from tests.test_gpu_delta_heads import inputs

pytestmark = pytest.mark.gpu
NAMES = ("Q", "K", "V", "g", "beta")


@pytest.fixture(scope="module")
def F():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2606_27748_amd as F
    F.load()
    return F


def _delta(F, t, off, Hk, H, T):
    desc = F.make_delta_desc(len(off) - 1, Hk, H, 128, T)
    saved = torch.empty(F.delta_saved_size(desc), dtype=torch.uint8, device="cuda")
    O, _ = F.flex_delta_fwd(desc, *(t[n] for n in NAMES), off, saved=saved)
    return {"O": O, **F.flex_delta_bwd(desc, *(t[n] for n in NAMES), off, t["dO"], saved)}


def _attn(F, q, k, v, dO, off, T):
    desc = F.make_attn_desc(len(off) - 1, q.shape[1], k.shape[1], q.shape[2], T, T)
    O, lse = F.flex_attn_fwd(desc, q, k, v, off, off)
    return {"O": O, "lse": lse, **F.flex_attn_bwd(desc, q, k, v, off, off, O, lse, dO)}


def test_rows_behind_four_gigabytes(F):
    """Sequences in the last rows of tensors of 2^18 rows of 8192 and more elements."""
    lengths, T = [130, 70], (1 << 18) + 200
    n, skip = sum(lengths), (1 << 18)
    x = dev(inputs(lengths, 1, 64, 128, 128, BF16, 91, (0.0, [0.3] * 64)))
    off = offsets(lengths, "cuda")
    near = _delta(F, x, off, 1, 64, n)

    def behind(y):
        z = torch.zeros(T, *y.shape[1:], dtype=y.dtype, device="cuda")
        z[skip:] = y
        return z

    far = {m: behind(x[m]) for m in (*NAMES, "dO")}
    assert far["V"].numel() * 2 > 1 << 32
    got = _delta(F, far, off + skip, 1, 64, T)
    for m, v in near.items():
        assert torch.equal(got[m][skip:], v), m
    del got, far
    g = torch.Generator().manual_seed(92)
    q, dO = (torch.randn(n, 64, 128, generator=g).to(BF16).cuda() for _ in range(2))
    k, v = (torch.randn(n, 64, 128, generator=g).to(BF16).cuda() for _ in range(2))
    near = _attn(F, q, k, v, dO, off, n)
    got = _attn(F, *(behind(y) for y in (q, k, v, dO)), off + skip, T)
    for m, y in near.items():
        assert torch.equal(got[m][skip:], y), m


def test_two_calls_at_once(F):
    """A training step of each operator on a stream of its own, both on their way at the same time, four times over."""
    lengths = [700, 30, 1, 400]
    n, off = sum(lengths), offsets(lengths, "cuda")
    x = dev(inputs(lengths, 2, 4, 128, 128, BF16, 93, (0.0, [0.3] * 4)))
    g = torch.Generator().manual_seed(94)
    q, dO, k, v = (torch.randn(n, h, 128, generator=g).to(BF16).cuda() for h in (4, 4, 2, 2))
    ref_d, ref_a = _delta(F, x, off, 2, 4, n), _attn(F, q, k, v, dO, off, n)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(4):
        with torch.cuda.stream(streams[0]):
            d = _delta(F, x, off, 2, 4, n)
        with torch.cuda.stream(streams[1]):
            a = _attn(F, q, k, v, dO, off, n)
        torch.cuda.synchronize()
        assert all(torch.equal(d[m], y) for m, y in ref_d.items()) and all(torch.equal(a[m], y) for m, y in ref_a.items())
