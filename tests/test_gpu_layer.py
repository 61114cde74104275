"""The operators of a selective state-space layer together, as a layer calls them: slices of one projection's rows
through the convolution, the scan and the gated norm; prompts, single tokens behind them, gradients; captured, on
another stream, two at once, and on rows behind 4 GB."""
import pytest
import torch

from tests.layer_util import near, wide
from tests.seq_util import BF16, F32, offsets

pytestmark = pytest.mark.gpu
G, H, N, P, K = 2, 4, 64, 64, 4
INNER, CONV = H * P, H * P + 2 * G * N
ROW = INNER + CONV + 8      # z, x and B and C, and a rest that belongs to neither


@pytest.fixture(scope="module")
def F():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2606_27748_amd as F
    F.load()
    return F


def make(lengths, dtype, seed):
    gen = torch.Generator().manual_seed(seed)
    T = sum(lengths)
    x = {"row": wide(gen, T, ROW, dtype), "off": offsets(lengths), "W": torch.randn(CONV, K, generator=gen) * 0.5,
         "bias": torch.randn(CONV, generator=gen) * 0.1, "dt": torch.rand(T, H, generator=gen) * 0.3 + 0.01,
         "D": torch.randn(H, generator=gen), "norm": 1 + 0.1 * torch.randn(INNER, generator=gen), "dY": wide(gen, T, INNER, dtype)}
    x["g"] = -x["dt"] * torch.tensor([0.3, 1.0, 4.0, 12.0])
    return x


class Layer:
    """Descriptors, workspaces and outputs of a layer's passes over T rows of B sequences."""
    def __init__(self, F, B, T, dtype, train=False):
        self.F, self.io = F, "bf16" if dtype == BF16 else "f32"
        s = dict(x_stride=ROW if T > 1 else 0)
        self.conv = F.make_conv_desc(B, T, CONV, K, io=self.io, dx_stride=ROW if T > 1 else 0, **s)
        c = dict.fromkeys(("x_stride", "b_stride", "c_stride", "dx_stride", "db_stride", "dc_stride"), CONV if T > 1 else 0)
        self.scan = F.make_scan_desc(B, G, H, N, P, T, io=self.io, **c)
        self.norm = F.make_norm_desc(T, INNER, INNER // 2, gate="first", io=self.io, z_stride=s["x_stride"], dz_stride=s["x_stride"])
        dev = dict(dtype=torch.uint8, device="cuda")
        need = [F.conv_workspace_size(self.conv), F.norm_workspace_size(self.norm)]
        need += [F.scan_workspace_size(self.scan, p) for p in (F.FLEX_PASS_FWD, F.FLEX_PASS_BWD)]
        self.ws = torch.empty(max(*need, 16), **dev)
        self.saved = torch.empty(F.scan_saved_size(self.scan), **dev) if train else None
        io = dict(dtype=dtype, device="cuda")
        self.xbc, self.y, self.out = torch.empty(T, CONV, **io), torch.empty(T, H, P, **io), torch.empty(T, INNER, **io)
        self.drow, self.dxbc, self.dy = torch.empty(T, ROW, **io), torch.empty(T, CONV, **io), torch.empty(T, INNER, **io)
        self.ddt, self.dg = torch.empty(T, H, **io), torch.empty(T, H, **io)
        f = dict(dtype=torch.float32, device="cuda")
        self.dW, self.dbias, self.dD, self.dnorm = (torch.empty(*n, **f) for n in ((CONV, K), (CONV,), (H,), (INNER,)))

    @staticmethod
    def split(x):
        a, b, c = x.split([INNER, G * N, G * N], 1)
        return a.unflatten(1, (H, P)), b.unflatten(1, (G, N)), c.unflatten(1, (G, N))

    def forward(self, t, conv_state=None, state=None, **kw):
        F, z, xbc = self.F, t["row"][:, :INNER], t["row"][:, INNER:INNER + CONV]
        _, conv_state = F.flex_conv_fwd(self.conv, xbc, t["W"], t["bias"], t["off"], state0=conv_state, Y=self.xbc, **kw)
        _, state = F.flex_scan_fwd(self.scan, *self.split(self.xbc), t["dt"], t["g"], t["D"], t["off"], state0=state, Y=self.y,
                                   saved=self.saved, ws=self.ws, **kw)
        F.flex_norm_fwd(self.norm, self.y.view(-1, INNER), z, t["norm"], Y=self.out)
        return conv_state, state

    def backward(self, t):
        F, z, xbc = self.F, t["row"][:, :INNER], t["row"][:, INNER:INNER + CONV]
        F.flex_norm_bwd(self.norm, self.y.view(-1, INNER), z, t["norm"], t["dY"], dX=self.dy, dZ=self.drow[:, :INNER], dW=self.dnorm,
                        ws=self.ws)
        dx, db, dc = self.split(self.dxbc)
        F.flex_scan_bwd(self.scan, *self.split(self.xbc), t["dt"], t["g"], t["D"], t["off"], self.dy.view(-1, H, P), self.saved, dX=dx,
                        dB=db, dC=dc, ddt=self.ddt, dg=self.dg, dD=self.dD, ws=self.ws)
        F.flex_conv_bwd(self.conv, xbc, t["W"], t["bias"], t["off"], self.dxbc, dX=self.drow[:, INNER:INNER + CONV], dW=self.dW,
                        dbias=self.dbias, ws=self.ws)

    def step(self, t, conv_state, state):
        F, z, xbc = self.F, t["row"][:, :INNER], t["row"][:, INNER:INNER + CONV]
        F.flex_conv_step(self.conv, xbc, t["W"], t["bias"], conv_state, y=self.xbc)
        F.flex_scan_step(self.scan, *self.split(self.xbc), t["dt"], t["g"], t["D"], state, y=self.y)
        F.flex_norm_fwd(self.norm, self.y.view(-1, INNER), z, t["norm"], Y=self.out)


def dev(x):
    return {k: v.cuda() for k, v in x.items()}


def reference(x, grads=False):
    """The layer in float64, from the definitions."""
    row = x["row"][:, :ROW].double().requires_grad_(grads)
    leaf = {k: x[k].double().clone().requires_grad_(grads) for k in ("W", "bias", "dt", "g", "D", "norm")}
    z, xbc = row[:, :INNER], row[:, INNER:INNER + CONV]
    off, outs = x["off"].tolist(), []
    for b in range(len(off) - 1):
        line = torch.cat([torch.zeros(K - 1, CONV, dtype=torch.float64), xbc[off[b]:off[b + 1]]])
        n = off[b + 1] - off[b]
        c = leaf["bias"] + sum(leaf["W"][:, k] * line[k:k + n] for k in range(K))
        outs.append(c * torch.sigmoid(c))
    xs, Bt, Ct = Layer.split(torch.cat(outs))
    head, rows = torch.arange(H) // (H // G), []
    for b in range(len(off) - 1):
        S = torch.zeros(H, N, P, dtype=torch.float64)
        for t in range(off[b], off[b + 1]):
            S = S * torch.exp(leaf["g"][t])[:, None, None] + Bt[t, head][:, :, None] * (leaf["dt"][t][:, None] * xs[t])[:, None, :]
            rows.append((S * Ct[t, head][:, :, None]).sum(1) + leaf["D"][:, None] * xs[t])
    u = (torch.stack(rows).reshape(-1, INNER) * z * torch.sigmoid(z)).reshape(-1, 2, INNER // 2)
    y = (u / torch.sqrt(u.square().mean(-1, keepdim=True) + 1e-5)).reshape(-1, INNER) * leaf["norm"]
    if not grads:
        return y.detach(), None
    y.backward(x["dY"].double())
    return y.detach(), {"row": row.grad, **{k: v.grad for k, v in leaf.items()}}


LENGTHS = [70, 1, 0, 200, 33]


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_layer_forward_and_backward(F, dtype):
    """Each operator is within 1e-2 (bf16) or 1.2e-5 (fp32) of its own results by 2-norm (their own tests), its inputs are
    off by what those before it left, and each passes an error on at most about as it passes its input: three
    operators forwards and three back, six times the tolerance of one, as sums of independent ones sqrt(6) < 2.5."""
    x = make(LENGTHS, dtype, 1)
    y, grads = reference(x, True)
    t, layer = dev(x), Layer(F, len(LENGTHS), sum(LENGTHS), dtype, train=True)
    layer.drow.fill_(7.0)
    layer.forward(t)
    layer.backward(t)
    tol = 2.5e-2 if dtype == BF16 else 3e-5
    near("out", layer.out, y, tol)
    near("dz", layer.drow[:, :INNER], grads["row"][:, :INNER], tol)
    near("dxbc", layer.drow[:, INNER:-8], grads["row"][:, INNER:-8], tol)
    assert (layer.drow[:, -8:] == 7).all()   # columns of no operator are left as they were
    for got, n in ((layer.dW, "W"), (layer.dbias, "bias"), (layer.ddt, "dt"), (layer.dg, "g"), (layer.dD, "D"), (layer.dnorm, "norm")):
        near(n, got, grads[n], tol)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_steps_behind_a_prompt(F, dtype):
    """Prompts, then tokens one by one, in place on the prompts' states: what the prompts with these tokens give."""
    n, more, B = 66, 3, 3
    x = make([n + more] * B, dtype, 2)
    whole, t = Layer(F, B, B * (n + more), dtype), dev(x)
    whole.forward(t)
    by = {k: t[k].view(B, n + more, -1) for k in ("row", "dt", "g")}
    head = {**t, **{k: v[:, :n].reshape(B * n, -1).contiguous() for k, v in by.items()}, "off": offsets([n] * B).cuda()}
    conv_state, state = Layer(F, B, B * n, dtype).forward(head, want_state=True)
    step = Layer(F, B, B, dtype)
    for i in range(n, n + more):
        step.step({**t, **{k: v[:, i].contiguous() for k, v in by.items()}}, conv_state, state)
        # the step's state and products are fp32, the prompt's have roundings to bf16 (tests of the scan): both are off, and
        # each operator's rows by one rounding
        near("step", step.out, whole.out.view(B, n + more, INNER)[:, i].double().cpu(), 1.2e-2 if dtype == BF16 else 1e-5)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_graph_replays(F, dtype):
    """A training step captured while an eager one's tensors live, replayed between eager work: bit for bit the eager
    step."""
    x, other = make(LENGTHS, dtype, 3), make(LENGTHS, dtype, 4)
    t, u, layer, eager = dev(x), dev(other), *(Layer(F, len(LENGTHS), sum(LENGTHS), dtype, train=True) for _ in range(2))
    outs = ("out", "dxbc", "ddt", "dg", "dW", "dbias", "dD", "dnorm")

    def run(a, b):
        a.drow.zero_()
        a.forward(b)
        a.backward(b)

    run(layer, t)
    torch.cuda.synchronize()
    want = {n: getattr(layer, n).clone() for n in outs + ("drow",)}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run(layer, t)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(layer, t)
    for _ in range(3):
        for n in want:
            getattr(layer, n).fill_(float("nan"))
        run(eager, u)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for n, v in want.items():
            assert torch.equal(getattr(layer, n), v), n


def test_two_streams_at_once(F):
    """Two layers on streams of their own, each with its workspace: the results of one after the other."""
    xs = [dev(make([500, 20, 300], BF16, s)) for s in (5, 6)]
    layers = [Layer(F, 3, 820, BF16, train=True) for _ in xs]
    want = []
    for layer, t in zip(layers, xs):
        layer.forward(t)
        layer.backward(t)
        want.append([x.clone() for x in (layer.out, layer.drow[:, :-8], layer.dW, layer.dg)])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    for layer in layers:
        layer.out.zero_()
        layer.drow.zero_()
    torch.cuda.synchronize()
    for _ in range(3):
        for s, layer, t in zip(streams, layers, xs):
            with torch.cuda.stream(s):
                layer.forward(t)
                layer.backward(t)
    torch.cuda.synchronize()
    for layer, w in zip(layers, want):
        for got, v in zip((layer.out, layer.drow[:, :-8], layer.dW, layer.dg), w):
            assert torch.equal(got, v)


def test_rows_behind_4_gb(F):
    """Rows a million elements apart: the last ones' places pass 32 bits.  The same values close together give the same
    results."""
    T, far = 2300, 1 << 20
    gen = torch.Generator(device="cuda").manual_seed(7)
    big = torch.empty(T, far, dtype=BF16, device="cuda")
    big[:, :CONV + INNER] = torch.randn(T, CONV + INNER, generator=gen, device="cuda")
    close = big[:, :CONV + INNER].contiguous()
    out = torch.empty(T, far, dtype=BF16, device="cuda")
    off = offsets([2000, 300]).cuda()
    W, bias = torch.randn(CONV, K, generator=gen, device="cuda") * 0.5, torch.zeros(CONV, device="cuda")
    dt = torch.rand(T, H, generator=gen, device="cuda") * 0.1
    D, w = torch.ones(H, device="cuda"), torch.ones(INNER, device="cuda")
    dY, dC = (torch.randn(T, n, generator=gen, device="cuda").to(BF16) for n in (INNER, CONV))
    got = []
    for rows, grads in ((big, out), (close, torch.empty_like(close))):
        s, r = rows.stride(0), []
        xbc, z, gx, gz = rows[:, :CONV], rows[:, CONV:CONV + INNER], grads[:, :CONV], grads[:, CONV:CONV + INNER]
        conv = F.make_conv_desc(2, T, CONV, K, x_stride=s, dx_stride=s)
        r += [F.flex_conv_fwd(conv, xbc, W, bias, off)[0], *F.flex_conv_bwd(conv, xbc, W, bias, off, dC, dX=gx).values()]
        r[1] = r[1].clone()
        scan = F.make_scan_desc(2, G, H, N, P, T, **dict.fromkeys(("x_stride", "b_stride", "c_stride", "dx_stride", "db_stride", "dc_stride"), s))
        saved = torch.empty(F.scan_saved_size(scan), dtype=torch.uint8, device="cuda")
        args = (scan, *Layer.split(xbc), dt, -dt, D, off)
        r += [*F.flex_scan_fwd(*args, saved=saved, want_state=True)]
        a, b, c = Layer.split(gx)
        F.flex_scan_bwd(*args, dY.view(T, H, P), saved, dX=a, dB=b, dC=c)
        r.append(gx.clone())
        norm = F.make_norm_desc(T, INNER, INNER, x_stride=s, z_stride=s, dx_stride=s, dz_stride=s)
        r.append(F.flex_norm_fwd(norm, xbc[:, :INNER], z, w))
        F.flex_norm_bwd(norm, xbc[:, :INNER], z, w, dY, dX=gx[:, :INNER], dZ=gz)
        r += [gx[:, :INNER].clone(), gz.clone()]
        got.append(r)
    for i, (a, b) in enumerate(zip(*got)):
        assert torch.isfinite(a.float()).all() and torch.equal(a, b), i


def test_offsets_that_are_not_in_order(F):
    """Offsets beyond the rows or falling lead nowhere outside the tensors; sequences that they leave whole keep their
    results."""
    x = make([100, 50, 80], BF16, 8)
    t = dev(x)
    ref = Layer(F, 3, 230, BF16, train=True)
    ref.forward(t)
    for off in ([0, 100, 150, 100000], [-5, 100, 150, 230], [0, 100, 60, 230], [400, 300, 200, 100], [0, 0, 0, 0]):
        layer = Layer(F, 3, 230, BF16, train=True)
        u = {**t, "off": torch.tensor(off, dtype=torch.int32, device="cuda")}
        layer.forward(u, want_state=True)
        layer.backward(u)
        torch.cuda.synchronize()
        if off[0] <= 0 and off[1] == 100:   # the first sequence is whole
            assert torch.equal(layer.out[:60], ref.out[:60])
