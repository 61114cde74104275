"""Helpers of the tests of selective state-space layers: seeded inputs, float64 oracles written from the definitions,
and the sums of absolute terms that the results' roundings scale with."""
from __future__ import annotations

import torch

from tests.seq_util import BF16, offsets

U32 = 2.0 ** -24   # half a step of fp32, relative to the value


def wide(gen, T, width, dtype, pad=0, scale=1.0):
    """[T, width] rows, `pad` more values between them (NaN there: they are never read)."""
    x = torch.full((T, width + pad), float("nan"), dtype=dtype)
    x[:, :width] = torch.randn(T, width, generator=gen, dtype=torch.float64).mul(scale).to(dtype)
    return x[:, :width]


def on(x, device="cuda"):
    """To the device with the row stride kept, the memory between rows too."""
    if x.dim() >= 2 and x.shape[0] > 1 and not x.is_contiguous():
        full = torch.full((x.shape[0], x.stride(0)), float("nan"), dtype=x.dtype, device=device)
        row = full[:, :x[0].numel()]
        row.copy_(x.reshape(len(x), -1))
        return row.unflatten(1, x.shape[1:])
    return x.contiguous().to(device)


def stride(x):
    return x.stride(0) if len(x) > 1 else 0


def io_of(dtype):
    return "bf16" if dtype == BF16 else "f32"


def within(name, got, ref, bound):
    got, ref, bound = got.detach().cpu().double(), ref.double(), bound.double() + 1e-30
    assert got.shape == ref.shape and torch.isfinite(got).all(), name
    bad = (got - ref).abs() > bound
    assert not bad.any(), (name, int(bad.sum()), float(((got - ref).abs() / bound).max()))


def near(name, got, ref, tol):
    """2-norm of the difference within tol of the result's, and no element further off than 40 tol of the larger of
    itself and the root mean square."""
    got, ref = got.detach().cpu().double(), ref.double()
    assert got.shape == ref.shape and torch.isfinite(got).all(), name
    if ref.numel() == 0:
        return
    rms = ref.square().mean().sqrt()
    assert (got - ref).norm() <= tol * ref.norm() + 1e-30, (name, float((got - ref).norm() / ref.norm()))
    assert ((got - ref).abs() <= 40 * tol * torch.maximum(ref.abs(), rms) + 1e-30).all(), name


# ---- short convolution ----
def conv_inputs(lengths, D, K, dtype, seed, pad=0, lead=0, extra=0):
    """`lead` rows before the first sequence, `extra` behind the last."""
    gen = torch.Generator().manual_seed(seed)
    T = lead + sum(lengths) + extra
    x = {"X": wide(gen, T, D, dtype, pad), "dY": wide(gen, T, D, dtype), "W": torch.randn(D, K, generator=gen),
         "bias": torch.randn(D, generator=gen) * 0.3, "off": (offsets(lengths) + lead).int()}
    x["state0"] = torch.randn(len(lengths), K - 1, D, generator=gen).to(dtype)
    return x


def conv_oracle(x, act, state0=True, grads=False, bias=True):
    """Y, state, dX, dW, dbias in float64 with the bounds of their fp32 roundings (without the one to the io type).

    z is a chain of K + 1 fused products and sums: K + 1 roundings of at most the sum of absolute terms.  The
    sigmoid's exponential has an argument of size 1.45 |z| rounded twice and an ulp of its own, then a sum and a
    reciprocal of one ulp: (6 + 3 |z|) roundings of itself, and |z sigmoid'| <= 1.1, |(z sigmoid)''| <= 0.5."""
    X, W, dY = x["X"].double(), x["W"].double(), x["dY"].double()
    T, D = X.shape
    K, off = W.shape[1], x["off"].tolist()
    B = len(off) - 1
    b = x["bias"].double() if bias else torch.zeros(D, dtype=torch.float64)
    r = {"Y": torch.zeros_like(X), "dX": torch.zeros_like(X), "dW": torch.zeros_like(W), "dbias": torch.zeros_like(b),
         "state": torch.zeros(B, K - 1, D, dtype=torch.float64)}
    e = {k: torch.zeros_like(v) for k, v in r.items()}
    for i in range(B):
        rows = slice(off[i], off[i + 1])
        n = off[i + 1] - off[i]
        past = x["state0"][i].double() if state0 else torch.zeros(K - 1, D, dtype=torch.float64)
        line = torch.cat([past, X[rows]])
        r["state"][i] = line[n:]
        if n == 0:
            continue
        taps = torch.stack([line[k:k + n] for k in range(K)])   # [K, n, D]
        z = b + (taps * W.T[:, None]).sum(0)
        mag = b.abs() + (taps.abs() * W.T[:, None].abs()).sum(0)
        ez = (K + 1) * U32 * mag
        sig = torch.sigmoid(z)
        if act:
            r["Y"][rows] = z * sig
            e["Y"][rows] = 1.1 * ez + U32 * (8 + 3 * z.abs()) * (z * sig).abs()
            slope, eslope = sig * (1 + z * (1 - sig)), 0.5 * ez + U32 * (10 + 4 * z.abs())
        else:
            r["Y"][rows], e["Y"][rows] = z, ez
            slope, eslope = torch.ones_like(z), torch.zeros_like(z)
        if not grads:
            continue
        dz, edz = dY[rows] * slope, dY[rows].abs() * (eslope + U32 * slope.abs())
        for k in range(K):
            w, s = W[:, k], K - 1 - k   # of row t, tap k reaches output t + s
            if s < n:
                r["dX"][rows][:n - s] += w * dz[s:]
                e["dX"][rows][:n - s] += w.abs() * (edz + (K + 1) * U32 * dz.abs())[s:]
            # fp32 sums of up to 64 rows, 4 of them, then 64 bits: 70 roundings
            r["dW"][:, k] += (taps[k] * dz).sum(0)
            e["dW"][:, k] += (taps[k].abs() * (edz + 70 * U32 * dz.abs())).sum(0)
        r["dbias"] += dz.sum(0)
        e["dbias"] += (edz + 70 * U32 * dz.abs()).sum(0)
    return r, e


# ---- selective scan ----
def scan_inputs(lengths, G, H, N, P, dtype, seed, pad=0, lead=0, extra=0, rate=1.0):
    gen = torch.Generator().manual_seed(seed)
    T = lead + sum(lengths) + extra
    x = {"X": wide(gen, T, H * P, dtype, pad).unflatten(1, (H, P)), "dY": wide(gen, T, H * P, dtype).unflatten(1, (H, P)),
         "Bt": wide(gen, T, G * N, dtype, pad).unflatten(1, (G, N)), "Ct": wide(gen, T, G * N, dtype, pad).unflatten(1, (G, N))}
    x["dt"] = torch.rand(T, H, generator=gen) * 0.5 + 0.01
    x["g"] = -torch.rand(T, H, generator=gen) * torch.logspace(-2.5, 0, H)[None] * rate
    x["D"] = torch.randn(H, generator=gen)
    x["off"] = (offsets(lengths) + lead).int()
    x["state0"] = torch.randn(len(lengths), H, N, P, generator=gen)
    return x


SCAN_ROWS = ("X", "Bt", "Ct", "dt", "g", "D")


def scan_oracle(x, state0=True, grads=False, D=True):
    """Y, final states and the gradients in float64: the recurrence token by token."""
    leaf = {n: x[n].double().clone().requires_grad_(grads) for n in SCAN_ROWS}
    T, H, P = x["X"].shape
    off = x["off"].tolist()
    B, N = len(off) - 1, x["Bt"].shape[2]
    head = torch.arange(H) // (H // x["Bt"].shape[1])
    Bt, Ct = leaf["Bt"][:, head], leaf["Ct"][:, head]
    rows, states = {}, []
    for b in range(B):
        S = x["state0"][b].double() if state0 else torch.zeros(H, N, P, dtype=torch.float64)
        for t in range(off[b], off[b + 1]):
            S = S * torch.exp(leaf["g"][t])[:, None, None] + Bt[t, :, :, None] * (leaf["dt"][t][:, None] * leaf["X"][t])[:, None, :]
            y = (S * Ct[t, :, :, None]).sum(1)
            rows[t] = y + leaf["D"][:, None] * leaf["X"][t] if D else y
        states.append(S.detach())
    out = {"Y": torch.zeros(T, H, P, dtype=torch.float64), "state": torch.stack(states)}
    if rows:
        at = list(rows)
        y = torch.stack([rows[t] for t in at])
        out["Y"][at] = y.detach()
        if grads:
            y.backward(x["dY"].double()[at])
    if grads:
        out.update({"d" + {"Bt": "B", "Ct": "C"}.get(n, n): torch.zeros_like(v) if v.grad is None else v.grad for n, v in leaf.items()})
    return out


def scan_desc(F, x, dtype, **kw):
    X, Bt = x["X"], x["Bt"]
    return F.make_scan_desc(len(x["off"]) - 1, Bt.shape[1], X.shape[1], Bt.shape[2], X.shape[2], len(X), io=io_of(dtype),
                            x_stride=stride(X), b_stride=stride(Bt), c_stride=stride(x["Ct"]), **kw)


# ---- gated norm ----
def norm_oracle(x, group, gate, eps):
    """Y, dX, dZ, dW in float64 with the bounds of their fp32 roundings (without the one to the io type).

    A group's sum of squares has terms of a few roundings each and is summed over 32 values in a lane and 8 levels of lanes:
    50 roundings, half of them in its root; the sigmoid's are as the convolution's."""
    X, Z, W, dY = (x[k].double() for k in ("X", "Z", "W", "dY"))
    T, D = X.shape

    def by_group(v):
        return v.reshape(*v.shape[:-1], D // group, group)

    def mean(v):
        return by_group(v).mean(-1, keepdim=True).expand(*v.shape[:-1], D // group, group).reshape(v.shape)

    sig = torch.sigmoid(Z)
    s, ds = Z * sig, sig * (1 + Z * (1 - sig))
    eds = U32 * (10 + 4 * Z.abs())              # of silu'
    k = U32 * (60 + 6 * (0 if gate == "none" else Z.abs() + mean(Z.abs() * s.square()) / (mean(s.square()) + 1e-300)))
    u = X * s if gate == "first" else X
    r = 1 / torch.sqrt(mean(u * u) + eps)
    n = u * r
    last = s if gate == "last" else torch.ones_like(X)
    y = n * W * last
    dn = dY * W * last
    m, am = mean(dn * n), mean((dn * n).abs())
    du = r * (dn - n * m)
    edu = k * r * (dn.abs() + n.abs() * am * 3)
    out = {"Y": y, "dX": du * s if gate == "first" else du, "dW": (dY * n * last).sum(0)}
    err = {"Y": k * y.abs(), "dX": (edu * s.abs() + k * (du * s).abs()) if gate == "first" else edu}
    # fp32 sums of a walk's rows, then 64 bits
    err["dW"] = ((k + U32 * T) * (dY * n * last).abs()).sum(0)
    if gate == "first":
        out["dZ"], err["dZ"] = du * X * ds, edu * (X * ds).abs() + k * (du * X * ds).abs() + (du * X).abs() * eds
    if gate == "last":
        out["dZ"], err["dZ"] = dY * n * W * ds, k * (dY * n * W * ds).abs() + (dY * n * W).abs() * eds
    return out, err
