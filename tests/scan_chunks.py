"""The selective scan in float64 in chunks of 64 tokens, on the device that its inputs are on: results of calls of any size, with the
sums of absolute terms that the kernels' roundings scale with, so that each value can be held to a bound of its own."""
from __future__ import annotations

import ctypes

import torch

from tests.seq_util import BF16, STEP

CHUNK = 64
LENGTHS = [1000, 0, 130, 1, 700, 65, 604]
# N, P, G, H and lengths whose sequences go in segments of several chunks, some of which end within one: heads of a workgroup by
# one, two and four, few sequences and many
MANY_CHUNKS = [(64, 64, 16, 16, LENGTHS), (128, 64, 1, 32, [2000] + LENGTHS[1:]), (128, 128, 2, 16, [2000] + LENGTHS[1:]),
               (64, 128, 4, 12, [1400] + LENGTHS[1:]), (64, 64, 64, 64, [300, 0, 130, 1, 400, 65, 204])]


def tokens_of_a_segment(F, B, T, G, H, N, P):
    """At least this many, from the workspace: a state for each of T / tokens + B segments, and each one's decays behind them.  A
    multiple of 64."""
    n = ctypes.c_size_t()
    assert F.load().flex_scan_workspace_size(ctypes.byref(F.make_scan_desc(B, G, H, N, P, T)), F.FLEX_PASS_FWD, ctypes.byref(n)) == F.FLEX_OK
    slots = n.value // (H * N * P * 4 + H * 4)
    return 1 << 30 if slots == 0 else T // (slots - B + 1) // CHUNK * CHUNK + CHUNK


def inputs(lengths, G, H, N, P, dtype, seed, device):
    gen = torch.Generator(device=device).manual_seed(seed)
    T = sum(lengths)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=device)

    x = {"X": normal(T, H, P).to(dtype), "Bt": normal(T, G, N).to(dtype), "Ct": normal(T, G, N).to(dtype)}
    x["dt"] = torch.rand(T, H, generator=gen, device=device) * 0.5 + 0.01
    x["g"] = -torch.rand(T, H, generator=gen, device=device) * torch.logspace(-2.5, 0, H, device=device)
    x["D"] = normal(H)
    x["off"] = torch.tensor([sum(lengths[:i]) for i in range(len(lengths) + 1)], dtype=torch.int32, device=device)
    x["state0"] = normal(len(lengths), H, N, P)
    x["dY"] = normal(T, H, P).to(dtype)
    return x


def results(x, start=True, grads=True):
    """Y, state, dX, dB, dC, ddt, dD, and in `mag` the absolute terms of each that have a factor which bf16 rows' kernels
    round: a chunk's matrix, the state that it reads, its gradient."""
    f = {k: x[k].double() for k in ("X", "Bt", "Ct", "dt", "g", "D", "dY", "state0")}
    T, H, P = f["X"].shape
    G, N = f["Bt"].shape[1:]
    off, dev = x["off"].tolist(), f["X"].device
    B, of = len(off) - 1, torch.arange(H, device=dev) // (H // G)

    def zeros(*shape):
        return torch.zeros(*shape, dtype=torch.float64, device=dev)

    out = {"Y": zeros(T, H, P), "state": zeros(B, H, N, P)}
    if grads:
        out.update(dX=zeros(T, H, P), dB=zeros(T, G, N), dC=zeros(T, G, N), ddt=zeros(T, H), dD=(f["dY"] * f["X"]).sum((0, 2)))
    mag = {k: zeros(*out[k].shape) for k in ("Y", "dX", "dB", "dC") if k in out}

    def by_head(v, rows):   # [rows, heads, n] -> [H, rows, n]
        return v[rows].transpose(0, 1).contiguous()

    def group(v):           # [H, rows, n] -> [rows, G, n], summed over a group's heads
        return v.view(G, H // G, *v.shape[1:]).sum(1).transpose(0, 1)

    def mm(a, b):
        return torch.matmul(a, b.contiguous())

    for b in range(B):
        S = f["state0"][b] if start else zeros(H, N, P)
        starts = []
        chunks = [slice(r, min(r + CHUNK, off[b + 1])) for r in range(off[b], off[b + 1], CHUNK)]

        def parts(rows):
            X, Bh, Ch = by_head(f["X"], rows), by_head(f["Bt"], rows)[of], by_head(f["Ct"], rows)[of]
            dt, L = f["dt"][rows].T[..., None], f["g"][rows].T.cumsum(1)[..., None]   # [H, rows, 1]
            n = X.shape[1]
            hidden = torch.ones(n, n, dtype=torch.bool, device=dev).triu(1)
            E = torch.exp((L - L.transpose(1, 2)).masked_fill(hidden, -float("inf")))
            return X, Bh, Ch, dt, L, E, mm(Ch, Bh.transpose(1, 2)) * E

        for rows in chunks:
            X, Bh, Ch, dt, L, E, CB = parts(rows)
            Pm = CB * dt.transpose(1, 2)
            starts.append(S)
            out["Y"][rows] = (mm(Pm, X) + torch.exp(L) * mm(Ch, S) + f["D"][:, None, None] * X).transpose(0, 1)
            mag["Y"][rows] = (mm(Pm.abs(), X.abs()) + torch.exp(L) * mm(Ch.abs(), S.abs())).transpose(0, 1)
            S = torch.exp(L[:, -1:]) * S + mm(Bh.transpose(1, 2).contiguous(), torch.exp(L[:, -1:] - L) * dt * X)
        out["state"][b] = S
        if not grads:
            continue
        dS = zeros(H, N, P)
        for rows, S in zip(chunks[::-1], starts[::-1]):
            X, Bh, Ch, dt, L, E, CB = parts(rows)
            dY, up, v = by_head(f["dY"], rows), torch.exp(L), torch.exp(L[:, -1:] - L)
            M = E * mm(dY, X.transpose(1, 2)) * dt.transpose(1, 2)
            dXt = mm(CB.transpose(1, 2).contiguous(), dY) + v * mm(Bh, dS)
            out["dX"][rows] = (dt * dXt + f["D"][:, None, None] * dY).transpose(0, 1)
            out["ddt"][rows] = (dXt * X).sum(-1).T
            out["dC"][rows] = group(mm(M, Bh) + up * mm(dY, S.transpose(1, 2)))
            out["dB"][rows] = group(mm(M.transpose(1, 2).contiguous(), Ch) + dt * v * mm(X, dS.transpose(1, 2)))
            mag["dX"][rows] = (dt * (mm(CB.abs().transpose(1, 2).contiguous(), dY.abs()) + v * mm(Bh.abs(), dS.abs()))).transpose(0, 1)
            mag["dC"][rows] = group(up * mm(dY.abs(), S.abs().transpose(1, 2)))
            mag["dB"][rows] = group(dt * v * mm(X.abs(), dS.abs().transpose(1, 2)))
            dS = torch.exp(L[:, -1:]) * dS + mm(Ch.transpose(1, 2).contiguous(), up * dY)
    return out, mag


def bounds(x, ref, mag, dtype, start=True, grads=True):
    """What each value may be off by.  A factor that is rounded to bf16 is off by half a step, 2^-8 of itself, and what is rounded by less
    than 2^-13 (a decay's argument is the difference of two floats below 2^7, 2^-18 each off; a few fp32 roundings); the rest of
    a result, its fp32 sums of 128 elements, 64 tokens and heads, the terms of a state and of a sum over heads with 16
    bits or more, is less than 512 roundings of the absolute terms, 2^-15; the result's own rounding."""
    every, _ = results({k: v if k in ("g", "off") else v.abs() for k, v in x.items()}, start, grads)
    e = {k: 2.0 ** -15 * every[k] + (2.0 ** -24 if k in ("state", "dD") else STEP[dtype]) * ref[k].abs() for k in ref}
    if dtype == BF16:
        for k, m in mag.items():
            e[k] += (2.0 ** -8 + 2.0 ** -13) * m
    return e


def hold(name, got, ref, bound):
    """Every value within its bound, on the device."""
    assert got.shape == ref.shape and torch.isfinite(got).all(), name
    off = (got.double() - ref).abs()
    bad = off > bound + 1e-30
    assert not bad.any(), (name, int(bad.sum()), float((off / (bound + 1e-30)).max()))
