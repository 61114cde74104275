"""Helpers of the packed-sequence tests: seeded inputs, float64 oracles written from the
definitions, and the error bounds that the tests hold results to."""
from __future__ import annotations

import math

import torch

BF16, F32 = torch.bfloat16, torch.float32
STEP = {BF16: 2.0 ** -8, F32: 2.0 ** -24}   # half a step relative to the value: what one rounding is off by at most


def offsets(lengths, device="cpu"):
    off = [0]
    for n in lengths:
        off.append(off[-1] + n)
    return torch.tensor(off, dtype=torch.int32, device=device)


def rows(gen, T, heads, d, dtype, pad=0, scale=1.0):
    """[T, heads, d] rows, `pad` extra heads' width between them (NaN there: it is never read)."""
    x = torch.full((T, heads + pad, d), float("nan"), dtype=dtype)
    x[:, :heads] = torch.randn(T, heads, d, generator=gen, dtype=torch.float64).mul(scale).to(dtype)
    return x[:, :heads]


def to_dev(x, device="cuda"):
    """To the device with the row stride kept."""
    if x.dim() == 3 and x.numel() and not x.is_contiguous():
        full = torch.full((x.shape[0], x.stride(0) // x.shape[2], x.shape[2]), float("nan"), dtype=x.dtype, device=device)
        full[:, :x.shape[1]] = x.to(device)
        return full[:, :x.shape[1]]
    return x.to(device)


def attn_oracle(Q, K, V, q_off, k_off, k_len=None, causal=True, scale=None, dO=None):
    """O, lse and, with dO, the gradients in float64, a sequence and a head at a time, only
    over the keys that a query sees; and with each result the sum of absolute terms that its
    roundings scale with."""
    Q, K, V = Q.double(), K.double(), V.double()
    Tq, Hq, d = Q.shape
    r = Hq // K.shape[1]
    scale = d ** -0.5 if scale is None else scale
    out = {"O": torch.zeros_like(Q), "lse": torch.full((Tq, Hq), -math.inf, dtype=torch.float64)}
    mag = {"O": torch.zeros_like(Q)}
    if dO is not None:
        dO = dO.double()
        for n, x in (("dQ", Q), ("dK", K), ("dV", V)):
            out[n], mag[n] = torch.zeros_like(x), torch.zeros_like(x)
    for b in range(len(q_off) - 1):
        q0, q1, k0, k1 = int(q_off[b]), int(q_off[b + 1]), int(k_off[b]), int(k_off[b + 1])
        if k_len is not None:
            k1 = k0 + min(max(int(k_len[b]), 0), k1 - k0)
        nq, nk = q1 - q0, k1 - k0
        seen = torch.ones(nq, nk, dtype=torch.bool)
        if causal:
            seen = seen.tril(nk - nq)
        some = seen.any(-1)
        for h in range(Hq):
            q, k, v = Q[q0:q1, h], K[k0:k1, h // r], V[k0:k1, h // r]
            s = torch.where(seen, scale * (q @ k.T), -math.inf)
            lse = torch.logsumexp(s, -1) if nk else torch.full((nq,), -math.inf, dtype=torch.float64)
            p = torch.where(some[:, None] & seen, torch.exp(s - torch.where(some, lse, 0.0)[:, None]), 0.0)
            out["lse"][q0:q1, h] = torch.where(some, lse, -math.inf)
            o = torch.where(p[:, :, None] > 0, p[:, :, None] * v, 0.0).sum(1) if not torch.isfinite(v).all() else p @ v
            out["O"][q0:q1, h] = o
            mag["O"][q0:q1, h] = p @ v.abs()
            if dO is None:
                continue
            g = dO[q0:q1, h]
            dp, delta = g @ v.T, (g * o).sum(-1, keepdim=True)
            ds = p * (dp - delta)
            dsm = p * (g.abs() @ v.abs().T + (g.abs() * (p @ v.abs())).sum(-1, keepdim=True))
            out["dQ"][q0:q1, h] += scale * ds @ k
            out["dK"][k0:k1, h // r] += scale * ds.T @ q
            out["dV"][k0:k1, h // r] += p.T @ g
            mag["dQ"][q0:q1, h] += scale * dsm @ k.abs()
            mag["dK"][k0:k1, h // r] += scale * dsm.T @ q.abs()
            mag["dV"][k0:k1, h // r] += p.T @ g.abs()
    return out, mag


def check(name, got, ref, mag, terms, dtype):
    """Every value within `terms` roundings of the sum of its absolute terms, and one of its own.

    A result sum_j a_j b_j whose factors carry relative roundings of u each and whose sum is held in
    fp32 is off by at most (number of rounded factors) u sum |a_j b_j| to first order, plus u of
    itself when it is stored."""
    got, u = got.detach().cpu().double(), STEP[dtype]
    bound = terms * u * mag + u * ref.abs() + 1e-30
    bad = ~((got - ref).abs() <= bound)
    assert not bad.any(), (name, int(bad.sum()), float(((got - ref).abs() / bound).nan_to_num(1e30).max()))


def delta_oracle(Q, K, V, g, beta, off, state0=None, scale=None, dO=None):
    """O, final states and, with dO, the gradients in float64: the recurrence token by token."""
    names = ("Q", "K", "V", "g", "beta")
    leaf = {n: x.double().clone().requires_grad_(dO is not None) for n, x in zip(names, (Q, K, V, g, beta))}
    T, Hk, d = Q.shape
    H, dv, B = V.shape[1], V.shape[2], len(off) - 1
    scale = d ** -0.5 if scale is None else scale
    head = torch.arange(H) // (H // Hk)
    q, k = leaf["Q"][:, head], leaf["K"][:, head]
    O, states = torch.zeros(T, H, dv, dtype=torch.float64), []
    rows = [None] * T
    for b in range(B):
        S = torch.zeros(H, d, dv, dtype=torch.float64) if state0 is None else state0[b].double()
        for t in range(int(off[b]), int(off[b + 1])):
            S = S * torch.exp(leaf["g"][t])[:, None, None]
            u = leaf["beta"][t, :, None] * (leaf["V"][t] - (S * k[t, :, :, None]).sum(1))
            S = S + k[t, :, :, None] * u[:, None, :]
            rows[t] = scale * (S * q[t, :, :, None]).sum(1)
        states.append(S.detach())
    kept = [t for t in range(T) if rows[t] is not None]
    out = {"state": torch.stack(states)}
    if kept:
        y = torch.stack([rows[t] for t in kept])
        O[kept] = y.detach()
        if dO is not None:
            y.backward(dO.double()[kept])
    out["O"] = O
    if dO is not None:
        out.update({"d" + n: torch.zeros_like(x) if x.grad is None else x.grad for n, x in leaf.items()})
    return out
