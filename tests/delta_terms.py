"""The gated delta rule token by token in float64, forward and backward by their formulas, and with each
gradient the quadrature of its terms: the root of the sum of their squares, which independent roundings of
the terms' factors scale with, also where the terms themselves cancel."""
from __future__ import annotations

import torch


def delta_terms(Q, K, V, g, beta, off, dO, state0=None, scale=None):
    """(results, quadratures): dicts of O, dQ, dK, dV, dg, dbeta, with dQ and dK per value head [T, H, d]."""
    Q, K, V, g, beta, dO = (x.double() for x in (Q, K, V, g, beta, dO))
    (T, Hk, d), (H, dv) = Q.shape, V.shape[1:]
    scale = d ** -0.5 if scale is None else scale
    head = torch.arange(H) // (H // Hk)
    q, k, a = Q[:, head], K[:, head], torch.exp(g)
    out = {n: torch.zeros(T, H, *s, dtype=torch.float64) for n, s in
           (("O", (dv,)), ("dQ", (d,)), ("dK", (d,)), ("dV", (dv,)), ("dg", ()), ("dbeta", ()))}
    quad = {n: torch.zeros_like(x) for n, x in out.items()}

    def put(n, t, *terms, over):
        """Sums of the terms (each [H, ...]) over an axis, and their squares'."""
        out[n][t] = sum(x.sum(over) for x in terms)
        quad[n][t] = sum(x.square().sum(over) for x in terms).sqrt()

    for b in range(len(off) - 1):
        rows = range(int(off[b]), int(off[b + 1]))
        S = torch.zeros(H, d, dv, dtype=torch.float64) if state0 is None else state0[b].double()
        before, write, read = {}, {}, {}
        for t in rows:
            before[t] = S * a[t, :, None, None]
            read[t] = (before[t] * k[t, :, :, None]).sum(1)
            write[t] = beta[t, :, None] * (V[t] - read[t])
            S = before[t] + k[t, :, :, None] * write[t][:, None]
            put("O", t, scale * S * q[t, :, :, None], over=1)
        dS = torch.zeros(H, d, dv, dtype=torch.float64)
        for t in reversed(rows):
            kt, qt, do = k[t, :, :, None], q[t, :, :, None], scale * dO[t][:, None]
            S = before[t] + kt * write[t][:, None]
            dS = dS + qt * do
            put("dQ", t, S * do, over=2)
            du = (dS * kt).sum(1)
            put("dV", t, beta[t, :, None, None] * dS * kt, over=1)
            put("dbeta", t, du * V[t], -du * read[t], over=1)
            dr = (-beta[t, :, None] * du)[:, None]
            put("dK", t, dS * write[t][:, None], before[t] * dr, over=2)
            dS = dS + kt * dr
            put("dg", t, (dS * before[t]).flatten(1), over=1)
            dS = dS * a[t, :, None, None]
    return out, quad


def by_key_head(x, Hk):
    """Per value head [T, H, d] -> the sum over each key head's group, and for quadratures its root of squares."""
    return x.reshape(len(x), Hk, -1, x.shape[-1])


def near_by_head(name, got, ref, quad, off, tol, few=16):
    """Of every head of every sequence by itself: the 2-norm of the difference within tol of that of the result and
    its terms, and no element further off than 8 tol of the largest of itself, its terms and their root mean
    squares.  tol is a root mean square; sequences of fewer than `few` tokens are held to what a rounding is
    off by at most, sqrt(3) of it."""
    got = got.detach().cpu().double()
    assert torch.isfinite(got).all(), name
    for b in range(len(off) - 1):
        at = slice(int(off[b]), int(off[b + 1]))
        n = at.stop - at.start
        if n == 0:
            continue
        t = tol if n >= few else tol * 3 ** 0.5
        for h in range(got.shape[1]):
            x, r, m = got[at, h], ref[at, h], quad[at, h]
            size = (r.square().sum() + m.square().sum()).sqrt()
            err = (x - r).norm()
            assert err <= t * size, (name, "sequence", b, "head", h, float(err / size), float(err / r.norm()))
            rms = size / max(r.numel(), 1) ** 0.5
            assert ((x - r).abs() <= 8 * t * torch.maximum(torch.maximum(r.abs(), m), rms)).all(), (name, b, h)
