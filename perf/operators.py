"""Cases of the packed-sequence operators: exact causal attention with grouped
heads, and the gated delta rule, each as a prompt's forward, a training step
(forward and backward) and a step of single tokens.

A case is a dict of plain values.  ``call`` names the entry point(s) of a pass:

  attn_fwd     flex_attn_fwd over packed prompts (``past`` keys before each
               sequence's first query: a prompt taken in pieces)
  attn_train   flex_attn_fwd, then flex_attn_bwd
  attn_decode  flex_attn_fwd of single tokens against a slotted cache
  delta_fwd    flex_delta_fwd over packed prompts, leaving the states
  delta_train  flex_delta_fwd, then flex_delta_bwd on what it saved
  delta_step   flex_delta_step: one token of every running sequence

B sequences, the longest of N tokens; ``mix`` 0 gives all of them N, any other
value is the seed of their lengths (shorter ones more often).  H value heads
(query heads of the attention), Hk heads that share keys (and for the delta
rule queries), d the head size, io "bf16" or "f32".  With ``fused`` the rows
are slices of one projection's output, with its row stride.

The plain forms pad the packed rows to a batch and work in 32 bits.
"""
from __future__ import annotations

import math
import random

import torch

own = False

C = 64   # chunk of the delta rule's plain form


def _case(name, call, B, N, H, Hk, d, io="bf16", mix=0, past=0, fused=False):
    return {"name": name, "call": call, "B": B, "N": N, "H": H, "Hk": Hk, "d": d, "io": io, "mix": mix,
            "past": past, "fused": fused}


def listed():
    return [
        # the smallest call: a short fp32 sequence (unit tests, notebooks); latency counts
        _case("attn_tiny_f32", "attn_fwd", 1, 33, 2, 1, 32, "f32"),
        # a serving batch's prompts of very different lengths, one layer
        _case("attn_packed", "attn_fwd", 16, 2048, 16, 4, 64, mix=5, fused=True),
        # one long prompt, one layer
        _case("attn_long", "attn_fwd", 1, 16384, 16, 2, 128),
        # one layer of language-model training, 8192-token sequences
        _case("attn_train", "attn_train", 2, 8192, 16, 4, 128),
        # the same over packed documents of odd lengths, heads of 64
        _case("attn_train_packed", "attn_train", 7, 3001, 12, 12, 64, mix=9, fused=True),
        # one layer of a decode step of a serving batch: bound by the cache
        _case("attn_decode", "attn_decode", 64, 8192, 16, 2, 128, mix=3),
        # one layer of a decode step of one long conversation
        _case("attn_decode_one", "attn_decode", 1, 40000, 16, 4, 128),
        # one layer of language-model training, 8192-token sequences
        _case("delta_train", "delta_train", 2, 8192, 16, 16, 128),
        # prompts of very different lengths, two value heads to a key head
        _case("delta_prefill", "delta_fwd", 9, 4096, 16, 8, 128, mix=7, fused=True),
        # training in full fp32 (small models, gradient checks), ragged length
        _case("delta_train_f32", "delta_train", 4, 1023, 8, 8, 64, "f32"),
        # one layer of a decode step of a full serving batch: bound by the state
        _case("delta_step", "delta_step", 256, 1, 16, 16, 128),
        # one layer of a decode step of a single sequence: bound by latency
        _case("delta_step_one", "delta_step", 1, 1, 12, 12, 64),
    ]


def _lengths(c):
    if not c["mix"]:
        return [c["N"]] * c["B"]
    r = random.Random(c["mix"])
    return [c["N"]] + [max(1, round(c["N"] * r.random() ** 1.5)) for _ in range(c["B"] - 1)]


def _cost(c):
    n = c["B"] * c["N"] * c["H"] * c["d"]
    if c["call"] == "attn_decode":
        return n / c["H"] * c["Hk"] * 3500   # at most twice the listed batch's cache
    if c["call"].startswith("attn"):
        return n * (c["N"] + 2 * c["past"]) * (3.5 if c["call"] == "attn_train" else 1) * (8 if c["io"] == "f32" else 1)
    return n * c["d"] * (60 if c["call"] == "delta_train" else 20) * (8 if c["io"] == "f32" else 1)


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    call = rng.choice(["attn_fwd", "attn_fwd", "attn_train", "attn_train", "attn_decode", "delta_fwd", "delta_train",
                       "delta_train", "delta_step"])
    while True:
        io = rng.choice(["bf16", "bf16", "bf16", "f32"])
        Hk, r = rng.choice([1, 2, 4, 8, 12]), rng.choice([1, 1, 2, 4, 8])
        B, N, mix, past = log_int(1, 24), log_int(20, 16000), rng.randrange(1000), 0
        if call.startswith("attn"):
            d = rng.choice([32, 64, 64, 128, 128])
            if call == "attn_fwd" and rng.random() < 0.3:
                past = log_int(1, 4000)
            if call == "attn_decode":
                B, N = log_int(1, 96), log_int(100, 60000)
        else:
            d = rng.choice([64, 128])
            r = rng.choice([1, 1, 2])
            if call == "delta_step":
                B, N = log_int(1, 256), 1
        c = {"call": call, "B": B, "N": N, "H": Hk * r, "Hk": Hk, "d": d, "io": io, "mix": mix, "past": past,
             "fused": rng.random() < 0.4}
        scores = 0 if call == "attn_decode" else B * Hk * r * N * (N + past)   # the plain form holds them all
        if call.startswith("delta"):
            scores = 0
        if Hk * r <= 32 and scores <= 2 ** 32 and _cost(c) <= _cost(listed()[3 if call[0] == "a" else 7]):
            return c


def prepare(case, seed):
    c, dev = case, torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(int(seed))
    io = torch.bfloat16 if c["io"] == "bf16" else torch.float32
    H, Hk, d, call = c["H"], c["Hk"], c["d"], c["call"]

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=dev, dtype=torch.float32)

    def offsets(ln):
        return torch.tensor([sum(ln[:i]) for i in range(len(ln) + 1)], dtype=torch.int32, device=dev)

    ln = _lengths(c)
    s = {"case": c}
    if call.startswith("attn"):
        nq = [1] * c["B"] if call == "attn_decode" else ln
        nk = ln if call == "attn_decode" else [n + c["past"] for n in ln]
        slots = [c["N"]] * c["B"] if call == "attn_decode" else nk   # a cache has room for the longest in every slot
        Tq, Tk = sum(nq), sum(slots)
        s["q_off"], s["k_off"] = offsets(nq), offsets(slots)
        s["k_len"] = torch.tensor(ln, dtype=torch.int32, device=dev) if call == "attn_decode" else None
        s["longest"] = (max(nq), max(nk))
        # queries and keys that attend: a logit's standard deviation is about two
        if c["fused"] and Tq == Tk:
            x = normal(Tq, H + 2 * Hk, d).to(io)
            x[:, :H + Hk] *= 2 ** 0.5
            s["Q"], s["K"], s["V"] = x[:, :H], x[:, H:H + Hk], x[:, H + Hk:]
        else:
            s["Q"] = (normal(Tq, H, d) * 2 ** 0.5).to(io)
            s["K"] = (normal(Tk, Hk, d) * 2 ** 0.5).to(io)
            s["V"] = normal(Tk, Hk, d).to(io)
        if call == "attn_train":
            s["dO"] = normal(Tq, H, d).to(io)
    else:
        T = c["B"] if call == "delta_step" else sum(ln)
        s["off"], s["longest"] = offsets(ln), max(ln)
        if c["fused"]:
            x = torch.empty(T, 2 * Hk + H, d, dtype=io, device=dev)
            s["Q"], s["K"], s["V"] = x[:, :Hk], x[:, Hk:2 * Hk], x[:, 2 * Hk:]
        else:
            s["Q"], s["K"] = (torch.empty(T, Hk, d, dtype=io, device=dev) for _ in range(2))
            s["V"] = torch.empty(T, H, d, dtype=io, device=dev)
        for name in ("Q", "K"):   # unit rows, with a part that they share, as after a convolution and its activation
            x = normal(T, Hk, d) + 0.3
            s[name].copy_(x / x.norm(dim=-1, keepdim=True))
        s["V"].copy_(normal(T, H, d))
        s["beta"] = torch.sigmoid(normal(T, H))
        # heads that forget over a few tokens to some hundreds
        rate = torch.exp(torch.linspace(math.log(0.003), math.log(0.7), H, device=dev))
        s["g"] = -rate * torch.nn.functional.softplus(normal(T, H) + 1.0)
        if call == "delta_train":
            s["dO"] = normal(T, H, d).to(io)
        if call == "delta_step":
            s["state"] = normal(T, H, d, d) * 0.3
    if own:
        _handles(s)
    return s


def work(case):
    c, e = case, 2 if case["io"] == "bf16" else 4
    ln, H, Hk, d = _lengths(c), c["H"], c["Hk"], c["d"]
    T = sum(ln)
    if c["call"] == "attn_decode":
        return {"bytes": e * d * (2 * c["B"] * H + 2 * T * Hk), "flops": 4 * d * H * T}
    if c["call"].startswith("attn"):
        past, train = c["past"], c["call"] == "attn_train"
        pairs = sum(n * (n + 1) // 2 + n * past for n in ln)
        rows = T * (2 * H) + (T + past * len(ln)) * 2 * Hk
        if train:   # q, k, v, o, do in; dq, dk, dv out
            rows += T * (4 * H) + T * 4 * Hk
        return {"bytes": e * d * rows + 4 * T * H, "flops": (14 if train else 4) * d * H * pairs}
    rows = T * (2 * Hk + 2 * H)
    if c["call"] == "delta_step":
        T = c["B"]
        return {"bytes": e * d * T * (2 * Hk + 2 * H) + 8 * T * H * d * d + 8 * T * H, "flops": 7 * T * H * d * d}
    if c["call"] == "delta_fwd":
        return {"bytes": e * d * rows + 8 * T * H + 4 * c["B"] * H * d * d, "flops": 7 * T * H * d * d}
    return {"bytes": e * d * (rows + T * (4 * Hk + 3 * H)) + (16 + 2 * e) * T * H, "flops": 21 * T * H * d * d}


# ---------------------------------------------------------------------------
# The framework's calls
# ---------------------------------------------------------------------------
def _handles(s):
    """Descriptor and workspaces, which a program makes once and keeps."""
    import paper_2606_27748_amd as flex
    c, call = s["case"], s["case"]["call"]
    strides = {"q_stride": s["Q"].stride(0), "k_stride": s["K"].stride(0), "v_stride": s["V"].stride(0)}
    if call.startswith("attn"):
        s["desc"] = flex.make_attn_desc(c["B"], c["H"], c["Hk"], c["d"], len(s["Q"]), len(s["K"]), causal=True,
                                        io=c["io"], **strides)
        passes = [flex.FLEX_PASS_FWD] + ([flex.FLEX_PASS_BWD] if call == "attn_train" else [])
        need = max(flex.attn_workspace_size(s["desc"], p) for p in passes)
    else:
        s["desc"] = flex.make_delta_desc(c["B"], c["Hk"], c["H"], c["d"], len(s["Q"]), io=c["io"], **strides)
        if call == "delta_step":
            return
        passes = [flex.FLEX_PASS_FWD] + ([flex.FLEX_PASS_BWD] if call == "delta_train" else [])
        need = max(flex.delta_workspace_size(s["desc"], p) for p in passes)
        if call == "delta_train":
            s["saved"] = torch.empty(flex.delta_saved_size(s["desc"]), dtype=torch.uint8, device=s["Q"].device)
    s["ws"] = torch.empty(max(need, 256), dtype=torch.uint8, device=s["Q"].device)


def _run_own(s):
    import paper_2606_27748_amd as flex
    call, d, Q, K, V = s["case"]["call"], s["desc"], s["Q"], s["K"], s["V"]
    if call.startswith("attn"):
        O, lse = flex.flex_attn_fwd(d, Q, K, V, s["q_off"], s["k_off"], k_len=s["k_len"], ws=s["ws"])
        if call != "attn_train":
            return {"O": O, "lse": lse}
        return {"O": O, **flex.flex_attn_bwd(d, Q, K, V, s["q_off"], s["k_off"], O, lse, s["dO"], ws=s["ws"])}
    if call == "delta_step":
        return {"O": flex.flex_delta_step(d, Q, K, V, s["g"], s["beta"], s["state"]), "state": s["state"]}
    if call == "delta_fwd":
        O, state = flex.flex_delta_fwd(d, Q, K, V, s["g"], s["beta"], s["off"], want_state=True, ws=s["ws"])
        return {"O": O, "state": state}
    O, _ = flex.flex_delta_fwd(d, Q, K, V, s["g"], s["beta"], s["off"], saved=s["saved"], ws=s["ws"])
    return {"O": O, **flex.flex_delta_bwd(d, Q, K, V, s["g"], s["beta"], s["off"], s["dO"], s["saved"], ws=s["ws"])}


# ---------------------------------------------------------------------------
# Plain forms
# ---------------------------------------------------------------------------
def _padded(x, start, length, n):
    """Packed rows [T, ...] -> [B, n, ...] in 32 bits, zeros behind each sequence."""
    j = torch.arange(n, device=x.device)
    y = x[(start[:, None] + j).clamp_(max=len(x) - 1)].float()
    return y * (j < length[:, None]).view(len(start), n, *[1] * (x.dim() - 1))


def _packed(y, start, T):
    """[B, n, ...] -> the packed rows [T, ...]."""
    t = torch.arange(T, device=y.device)
    b = torch.searchsorted(start, t, right=True) - 1
    return y[b, t - start[b]]


def _mm(a, b):
    return torch.matmul(a, b.contiguous())


def _attn(s):
    c, io = s["case"], s["Q"].dtype
    q0, k0 = s["q_off"].long(), s["k_off"].long()
    qn = q0[1:] - q0[:-1]
    kn = k0[1:] - k0[:-1] if s["k_len"] is None else s["k_len"].long()
    q0, k0, (nq, nk) = q0[:-1], k0[:-1], s["longest"]
    B, H, Hk, d, r = c["B"], c["H"], c["Hk"], c["d"], c["H"] // c["Hk"]

    def by_head(x, heads, start, length, n):
        return _padded(x, start, length, n).transpose(1, 2).reshape(B, Hk, heads // Hk * n, d)

    q = by_head(s["Q"], H, q0, qn, nq) * (1 / math.sqrt(d))
    k, v = by_head(s["K"], Hk, k0, kn, nk), by_head(s["V"], Hk, k0, kn, nk)
    i, j = torch.arange(nq, device=q.device)[:, None], torch.arange(nk, device=q.device)
    seen = (j < kn[:, None, None]) & (j <= i + (kn - qn)[:, None, None])
    p = _mm(q, k.transpose(-1, -2)).view(B, Hk, r, nq, nk).masked_fill_(~seen[:, None, None], -math.inf)
    top = p.amax(-1, keepdim=True)
    top = torch.where(torch.isfinite(top), top, torch.zeros_like(top))
    p = p.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    lse = (top + total.log())[..., 0]
    p = p.div_(total.clamp(min=1e-30)).view(B, Hk, r * nq, nk)
    o = _mm(p, v)

    def rows(x, heads, start, T, n):
        return _packed(x.reshape(B, heads, n, d).transpose(1, 2), start, T).to(io)

    out = {"O": rows(o, H, q0, len(s["Q"]), nq)}
    if c["call"] != "attn_train":
        out["lse"] = _packed(lse.reshape(B, H, nq).transpose(1, 2), q0, len(s["Q"]))
        return out
    do = by_head(s["dO"], H, q0, qn, nq)
    dv = _mm(p.transpose(-1, -2), do)
    ds = _mm(do, v.transpose(-1, -2)).sub_((do * o).sum(-1, keepdim=True)).mul_(p)
    out["dQ"] = rows(_mm(ds, k) * (1 / math.sqrt(d)), H, q0, len(s["Q"]), nq)
    out["dK"] = rows(_mm(ds.transpose(-1, -2), q), Hk, k0, len(s["K"]), nk)
    out["dV"] = rows(dv, Hk, k0, len(s["K"]), nk)
    return out


def _delta(s):
    c, io = s["case"], s["Q"].dtype
    B, H, Hk, d, train = c["B"], c["H"], c["Hk"], c["d"], c["call"] == "delta_train"
    start, T = s["off"].long(), len(s["Q"])
    length, start, n = start[1:] - start[:-1], start[:-1], -(-s["longest"] // C) * C
    leaves = {k: _padded(s[k], start, length, n).requires_grad_(train) for k in ("Q", "K", "V", "g", "beta")}

    with torch.set_grad_enabled(train):
        def chunks(x, heads):
            return x.transpose(1, 2).reshape(B, heads, n // C, C, -1)

        q, k = (chunks(leaves[x], Hk).repeat_interleave(H // Hk, 1) for x in ("Q", "K"))
        v, b, g = chunks(leaves["V"], H), chunks(leaves["beta"], H), chunks(leaves["g"], H)
        G = g.double().cumsum(-2)
        D = torch.exp((G - G.transpose(-1, -2)).tril()).float().tril()
        grow, last, left = torch.exp(G).float(), torch.exp(G[..., -1:, :]).float(), torch.exp(G[..., -1:, :] - G).float()
        kt = k.transpose(-1, -2)
        P = _mm(q, kt) * D
        A = -(_mm(k, kt) * D * b).tril(-1)
        eye = torch.eye(C, device=A.device)
        inv = eye + A
        for _ in range(5):   # (1 - A)^-1 = (1 + A)(1 + A^2)(1 + A^4)...: A^64 = 0
            A = _mm(A, A)
            inv = inv + _mm(A, inv)
        u0, w = _mm(inv, b * v), _mm(inv, b * grow * k)
        S, o = q.new_zeros(B, H, d, d), []
        for i in range(n // C):
            u = u0[:, :, i] - _mm(w[:, :, i], S)
            o.append(grow[:, :, i] * _mm(q[:, :, i], S) + _mm(P[:, :, i], u))
            S = last[:, :, i] * S + _mm(kt[:, :, i], left[:, :, i] * u)
        o = torch.stack(o, 2).reshape(B, H, n, d).transpose(1, 2) * (1 / math.sqrt(d))
    out = {"O": _packed(o.detach(), start, T).to(io)}
    if not train:
        return {**out, "state": S}
    got = torch.autograd.grad(o, list(leaves.values()), _padded(s["dO"], start, length, n))
    return {**out, **{"d" + k: _packed(x, start, T).to(io) for k, x in zip(leaves, got)}}


def _step(s):
    c, r, S = s["case"], s["case"]["H"] // s["case"]["Hk"], s["state"]
    q, k = (s[x].float().repeat_interleave(r, 1) for x in ("Q", "K"))
    S.mul_(torch.exp(s["g"])[..., None, None])
    u = s["beta"][..., None] * (s["V"].float() - (S * k[..., None]).sum(-2))
    S.add_(k[..., None] * u[..., None, :])
    return {"O": ((S * q[..., None]).sum(-2) / math.sqrt(c["d"])).to(s["Q"].dtype), "state": S}


def run(state):
    if own:
        return _run_own(state)
    call = state["case"]["call"]
    return _step(state) if call == "delta_step" else _attn(state) if call.startswith("attn") else _delta(state)


# ---------------------------------------------------------------------------
# The same outputs in 64 bits, a sequence and a head at a time
# ---------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    call, H, Hk, d = case["call"], case["H"], case["Hk"], case["d"]
    r, train = H // Hk, call.endswith("train")
    x = {k: s[k].double() for k in ("Q", "K", "V", "g", "beta", "dO", "state") if s.get(k) is not None}
    if call == "delta_step":
        q, k = (x[n][:, torch.arange(H, device=x[n].device) // r] for n in ("Q", "K"))
        S = x["state"] * torch.exp(x["g"])[:, :, None, None]
        read = torch.matmul(k[:, :, None], S)[:, :, 0]
        S = S + k[..., None] * (x["beta"][..., None] * (x["V"] - read))[:, :, None]
        return {"O": torch.matmul(q[:, :, None], S)[:, :, 0] / math.sqrt(d), "state": S}
    out = {"O": torch.zeros_like(x["Q"] if call.startswith("attn") else x["V"])}
    grads = {"d" + k: torch.zeros_like(x[k]) for k in ("Q", "K", "V", "g", "beta") if k in x} if train else {}
    if call.startswith("attn"):
        out["lse"] = torch.zeros_like(out["O"][..., 0])
        q0, k0 = s["q_off"].tolist(), s["k_off"].tolist()
        for b, n in enumerate(_lengths(case)):
            nq = q0[b + 1] - q0[b]
            nk = n if call == "attn_decode" else k0[b + 1] - k0[b]
            rq, rk = slice(q0[b], q0[b] + nq), slice(k0[b], k0[b] + nk)
            hidden = torch.ones(nq, nk, dtype=torch.bool, device=x["Q"].device).triu(nk - nq + 1)
            for h in range(H):
                at = {"Q": (rq, h), "K": (rk, h // r), "V": (rk, h // r)}
                leaf = {k: x[k][i].clone().requires_grad_(train) for k, i in at.items()}
                z = (leaf["Q"] @ leaf["K"].T / math.sqrt(d)).masked_fill(hidden, -math.inf)
                o = torch.softmax(z, -1) @ leaf["V"]
                out["O"][rq, h], out["lse"][rq, h] = o.detach(), torch.logsumexp(z.detach(), -1)
                if train:
                    o.backward(x["dO"][rq, h])
                    for k, i in at.items():
                        grads["d" + k][i] += leaf[k].grad
        if train:
            del out["lse"]
        return {**out, **grads}
    if not train:
        out["state"] = torch.zeros(case["B"], H, d, d, dtype=torch.float64, device=x["Q"].device)
    M, off = 128, s["off"].tolist()
    for b, n in enumerate(_lengths(case)):
        row = slice(off[b], off[b + 1])
        leaf = {k: x[k][row].transpose(0, 1).clone().requires_grad_(train) for k in ("Q", "K", "V", "g", "beta")}
        q, k = leaf["Q"].repeat_interleave(r, 0), leaf["K"].repeat_interleave(r, 0)
        S, o = torch.zeros(H, d, d, dtype=torch.float64, device=q.device), []
        for t in range(0, n, M):
            e = min(n, t + M)
            kc, beta, G = k[:, t:e], leaf["beta"][:, t:e, None], leaf["g"][:, t:e].cumsum(-1)
            D = torch.exp((G[:, :, None] - G[:, None]).tril()).tril()
            low = torch.eye(e - t, dtype=torch.float64, device=q.device) + (beta * D * (kc @ kc.mT)).tril(-1)
            # the writes u: u_i + sum_{j<i} b_i D_ij (k_i.k_j) u_j = b_i (v_i - e^G_i S^T k_i)
            known = beta * (leaf["V"][:, t:e] - torch.exp(G)[..., None] * (kc @ S))
            u = torch.linalg.solve_triangular(low, known, upper=False, unitriangular=True)
            o.append(torch.exp(G)[..., None] * (q[:, t:e] @ S) + (D * (q[:, t:e] @ kc.mT)) @ u)
            S = torch.exp(G[:, -1])[:, None, None] * S + kc.mT @ (torch.exp(G[:, -1:] - G)[..., None] * u)
        o = torch.cat(o, 1) / math.sqrt(d)
        out["O"][row] = o.detach().transpose(0, 1)
        if train:
            o.backward(x["dO"][row].transpose(0, 1))
            for name, v in leaf.items():
                grads["d" + name][row] = v.grad.transpose(0, 1)
        else:
            out["state"][b] = S
    return {**out, **grads}
