"""Cases of the operators of a selective state-space layer over packed sequences: the
short causal convolution in front of it, the scan, and the gated norm behind it.

A case is a dict of plain values.  ``call`` names the entry point(s) of a pass:

  conv_fwd    flex_conv_fwd over packed prompts, leaving the last rows
  conv_train  flex_conv_fwd, then flex_conv_bwd
  conv_step   flex_conv_step: one token of every running sequence
  scan_fwd    flex_scan_fwd over packed prompts, leaving the states
  scan_train  flex_scan_fwd, then flex_scan_bwd on what it saved
  scan_step   flex_scan_step: one token of every running sequence
  norm_fwd    flex_norm_fwd
  norm_train  flex_norm_fwd, then flex_norm_bwd

B sequences, the longest of N tokens; ``mix`` 0 gives all of them N, any other
value is the seed of their lengths (shorter ones more often).  io "bf16" or
"f32".  With ``start`` the sequences continue from given states; with ``fused``
rows are slices of a wider row, as one projection or convolution puts them out,
and so are the gradients' rows.
Convolution: D channels, K taps, ``act`` for SiLU behind it.  Scan: H heads of P
columns on G groups of keys and queries of S elements.  Norm: D channels in groups of
``group``, ``gate`` "first" (before the norm) or "last".

The plain forms work in 32 bits (decays in 64); the scan's pads the packed rows to a batch.
"""
from __future__ import annotations

import math
import random

import torch

own = False

C = 64       # chunk of the scan's plain form
EPS = 1e-5   # of the norm


def _conv(name, call, B, N, D, K=4, io="bf16", mix=0, act=True, start=False, fused=False):
    return {"name": name, "call": call, "B": B, "N": N, "D": D, "K": K, "io": io, "mix": mix, "act": act,
            "start": start, "fused": fused}


def _scan(name, call, B, N, H, G, S, P, io="bf16", mix=0, start=False, fused=False):
    return {"name": name, "call": call, "B": B, "N": N, "H": H, "G": G, "S": S, "P": P, "io": io, "mix": mix,
            "start": start, "fused": fused}


def _norm(name, call, N, D, group, gate, io="bf16", fused=False):
    return {"name": name, "call": call, "B": 1, "N": N, "D": D, "group": group, "gate": gate, "io": io, "fused": fused}


def listed():
    return [
        # a serving batch's prompts of very different lengths, pieces of longer ones among them, one layer
        _conv("conv_prompts", "conv_fwd", 16, 4096, 4352, mix=5, start=True, fused=True),
        # one layer of language-model training, 8192-token sequences
        _conv("conv_train", "conv_train", 2, 8192, 4352, fused=True),
        # one layer of a decode step of a full serving batch: bound by latency
        _conv("conv_step", "conv_step", 256, 1, 4352),
        # the smallest call: a short fp32 sequence (unit tests, notebooks); latency counts
        _scan("scan_tiny_f32", "scan_fwd", 1, 33, 2, 1, 64, 64, "f32"),
        # a serving batch's prompts of very different lengths, one layer
        _scan("scan_prompts", "scan_fwd", 16, 4096, 64, 1, 128, 64, mix=7, start=True, fused=True),
        # one long prompt of a model of few, wide heads
        _scan("scan_long", "scan_fwd", 1, 32768, 16, 2, 128, 128),
        # one layer of language-model training, 8192-token sequences
        _scan("scan_train", "scan_train", 2, 8192, 64, 1, 128, 64, fused=True),
        # training in full fp32 over documents of odd lengths (small models, gradient checks)
        _scan("scan_train_f32", "scan_train", 5, 1023, 8, 4, 64, 64, "f32", mix=3),
        # one layer of a decode step of a full serving batch: bound by the states
        _scan("scan_step", "scan_step", 256, 1, 32, 1, 128, 64),
        # one layer of a decode step of a single sequence: bound by latency
        _scan("scan_step_one", "scan_step", 1, 1, 24, 1, 64, 64),
        # a serving batch's prompts behind the scan, one norm over a row
        _norm("norm_prompts", "norm_fwd", 17973, 4096, 4096, "first", fused=True),
        # one layer of language-model training behind a recurrence with heads of 128, a norm each
        _norm("norm_train", "norm_train", 16384, 2048, 128, "last", fused=True),
    ]


def _lengths(c):
    if not c.get("mix"):
        return [c["N"]] * c["B"]
    r = random.Random(c["mix"])
    return [c["N"]] + [max(1, round(c["N"] * r.random() ** 1.5)) for _ in range(c["B"] - 1)]


def _cost(c):
    """Of a pass of the plain form, which pads to the longest; comparable within one kind of call."""
    n = c["B"] * c["N"]
    if not c["call"].startswith("scan"):
        return n * c["D"] * (2 if c["io"] == "f32" else 1)
    if c["call"] == "scan_step":
        return n * c["H"] * c["S"] * c["P"] / 4
    chunks = c["N"] / C
    each = c["P"] * (C + 3 * c["S"] + c["S"] * chunks / C) + C * (c["S"] + 8 * 10) + 40 * c["P"]
    return n * c["H"] * each * (3 if c["call"] == "scan_train" else 1)


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    call = rng.choice(["conv_fwd", "conv_train", "conv_step", "scan_fwd", "scan_fwd", "scan_train", "scan_train",
                       "scan_step", "norm_fwd", "norm_train"])
    top = max(_cost(c) for c in listed() if (c["call"][:4], c["call"].endswith("step")) == (call[:4], call.endswith("step")))
    while True:
        io = rng.choice(["bf16", "bf16", "bf16", "f32"])
        B, N, mix = log_int(1, 24), log_int(20, 16000), rng.randrange(1000)
        start, fused = rng.random() < 0.4, rng.random() < 0.5
        if call.endswith("step"):
            B, N, mix, start = log_int(1, 256), 1, 0, False
        if call.startswith("conv"):
            c = _conv("", call, B, N, 8 * log_int(8, 900), rng.choice([2, 3, 4, 4]), io, mix, rng.random() < 0.8, start, fused)
        elif call.startswith("scan"):
            G, r = rng.choice([1, 1, 2, 4, 8]), rng.choice([1, 2, 3, 4, 8, 24, 64])
            c = _scan("", call, B, N, G * r, G, rng.choice([64, 128]), rng.choice([64, 64, 128]), io, mix, start, fused)
            if G * r > 64:
                continue
        else:
            group = 8 * log_int(4, 512)
            c = _norm("", call, log_int(1, 20000), group * rng.randint(1, max(1, min(16, 8192 // group))), group,
                      rng.choice(["first", "last"]), io, fused)
        del c["name"]
        if _cost(c) <= top:
            return c


def prepare(case, seed):
    c, dev = case, torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(int(seed))
    io = torch.bfloat16 if c["io"] == "bf16" else torch.float32
    ln, call = _lengths(c), c["call"]
    T, train = sum(ln), call.endswith("train")

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=dev, dtype=torch.float32)

    def row(*widths):
        """Rows of io values of the given widths, in one wider row or each for itself."""
        if c["fused"]:
            x = normal(T, sum(widths)).to(io)
            return list(x.split(widths, 1))
        return [normal(T, w).to(io) for w in widths]

    s = {"case": c, "T": T, "lengths": ln}
    s["off"] = torch.tensor([sum(ln[:i]) for i in range(len(ln) + 1)], dtype=torch.int32, device=dev)
    if call.startswith("conv"):
        D, K = c["D"], c["K"]
        s["X"] = row(D, 64)[0]   # a projection's output has other columns behind the convolution's
        s["W"] = (torch.rand(D, K, generator=gen, device=dev) - 0.5) * (2 / math.sqrt(K))
        s["bias"] = normal(D) * 0.1
        if c["start"] or call == "conv_step":
            s["state"] = normal(c["B"], K - 1, D).to(io)
        if train:
            s["dY"] = normal(T, D).to(io)
    elif call.startswith("scan"):
        H, G, S, P = c["H"], c["G"], c["S"], c["P"]
        rows = row(H * P, G * S, G * S)
        for x in rows:   # behind the convolution's SiLU
            x.copy_(torch.nn.functional.silu(x.float()))
        s["X"], s["Bt"], s["Ct"] = (x.unflatten(1, shape) for x, shape in zip(rows, ((H, P), (G, S), (G, S))))
        # step sizes of 0.001 to 0.1 and rates of 1 to 16: heads that forget over one token to a thousand
        mean = torch.exp(torch.linspace(math.log(0.001), math.log(0.1), H, device=dev))
        rate = torch.linspace(1.0, 16.0, H, device=dev)[torch.randperm(H, generator=gen, device=dev)]
        s["dt"] = torch.nn.functional.softplus(normal(T, H) + torch.log(torch.expm1(mean)))
        s["g"] = -s["dt"] * rate
        s["D"] = 1.0 + 0.1 * normal(H)
        if c["start"] or call == "scan_step":
            s["state"] = normal(c["B"], H, S, P) * 0.3
        if train:
            s["dY"] = normal(T, H, P).to(io)
    else:
        D = c["D"]
        s["Z"], s["X"] = row(D, D) if c["fused"] else (normal(T, D).to(io) for _ in range(2))
        s["W"] = 1.0 + 0.1 * normal(D)
        if train:
            s["dY"] = normal(T, D).to(io)
    if own:
        _handles(s)
    return s


def work(case):
    c, e, T = case, 2 if case["io"] == "bf16" else 4, sum(_lengths(case))
    call, train = c["call"], case["call"].endswith("train")
    if call.startswith("conv"):
        D, K = c["D"], c["K"]
        states = 2 if call == "conv_step" else 1 if train else 1 + c["start"]
        return {"bytes": e * D * (T * (4 if train else 2) + (0 if train and not c["start"] else states * c["B"] * (K - 1)))
                + 4 * D * (K + 1) * (2 if train else 1),
                "flops": T * D * (2 * K + 4) * (3 if train else 1)}
    if call.startswith("norm"):
        D = c["D"]
        return {"bytes": e * T * D * (6 if train else 3) + 4 * D * (2 if train else 1), "flops": T * D * (30 if train else 10)}
    H, G, S, P = c["H"], c["G"], c["S"], c["P"]
    rows = T * (2 * H * P + 2 * G * S)   # x, B, C in; y out
    if train:
        rows += T * (2 * H * P + 2 * G * S + 2 * H)   # dy in; dx, dB, dC, ddt, dg out
    states = 2 if call == "scan_step" else c["start"] + (not train)
    return {"bytes": e * rows + 8 * T * H + 4 * states * c["B"] * H * S * P, "flops": (12 if train else 4) * T * H * S * P}


# ---------------------------------------------------------------------------
# The framework's calls
# ---------------------------------------------------------------------------
def _stride(x):
    return x.stride(0) if len(x) > 1 else 0


def _handles(s):
    """Descriptor and workspaces, which a program makes once and keeps."""
    import paper_2606_27748_amd as flex
    c, T, call = s["case"], s["T"], s["case"]["call"]
    train, dev = call.endswith("train"), s["X"].device

    def buffer(n):
        return torch.empty(max(n, 256), dtype=torch.uint8, device=dev)

    if call.startswith("conv"):
        s["desc"] = flex.make_conv_desc(c["B"], T, c["D"], c["K"], act="silu" if c["act"] else "none", io=c["io"],
                                        x_stride=_stride(s["X"]), dx_stride=_stride(s["X"]) if train else 0)
        if train:
            s["ws"] = buffer(flex.conv_workspace_size(s["desc"]))
    elif call.startswith("scan"):
        strides = {n + "_stride": _stride(s[t]) for n, t in (("x", "X"), ("b", "Bt"), ("c", "Ct"))}
        if train:
            strides.update({"d" + n: x for n, x in strides.items()})
        s["desc"] = flex.make_scan_desc(c["B"], c["G"], c["H"], c["S"], c["P"], T, io=c["io"], **strides)
        if call == "scan_step":
            return
        passes = [flex.FLEX_PASS_FWD] + ([flex.FLEX_PASS_BWD] if train else [])
        s["ws"] = buffer(max(flex.scan_workspace_size(s["desc"], p) for p in passes))
        s["saved"] = buffer(flex.scan_saved_size(s["desc"])) if train else None
    else:
        wide = {n + "_stride": _stride(s[n.upper()]) for n in "xz"}
        if train:
            wide.update({"d" + n: x for n, x in wide.items()})
        s["desc"] = flex.make_norm_desc(T, c["D"], c["group"], gate=c["gate"], io=c["io"], eps=EPS, **wide)
        if train:
            s["ws"] = buffer(flex.norm_workspace_size(s["desc"]))


def _wide(x, *widths):
    """Gradients of rows that are slices of a wider row: slices of one like it."""
    return torch.empty(len(x), sum(widths), dtype=x.dtype, device=x.device).split(widths, 1)


def _run_own(s):
    import paper_2606_27748_amd as flex
    c, d, call, X, fused = s["case"], s["desc"], s["case"]["call"], s["X"], s["case"]["fused"]
    if call == "conv_step":
        return {"Y": flex.flex_conv_step(d, X, s["W"], s["bias"], s["state"]), "state": s["state"]}
    if call.startswith("conv"):
        args = (d, X, s["W"], s["bias"], s["off"])
        Y, state = flex.flex_conv_fwd(*args, state0=s.get("state"), want_state=call == "conv_fwd")
        if call == "conv_fwd":
            return {"Y": Y, "state": state}
        dX = _wide(X, c["D"], 64)[0] if fused else None
        return {"Y": Y, **flex.flex_conv_bwd(*args, s["dY"], state0=s.get("state"), dX=dX, ws=s["ws"])}
    if call.startswith("norm"):
        args = (d, X, s["Z"], s["W"])
        Y = flex.flex_norm_fwd(*args)
        if call == "norm_fwd":
            return {"Y": Y}
        dZ, dX = _wide(X, c["D"], c["D"]) if fused else (None, None)
        return {"Y": Y, **flex.flex_norm_bwd(*args, s["dY"], dX=dX, dZ=dZ, ws=s["ws"])}
    rows = (d, X, s["Bt"], s["Ct"], s["dt"], s["g"], s["D"])
    if call == "scan_step":
        return {"Y": flex.flex_scan_step(*rows, s["state"]), "state": s["state"]}
    if call == "scan_fwd":
        Y, state = flex.flex_scan_fwd(*rows, s["off"], state0=s.get("state"), want_state=True, ws=s["ws"])
        return {"Y": Y, "state": state}
    Y, _ = flex.flex_scan_fwd(*rows, s["off"], state0=s.get("state"), saved=s["saved"], ws=s["ws"])
    out = {}
    if fused:
        H, G, S, P = (c[k] for k in "HGSP")
        wide = _wide(X, H * P, G * S, G * S)
        out = {n: x.unflatten(1, t.shape[1:]) for n, x, t in zip(("dX", "dB", "dC"), wide, (X, s["Bt"], s["Ct"]))}
    return {"Y": Y, **flex.flex_scan_bwd(*rows, s["off"], s["dY"], s["saved"], ws=s["ws"], **out)}


# ---------------------------------------------------------------------------
# Plain forms
# ---------------------------------------------------------------------------
def _place(s):
    """Sequence of each packed row, and its place in it."""
    off, t = s["off"].long(), torch.arange(s["T"], device=s["off"].device)
    b = torch.searchsorted(off, t, right=True) - 1
    return b, t - off[b]


def _silu(x):
    return x / (1 + torch.exp(-x))


def _dsilu(x):
    sig = 1 / (1 + torch.exp(-x))
    return sig * (1 + x * (1 - sig))


def _conv_step(s):
    X, W, state = s["X"], s["W"], s["state"]
    rows = torch.cat([state, X[:, None]], 1)   # [B, K, D]
    z = (rows.float() * W.T).sum(1) + s["bias"]
    state.copy_(rows[:, 1:])
    return {"Y": (_silu(z) if s["case"]["act"] else z).to(X.dtype), "state": state}


def _conv_plain(s):
    c, X, W, off = s["case"], s["X"], s["W"], s["off"].long()
    B, K, D, T = c["B"], c["K"], c["D"], s["T"]
    before = s["state"] if c["start"] else X.new_zeros(B, K - 1, D)
    # every sequence's rows behind its K-1 earlier ones
    b, _ = _place(s)
    at = torch.arange(T, device=X.device) + (K - 1) * (b + 1)   # of the packed rows among them
    first = off[:-1, None] + (K - 1) * torch.arange(B, device=X.device)[:, None] + torch.arange(K - 1, device=X.device)
    rows = X.new_empty(T + B * (K - 1), D, dtype=torch.float32)
    rows[at], rows[first] = X.float(), before.float()
    z = s["bias"].expand(T, D)
    taps = at[:, None] - (K - 1) + torch.arange(K, device=X.device)   # [T, K]
    z = z + (rows[taps.T] * W.T[:, None]).sum(0)
    out = {"Y": (_silu(z) if c["act"] else z).to(X.dtype)}
    if c["call"] == "conv_fwd":
        last = off[1:, None] + (K - 1) * torch.arange(B, device=X.device)[:, None] + torch.arange(K - 1, device=X.device)
        return {**out, "state": rows[last].to(X.dtype)}
    dz = s["dY"].float() * (_dsilu(z) if c["act"] else 1.0)
    down = torch.zeros_like(rows)
    down[at] = dz
    back = torch.cat([down, down.new_zeros(K - 1, D)])
    # of row at[t] - (K-1) + k, tap k reaches output t; the rows behind a sequence's last belong to the next one's past
    later = at[:, None] + (K - 1) - torch.arange(K, device=X.device)
    out["dX"] = (back[later.T] * W.T[:, None]).sum(0).to(X.dtype)
    out["dW"] = (rows[taps.T] * dz).sum(1, dtype=torch.float64).T.float()
    out["dbias"] = dz.sum(0, dtype=torch.float64).float()
    return out


def _mm(a, b):
    return torch.matmul(a, b.contiguous())


def _scan_plain(s):
    c, io, train = s["case"], s["X"].dtype, s["case"]["call"] == "scan_train"
    B, H, G, S, P, T = c["B"], c["H"], c["G"], c["S"], c["P"], s["T"]
    r, n = H // G, -(-c["N"] // C)
    b, j = _place(s)
    names = ("X", "Bt", "Ct", "dt", "g", "D")
    leaves = {k: s[k].float().requires_grad_(train) for k in names}

    with torch.set_grad_enabled(train):
        def chunks(x, heads, width):   # [T, heads, width] -> [B, G, heads / G, n, C, width], zeros behind each sequence
            y = x.new_zeros(B, n * C, heads, width).index_put((b, j), x)
            return y.view(B, n, C, G, heads // G, width).permute(0, 3, 4, 1, 2, 5)

        x, Bt, Ct = chunks(leaves["X"], H, P), chunks(leaves["Bt"], G, S), chunks(leaves["Ct"], G, S)
        dt, g = chunks(leaves["dt"][..., None], H, 1), chunks(leaves["g"].double()[..., None], H, 1)
        xt = x * dt
        L = g.cumsum(-2)
        D = torch.exp((L - L.transpose(-1, -2)).tril()).float().tril()
        y = _mm(_mm(Ct, Bt.transpose(-1, -2)) * D, xt)
        # each chunk's part of the state, and what is left of it at the start of each later one (and at the end)
        U = _mm(Bt.transpose(-1, -2).expand(B, G, r, n, S, C), torch.exp(L[..., -1:, :] - L).float() * xt).reshape(B, G, r, n, S * P)
        whole = torch.cat([torch.zeros_like(L[..., :1, 0, 0]), L[..., -1, 0].cumsum(-1)], -1)   # [B, G, r, n + 1]
        left = whole[..., :, None] - whole[..., None, 1:]
        lower = torch.ones(n + 1, n, dtype=torch.bool, device=x.device).tril(-1)
        states = _mm(torch.exp(torch.where(lower, left, -math.inf)).float(), U)
        if c["start"]:
            states = states + torch.exp(whole).float()[..., None] * s["state"].view(B, G, r, 1, S * P)
        states = states.view(B, G, r, n + 1, S, P)
        y = y + torch.exp(L).float() * _mm(Ct.expand(B, G, r, n, C, S), states[..., :n, :, :])
        y = y.permute(0, 3, 4, 1, 2, 5).reshape(B, n * C, H, P)[b, j] + leaves["D"][:, None] * leaves["X"]
    out = {"Y": y.detach().to(io)}
    if not train:
        return {**out, "state": states[..., n, :, :].reshape(B, H, S, P).clone()}
    got = dict(zip(names, torch.autograd.grad(y, list(leaves.values()), s["dY"].float())))
    skip = (s["dY"].double() * s["X"].double()).sum((0, 2))   # a sum over all rows
    return {**out, "dX": got["X"].to(io), "dB": got["Bt"].to(io), "dC": got["Ct"].to(io), "ddt": got["dt"].to(io),
            "dg": got["g"].to(io), "dD": skip.float()}


def _scan_step(s):
    c, state, x = s["case"], s["state"], s["X"].float()
    Bt, Ct = (s[k].float().repeat_interleave(c["H"] // c["G"], 1) for k in ("Bt", "Ct"))
    state.mul_(torch.exp(s["g"])[..., None, None])
    state.add_(Bt[..., None] * (s["dt"][..., None] * x)[..., None, :])
    y = (state * Ct[..., None]).sum(-2) + s["D"][:, None] * x
    return {"Y": y.to(s["X"].dtype), "state": state}


def _norm_plain(s):
    c, io, T = s["case"], s["X"].dtype, s["T"]

    def groups(x):
        return x.float().view(-1, c["D"] // c["group"], c["group"]) if x.is_contiguous() else x.float().unflatten(1, (-1, c["group"]))

    x, z, w = groups(s["X"]), groups(s["Z"]), groups(s["W"])
    gate = _silu(z)
    u = x * gate if c["gate"] == "first" else x
    rs = torch.rsqrt(u.square().mean(-1, keepdim=True) + EPS)
    n = u * rs
    out = {"Y": (n * w * (gate if c["gate"] == "last" else 1.0)).view(T, -1).to(io)}
    if c["call"] == "norm_fwd":
        return out
    dy = groups(s["dY"])
    dn = dy * w * (gate if c["gate"] == "last" else 1.0)
    du = rs * (dn - n * (dn * n).mean(-1, keepdim=True))
    dgate = du * x if c["gate"] == "first" else dy * n * w
    out["dX"] = (du * gate if c["gate"] == "first" else du).view(T, -1).to(io)
    out["dZ"] = (dgate * _dsilu(z)).view(T, -1).to(io)
    out["dW"] = (dy * n * (gate if c["gate"] == "last" else 1.0)).sum(0, dtype=torch.float64).view(-1).float()
    return out


def run(state):
    if own:
        return _run_own(state)
    call = state["case"]["call"]
    if call == "conv_step":
        return _conv_step(state)
    if call == "scan_step":
        return _scan_step(state)
    return {"conv": _conv_plain, "scan": _scan_plain, "norm": _norm_plain}[call[:4]](state)


# ---------------------------------------------------------------------------
# The same outputs in 64 bits, from the definitions, a sequence at a time
# ---------------------------------------------------------------------------
def _exact_conv(s, x):
    c, K = s["case"], s["case"]["K"]
    train, step = c["call"] == "conv_train", c["call"] == "conv_step"
    out = {"Y": torch.empty_like(x["X"])}
    leaf = {k: x[k].clone().requires_grad_(train) for k in ("W", "bias")}
    if train:
        out["dX"] = torch.empty_like(x["X"])
        total = {k: torch.zeros_like(v) for k, v in leaf.items()}
    else:
        out["state"] = torch.empty(c["B"], K - 1, c["D"], dtype=torch.float64, device=x["X"].device)
    off = list(range(c["B"] + 1)) if step else s["off"].tolist()
    for b in range(c["B"]):
        rows = slice(off[b], off[b + 1])
        own_rows = x["X"][rows].T.clone().requires_grad_(train)   # [D, n]
        past = x["state"][b].T if "state" in x else torch.zeros(c["D"], K - 1, dtype=torch.float64, device=own_rows.device)
        line = torch.cat([past, own_rows], 1)
        n = own_rows.shape[1]
        z = leaf["bias"][:, None]
        for k in range(K):
            z = z + leaf["W"][:, k:k + 1] * line[:, k:k + n]
        y = z * torch.sigmoid(z) if c["act"] else z
        out["Y"][rows] = y.detach().T
        if train:
            got = torch.autograd.grad(y, [own_rows, leaf["W"], leaf["bias"]], x["dY"][rows].T)
            out["dX"][rows] = got[0].T
            total["W"] += got[1]
            total["bias"] += got[2]
        else:
            out["state"][b] = line[:, n:].T
    return {**out, **({"dW": total["W"], "dbias": total["bias"]} if train else {})}


def _exact_scan(s, x):
    c, H, r = s["case"], s["case"]["H"], s["case"]["H"] // s["case"]["G"]
    train, dev = c["call"] == "scan_train", x["X"].device
    if c["call"] == "scan_step":
        head = torch.arange(H, device=dev) // r
        S = torch.exp(x["g"])[..., None, None] * x["state"] + torch.einsum("bhn,bhp,bh->bhnp", x["Bt"][:, head], x["X"], x["dt"])
        return {"Y": torch.matmul(x["Ct"][:, head][:, :, None], S)[:, :, 0] + x["D"][:, None] * x["X"], "state": S}
    ln = s["lengths"]
    if H * sum(n * n for n in ln) * (4 if train else 1) > 1e11:
        return None
    names = ("X", "Bt", "Ct", "dt", "g")
    out = {"Y": torch.zeros_like(x["X"])}
    grad = {k: torch.zeros_like(x[k]) for k in names}
    state = torch.zeros(c["B"], H, c["S"], c["P"], dtype=torch.float64, device=dev)
    dD, off = torch.zeros(H, dtype=torch.float64, device=dev), s["off"].tolist()
    for b, n in enumerate(ln):
        rows = slice(off[b], off[b + 1])
        hidden = torch.ones(n, n, dtype=torch.bool, device=dev).triu(1)
        for h in range(H):
            at = {k: (rows, h // r if k in ("Bt", "Ct") else h) for k in names}
            leaf = {k: x[k][i].clone().requires_grad_(train) for k, i in at.items()}
            skip = x["D"][h].clone().requires_grad_(train)
            L = leaf["g"].cumsum(0)
            w = torch.exp((L[:, None] - L[None]).masked_fill(hidden, -math.inf)) * (leaf["Ct"] @ leaf["Bt"].T) * leaf["dt"]
            y = w @ leaf["X"] + skip * leaf["X"]
            del w
            if c["start"]:
                y = y + torch.exp(L)[:, None] * (leaf["Ct"] @ x["state"][b, h])
            out["Y"][rows, h] = y.detach()
            if train:
                got = torch.autograd.grad(y, [*leaf.values(), skip], x["dY"][rows, h])
                for k, v in zip(names, got):
                    grad[k][at[k]] += v
                dD[h] += got[-1]
            else:
                state[b, h] = leaf["Bt"].T @ ((torch.exp(L[-1] - L) * leaf["dt"])[:, None] * leaf["X"])
                if c["start"]:
                    state[b, h] += torch.exp(L[-1]) * x["state"][b, h]
    if not train:
        return {**out, "state": state}
    return {**out, "dX": grad["X"], "dB": grad["Bt"], "dC": grad["Ct"], "ddt": grad["dt"], "dg": grad["g"], "dD": dD}


def _exact_norm(s, x):
    c, train = s["case"], s["case"]["call"] == "norm_train"
    leaf = {k: x[k].clone().requires_grad_(train) for k in ("X", "Z", "W")}
    gate = leaf["Z"] * torch.sigmoid(leaf["Z"])
    u = (leaf["X"] * gate if c["gate"] == "first" else leaf["X"]).reshape(len(gate), -1, c["group"])
    y = (u / torch.sqrt((u * u).mean(-1, keepdim=True) + EPS)).reshape(gate.shape) * leaf["W"]
    if c["gate"] == "last":
        y = y * gate
    if not train:
        return {"Y": y}
    got = torch.autograd.grad(y, list(leaf.values()), x["dY"])
    return {"Y": y.detach(), "dX": got[0], "dZ": got[1], "dW": got[2]}


def exact(case, seed):
    s = prepare(case, seed)
    x = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor) and v.is_floating_point()}
    return {"conv": _exact_conv, "scan": _exact_scan, "norm": _exact_norm}[case["call"][:4]](s, x)
