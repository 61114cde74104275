"""ctypes binding of libflexattn.so (the C ABI declared in include/flex.h).

Argument marshalling only: torch tensors supply device pointers and the
current HIP stream; every step of the computation runs in the library's HIP
kernels.  There is no CPU or PyTorch fallback: if the library is missing the
calls raise.
"""
from __future__ import annotations

import ctypes
import os

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libflexattn.so")

FLEX_OK, FLEX_ERR_INVALID_ARG, FLEX_ERR_UNSUPPORTED, FLEX_ERR_WORKSPACE, FLEX_ERR_HIP = range(5)
FLEX_F32, FLEX_BF16 = 0, 1
FLEX_STATIONARY, FLEX_NONSTATIONARY = 0, 1
FLEX_PASS_FEATURE_MAP, FLEX_PASS_FWD, FLEX_PASS_BWD, FLEX_PASS_AWD = 0, 1, 2, 3
EXPORTS = ("flex_abi_version", "flex_status_string", "flex_workspace_size",
           "flex_feature_map", "flex_linattn_fwd", "flex_linattn_prefill", "flex_linattn_fwd_noalloc",
           "flex_linattn_bwd",
           "flex_decode_step",
           "flex_awd_loss", "flex_attn_workspace_size", "flex_attn_fwd", "flex_attn_bwd",
           "flex_delta_workspace_size", "flex_delta_saved_size", "flex_delta_fwd", "flex_delta_bwd",
           "flex_delta_step",
           "flex_timing_enable", "flex_timing_read")
KERNELS = {"none": 0, "fwd_state": 1, "fwd_sweep": 2, "scan": 3, "bwd_prepass": 4,
           "bwd_dq": 5, "bwd_dkv": 6, "bwd_reduce": 7, "feature_map": 8, "decode_step": 9,
           "awd_fwd": 10, "awd_bwd_k": 11, "awd_wgrad": 12,
           "attn_fwd": 13, "attn_bwd": 14, "delta_fwd": 15, "delta_bwd": 16, "delta_step": 17}


class FlexError(RuntimeError):
    def __init__(self, status: int, what: str):
        super().__init__(f"{what}: {status_string(status)} (status {status})")
        self.status = status


class flex_desc(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("H", ctypes.c_int32), ("N", ctypes.c_int32),
                ("d", ctypes.c_int32), ("dv", ctypes.c_int32), ("m", ctypes.c_int32),
                ("variant", ctypes.c_int32), ("causal", ctypes.c_int32),
                ("chunk", ctypes.c_int32), ("segments", ctypes.c_int32),
                ("io_dtype", ctypes.c_int32), ("grad_dtype", ctypes.c_int32),
                ("sigma", ctypes.c_float)]


class flex_attn_desc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "Hq", "Hkv", "d", "Tq", "Tk", "causal", "io_dtype",
                                              "q_stride", "k_stride", "v_stride")] + [("scale", ctypes.c_float)]


class flex_delta_desc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "T", "Hk", "H", "d", "dv", "io_dtype", "q_stride", "k_stride",
                                              "v_stride")] + [("scale", ctypes.c_float)]


_lib = None


def load(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load the shared library (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise FileNotFoundError(
            f"{path} not found: build it with `python -m paper_2606_27748_amd.build` "
            "or __graft_entry__.build()")
    # The calls take device pointers and streams from torch, so the library must
    # bind to the HIP runtime torch loads (torch ships its own copy): importing
    # torch first makes the dynamic linker reuse that runtime.  Loaded the other
    # way round, torch brings a second runtime whose streams the library's
    # launches reject.
    import torch  # noqa: F401
    lib = ctypes.CDLL(path)
    P, S, I = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32
    D = ctypes.POINTER(flex_desc)
    lib.flex_abi_version.restype = I
    lib.flex_abi_version.argtypes = []
    lib.flex_status_string.restype = ctypes.c_char_p
    lib.flex_status_string.argtypes = [I]
    lib.flex_workspace_size.restype = I
    lib.flex_workspace_size.argtypes = [D, I, ctypes.POINTER(S)]
    lib.flex_feature_map.restype = I
    lib.flex_feature_map.argtypes = [D, P, P, P, P, P, P, S, P]
    lib.flex_linattn_fwd.restype = I
    lib.flex_linattn_fwd.argtypes = [D, P, P, P, P, P, P, P, P, P, S, P]
    lib.flex_linattn_prefill.restype = I
    lib.flex_linattn_prefill.argtypes = [D, P, P, P, P, P, P, P, P, P, P, S, P]
    lib.flex_linattn_fwd_noalloc.restype = I
    lib.flex_linattn_fwd_noalloc.argtypes = [D, P, P, P, P, P, P, P, P, P]
    lib.flex_linattn_bwd.restype = I
    lib.flex_linattn_bwd.argtypes = [D] + [P] * 15 + [P, S] + [P, S, P]
    lib.flex_decode_step.restype = I
    lib.flex_decode_step.argtypes = [D] + [P] * 10
    lib.flex_awd_loss.restype = I
    lib.flex_awd_loss.argtypes = [D] + [P] * 10 + [S, P]
    A = ctypes.POINTER(flex_attn_desc)
    lib.flex_attn_workspace_size.restype = I
    lib.flex_attn_workspace_size.argtypes = [A, I, ctypes.POINTER(S)]
    lib.flex_attn_fwd.restype = I
    lib.flex_attn_fwd.argtypes = [A] + [P] * 9 + [S, P]
    lib.flex_attn_bwd.restype = I
    lib.flex_attn_bwd.argtypes = [A] + [P] * 12 + [S, P]
    G = ctypes.POINTER(flex_delta_desc)
    lib.flex_delta_workspace_size.restype = I
    lib.flex_delta_workspace_size.argtypes = [G, I, ctypes.POINTER(S)]
    lib.flex_delta_saved_size.restype = I
    lib.flex_delta_saved_size.argtypes = [G, ctypes.POINTER(S)]
    lib.flex_delta_fwd.restype = I
    lib.flex_delta_fwd.argtypes = [G] + [P] * 10 + [S, P, S, P]
    lib.flex_delta_bwd.restype = I
    lib.flex_delta_bwd.argtypes = [G] + [P] * 7 + [S] + [P] * 7 + [S, P]
    lib.flex_delta_step.restype = I
    lib.flex_delta_step.argtypes = [G] + [P] * 8
    lib.flex_timing_enable.restype = I
    lib.flex_timing_enable.argtypes = [I]
    lib.flex_timing_read.restype = I
    lib.flex_timing_read.argtypes = [ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int64)]
    _lib = lib
    return lib


def status_string(status: int) -> str:
    return load().flex_status_string(int(status)).decode()


def make_desc(B, H, N, d, m, variant="stationary", causal=False, io="bf16",
              dv=None, sigma=1.0, segments=0, chunk=0) -> flex_desc:
    return flex_desc(B, H, N, d, d if dv is None else dv, m,
                     FLEX_NONSTATIONARY if variant == "nonstationary" else FLEX_STATIONARY,
                     1 if causal else 0, chunk, segments,
                     FLEX_BF16 if io == "bf16" else FLEX_F32, FLEX_F32, float(sigma))


def workspace_size(desc: flex_desc, pass_: int) -> int:
    n = ctypes.c_size_t(0)
    st = load().flex_workspace_size(ctypes.byref(desc), pass_, ctypes.byref(n))
    if st != FLEX_OK:
        raise FlexError(st, "flex_workspace_size")
    return n.value


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream():
    import torch
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _check(st, what):
    if st != FLEX_OK:
        raise FlexError(st, what)


def _workspace(desc, pass_, ws, device):
    import torch
    need = workspace_size(desc, pass_)
    if ws is None or ws.numel() * ws.element_size() < need:
        ws = torch.empty(max(need, 256), dtype=torch.uint8, device=device)
    return ws


def flex_feature_map(desc: flex_desc, X, W1, W2, tau, Phi=None):
    """phi~(X) -> Phi [B,H,N,2m] (io dtype).  Tensors on the GPU."""
    import torch
    if Phi is None:
        Phi = torch.empty(desc.B, desc.H, desc.N, 2 * desc.m, dtype=X.dtype, device=X.device)
    st = load().flex_feature_map(ctypes.byref(desc), _ptr(X), _ptr(W1), _ptr(W2), _ptr(tau),
                                 _ptr(Phi), None, 0, _stream())
    _check(st, "flex_feature_map")
    return Phi


def flex_linattn_fwd(desc: flex_desc, Q, K, V, W1, W2, tau, O=None, den=None, ws=None,
                     want_den=True):
    """Forward linear attention.  Returns (O, den)."""
    import torch
    dev = Q.device
    if O is None:
        O = torch.empty(desc.B, desc.H, desc.N, desc.dv, dtype=Q.dtype, device=dev)
    if den is None and want_den:
        den = torch.empty(desc.B, desc.H, desc.N, dtype=torch.float32, device=dev)
    ws = _workspace(desc, FLEX_PASS_FWD, ws, dev)
    st = load().flex_linattn_fwd(ctypes.byref(desc), _ptr(Q), _ptr(K), _ptr(V), _ptr(W1),
                                 _ptr(W2), _ptr(tau), _ptr(O), _ptr(den), _ptr(ws),
                                 ws.numel(), _stream())
    _check(st, "flex_linattn_fwd")
    return O, den


def flex_linattn_prefill(desc: flex_desc, Q, K, V, W1, W2, tau, state=None, O=None, den=None,
                         ws=None, want_den=True):
    """Causal forward that also writes the prefix's state in the decode layout
    (decode_state).  Returns (O, den, state)."""
    import torch
    dev = Q.device
    if O is None:
        O = torch.empty(desc.B, desc.H, desc.N, desc.dv, dtype=Q.dtype, device=dev)
    if den is None and want_den:
        den = torch.empty(desc.B, desc.H, desc.N, dtype=torch.float32, device=dev)
    if state is None:
        state = torch.empty(desc.B, desc.H, 2 * desc.m * (desc.dv + 1), dtype=torch.float32, device=dev)
    if state.numel() != desc.B * desc.H * 2 * desc.m * (desc.dv + 1) or state.dtype != torch.float32:
        raise FlexError(FLEX_ERR_INVALID_ARG, "flex_linattn_prefill: state must hold B*H*2m*(dv+1) fp32")
    ws = _workspace(desc, FLEX_PASS_FWD, ws, dev)
    st = load().flex_linattn_prefill(ctypes.byref(desc), _ptr(Q), _ptr(K), _ptr(V), _ptr(W1),
                                     _ptr(W2), _ptr(tau), _ptr(O), _ptr(den), _ptr(state), _ptr(ws),
                                     ws.numel(), _stream())
    _check(st, "flex_linattn_prefill")
    return O, den, state


def flex_linattn_fwd_noalloc(desc: flex_desc, Q, K, V, W1, W2, tau, O, den=None):
    """Forward linear attention with the library's static scratch as its
    workspace: O (and den, if given) are caller-allocated, nothing else is.
    Returns (O, den)."""
    st = load().flex_linattn_fwd_noalloc(ctypes.byref(desc), _ptr(Q), _ptr(K), _ptr(V), _ptr(W1),
                                         _ptr(W2), _ptr(tau), _ptr(O), _ptr(den), _stream())
    _check(st, "flex_linattn_fwd_noalloc")
    return O, den


def flex_linattn_bwd(desc: flex_desc, Q, K, V, W1, W2, tau, O, den, dO, dQ=None, dK=None,
                     dV=None, dW1=None, dW2=None, dtau=None, ws=None, want_dtau=True, fwd_ws=None):
    """Backward linear attention.  Returns dict of fp32 gradients.

    fwd_ws: optionally the workspace tensor of the matching flex_linattn_fwd
    call (same descriptor and inputs, unchanged since): its segment states are
    then reused instead of recomputed."""
    import torch
    dev = Q.device
    f32 = torch.float32
    if dQ is None:
        dQ = torch.empty(desc.B, desc.H, desc.N, desc.d, dtype=f32, device=dev)
    if dK is None:
        dK = torch.empty(desc.B, desc.H, desc.N, desc.d, dtype=f32, device=dev)
    if dV is None:
        dV = torch.empty(desc.B, desc.H, desc.N, desc.dv, dtype=f32, device=dev)
    if dW1 is None:
        dW1 = torch.empty(desc.H, desc.m, desc.d, dtype=f32, device=dev)
    if dW2 is None and desc.variant == FLEX_NONSTATIONARY:
        dW2 = torch.empty(desc.H, desc.m, desc.d, dtype=f32, device=dev)
    if dtau is None and want_dtau:
        dtau = torch.empty(desc.H, dtype=f32, device=dev)
    ws = _workspace(desc, FLEX_PASS_BWD, ws, dev)
    st = load().flex_linattn_bwd(ctypes.byref(desc), _ptr(Q), _ptr(K), _ptr(V), _ptr(W1),
                                 _ptr(W2), _ptr(tau), _ptr(O), _ptr(den), _ptr(dO), _ptr(dQ),
                                 _ptr(dK), _ptr(dV), _ptr(dW1), _ptr(dW2), _ptr(dtau),
                                 _ptr(fwd_ws), 0 if fwd_ws is None else fwd_ws.numel(),
                                 _ptr(ws), ws.numel(), _stream())
    _check(st, "flex_linattn_bwd")
    return dict(dQ=dQ, dK=dK, dV=dV, dW1=dW1, dW2=dW2, dtau=dtau)


def decode_state(desc: flex_desc, device="cuda"):
    """A zero decode state: fp32 [B,H,2m*dv + 2m], per slice S [2m][dv] then z [2m]."""
    import torch
    F = 2 * desc.m
    return torch.zeros(desc.B, desc.H, F * desc.dv + F, dtype=torch.float32, device=device)


def decode_state_views(desc: flex_desc, state):
    """(S [B,H,2m,dv], z [B,H,2m]) views of a decode state."""
    F = 2 * desc.m
    st = state.reshape(desc.B, desc.H, F * (desc.dv + 1))
    return st[..., :F * desc.dv].unflatten(-1, (F, desc.dv)), st[..., F * desc.dv:]


def flex_decode_step(desc: flex_desc, q, k, v, W1, W2, tau, state, o=None, den=None, want_den=True):
    """One decode step: state (fp32, B*H*2m*(dv+1) floats laid out as in
    decode_state, updated in place) takes the new token k, v; returns (o, den)
    for the new token's query q."""
    import torch
    if state.numel() != desc.B * desc.H * 2 * desc.m * (desc.dv + 1) or state.dtype != torch.float32:
        raise FlexError(FLEX_ERR_INVALID_ARG, "flex_decode_step: state must hold B*H*2m*(dv+1) fp32")
    if o is None:
        o = torch.empty(desc.B, desc.H, desc.dv, dtype=q.dtype, device=q.device)
    if den is None and want_den:
        den = torch.empty(desc.B, desc.H, dtype=torch.float32, device=q.device)
    st = load().flex_decode_step(ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(v), _ptr(W1), _ptr(W2),
                                 _ptr(tau), _ptr(state), _ptr(o), _ptr(den), _stream())
    _check(st, "flex_decode_step")
    return o, den


def flex_awd_loss(desc: flex_desc, Q, K, W1, W2, tau, grads=True, loss=None, dW1=None, dW2=None,
                  dtau=None, ws=None, want_dtau=True):
    """Attention-weight distillation loss per (b,h) slice and, with grads, the
    gradients of its sum over slices with respect to W1, W2 and tau.
    Returns dict(loss [B,H], dW1, dW2, dtau) (fp32; gradients None without grads)."""
    import torch
    dev = Q.device
    f32 = torch.float32
    if loss is None:
        loss = torch.empty(desc.B, desc.H, dtype=f32, device=dev)
    if grads:
        if dW1 is None:
            dW1 = torch.empty(desc.H, desc.m, desc.d, dtype=f32, device=dev)
        if dW2 is None and desc.variant == FLEX_NONSTATIONARY:
            dW2 = torch.empty(desc.H, desc.m, desc.d, dtype=f32, device=dev)
        if dtau is None and want_dtau:
            dtau = torch.empty(desc.H, dtype=f32, device=dev)
    else:
        dW1 = dW2 = dtau = None
    ws = _workspace(desc, FLEX_PASS_AWD, ws, dev)
    st = load().flex_awd_loss(ctypes.byref(desc), _ptr(Q), _ptr(K), _ptr(W1), _ptr(W2), _ptr(tau),
                              _ptr(loss), _ptr(dW1), _ptr(dW2), _ptr(dtau), _ptr(ws), ws.numel(),
                              _stream())
    _check(st, "flex_awd_loss")
    return dict(loss=loss, dW1=dW1, dW2=dW2, dtau=dtau)


# ---------------------------------------------------------------------------
# Packed sequences
# ---------------------------------------------------------------------------
def _size(fn, desc, *args):
    n = ctypes.c_size_t(0)
    _check(getattr(load(), fn)(ctypes.byref(desc), *args, ctypes.byref(n)), fn)
    return n.value


def _device(what, Q):
    if Q is None:
        raise FlexError(FLEX_ERR_INVALID_ARG, f"{what}: the first tensor is missing")
    return Q.device


def _expect(what, dev, tensors, optional=()):
    """Each (name, tensor, shape, dtype, row stride or 0 for contiguous) as it must be; the optional ones may
    be None."""
    if dev.type != "cuda":
        raise FlexError(FLEX_ERR_INVALID_ARG, f"{what}: tensors must be on the GPU")
    for name, t, _, _, _ in tensors:
        if t is None:
            raise FlexError(FLEX_ERR_INVALID_ARG, f"{what}: {name} is missing")
    for name, t, shape, dtype, stride in (*tensors, *optional):
        if t is None:
            continue
        ok = t.shape == shape and t.dtype is dtype and t.device == dev
        if ok and stride and shape[0] > 1:
            ok = t.stride() == (stride, shape[2], 1)
        elif ok:
            ok = t.is_contiguous()
        if not ok:
            raise FlexError(FLEX_ERR_INVALID_ARG, f"{what}: {name} must be {dtype} {list(shape)} on {dev}, rows "
                            + (f"{stride} elements apart" if stride else "contiguous"))


def _io(desc):
    import torch
    return torch.bfloat16 if desc.io_dtype == FLEX_BF16 else torch.float32


def _at(t):
    return None if t is None else t.data_ptr()


def _run(fn, dev, desc, *args):
    """The call on the current stream of the tensors' device, with that device current."""
    import torch
    f = getattr(load(), fn)
    if dev.index == torch.cuda.current_device():
        st = f(ctypes.byref(desc), *args, torch._C._cuda_getCurrentRawStream(dev.index))
    else:
        with torch.cuda.device(dev):
            st = f(ctypes.byref(desc), *args, torch.cuda.current_stream().cuda_stream)
    if st != FLEX_OK:
        raise FlexError(st, fn)


def _seq_workspace(need, ws, dev):
    """The workspace of a call, or None where it needs none.  The caller keeps the tensor until the call has
    returned: memory freed earlier could be another thread's by the time the kernels are queued."""
    if ws is not None and (ws.device != dev or not ws.is_contiguous()):
        raise FlexError(FLEX_ERR_WORKSPACE, f"ws must be contiguous on {dev}")
    if ws is None or ws.numel() * ws.element_size() < need:
        if not need:
            return None
        import torch
        ws = torch.empty(need, dtype=torch.uint8, device=dev)
    return ws


def _span(t):
    return (None, 0) if t is None else (t.data_ptr(), t.numel() * t.element_size())


def make_attn_desc(B, Hq, Hkv, d, Tq, Tk, causal=True, io="bf16", scale=None, q_stride=0, k_stride=0,
                   v_stride=0) -> flex_attn_desc:
    """B sequences packed in Tq query and Tk key rows; strides in elements between rows (0: contiguous)."""
    return flex_attn_desc(B, Hq, Hkv, d, Tq, Tk, 1 if causal else 0, FLEX_BF16 if io == "bf16" else FLEX_F32,
                          q_stride, k_stride, v_stride, float(d ** -0.5 if scale is None else scale))


def attn_workspace_size(desc: flex_attn_desc, pass_: int) -> int:
    return _size("flex_attn_workspace_size", desc, pass_)


def _attn_inputs(what, desc, Q, K, V, q_off, k_off, more, optional):
    import torch
    io, dev, i32, off = _io(desc), _device(what, Q), torch.int32, (desc.B + 1,)
    kv = (desc.Tk, desc.Hkv, desc.d)
    _expect(what, dev, (("Q", Q, (desc.Tq, desc.Hq, desc.d), io, desc.q_stride), ("K", K, kv, io, desc.k_stride),
                        ("V", V, kv, io, desc.v_stride), ("q_off", q_off, off, i32, 0),
                        ("k_off", k_off, off, i32, 0)) + more, optional)
    return io, dev


def flex_attn_fwd(desc: flex_attn_desc, Q, K, V, q_off, k_off, k_len=None, O=None, lse=None, ws=None,
                  want_lse=True):
    """Exact attention of packed sequences: Q [Tq,Hq,d] against K, V [Tk,Hkv,d], int32
    offsets [B+1] (and the used key lengths k_len [B] of a slotted cache) on the
    device.  Returns (O, lse)."""
    import torch
    rows, f32 = (desc.Tq, desc.Hq, desc.d), torch.float32
    io, dev = _attn_inputs("flex_attn_fwd", desc, Q, K, V, q_off, k_off, (),
                           (("k_len", k_len, (desc.B,), torch.int32, 0), ("O", O, rows, _io(desc), 0),
                            ("lse", lse, rows[:2], f32, 0)))
    if O is None:
        O = torch.empty(rows, dtype=io, device=dev)
    if lse is None and want_lse:
        lse = torch.empty(rows[:2], dtype=f32, device=dev)
    ws = _seq_workspace(attn_workspace_size(desc, FLEX_PASS_FWD), ws, dev)
    _run("flex_attn_fwd", dev, desc, Q.data_ptr(), K.data_ptr(), V.data_ptr(), q_off.data_ptr(), k_off.data_ptr(),
         _at(k_len), O.data_ptr(), _at(lse), *_span(ws))
    return O, lse


def flex_attn_bwd(desc: flex_attn_desc, Q, K, V, q_off, k_off, O, lse, dO, dQ=None, dK=None, dV=None, ws=None):
    """Backward of flex_attn_fwd (k_len None) from its O and lse.  Returns dict(dQ, dK, dV)
    in the io dtype; rows of no sequence are not written."""
    import torch
    rows, krow, io = (desc.Tq, desc.Hq, desc.d), (desc.Tk, desc.Hkv, desc.d), _io(desc)
    _, dev = _attn_inputs("flex_attn_bwd", desc, Q, K, V, q_off, k_off,
                          (("O", O, rows, io, 0), ("dO", dO, rows, io, 0), ("lse", lse, rows[:2], torch.float32, 0)),
                          (("dQ", dQ, rows, io, 0), ("dK", dK, krow, io, 0), ("dV", dV, krow, io, 0)))
    dQ = torch.empty(rows, dtype=io, device=dev) if dQ is None else dQ
    dK = torch.empty(krow, dtype=io, device=dev) if dK is None else dK
    dV = torch.empty(krow, dtype=io, device=dev) if dV is None else dV
    ws = _seq_workspace(attn_workspace_size(desc, FLEX_PASS_BWD), ws, dev)
    _run("flex_attn_bwd", dev, desc, *(t.data_ptr() for t in (Q, K, V, q_off, k_off, O, lse, dO, dQ, dK, dV)), *_span(ws))
    return dict(dQ=dQ, dK=dK, dV=dV)


def make_delta_desc(B, Hk, H, d, T, dv=None, io="bf16", scale=None, q_stride=0, k_stride=0,
                    v_stride=0) -> flex_delta_desc:
    """B sequences packed in T rows of Hk query/key heads and H value heads; strides in elements
    between rows (0: contiguous)."""
    return flex_delta_desc(B, T, Hk, H, d, d if dv is None else dv, FLEX_BF16 if io == "bf16" else FLEX_F32,
                           q_stride, k_stride, v_stride, float(d ** -0.5 if scale is None else scale))


def delta_workspace_size(desc: flex_delta_desc, pass_: int) -> int:
    return _size("flex_delta_workspace_size", desc, pass_)


def delta_saved_size(desc: flex_delta_desc) -> int:
    """Bytes of the buffer in which a forward keeps what its backward reads."""
    return _size("flex_delta_saved_size", desc)


def _delta_inputs(what, desc, T, Q, K, V, g, beta, more, optional):
    import torch
    io, dev, f32, qk = _io(desc), _device(what, Q), torch.float32, (T, desc.Hk, desc.d)
    _expect(what, dev, (("Q", Q, qk, io, desc.q_stride), ("K", K, qk, io, desc.k_stride),
                        ("V", V, (T, desc.H, desc.dv), io, desc.v_stride), ("g", g, (T, desc.H), f32, 0),
                        ("beta", beta, (T, desc.H), f32, 0)) + more, optional)
    return io, dev


def _check_saved(what, desc, saved, dev):
    if saved is None or _span(saved)[1] < delta_saved_size(desc) or not saved.is_contiguous() or saved.device != dev:
        raise FlexError(FLEX_ERR_WORKSPACE, f"{what}: saved must hold delta_saved_size bytes on {dev}")


def flex_delta_fwd(desc: flex_delta_desc, Q, K, V, g, beta, off, state0=None, O=None, state=None, saved=None,
                   ws=None, want_state=False):
    """Gated delta rule over packed sequences: Q, K [T,Hk,d], V [T,H,dv], g (log decay) and beta
    [T,H] fp32, int32 offsets [B+1] on the device.  saved: a buffer of delta_saved_size bytes
    for flex_delta_bwd.  Returns (O, state), state [B,H,d,dv] fp32 where one was given or
    want_state."""
    import torch
    sshape, rows, f32 = (desc.B, desc.H, desc.d, desc.dv), (desc.T, desc.H, desc.dv), torch.float32
    io, dev = _delta_inputs("flex_delta_fwd", desc, desc.T, Q, K, V, g, beta, (("off", off, (desc.B + 1,), torch.int32, 0),),
                            (("O", O, rows, _io(desc), 0), ("state0", state0, sshape, f32, 0),
                             ("state", state, sshape, f32, 0)))
    if O is None:
        O = torch.empty(rows, dtype=io, device=dev)
    if state is None and want_state:
        state = torch.empty(sshape, dtype=f32, device=dev)
    if saved is not None:
        _check_saved("flex_delta_fwd", desc, saved, dev)
        ws = None
    else:
        ws = _seq_workspace(delta_workspace_size(desc, FLEX_PASS_FWD), ws, dev)
    _run("flex_delta_fwd", dev, desc, *(t.data_ptr() for t in (Q, K, V, g, beta, off)), _at(state0), O.data_ptr(),
         _at(state), *_span(saved), *_span(ws))
    return O, state


def flex_delta_bwd(desc: flex_delta_desc, Q, K, V, g, beta, off, dO, saved, dQ=None, dK=None, dV=None, dg=None,
                   dbeta=None, ws=None):
    """Backward of flex_delta_fwd from what it kept in saved, its state0 a constant.  Returns dict(dQ,
    dK, dV, dg, dbeta) in the io dtype; rows of no sequence are not written."""
    import torch
    io, qk, rows, gates = _io(desc), (desc.T, desc.Hk, desc.d), (desc.T, desc.H, desc.dv), (desc.T, desc.H)
    out = (("dQ", dQ, qk, io, 0), ("dK", dK, qk, io, 0), ("dV", dV, rows, io, 0), ("dg", dg, gates, io, 0),
           ("dbeta", dbeta, gates, io, 0))
    _, dev = _delta_inputs("flex_delta_bwd", desc, desc.T, Q, K, V, g, beta,
                           (("off", off, (desc.B + 1,), torch.int32, 0), ("dO", dO, rows, io, 0)), out)
    grads = {n: torch.empty(shape, dtype=io, device=dev) if t is None else t for n, t, shape, _, _ in out}
    _check_saved("flex_delta_bwd", desc, saved, dev)
    ws = _seq_workspace(delta_workspace_size(desc, FLEX_PASS_BWD), ws, dev)
    _run("flex_delta_bwd", dev, desc, *(t.data_ptr() for t in (Q, K, V, g, beta, off)), *_span(saved), dO.data_ptr(),
         *(t.data_ptr() for t in grads.values()), *_span(ws))
    return grads


def flex_delta_step(desc: flex_delta_desc, q, k, v, g, beta, state, o=None):
    """One token of every sequence: q, k [B,Hk,d], v [B,H,dv], g, beta [B,H], state [B,H,d,dv]
    fp32 updated in place.  Returns o [B,H,dv]."""
    import torch
    rows = (desc.B, desc.H, desc.dv)
    io, dev = _delta_inputs("flex_delta_step", desc, desc.B, q, k, v, g, beta,
                            (("state", state, (desc.B, desc.H, desc.d, desc.dv), torch.float32, 0),),
                            (("o", o, rows, _io(desc), 0),))
    if o is None:
        o = torch.empty(rows, dtype=io, device=dev)
    _run("flex_delta_step", dev, desc, *(t.data_ptr() for t in (q, k, v, g, beta, state, o)))
    return o


def flex_timing_enable(kernel: str) -> None:
    """Time every launch of one kernel class with HIP events ("none" disables)."""
    _check(load().flex_timing_enable(KERNELS[kernel]), "flex_timing_enable")


def flex_timing_read():
    """(summed milliseconds, number of launches) since the last enable/read."""
    ms = ctypes.c_double(0.0)
    n = ctypes.c_int64(0)
    _check(load().flex_timing_read(ctypes.byref(ms), ctypes.byref(n)), "flex_timing_read")
    return ms.value, n.value
