"""ctypes binding of libflexattn.so (the C ABI declared in include/flex.h).

Argument marshalling only: torch tensors supply device pointers and the
current HIP stream; every step of the computation runs in the library's HIP
kernels.  There is no CPU or PyTorch fallback: if the library is missing the
calls raise.
"""
from __future__ import annotations

import ctypes
import math
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
           "flex_conv_workspace_size", "flex_conv_fwd", "flex_conv_bwd", "flex_conv_step",
           "flex_scan_workspace_size", "flex_scan_saved_size", "flex_scan_fwd", "flex_scan_bwd", "flex_scan_step",
           "flex_norm_workspace_size", "flex_norm_fwd", "flex_norm_bwd",
           "flex_timing_enable", "flex_timing_read")
KERNELS = {"none": 0, "fwd_state": 1, "fwd_sweep": 2, "scan": 3, "bwd_prepass": 4,
           "bwd_dq": 5, "bwd_dkv": 6, "bwd_reduce": 7, "feature_map": 8, "decode_step": 9,
           "awd_fwd": 10, "awd_bwd_k": 11, "awd_wgrad": 12,
           "attn_fwd": 13, "attn_bwd": 14, "delta_fwd": 15, "delta_bwd": 16, "delta_step": 17,
           "conv_fwd": 18, "conv_bwd": 19, "conv_step": 20, "scan_fwd": 21, "scan_bwd": 22, "scan_step": 23,
           "norm_fwd": 24, "norm_bwd": 25}


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


class flex_conv_desc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "T", "D", "K", "act", "io_dtype", "x_stride", "dx_stride")]


class flex_scan_desc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "T", "G", "H", "N", "P", "io_dtype", "x_stride", "b_stride", "c_stride",
                                              "dx_stride", "db_stride", "dc_stride")]


class flex_norm_desc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("T", "D", "group", "gate", "io_dtype", "x_stride", "z_stride", "dx_stride",
                                              "dz_stride")] + [("eps", ctypes.c_float)]


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
    C, N, M = (ctypes.POINTER(x) for x in (flex_conv_desc, flex_scan_desc, flex_norm_desc))
    lib.flex_conv_workspace_size.restype = I
    lib.flex_conv_workspace_size.argtypes = [C, ctypes.POINTER(S)]
    lib.flex_conv_fwd.restype = I
    lib.flex_conv_fwd.argtypes = [C] + [P] * 8
    lib.flex_conv_bwd.restype = I
    lib.flex_conv_bwd.argtypes = [C] + [P] * 10 + [S, P]
    lib.flex_conv_step.restype = I
    lib.flex_conv_step.argtypes = [C] + [P] * 6
    lib.flex_scan_workspace_size.restype = I
    lib.flex_scan_workspace_size.argtypes = [N, I, ctypes.POINTER(S)]
    lib.flex_scan_saved_size.restype = I
    lib.flex_scan_saved_size.argtypes = [N, ctypes.POINTER(S)]
    lib.flex_scan_fwd.restype = I
    lib.flex_scan_fwd.argtypes = [N] + [P] * 11 + [S, P, S, P]
    lib.flex_scan_bwd.restype = I
    lib.flex_scan_bwd.argtypes = [N] + [P] * 8 + [S] + [P] * 8 + [S, P]
    lib.flex_scan_step.restype = I
    lib.flex_scan_step.argtypes = [N] + [P] * 9
    lib.flex_norm_workspace_size.restype = I
    lib.flex_norm_workspace_size.argtypes = [M, ctypes.POINTER(S)]
    lib.flex_norm_fwd.restype = I
    lib.flex_norm_fwd.argtypes = [M] + [P] * 5
    lib.flex_norm_bwd.restype = I
    lib.flex_norm_bwd.argtypes = [M] + [P] * 8 + [S, P]
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
            ok = t.stride() == (stride, *shape[2:], 1)
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


# ---------------------------------------------------------------------------
# Selective state-space layers
# ---------------------------------------------------------------------------
_ACTS = {"none": 0, "silu": 1}
_GATES = {"none": 0, "first": 1, "last": 2}


def _make(out, dev):
    """The tensors of (name, tensor or None, shape, dtype, row stride), new ones for None: contiguous, or with the
    stride that the descriptor asks for, as the first columns of wider rows."""
    import torch
    made = {}
    for n, t, shape, dtype, stride in out:
        if t is None:
            row = math.prod(shape[1:])
            t = torch.empty(shape, dtype=dtype, device=dev)
            if stride and stride != row and shape[0] > 1:
                t = torch.empty(shape[0], stride, dtype=dtype, device=dev)[:, :row].unflatten(1, shape[1:])
        made[n] = t
    return made


def make_conv_desc(B, T, D, K, act="silu", io="bf16", x_stride=0, dx_stride=0) -> flex_conv_desc:
    """Short causal convolution of B sequences packed in T rows of D channels, K taps each, act "silu" or
    "none" behind it; strides in elements between rows (0: contiguous)."""
    return flex_conv_desc(B, T, D, K, _ACTS.get(act, -1), FLEX_BF16 if io == "bf16" else FLEX_F32, x_stride, dx_stride)


def conv_workspace_size(desc: flex_conv_desc) -> int:
    """Bytes of workspace of flex_conv_bwd."""
    return _size("flex_conv_workspace_size", desc)


def _conv_inputs(what, desc, T, X, W, bias, more, optional):
    import torch
    io, dev, f32 = _io(desc), _device(what, X), torch.float32
    _expect(what, dev, (("X", X, (T, desc.D), io, desc.x_stride), ("W", W, (desc.D, desc.K), f32, 0)) + more,
            (("bias", bias, (desc.D,), f32, 0),) + optional)
    return io, dev


def flex_conv_fwd(desc: flex_conv_desc, X, W, bias, off, state0=None, Y=None, state=None, want_state=False):
    """Short causal convolution over packed sequences: X [T,D], W [D,K] and bias [D] (or None) fp32, int32
    offsets [B+1] on the device, the K-1 rows before each sequence in state0 [B,K-1,D] (None: zeros).  Returns
    (Y, state), the last K-1 rows of each sequence where a state was given or want_state."""
    import torch
    io, sshape = _io(desc), (desc.B, desc.K - 1, desc.D)
    _, dev = _conv_inputs("flex_conv_fwd", desc, desc.T, X, W, bias, (("off", off, (desc.B + 1,), torch.int32, 0),),
                          (("state0", state0, sshape, io, 0), ("Y", Y, (desc.T, desc.D), io, 0),
                           ("state", state, sshape, io, 0)))
    if Y is None:
        Y = torch.empty(desc.T, desc.D, dtype=io, device=dev)
    if state is None and want_state:
        state = torch.empty(sshape, dtype=io, device=dev)
    _run("flex_conv_fwd", dev, desc, X.data_ptr(), W.data_ptr(), _at(bias), off.data_ptr(), _at(state0), Y.data_ptr(),
         _at(state))
    return Y, state


def flex_conv_bwd(desc: flex_conv_desc, X, W, bias, off, dY, state0=None, dX=None, dW=None, dbias=None, ws=None):
    """Backward of flex_conv_fwd, its state0 a constant, as it was before a forward in place.  Returns dict(dX, dW, dbias): dX in the io dtype (rows of no
    sequence are not written), dW [D,K] and dbias [D] (None without a bias) fp32."""
    import torch
    io, f32, rows = _io(desc), torch.float32, (desc.T, desc.D)
    out = (("dX", dX, rows, io, desc.dx_stride), ("dW", dW, (desc.D, desc.K), f32, 0))
    more = (("dbias", dbias, (desc.D,), f32, 0),)
    _, dev = _conv_inputs("flex_conv_bwd", desc, desc.T, X, W, bias,
                          (("off", off, (desc.B + 1,), torch.int32, 0), ("dY", dY, rows, io, 0)),
                          (("state0", state0, (desc.B, desc.K - 1, desc.D), io, 0),) + out + more)
    grads = _make(out + (more if bias is not None else ()), dev)
    grads.setdefault("dbias", dbias)
    ws = _seq_workspace(conv_workspace_size(desc), ws, dev)
    _run("flex_conv_bwd", dev, desc, X.data_ptr(), W.data_ptr(), _at(bias), off.data_ptr(), _at(state0), dY.data_ptr(),
         *(_at(t) for t in grads.values()), *_span(ws))
    return grads


def flex_conv_step(desc: flex_conv_desc, x, W, bias, state, y=None):
    """One token of every sequence: x [B,D], state [B,K-1,D] (the rows before, oldest first) updated in
    place.  Returns y [B,D]."""
    import torch
    io, rows = _io(desc), (desc.B, desc.D)
    _, dev = _conv_inputs("flex_conv_step", desc, desc.B, x, W, bias, (("state", state, (desc.B, desc.K - 1, desc.D), io, 0),),
                          (("y", y, rows, io, 0),))
    if y is None:
        y = torch.empty(rows, dtype=io, device=dev)
    _run("flex_conv_step", dev, desc, x.data_ptr(), W.data_ptr(), _at(bias), state.data_ptr(), y.data_ptr())
    return y


def make_scan_desc(B, G, H, N, P, T, io="bf16", x_stride=0, b_stride=0, c_stride=0, dx_stride=0, db_stride=0,
                   dc_stride=0) -> flex_scan_desc:
    """Selective scan of B sequences packed in T rows: H heads of P columns on G groups of B and C of N elements;
    strides in elements between rows (0: contiguous)."""
    return flex_scan_desc(B, T, G, H, N, P, FLEX_BF16 if io == "bf16" else FLEX_F32, x_stride, b_stride, c_stride,
                          dx_stride, db_stride, dc_stride)


def scan_workspace_size(desc: flex_scan_desc, pass_: int) -> int:
    return _size("flex_scan_workspace_size", desc, pass_)


def scan_saved_size(desc: flex_scan_desc) -> int:
    """Bytes of the buffer in which a forward keeps what its backward reads."""
    return _size("flex_scan_saved_size", desc)


def _scan_inputs(what, desc, T, X, Bt, Ct, dt, g, D, more, optional):
    import torch
    io, dev, f32, bc = _io(desc), _device(what, X), torch.float32, (T, desc.G, desc.N)
    _expect(what, dev, (("X", X, (T, desc.H, desc.P), io, desc.x_stride), ("Bt", Bt, bc, io, desc.b_stride),
                        ("Ct", Ct, bc, io, desc.c_stride), ("dt", dt, (T, desc.H), f32, 0),
                        ("g", g, (T, desc.H), f32, 0)) + more, (("D", D, (desc.H,), f32, 0),) + optional)
    return io, dev


def _scan_saved(what, desc, saved, dev):
    if saved is None or _span(saved)[1] < scan_saved_size(desc) or not saved.is_contiguous() or saved.device != dev:
        raise FlexError(FLEX_ERR_WORKSPACE, f"{what}: saved must hold scan_saved_size bytes on {dev}")


def flex_scan_fwd(desc: flex_scan_desc, X, Bt, Ct, dt, g, D, off, state0=None, Y=None, state=None, saved=None, ws=None,
                  want_state=False):
    """Selective scan over packed sequences: X [T,H,P], Bt and Ct [T,G,N], dt and g (log decay) [T,H] fp32, D [H]
    fp32 or None, int32 offsets [B+1] on the device.  saved: a buffer of scan_saved_size bytes for
    flex_scan_bwd.  Returns (Y, state), state [B,H,N,P] fp32 where one was given or want_state."""
    import torch
    sshape, rows, f32 = (desc.B, desc.H, desc.N, desc.P), (desc.T, desc.H, desc.P), torch.float32
    io, dev = _scan_inputs("flex_scan_fwd", desc, desc.T, X, Bt, Ct, dt, g, D, (("off", off, (desc.B + 1,), torch.int32, 0),),
                           (("Y", Y, rows, _io(desc), 0), ("state0", state0, sshape, f32, 0),
                            ("state", state, sshape, f32, 0)))
    if Y is None:
        Y = torch.empty(rows, dtype=io, device=dev)
    if state is None and want_state:
        state = torch.empty(sshape, dtype=f32, device=dev)
    if saved is not None:
        _scan_saved("flex_scan_fwd", desc, saved, dev)
    ws = _seq_workspace(scan_workspace_size(desc, FLEX_PASS_FWD), ws, dev)
    _run("flex_scan_fwd", dev, desc, *(t.data_ptr() for t in (X, Bt, Ct, dt, g)), _at(D), off.data_ptr(), _at(state0),
         Y.data_ptr(), _at(state), *_span(saved), *_span(ws))
    return Y, state


def flex_scan_bwd(desc: flex_scan_desc, X, Bt, Ct, dt, g, D, off, dY, saved, dX=None, dB=None, dC=None, ddt=None, dg=None,
                  dD=None, ws=None):
    """Backward of flex_scan_fwd from what it kept in saved, its state0 a constant.  Returns dict(dX, dB, dC,
    ddt, dg) in the io dtype (rows of no sequence are not written) and dD [H] fp32 (None without a D)."""
    import torch
    io, rows, bc, gates = _io(desc), (desc.T, desc.H, desc.P), (desc.T, desc.G, desc.N), (desc.T, desc.H)
    out = (("dX", dX, rows, io, desc.dx_stride), ("dB", dB, bc, io, desc.db_stride), ("dC", dC, bc, io, desc.dc_stride),
           ("ddt", ddt, gates, io, 0), ("dg", dg, gates, io, 0))
    more = (("dD", dD, (desc.H,), torch.float32, 0),)
    _, dev = _scan_inputs("flex_scan_bwd", desc, desc.T, X, Bt, Ct, dt, g, D,
                          (("off", off, (desc.B + 1,), torch.int32, 0), ("dY", dY, rows, io, 0)), out + more)
    grads = _make(out + (more if D is not None else ()), dev)
    grads.setdefault("dD", dD)
    _scan_saved("flex_scan_bwd", desc, saved, dev)
    ws = _seq_workspace(scan_workspace_size(desc, FLEX_PASS_BWD), ws, dev)
    _run("flex_scan_bwd", dev, desc, *(t.data_ptr() for t in (X, Bt, Ct, dt, g)), _at(D), off.data_ptr(), *_span(saved),
         dY.data_ptr(), *(_at(t) for t in grads.values()), *_span(ws))
    return grads


def flex_scan_step(desc: flex_scan_desc, x, Bt, Ct, dt, g, D, state, y=None):
    """One token of every sequence: x [B,H,P], Bt and Ct [B,G,N], dt and g [B,H], state [B,H,N,P] fp32 updated
    in place.  Returns y [B,H,P]."""
    import torch
    rows = (desc.B, desc.H, desc.P)
    io, dev = _scan_inputs("flex_scan_step", desc, desc.B, x, Bt, Ct, dt, g, D,
                           (("state", state, (desc.B, desc.H, desc.N, desc.P), torch.float32, 0),),
                           (("y", y, rows, _io(desc), 0),))
    if y is None:
        y = torch.empty(rows, dtype=io, device=dev)
    _run("flex_scan_step", dev, desc, *(t.data_ptr() for t in (x, Bt, Ct, dt, g)), _at(D), state.data_ptr(), y.data_ptr())
    return y


def make_norm_desc(T, D, group, gate="first", io="bf16", eps=1e-5, x_stride=0, z_stride=0, dx_stride=0,
                   dz_stride=0) -> flex_norm_desc:
    """Gated norm of T rows of D channels in groups of `group`; gate "first" (before the norm), "last" or "none";
    strides in elements between rows (0: contiguous)."""
    return flex_norm_desc(T, D, group, _GATES.get(gate, -1), FLEX_BF16 if io == "bf16" else FLEX_F32, x_stride, z_stride, dx_stride,
                          dz_stride, float(eps))


def norm_workspace_size(desc: flex_norm_desc) -> int:
    """Bytes of workspace of flex_norm_bwd."""
    return _size("flex_norm_workspace_size", desc)


def _norm_inputs(what, desc, X, Z, W, more, optional):
    import torch
    io, dev, rows = _io(desc), _device(what, X), (desc.T, desc.D)
    gate = (("Z", Z, rows, io, desc.z_stride),)
    if desc.gate == 0 and Z is not None:
        raise FlexError(FLEX_ERR_INVALID_ARG, f"{what}: Z without a gate")
    _expect(what, dev, (("X", X, rows, io, desc.x_stride), ("W", W, (desc.D,), torch.float32, 0))
            + (gate if desc.gate else ()) + more, optional)
    return io, dev


def flex_norm_fwd(desc: flex_norm_desc, X, Z, W, Y=None):
    """Gated norm of rows: X, Z [T,D] (Z None without a gate), W [D] fp32.  Returns Y [T,D]."""
    import torch
    rows = (desc.T, desc.D)
    io, dev = _norm_inputs("flex_norm_fwd", desc, X, Z, W, (), (("Y", Y, rows, _io(desc), 0),))
    if Y is None:
        Y = torch.empty(rows, dtype=io, device=dev)
    _run("flex_norm_fwd", dev, desc, X.data_ptr(), _at(Z), W.data_ptr(), Y.data_ptr())
    return Y


def flex_norm_bwd(desc: flex_norm_desc, X, Z, W, dY, dX=None, dZ=None, dW=None, ws=None):
    """Backward of flex_norm_fwd.  Returns dict(dX, dZ, dW): dX and dZ (None without a gate) in the io dtype, dW
    [D] fp32."""
    import torch
    io, rows = _io(desc), (desc.T, desc.D)
    out = (("dX", dX, rows, io, desc.dx_stride), ("dZ", dZ, rows, io, desc.dz_stride),
           ("dW", dW, (desc.D,), torch.float32, 0))
    _, dev = _norm_inputs("flex_norm_bwd", desc, X, Z, W, (("dY", dY, rows, io, 0),), out)
    if desc.gate == 0:
        if dZ is not None:
            raise FlexError(FLEX_ERR_INVALID_ARG, "flex_norm_bwd: dZ without a gate")
        out = (out[0], out[2])
    made = _make(out, dev)
    grads = {n: made.get(n) for n in ("dX", "dZ", "dW")}
    ws = _seq_workspace(norm_workspace_size(desc), ws, dev)
    _run("flex_norm_bwd", dev, desc, X.data_ptr(), _at(Z), W.data_ptr(), dY.data_ptr(), *(_at(t) for t in grads.values()),
         *_span(ws))
    return grads


def flex_timing_enable(kernel: str) -> None:
    """Time every launch of one kernel class with HIP events ("none" disables)."""
    _check(load().flex_timing_enable(KERNELS[kernel]), "flex_timing_enable")


def flex_timing_read():
    """(summed milliseconds, number of launches) since the last enable/read."""
    ms = ctypes.c_double(0.0)
    n = ctypes.c_int64(0)
    _check(load().flex_timing_read(ctypes.byref(ms), ctypes.byref(n)), "flex_timing_read")
    return ms.value, n.value
