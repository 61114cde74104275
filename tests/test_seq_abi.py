"""Refusals of the packed-sequence entry points, without a GPU: descriptors and arguments are
checked before any device work, sizes are what the kernels index, and the host code of the
ABI runs clean under AddressSanitizer."""
import ctypes
import os
import subprocess

import pytest

import paper_2606_27748_amd as F
from paper_2606_27748_amd import build as B

FAKE = 0x10000   # aligned, never dereferenced: every call below is refused
NO_GPU = not os.path.exists("/dev/kfd")
BAD, UNS, WS, OK = F.FLEX_ERR_INVALID_ARG, F.FLEX_ERR_UNSUPPORTED, F.FLEX_ERR_WORKSPACE, F.FLEX_OK


def _size(fn, desc, *args):
    n = ctypes.c_size_t(7)
    return getattr(F.load(), fn)(ctypes.byref(desc) if desc is not None else None, *args, ctypes.byref(n)), n.value


@pytest.mark.parametrize("field,value,status", [
    ("B", 0, BAD), ("Hq", 0, BAD), ("Hq", 6, BAD), ("Hkv", 0, BAD), ("Tq", -1, BAD), ("Tk", -1, BAD), ("causal", 2, BAD),
    ("io_dtype", 3, BAD), ("scale", 0.0, BAD), ("scale", -1.0, BAD), ("scale", float("nan"), BAD),
    ("scale", float("inf"), BAD), ("d", 48, UNS), ("d", 256, UNS), ("d", 0, BAD), ("q_stride", 8, BAD),
    ("q_stride", 8 * 64 + 4, BAD), ("q_stride", 8 * 64 + 8, OK), ("k_stride", 4 * 64, OK), ("k_stride", (1 << 20) + 8, BAD),
    ("v_stride", -8, BAD), ("Tq", 0, OK), ("Tk", 0, OK), ("Hq", 1 << 20, UNS), ("d", 32, OK), ("d", 128, OK),
    ("Tq", (1 << 31) - 1, BAD)])
def test_attention_descriptor(field, value, status):
    d = F.make_attn_desc(3, 8, 4, 64, 100, 200)
    setattr(d, field, value)
    for p in (F.FLEX_PASS_FWD, F.FLEX_PASS_BWD):
        st, n = _size("flex_attn_workspace_size", d, p)
        assert st == status and (st == OK or n == 0)


@pytest.mark.parametrize("field,value,status", [
    ("B", 0, BAD), ("T", -1, BAD), ("T", 0, OK), ("Hk", 0, BAD), ("H", 0, BAD), ("H", 5, BAD), ("io_dtype", -1, BAD),
    ("scale", 0.0, BAD), ("scale", float("nan"), BAD), ("d", 32, UNS), ("d", 96, UNS), ("dv", 32, UNS), ("dv", 128, OK),
    ("dv", 0, BAD), ("q_stride", 2 * 64 - 8, BAD), ("k_stride", 2 * 64 + 4, BAD), ("v_stride", 4 * 64 + 16, OK),
    ("v_stride", 1 << 21, BAD), ("H", 1 << 15, UNS)])
def test_delta_descriptor(field, value, status):
    d = F.make_delta_desc(3, 2, 4, 64, 100)
    setattr(d, field, value)
    assert _size("flex_delta_saved_size", d)[0] == status
    for p in (F.FLEX_PASS_FWD, F.FLEX_PASS_BWD):
        assert _size("flex_delta_workspace_size", d, p)[0] == status


def test_sizes():
    """What the kernels write: parts of few rows per sequence, statistics of the backward, blocks of chunk slots."""
    few = F.make_attn_desc(2, 8, 2, 128, 2, 20000)
    parts = _size("flex_attn_workspace_size", few, F.FLEX_PASS_FWD)[1]
    rows = 2 * 8
    assert parts >= 2 * rows * (128 + 2) * 4 and parts % rows == 0   # two parts of each row at least
    assert _size("flex_attn_workspace_size", F.make_attn_desc(2, 8, 2, 128, 5000, 20000), F.FLEX_PASS_FWD) == (OK, 0)
    assert _size("flex_attn_workspace_size", few, F.FLEX_PASS_BWD)[1] == 2 * rows * 4
    for T in (1, 63, 64, 65, 1000):
        for B_ in (1, 7):
            d = F.make_delta_desc(B_, 2, 4, 128, T, dv=64)
            blocks = (T // 64 + B_) * 4
            prep = 2 * (32 * 32 + 32 * 64) * 4 + 2048
            assert _size("flex_delta_workspace_size", d, F.FLEX_PASS_FWD)[1] == blocks * prep
            assert _size("flex_delta_saved_size", d)[1] == blocks * (prep + 128 * 64 * 2 + 64 * 64 * 4)
            assert _size("flex_delta_workspace_size", d, F.FLEX_PASS_BWD)[1] == blocks * (128 * 64 * 2 + 64 * 64 * 4)
    for fn, d in (("flex_attn_workspace_size", few), ("flex_delta_workspace_size", F.make_delta_desc(1, 1, 1, 64, 5))):
        assert _size(fn, None, F.FLEX_PASS_FWD)[0] == BAD and _size(fn, d, F.FLEX_PASS_AWD)[0] == BAD
        assert getattr(F.load(), fn)(ctypes.byref(d), F.FLEX_PASS_FWD, None) == BAD


@pytest.mark.skipif(not NO_GPU, reason="fake pointers are only passed where no GPU is visible")
def test_calls_are_refused():
    lib, big = F.load(), 1 << 40
    d = F.make_attn_desc(2, 8, 2, 64, 2, 20000)
    r = ctypes.byref(d)
    fwd = lambda a, ws=FAKE, n=big: lib.flex_attn_fwd(r, *a, ws, n, None)  # noqa: E731
    ok = [FAKE] * 8   # Q K V q_off k_off k_len O lse
    for i in (0, 1, 2, 3, 4, 6):
        assert fwd(ok[:i] + [None] + ok[i + 1:]) == BAD, i
    for i in (0, 1, 2, 6, 7):
        assert fwd(ok[:i] + [FAKE + 2] + ok[i + 1:]) == BAD, i
    assert lib.flex_attn_fwd(None, *ok, FAKE, big, None) == BAD
    assert fwd(ok, None) == WS and fwd(ok, FAKE, 16) == WS and fwd(ok, FAKE + 4) == WS
    ok = [FAKE] * 11   # Q K V q_off k_off O lse dO dQ dK dV
    for i in range(11):
        assert lib.flex_attn_bwd(r, *ok[:i], None, *ok[i + 1:], FAKE, big, None) == BAD, i
    assert lib.flex_attn_bwd(r, *ok, FAKE, 8, None) == WS
    d = F.make_delta_desc(2, 2, 4, 64, 100)
    r = ctypes.byref(d)
    ok = [FAKE] * 9   # Q K V g beta off state0 O state
    for i in (0, 1, 2, 3, 4, 5, 7):
        assert lib.flex_delta_fwd(r, *ok[:i], None, *ok[i + 1:], None, 0, FAKE, big, None) == BAD, i
    assert lib.flex_delta_fwd(r, *ok, None, 0, None, 0, None) == WS
    assert lib.flex_delta_fwd(r, *ok, None, 0, FAKE, 100, None) == WS
    assert lib.flex_delta_fwd(r, *ok, FAKE, 100, FAKE, big, None) == WS
    ok = [FAKE] * 6 + [FAKE, big] + [FAKE] * 6   # Q K V g beta off saved bytes dO dQ dK dV dg dbeta
    for i in (0, 1, 2, 3, 4, 5, 8, 9, 10, 11, 12, 13):
        assert lib.flex_delta_bwd(r, *ok[:i], None, *ok[i + 1:], FAKE, big, None) == BAD, i
    assert lib.flex_delta_bwd(r, *ok[:6], FAKE, 100, *ok[8:], FAKE, big, None) == WS
    assert lib.flex_delta_bwd(r, *ok[:6], None, big, *ok[8:], FAKE, big, None) == WS
    assert lib.flex_delta_bwd(r, *ok, FAKE, 100, None) == WS
    ok = [FAKE] * 7
    for i in range(7):
        assert lib.flex_delta_step(r, *ok[:i], None, *ok[i + 1:], None) == BAD, i
    # nothing to do: no rows
    e = ctypes.byref(F.make_attn_desc(2, 8, 2, 64, 0, 0))
    assert lib.flex_attn_fwd(e, None, None, None, FAKE, FAKE, None, None, None, None, 0, None) == OK
    assert lib.flex_attn_bwd(e, None, None, None, FAKE, FAKE, *[None] * 6, None, 0, None) == OK


def test_binding_checks_tensors():
    """The Python binding refuses tensors that are not what the descriptor says, before the library sees them."""
    import torch
    d = F.make_attn_desc(1, 2, 1, 32, 5, 5)
    q, k = torch.zeros(5, 2, 32, dtype=torch.bfloat16), torch.zeros(5, 1, 32, dtype=torch.bfloat16)
    off = torch.tensor([0, 5], dtype=torch.int32)
    for args in ((q.float(), k, k, off, off), (q[:4], k, k, off, off), (q, k, k, off.long(), off),
                 (q.transpose(0, 1).contiguous().transpose(0, 1), k, k, off, off), (q, k, k, off, off)):
        with pytest.raises(F.FlexError) as e:   # the last: tensors of the CPU
            F.flex_attn_fwd(d, *args)
        assert e.value.status == BAD


def test_largest_launches():
    """Sizes whose launches would have 2^32 threads are refused, the next below are not."""
    size = lambda fn, d: _size(fn, d, F.FLEX_PASS_FWD)[0]  # noqa: E731
    for B_, status in ((174762, OK), (174763, BAD)):   # 384 threads per 32 of 128 columns of 16 states
        assert size("flex_delta_workspace_size", F.make_delta_desc(B_, 16, 16, 128, 1000)) == status
    for B_, status in ((524280, OK), (524288, BAD)):   # 512 threads per sequence and key head
        assert size("flex_attn_workspace_size", F.make_attn_desc(B_, 16, 16, 128, 1000, 1000)) == status
    for Tq, status in ((1 << 23, OK), (1 << 24, BAD)):   # d / 8 threads per row and head
        assert size("flex_attn_workspace_size", F.make_attn_desc(1, 16, 1, 128, Tq, 1000)) == status


def test_workspace_of_another_device():
    import torch
    from paper_2606_27748_amd import _lib
    for need in (0, 16):
        with pytest.raises(F.FlexError) as e:
            _lib._seq_workspace(need, torch.empty(64, dtype=torch.uint8), torch.device("cuda", 0))
        assert e.value.status == WS


ASAN_DRIVER = r"""
#include <cstdio>
#include <cstring>
#include "flex.h"
int main() {
  size_t n = 0; int bad = 0;
  void* p = reinterpret_cast<void*>(0x10000);
  const int32_t* o = static_cast<const int32_t*>(p);
  float* f = static_cast<float*>(p);
  for (int B = 1; B < 5; ++B) for (int d = 32; d <= 128; d *= 2) for (int T = 0; T < 300; T += 37) for (int io = 0; io < 2; ++io) {
    flex_attn_desc a; std::memset(&a, 0, sizeof(a));
    a.B = B; a.Hq = 4; a.Hkv = 2; a.d = d; a.Tq = T; a.Tk = 3 * T; a.causal = 1; a.io_dtype = io; a.scale = 1.f;
    bad += flex_attn_workspace_size(&a, FLEX_PASS_FWD, &n) != FLEX_OK;
    bad += flex_attn_workspace_size(&a, FLEX_PASS_BWD, &n) != FLEX_OK;
    bad += flex_attn_fwd(&a, p, p, p, nullptr, o, o, p, f, p, 1u << 30, nullptr) != FLEX_ERR_INVALID_ARG;
    bad += flex_attn_bwd(&a, p, p, p, o, nullptr, p, f, p, p, p, p, p, 1u << 30, nullptr) != FLEX_ERR_INVALID_ARG;
    flex_delta_desc g; std::memset(&g, 0, sizeof(g));
    g.B = B; g.T = T; g.Hk = 2; g.H = 4; g.d = d; g.dv = 64; g.io_dtype = io; g.scale = 1.f;
    const int want = d == 32 ? FLEX_ERR_UNSUPPORTED : FLEX_OK;
    bad += flex_delta_workspace_size(&g, FLEX_PASS_FWD, &n) != want;
    bad += flex_delta_saved_size(&g, &n) != want;
    bad += flex_delta_fwd(&g, p, p, p, f, f, nullptr, f, p, f, p, 1, p, 1, nullptr) == FLEX_OK;
    bad += flex_delta_bwd(&g, p, p, p, f, f, o, p, 1, p, p, p, p, p, p, p, 1, nullptr) == FLEX_OK;
    bad += flex_delta_step(&g, p, p, p, f, f, nullptr, p, nullptr) == FLEX_OK;
  }
  std::printf("%d\n", bad);
  return bad != 0;
}
"""


@pytest.mark.skipif(not os.path.exists("/opt/rocm/llvm/bin/clang++"), reason="needs hipcc and clang++")
def test_host_code_under_asan(tmp_path):
    objs = [os.path.join(B.BUILD, s.replace(".hip", ".o")) for s in B.SOURCES if s != "flex_seq_api.hip"]
    if not all(os.path.exists(o) for o in objs):
        B.build()
    api, drv, exe = (str(tmp_path / n) for n in ("api.o", "drv.o", "drv"))
    inc, host = os.path.join(B.ROOT, "include"), ["-Xarch_host", "-fsanitize=address"]
    subprocess.run([B.HIPCC, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-fPIC", "-Xclang", "-target-feature",
                    "-Xclang", "-packed-fp32-ops", *host, "-I", inc, "-c", os.path.join(B.CSRC, "flex_seq_api.hip"),
                    "-o", api], check=True, capture_output=True)
    (tmp_path / "drv.cpp").write_text(ASAN_DRIVER)
    clang = "/opt/rocm/llvm/bin/clang++"
    subprocess.run([clang, "-std=c++17", "-g", "-fsanitize=address", "-I", inc, "-c", str(tmp_path / "drv.cpp"), "-o", drv],
                   check=True, capture_output=True)
    subprocess.run([clang, "-fsanitize=address", drv, api, *objs, "-L/opt/rocm/lib", "-lamdhip64",
                    "-Wl,-rpath,/opt/rocm/lib", "-o", exe], check=True, capture_output=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120, env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0"))
    assert r.returncode == 0 and r.stdout.strip() == "0", (r.stdout, r.stderr[-2000:])
