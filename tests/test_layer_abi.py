"""Refusals of the entry points of selective state-space layers, without a GPU: descriptors and arguments are checked
before any device work, sizes are what the kernels index, and the host code runs clean under AddressSanitizer."""
import ctypes
import os
import subprocess

import pytest

import paper_2606_27748_amd as F
from paper_2606_27748_amd import build as B

FAKE = 0x10000   # aligned, never dereferenced: every call below is refused
NO_GPU = not os.path.exists("/dev/kfd")
BAD, UNS, WS, OK = F.FLEX_ERR_INVALID_ARG, F.FLEX_ERR_UNSUPPORTED, F.FLEX_ERR_WORKSPACE, F.FLEX_OK
PASSES = (F.FLEX_PASS_FWD, F.FLEX_PASS_BWD)


def _size(fn, desc, *args):
    n = ctypes.c_size_t(7)
    return getattr(F.load(), fn)(ctypes.byref(desc) if desc is not None else None, *args, ctypes.byref(n)), n.value


@pytest.mark.parametrize("field,value,status", [
    ("B", 0, BAD), ("T", -1, BAD), ("T", 0, OK), ("D", 0, BAD), ("D", 12, UNS), ("D", 8, OK), ("D", (1 << 20) + 8, UNS),
    ("K", 0, BAD), ("K", 1, UNS), ("K", 5, UNS), ("K", 2, OK), ("act", 2, BAD), ("act", -1, BAD), ("io_dtype", 2, BAD),
    ("x_stride", 56, BAD), ("x_stride", 68, BAD), ("x_stride", 72, OK), ("dx_stride", -64, BAD), ("dx_stride", 1 << 21, BAD),
    ("T", (1 << 31) - 1, BAD), ("B", (1 << 31) - 1, BAD)])
def test_convolution_descriptor(field, value, status):
    d = F.make_conv_desc(3, 100, 64, 4)
    setattr(d, field, value)
    st, n = _size("flex_conv_workspace_size", d)
    assert st == status and (st == OK or n == 0)


@pytest.mark.parametrize("field,value,status", [
    ("B", 0, BAD), ("T", -1, BAD), ("T", 0, OK), ("G", 0, BAD), ("H", 0, BAD), ("H", 5, BAD), ("H", 6, OK), ("N", 32, UNS),
    ("N", 0, BAD), ("N", 128, OK), ("P", 96, UNS), ("P", 128, OK), ("io_dtype", -1, BAD), ("x_stride", 4 * 64 - 8, BAD),
    ("x_stride", 4 * 64 + 4, BAD), ("x_stride", 4 * 64 + 8, OK), ("b_stride", 2 * 64 + 16, OK), ("c_stride", 64, BAD),
    ("dx_stride", 1 << 21, BAD), ("db_stride", 2 * 64 + 4, BAD), ("dc_stride", -8, BAD), ("H", 1 << 15, UNS),
    ("T", (1 << 31) - 1, BAD), ("B", 1 << 30, BAD)])
def test_scan_descriptor(field, value, status):
    d = F.make_scan_desc(3, 2, 4, 64, 64, 100)
    setattr(d, field, value)
    assert _size("flex_scan_saved_size", d)[0] == status
    for p in PASSES:
        assert _size("flex_scan_workspace_size", d, p)[0] == status


@pytest.mark.parametrize("field,value,status", [
    ("T", -1, BAD), ("T", 0, OK), ("D", 0, BAD), ("D", 100, BAD), ("group", 0, BAD), ("group", 40, BAD), ("group", 12, UNS),
    ("group", 192, OK), ("gate", 3, BAD), ("gate", -1, BAD), ("gate", 0, OK), ("io_dtype", 7, BAD), ("eps", -1.0, BAD),
    ("eps", float("nan"), BAD), ("eps", float("inf"), BAD), ("eps", 0.0, OK), ("x_stride", 184, BAD), ("z_stride", 196, BAD),
    ("z_stride", 200, OK), ("dx_stride", 1 << 21, BAD), ("dz_stride", -8, BAD), ("T", (1 << 31) - 1, BAD)])
def test_norm_descriptor(field, value, status):
    d = F.make_norm_desc(100, 192, 64)
    setattr(d, field, value)
    st, n = _size("flex_norm_workspace_size", d)
    assert st == status and (st == OK or n == 0)


def test_largest_group():
    for group, status in ((8192, OK), (8200, UNS)):
        assert _size("flex_norm_workspace_size", F.make_norm_desc(10, group, group))[0] == status


def test_names_that_are_not_known_are_refused():
    assert _size("flex_conv_workspace_size", F.make_conv_desc(1, 5, 8, 4, act="gelu"))[0] == BAD
    assert _size("flex_norm_workspace_size", F.make_norm_desc(5, 8, 8, gate="both"))[0] == BAD


def test_sizes():
    """What the kernels write: sums of 256 rows each, of the rows that are walked at once, states of chunk and segment slots."""
    for T in (1, 255, 256, 257, 5000):
        d = F.make_conv_desc(3, T, 64, 3)
        assert _size("flex_conv_workspace_size", d) == (OK, -(-T // 256) * 4 * 64 * 4)
        n = _size("flex_norm_workspace_size", F.make_norm_desc(T, 1024, 128))[1]
        assert n == min(T, 4096 * 64 // 128) * 1024 * 4
        for io, e in (("bf16", 2), ("f32", 4)):
            d = F.make_scan_desc(3, 2, 8, 128, 64, T, io=io)
            state = 8 * 128 * 64
            assert _size("flex_scan_saved_size", d) == (OK, (T // 64 + 3) * state * e)
            fwd, bwd = (_size("flex_scan_workspace_size", d, p)[1] for p in PASSES)
            segments = fwd // (state * 4)   # and a decay of each and head, in units of 256 bytes
            assert fwd == (segments * state * 4 + -(-segments * 8 * 4 // 256) * 256 if T > 64 else 0)
            assert bwd >= fwd + (T // 64 + 3) * (state * e + 8 * 4)
            assert T <= 64 or T // 64 + 3 >= segments >= 4
    for fn, d in (("flex_conv_workspace_size", F.make_conv_desc(1, 5, 8, 4)), ("flex_norm_workspace_size", F.make_norm_desc(5, 8, 8)),
                  ("flex_scan_saved_size", F.make_scan_desc(1, 1, 1, 64, 64, 5))):
        assert _size(fn, None)[0] == BAD and getattr(F.load(), fn)(ctypes.byref(d), None) == BAD
    d = F.make_scan_desc(1, 1, 1, 64, 64, 5)
    assert _size("flex_scan_workspace_size", None, PASSES[0])[0] == BAD
    assert _size("flex_scan_workspace_size", d, F.FLEX_PASS_AWD)[0] == BAD


@pytest.mark.parametrize("T", [0, 1, 300, 100000])
def test_norm_sums_of_every_width(T):
    """A row of partial sums for each row that is walked, or for each workgroup of rows that a wave's lanes hold, a piece of 8
    channels each."""
    for group, D in ((8, 8), (24, 24), (24, 72), (512, 512), (520, 520), (1048, 1048), (1024, 1024), (2056, 2056), (8192, 8192), (40, 360)):
        team = 1
        while team < group // 8 and team < 64:
            team *= 2
        rows = max(1, min(T, 4096 * 64 // (D // 8)))
        if group <= 512 and team * (D // group) <= 64:
            rows = max(1, min(-(-T // (256 // (team * (D // group)))), 1024))
        assert _size("flex_norm_workspace_size", F.make_norm_desc(T, D, group)) == (OK, rows * D * 4), (group, D)


@pytest.mark.skipif(not NO_GPU, reason="fake pointers are only passed where no GPU is visible")
def test_calls_are_refused():
    lib, big = F.load(), 1 << 40

    def each(call, ok, needed, loose):
        """Every needed argument missing, every one but the offsets unaligned."""
        for i in needed:
            assert call(*ok[:i], None, *ok[i + 1:]) == BAD, i
        for i in range(len(ok)):
            if i not in loose:
                assert call(*ok[:i], FAKE + 2, *ok[i + 1:]) == BAD, i

    r = ctypes.byref(F.make_conv_desc(2, 100, 64, 4))
    each(lambda *a: lib.flex_conv_fwd(r, *a, None), [FAKE] * 7, (0, 1, 3, 5), (3,))   # X W bias off state0 Y state
    each(lambda *a: lib.flex_conv_bwd(r, *a, FAKE, big, None), [FAKE] * 9, (0, 1, 3, 5, 6, 7), (3,))   # .. dY dX dW dbias
    assert lib.flex_conv_bwd(r, *[FAKE] * 9, None, big, None) == WS and lib.flex_conv_bwd(r, *[FAKE] * 9, FAKE, 64, None) == WS
    each(lambda *a: lib.flex_conv_step(r, *a, None), [FAKE] * 5, (0, 1, 3, 4), ())   # x W bias state y
    assert lib.flex_conv_fwd(None, *[FAKE] * 7, None) == BAD

    r = ctypes.byref(F.make_scan_desc(2, 2, 4, 64, 64, 100))
    each(lambda *a: lib.flex_scan_fwd(r, *a, None, 0, FAKE, big, None), [FAKE] * 10, (0, 1, 2, 3, 4, 6, 8), (6,))
    ok = [FAKE] * 10   # X Bt Ct dt g D off state0 Y state
    assert lib.flex_scan_fwd(r, *ok, None, 0, None, 0, None) == WS
    assert lib.flex_scan_fwd(r, *ok, None, 0, FAKE, 100, None) == WS
    assert lib.flex_scan_fwd(r, *ok, FAKE, 100, FAKE, big, None) == WS
    assert lib.flex_scan_fwd(r, *ok, FAKE + 4, big, FAKE, big, None) == WS
    ok, out = [FAKE] * 7, [FAKE] * 7   # X Bt Ct dt g D off; dY dX dB dC ddt dg dD
    for i in (0, 1, 2, 3, 4, 6):
        assert lib.flex_scan_bwd(r, *ok[:i], None, *ok[i + 1:], FAKE, big, *out, FAKE, big, None) == BAD, i
    for i in range(6):
        assert lib.flex_scan_bwd(r, *ok, FAKE, big, *out[:i], None, *out[i + 1:], FAKE, big, None) == BAD, i
    assert lib.flex_scan_bwd(r, *ok, None, big, *out, FAKE, big, None) == WS
    assert lib.flex_scan_bwd(r, *ok, FAKE, 100, *out, FAKE, big, None) == WS
    assert lib.flex_scan_bwd(r, *ok, FAKE, big, *out, FAKE, 100, None) == WS
    each(lambda *a: lib.flex_scan_step(r, *a, None), [FAKE] * 8, (0, 1, 2, 3, 4, 6, 7), ())   # x Bt Ct dt g D state y

    r = ctypes.byref(F.make_norm_desc(100, 64, 64))
    each(lambda *a: lib.flex_norm_fwd(r, *a, None), [FAKE] * 4, (0, 1, 2, 3), ())   # X Z W Y
    each(lambda *a: lib.flex_norm_bwd(r, *a, FAKE, big, None), [FAKE] * 7, range(7), ())   # X Z W dY dX dZ dW
    assert lib.flex_norm_bwd(r, *[FAKE] * 7, FAKE, 100, None) == WS
    n = ctypes.byref(F.make_norm_desc(100, 64, 64, gate="none"))   # no gate: no Z and no dZ
    assert lib.flex_norm_fwd(n, *[FAKE] * 4, None) == BAD
    assert lib.flex_norm_bwd(n, FAKE, None, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, big, None) == BAD

    # nothing to do: no rows
    assert lib.flex_conv_fwd(ctypes.byref(F.make_conv_desc(2, 0, 64, 4)), None, FAKE, None, FAKE, None, None, None, None) == OK
    assert lib.flex_norm_fwd(ctypes.byref(F.make_norm_desc(0, 64, 64)), None, None, FAKE, None, None) == OK
    e = ctypes.byref(F.make_scan_desc(2, 2, 4, 64, 64, 0))
    assert lib.flex_scan_fwd(e, *[None] * 6, FAKE, *[None] * 3, None, 0, None, 0, None) == OK


def test_largest_launches():
    """Sizes whose launches would have 2^32 threads are refused, the next below are not."""
    for B_, status in ((16383, OK), (16384, BAD)):   # 4096 threads per state of 128 x 128
        assert _size("flex_scan_saved_size", F.make_scan_desc(B_, 16, 64, 128, 128, 1000))[0] == status
    for T, status in ((1 << 23, OK), (1 << 24, BAD)):   # 128 waves for 32 rows of 2^15 channels
        assert _size("flex_conv_workspace_size", F.make_conv_desc(1, T, 1 << 15, 4))[0] == status


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
    flex_conv_desc c; std::memset(&c, 0, sizeof(c));
    c.B = B; c.T = T; c.D = d; c.K = 2 + B % 3; c.act = io; c.io_dtype = io;
    bad += flex_conv_workspace_size(&c, &n) != FLEX_OK;
    bad += flex_conv_fwd(&c, p, f, f, nullptr, p, p, p, nullptr) != FLEX_ERR_INVALID_ARG;
    bad += flex_conv_bwd(&c, p, f, f, o, p, p, p, nullptr, f, p, 1u << 30, nullptr) != FLEX_ERR_INVALID_ARG;
    bad += flex_conv_step(&c, p, f, f, nullptr, p, nullptr) != FLEX_ERR_INVALID_ARG;
    flex_scan_desc s; std::memset(&s, 0, sizeof(s));
    s.B = B; s.T = T; s.G = 2; s.H = 4; s.N = d; s.P = 64; s.io_dtype = io;
    const int want = d == 32 ? FLEX_ERR_UNSUPPORTED : FLEX_OK;
    bad += flex_scan_workspace_size(&s, FLEX_PASS_FWD, &n) != want;
    bad += flex_scan_workspace_size(&s, FLEX_PASS_BWD, &n) != want;
    bad += flex_scan_saved_size(&s, &n) != want;
    bad += flex_scan_fwd(&s, p, p, p, f, f, f, nullptr, f, p, f, p, 1, p, 1, nullptr) == FLEX_OK;
    bad += flex_scan_bwd(&s, p, p, p, f, f, f, o, p, 1, p, p, p, p, p, p, f, p, 1, nullptr) == FLEX_OK;
    bad += flex_scan_step(&s, p, p, p, f, f, f, nullptr, p, nullptr) == FLEX_OK;
    flex_norm_desc m; std::memset(&m, 0, sizeof(m));
    m.T = T; m.D = 2 * d; m.group = d; m.gate = B % 3; m.io_dtype = io;
    bad += flex_norm_workspace_size(&m, &n) != FLEX_OK;
    bad += flex_norm_fwd(&m, p, p, nullptr, p, nullptr) != FLEX_ERR_INVALID_ARG;
    bad += flex_norm_bwd(&m, p, p, f, p, p, p, nullptr, p, 1u << 30, nullptr) != FLEX_ERR_INVALID_ARG;
  }
  std::printf("%d\n", bad);
  return bad != 0;
}
"""


@pytest.mark.skipif(not os.path.exists("/opt/rocm/llvm/bin/clang++"), reason="needs hipcc and clang++")
def test_host_code_under_asan(tmp_path):
    objs = [os.path.join(B.BUILD, s.replace(".hip", ".o")) for s in B.SOURCES if s != "flex_layer_api.hip"]
    if not all(os.path.exists(o) for o in objs):
        B.build()
    api, drv, exe = (str(tmp_path / n) for n in ("api.o", "drv.o", "drv"))
    inc, host = os.path.join(B.ROOT, "include"), ["-Xarch_host", "-fsanitize=address"]
    subprocess.run([B.HIPCC, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-fPIC", "-Xclang", "-target-feature",
                    "-Xclang", "-packed-fp32-ops", *host, "-I", inc, "-c", os.path.join(B.CSRC, "flex_layer_api.hip"),
                    "-o", api], check=True, capture_output=True)
    (tmp_path / "drv.cpp").write_text(ASAN_DRIVER)
    clang = "/opt/rocm/llvm/bin/clang++"
    subprocess.run([clang, "-std=c++17", "-g", "-fsanitize=address", "-I", inc, "-c", str(tmp_path / "drv.cpp"), "-o", drv],
                   check=True, capture_output=True)
    subprocess.run([clang, "-fsanitize=address", drv, api, *objs, "-L/opt/rocm/lib", "-lamdhip64",
                    "-Wl,-rpath,/opt/rocm/lib", "-o", exe], check=True, capture_output=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120, env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0"))
    assert r.returncode == 0 and r.stdout.strip() == "0", (r.stdout, r.stderr[-2000:])
