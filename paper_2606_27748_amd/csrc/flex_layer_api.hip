// C ABI of the operators of selective state-space layers (short convolution, selective scan, gated
// norm): argument validation, workspace sizing and how the work is cut.
#include "../../include/flex.h"
#include "flex_layer_kernels.hpp"

#include <math.h>
#include <string.h>

using namespace flex;

namespace {

constexpr int kMaxStride = 1 << 20;   // elements: a tile's window of rows stays within 32-bit byte offsets
constexpr int64_t kMaxThreads = (1LL << 32) - 1;   // of a launch

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }
int esize(int32_t io_dtype) { return io_dtype == FLEX_BF16 ? 2 : 4; }
bool io_ok(int32_t io_dtype) { return io_dtype == FLEX_F32 || io_dtype == FLEX_BF16; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// A row stride: 0 (contiguous rows of `row` elements), or a whole number of 16-byte
// units that rows fit in.
bool stride_ok(int32_t stride, int64_t row, int e) {
  if (stride == 0) return true;
  return stride >= row && stride <= kMaxStride && (int64_t)stride * e % 16 == 0;
}
int stride_of(int32_t stride, int64_t row) { return stride ? stride : (int)row; }
// a required tensor of `rows` rows, an optional one
bool tensor_ok(const void* p, int64_t rows) { return rows == 0 || (p && aligned16(p)); }
bool maybe_ok(const void* p) { return !p || aligned16(p); }

// ---- short convolution ----
int32_t check_conv(const flex_conv_desc* d, bool step) {
  if (!d) return FLEX_ERR_INVALID_ARG;
  if (d->B <= 0 || d->T < 0 || d->D <= 0 || d->K <= 0) return FLEX_ERR_INVALID_ARG;
  if (d->act != FLEX_ACT_NONE && d->act != FLEX_ACT_SILU) return FLEX_ERR_INVALID_ARG;
  if (!io_ok(d->io_dtype)) return FLEX_ERR_INVALID_ARG;
  if (d->D % 8 != 0 || d->D > kMaxStride || d->K < 2 || d->K > 4) return FLEX_ERR_UNSUPPORTED;
  const int e = esize(d->io_dtype);
  if (!stride_ok(d->x_stride, d->D, e) || !stride_ok(d->dx_stride, d->D, e)) return FLEX_ERR_INVALID_ARG;
  // the threads of a launch: a wave per tile of rows (and sequence, for the last rows) and 64 lanes' channels; a step's
  // thread per piece; indexes of rows fit 31 bits
  const int64_t units = d->D / (16 / e), spans = ceil_div(units, 64);
  const int64_t back = ceil_div(d->T, CONV_BWD_ROWS * CONV_BWD_WAVES) * CONV_BWD_WAVES * ceil_div(d->D / CONV_BWD_CH, 64);
  int64_t waves = step ? ceil_div((int64_t)d->B * units, 64) : (ceil_div(d->T, CONV_ROWS) + d->B + 4) * spans;
  if (!step && back > waves) waves = back;
  if ((waves + 4) * 64 > kMaxThreads || (int64_t)d->T + CONV_BWD_ROWS * CONV_BWD_WAVES >= (1LL << 31)) return FLEX_ERR_INVALID_ARG;
  return FLEX_OK;
}
int conv_parts(const flex_conv_desc* d) { return (int)ceil_div(d->T, CONV_BWD_ROWS * CONV_BWD_WAVES); }
size_t conv_ws_bytes(const flex_conv_desc* d) { return (size_t)conv_parts(d) * (d->K + 1) * d->D * sizeof(float); }
ConvArgs conv_args(const flex_conv_desc* d, const void* X, const float* W, const float* bias, const int32_t* off,
                   const void* state0) {
  ConvArgs a;
  memset(&a, 0, sizeof(a));
  a.X = X; a.W = W; a.bias = bias; a.off = off; a.state0 = state0;
  a.B = d->B; a.T = d->T; a.D = d->D; a.K = d->K; a.act = d->act;
  a.xs = stride_of(d->x_stride, d->D);
  a.dxs = stride_of(d->dx_stride, d->D);
  return a;
}

// ---- gated norm ----
constexpr int64_t kNormWaves = 4096;   // 16 per CU
int32_t check_norm(const flex_norm_desc* d) {
  if (!d) return FLEX_ERR_INVALID_ARG;
  if (d->T < 0 || d->D <= 0 || d->group <= 0 || d->D % d->group != 0) return FLEX_ERR_INVALID_ARG;
  if (d->gate < FLEX_GATE_NONE || d->gate > FLEX_GATE_LAST || !io_ok(d->io_dtype)) return FLEX_ERR_INVALID_ARG;
  if (!(d->eps >= 0.0f) || !isfinite(d->eps)) return FLEX_ERR_INVALID_ARG;
  if (d->group % 8 != 0 || d->group > NORM_MAX || d->D > kMaxStride) return FLEX_ERR_UNSUPPORTED;
  const int e = esize(d->io_dtype);
  const int32_t s[] = {d->x_stride, d->z_stride, d->dx_stride, d->dz_stride};
  for (int32_t x : s)
    if (!stride_ok(x, d->D, e)) return FLEX_ERR_INVALID_ARG;
  if ((int64_t)d->T + kNormWaves * 64 >= (1LL << 31)) return FLEX_ERR_INVALID_ARG;   // row indexes fit 31 bits
  return FLEX_OK;
}
// Rows that are walked at once: as many as give the card kNormWaves waves.
int norm_rows(const flex_norm_desc* d) {
  const int64_t n = kNormWaves * 64 / (d->D / 8);
  return (int)(n < 1 ? 1 : n > d->T ? (d->T > 0 ? d->T : 1) : n);
}
// Rows of a workgroup of the backward at a time, which leaves one row of partial sums of dW: of rows that up to a wave's
// lanes have, a piece each.  Wider ones leave a row of sums for each that is walked.
// (2^20 rows of 64 channels, bf16: backward 137 us, forward 76; with a row of sums each, and so 4096 rows at once, 261 and 194.)
int norm_wg_rows(const flex_norm_desc* d) {
  const int64_t lanes = (int64_t)norm_team(d->group) * (d->D / d->group);
  return lanes <= 64 && d->group <= 64 * 8 ? (int)(256 / lanes) : 1;
}
int norm_parts(const flex_norm_desc* d) {
  const int r = norm_wg_rows(d);
  if (r == 1) return norm_rows(d);
  const int64_t wgs = ceil_div(d->T, r);
  return (int)(wgs < 1 ? 1 : wgs > kNormWaves / 4 ? kNormWaves / 4 : wgs);
}
size_t norm_ws_bytes(const flex_norm_desc* d) { return (size_t)norm_parts(d) * d->D * sizeof(float); }
NormArgs norm_args(const flex_norm_desc* d, const void* X, const void* Z, const float* W) {
  NormArgs a;
  memset(&a, 0, sizeof(a));
  a.X = X; a.Z = Z; a.W = W;
  a.T = d->T; a.D = d->D; a.group = d->group; a.gate = d->gate; a.eps = d->eps;
  a.xs = stride_of(d->x_stride, d->D);
  a.zs = stride_of(d->z_stride, d->D);
  a.dxs = stride_of(d->dx_stride, d->D);
  a.dzs = stride_of(d->dz_stride, d->D);
  a.rows = norm_rows(d);
  return a;
}

// ---- selective scan ----
// Heads of a sweep's workgroup: as many of a group as eight waves of 32 columns hold, by halves.
int scan_heads(const flex_scan_desc* d) {
  const int r = d->H / d->G;
  int n = 256 / d->P;
  while (n > 1 && r % n != 0) n /= 2;
  return n;
}
int64_t scan_slots(const flex_scan_desc* d, int rows) { return (int64_t)d->T / rows + d->B; }

// Parts of a group's heads in the gradients, each a workgroup's: as many as give the card two workgroups per CU.
int scan_parts(const flex_scan_desc* d) {
  const int r = d->H / d->G;
  const int64_t wgs = scan_slots(d, SCAN_CHUNK) * d->G;
  int n = 1;
  while (n < r && (r % (2 * n) == 0) && wgs * n < 512) n *= 2;
  return n;
}
int32_t check_scan(const flex_scan_desc* d, bool step) {
  if (!d) return FLEX_ERR_INVALID_ARG;
  if (d->B <= 0 || d->T < 0 || d->G <= 0 || d->H <= 0 || d->N <= 0 || d->P <= 0) return FLEX_ERR_INVALID_ARG;
  if (d->H % d->G != 0 || !io_ok(d->io_dtype)) return FLEX_ERR_INVALID_ARG;
  if ((d->N != 64 && d->N != 128) || (d->P != 64 && d->P != 128)) return FLEX_ERR_UNSUPPORTED;
  const int64_t x = (int64_t)d->H * d->P, b = (int64_t)d->G * d->N;
  if (x > kMaxStride || b > kMaxStride) return FLEX_ERR_UNSUPPORTED;
  const int e = esize(d->io_dtype);
  if (!stride_ok(d->x_stride, x, e) || !stride_ok(d->dx_stride, x, e) || !stride_ok(d->b_stride, b, e) ||
      !stride_ok(d->db_stride, b, e) || !stride_ok(d->c_stride, b, e) || !stride_ok(d->dc_stride, b, e))
    return FLEX_ERR_INVALID_ARG;
  // the threads of a launch: a state's in the step and where carries meet, its columns' waves in the sweeps,
  // a chunk's for each part of a group's heads; row and slot indexes fit 31 bits
  const int64_t states = (int64_t)d->B * d->H, slots = step ? 0 : scan_slots(d, SCAN_CHUNK);
  if (states * 4096 > kMaxThreads || slots * d->H * 512 > kMaxThreads || (int64_t)d->T + d->B >= (1LL << 30))
    return FLEX_ERR_INVALID_ARG;
  // the gradients' chunks go by as many at once as there are XCDs
  if (!step && ceil_div(slots, 8) * 8 * d->G * scan_parts(d) * 512 > kMaxThreads) return FLEX_ERR_INVALID_ARG;
  return FLEX_OK;
}

// Tokens of a segment.  A sweep's workgroup takes a CU, its sequences are walked in order, and a
// segment that is not its sequence's last has its rows read twice: segments so long that the card has one
// workgroup per CU of them, 64 to 4096 tokens (a prompt of 32768 tokens, 16 heads of 128: 207 us; with twice as many
// 235).  Many sequences, whose ends leave workgroups of any length, have twice as many.  Heads of 64, N = 128, forward with twice as
// many against one per CU: 16 prompts of 17152 tokens 253 and 265 us, of 31149 393 and 484, of 26818 360 and 349; 24 of 47020 610 and 686;
// training of 12 of 15190 689 and 716.  Where as few as eight are of one length, one per CU is better (8 x 2048: 197 and 179,
// training 665 and 609), but the host knows no lengths.
int scan_seg(const flex_scan_desc* d) {
  const int64_t sets = d->H / scan_heads(d), wgs = d->B * sets < 128 ? 256 : 512;
  int64_t n = ceil_div((int64_t)d->T * sets, wgs * SCAN_CHUNK) * SCAN_CHUNK;
  if (n < SCAN_CHUNK) n = SCAN_CHUNK;
  if (n > 4096) n = 4096;
  return (int)n;
}
bool scan_split(const flex_scan_desc* d) { return d->T > scan_seg(d); }
size_t scan_state(const flex_scan_desc* d) { return (size_t)d->H * d->N * d->P; }
size_t scan_carry_bytes(const flex_scan_desc* d) {
  return scan_split(d) ? (size_t)scan_slots(d, scan_seg(d)) * scan_state(d) * sizeof(float) : 0;
}
size_t scan_tot_bytes(const flex_scan_desc* d) {
  return scan_split(d) ? align256((size_t)scan_slots(d, scan_seg(d)) * d->H * sizeof(float)) : 0;
}
size_t scan_saved_bytes(const flex_scan_desc* d) {
  return (size_t)scan_slots(d, SCAN_CHUNK) * scan_state(d) * esize(d->io_dtype);
}
size_t scan_part_bytes(const flex_scan_desc* d) {
  return scan_parts(d) > 1 ? (size_t)scan_parts(d) * scan_slots(d, SCAN_CHUNK) * SCAN_CHUNK * d->G * d->N * sizeof(float) : 0;
}
size_t scan_ws_bytes(const flex_scan_desc* d, int32_t pass) {
  size_t n = scan_carry_bytes(d) + scan_tot_bytes(d);
  if (pass == FLEX_PASS_BWD)
    n += scan_saved_bytes(d) + 2 * scan_part_bytes(d) + (size_t)scan_slots(d, SCAN_CHUNK) * d->H * sizeof(float);
  return n;
}
ScanArgs scan_args(const flex_scan_desc* d, const void* X, const void* Bt, const void* Ct, const float* dt,
                   const float* g, const float* D, const int32_t* off) {
  ScanArgs a;
  memset(&a, 0, sizeof(a));
  a.X = X; a.Bt = Bt; a.Ct = Ct; a.dt = dt; a.g = g; a.D = D; a.off = off;
  a.B = d->B; a.T = d->T; a.G = d->G; a.H = d->H; a.N = d->N; a.P = d->P;
  const int64_t x = (int64_t)d->H * d->P, b = (int64_t)d->G * d->N;
  a.xs = stride_of(d->x_stride, x);
  a.bs = stride_of(d->b_stride, b);
  a.cs = stride_of(d->c_stride, b);
  a.dxs = stride_of(d->dx_stride, x);
  a.dbs = stride_of(d->db_stride, b);
  a.dcs = stride_of(d->dc_stride, b);
  a.heads = scan_heads(d);
  a.seg = scan_seg(d);
  return a;
}
char* scan_carry(ScanArgs& a, const flex_scan_desc* d, void* ws) {
  char* p = static_cast<char*>(ws);
  if (scan_split(d)) {
    a.carry = reinterpret_cast<float*>(p);
    a.tot = reinterpret_cast<float*>(p + scan_carry_bytes(d));
  }
  return p + scan_carry_bytes(d) + scan_tot_bytes(d);
}

int32_t done(hipError_t e) { return e == hipSuccess ? FLEX_OK : FLEX_ERR_HIP; }

}  // namespace

extern "C" {

int32_t flex_conv_workspace_size(const flex_conv_desc* desc, size_t* bytes) {
  if (!bytes) return FLEX_ERR_INVALID_ARG;
  *bytes = 0;
  const int32_t st = check_conv(desc, false);
  if (st != FLEX_OK) return st;
  *bytes = conv_ws_bytes(desc);
  return FLEX_OK;
}

int32_t flex_conv_fwd(const flex_conv_desc* desc, const void* X, const float* W, const float* bias, const int32_t* off,
                      const void* state0, void* Y, void* state, void* stream) {
  const int32_t st = check_conv(desc, false);
  if (st != FLEX_OK) return st;
  if (!off || !W || !aligned16(W) || !maybe_ok(bias) || !maybe_ok(state0) || !maybe_ok(state) || !tensor_ok(X, desc->T) ||
      !tensor_ok(Y, desc->T))
    return FLEX_ERR_INVALID_ARG;
  if (desc->T == 0 && !state) return FLEX_OK;
  ConvArgs a = conv_args(desc, X, W, bias, off, state0);
  a.Y = Y; a.state = state;
  return done(launch_conv_fwd(a, desc->io_dtype == FLEX_BF16, (hipStream_t)stream));
}

int32_t flex_conv_bwd(const flex_conv_desc* desc, const void* X, const float* W, const float* bias, const int32_t* off,
                      const void* state0, const void* dY, void* dX, float* dW, float* dbias, void* ws, size_t ws_bytes,
                      void* stream) {
  const int32_t st = check_conv(desc, false);
  if (st != FLEX_OK) return st;
  if (!off || !W || !aligned16(W) || !maybe_ok(bias) || !maybe_ok(state0) || !dW || !aligned16(dW) || !maybe_ok(dbias) ||
      !tensor_ok(X, desc->T) || !tensor_ok(dY, desc->T) || !tensor_ok(dX, desc->T))
    return FLEX_ERR_INVALID_ARG;
  const size_t need = conv_ws_bytes(desc);
  if (need > 0 && (!ws || ws_bytes < need || !aligned16(ws))) return FLEX_ERR_WORKSPACE;
  ConvArgs a = conv_args(desc, X, W, bias, off, state0);
  a.dY = dY; a.dX = dX; a.dW = dW; a.dbias = dbias;
  a.part = static_cast<float*>(ws);
  a.parts = conv_parts(desc);
  return done(launch_conv_bwd(a, desc->io_dtype == FLEX_BF16, (hipStream_t)stream));
}

int32_t flex_conv_step(const flex_conv_desc* desc, const void* x, const float* W, const float* bias, void* state, void* y,
                       void* stream) {
  const int32_t st = check_conv(desc, true);
  if (st != FLEX_OK) return st;
  const void* need[] = {x, W, state, y};
  for (const void* p : need)
    if (!p || !aligned16(p)) return FLEX_ERR_INVALID_ARG;
  if (!maybe_ok(bias)) return FLEX_ERR_INVALID_ARG;
  ConvArgs a = conv_args(desc, x, W, bias, nullptr, nullptr);
  a.Y = y; a.state = state;
  return done(launch_conv_step(a, desc->io_dtype == FLEX_BF16, (hipStream_t)stream));
}

int32_t flex_norm_workspace_size(const flex_norm_desc* desc, size_t* bytes) {
  if (!bytes) return FLEX_ERR_INVALID_ARG;
  *bytes = 0;
  const int32_t st = check_norm(desc);
  if (st != FLEX_OK) return st;
  *bytes = norm_ws_bytes(desc);
  return FLEX_OK;
}

int32_t flex_norm_fwd(const flex_norm_desc* desc, const void* X, const void* Z, const float* W, void* Y, void* stream) {
  const int32_t st = check_norm(desc);
  if (st != FLEX_OK) return st;
  if (!W || !aligned16(W) || !tensor_ok(X, desc->T) || !tensor_ok(Y, desc->T)) return FLEX_ERR_INVALID_ARG;
  if (desc->gate == FLEX_GATE_NONE ? Z != nullptr : !tensor_ok(Z, desc->T)) return FLEX_ERR_INVALID_ARG;
  if (desc->T == 0) return FLEX_OK;
  NormArgs a = norm_args(desc, X, Z, W);
  a.Y = Y;
  return done(launch_norm_fwd(a, desc->io_dtype == FLEX_BF16, (hipStream_t)stream));
}

int32_t flex_norm_bwd(const flex_norm_desc* desc, const void* X, const void* Z, const float* W, const void* dY, void* dX,
                      void* dZ, float* dW, void* ws, size_t ws_bytes, void* stream) {
  const int32_t st = check_norm(desc);
  if (st != FLEX_OK) return st;
  if (!W || !aligned16(W) || !dW || !aligned16(dW) || !tensor_ok(X, desc->T) || !tensor_ok(dY, desc->T) ||
      !tensor_ok(dX, desc->T))
    return FLEX_ERR_INVALID_ARG;
  if (desc->gate == FLEX_GATE_NONE ? Z || dZ : !tensor_ok(Z, desc->T) || !tensor_ok(dZ, desc->T)) return FLEX_ERR_INVALID_ARG;
  const size_t need = norm_ws_bytes(desc);
  if (!ws || ws_bytes < need || !aligned16(ws)) return FLEX_ERR_WORKSPACE;
  NormArgs a = norm_args(desc, X, Z, W);
  a.dY = dY; a.dX = dX; a.dZ = dZ; a.dW = dW;
  a.part = static_cast<float*>(ws);
  a.parts = norm_parts(desc);
  a.wg_rows = norm_wg_rows(desc);
  if (a.wg_rows > 1) a.rows = a.parts * a.wg_rows;
  return done(launch_norm_bwd(a, desc->io_dtype == FLEX_BF16, (hipStream_t)stream));
}

int32_t flex_scan_workspace_size(const flex_scan_desc* desc, int32_t pass, size_t* bytes) {
  if (!bytes) return FLEX_ERR_INVALID_ARG;
  *bytes = 0;
  if (pass != FLEX_PASS_FWD && pass != FLEX_PASS_BWD) return FLEX_ERR_INVALID_ARG;
  const int32_t st = check_scan(desc, false);
  if (st != FLEX_OK) return st;
  *bytes = scan_ws_bytes(desc, pass);
  return FLEX_OK;
}

int32_t flex_scan_saved_size(const flex_scan_desc* desc, size_t* bytes) {
  if (!bytes) return FLEX_ERR_INVALID_ARG;
  *bytes = 0;
  const int32_t st = check_scan(desc, false);
  if (st != FLEX_OK) return st;
  *bytes = scan_saved_bytes(desc);
  return FLEX_OK;
}

int32_t flex_scan_fwd(const flex_scan_desc* desc, const void* X, const void* Bt, const void* Ct, const float* dt,
                      const float* g, const float* D, const int32_t* off, const float* state0, void* Y, float* state,
                      void* saved, size_t saved_bytes, void* ws, size_t ws_bytes, void* stream) {
  const int32_t st = check_scan(desc, false);
  if (st != FLEX_OK) return st;
  if (!off) return FLEX_ERR_INVALID_ARG;
  const void* rows[] = {X, Bt, Ct, dt, g, Y};
  for (const void* p : rows)
    if (!tensor_ok(p, desc->T)) return FLEX_ERR_INVALID_ARG;
  if (!maybe_ok(D) || !maybe_ok(state0) || !maybe_ok(state)) return FLEX_ERR_INVALID_ARG;
  if (saved && (saved_bytes < scan_saved_bytes(desc) || !aligned16(saved))) return FLEX_ERR_WORKSPACE;
  const size_t need = scan_ws_bytes(desc, FLEX_PASS_FWD);
  if (need > 0 && (!ws || ws_bytes < need || !aligned16(ws))) return FLEX_ERR_WORKSPACE;
  if (desc->T == 0 && !state) return FLEX_OK;
  ScanArgs a = scan_args(desc, X, Bt, Ct, dt, g, D, off);
  a.state0 = state0; a.state = state; a.Y = Y; a.st = saved;
  scan_carry(a, desc, ws);
  return done(launch_scan_fwd(a, desc->io_dtype == FLEX_BF16, (hipStream_t)stream));
}

int32_t flex_scan_bwd(const flex_scan_desc* desc, const void* X, const void* Bt, const void* Ct, const float* dt,
                      const float* g, const float* D, const int32_t* off, const void* saved, size_t saved_bytes,
                      const void* dY, void* dX, void* dB, void* dC, void* ddt, void* dg, float* dD, void* ws,
                      size_t ws_bytes, void* stream) {
  const int32_t st = check_scan(desc, false);
  if (st != FLEX_OK) return st;
  if (!off) return FLEX_ERR_INVALID_ARG;
  const void* rows[] = {X, Bt, Ct, dt, g, dY, dX, dB, dC, ddt, dg};
  for (const void* p : rows)
    if (!tensor_ok(p, desc->T)) return FLEX_ERR_INVALID_ARG;
  if (!maybe_ok(D) || !maybe_ok(dD)) return FLEX_ERR_INVALID_ARG;
  if (!saved || saved_bytes < scan_saved_bytes(desc) || !aligned16(saved)) return FLEX_ERR_WORKSPACE;
  const size_t need = scan_ws_bytes(desc, FLEX_PASS_BWD);
  if (!ws || ws_bytes < need || !aligned16(ws)) return FLEX_ERR_WORKSPACE;
  if (desc->T == 0 && !dD) return FLEX_OK;
  ScanArgs a = scan_args(desc, X, Bt, Ct, dt, g, D, off);
  a.st = const_cast<void*>(saved);
  a.dY = dY; a.dX = dX; a.dB = dB; a.dC = dC; a.ddt = ddt; a.dg = dg; a.dD = dD;
  char* p = scan_carry(a, desc, ws);
  a.dst = p;
  p += scan_saved_bytes(desc);
  a.parts = scan_parts(desc);
  if (a.parts > 1) {
    a.part_b = reinterpret_cast<float*>(p);
    a.part_c = reinterpret_cast<float*>(p + scan_part_bytes(desc));
  }
  a.part_d = reinterpret_cast<float*>(p + 2 * scan_part_bytes(desc));
  return done(launch_scan_bwd(a, desc->io_dtype == FLEX_BF16, (hipStream_t)stream));
}

int32_t flex_scan_step(const flex_scan_desc* desc, const void* x, const void* Bt, const void* Ct, const float* dt,
                       const float* g, const float* D, float* state, void* y, void* stream) {
  const int32_t st = check_scan(desc, true);
  if (st != FLEX_OK) return st;
  const void* rows[] = {x, Bt, Ct, dt, g, state, y};
  for (const void* p : rows)
    if (!p || !aligned16(p)) return FLEX_ERR_INVALID_ARG;
  if (!maybe_ok(D)) return FLEX_ERR_INVALID_ARG;
  ScanArgs a = scan_args(desc, x, Bt, Ct, dt, g, D, nullptr);
  a.state = state; a.Y = y;
  return done(launch_scan_step(a, desc->io_dtype == FLEX_BF16, (hipStream_t)stream));
}

}  // extern "C"
