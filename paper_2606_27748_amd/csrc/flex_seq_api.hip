// C ABI of the packed-sequence operators: argument validation, workspace sizing and
// the choice of kernels.
#include "../../include/flex.h"
#include "flex_seq_kernels.hpp"

#include <math.h>
#include <string.h>

using namespace flex;

namespace {

constexpr int kMaxStride = 1 << 20;   // elements: a tile's window of rows stays within 32-bit byte offsets
constexpr int64_t kMaxThreads = (1LL << 32) - 1;   // of a launch

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }
int esize(int32_t io_dtype) { return io_dtype == FLEX_BF16 ? 2 : 4; }

// A row stride: 0 (contiguous rows of `row` elements), or a whole number of 16-byte
// units that rows fit in.
bool stride_ok(int32_t stride, int64_t row, int e) {
  if (stride == 0) return true;
  return stride >= row && stride <= kMaxStride && (int64_t)stride * e % 16 == 0;
}
int stride_of(int32_t stride, int64_t row) { return stride ? stride : (int)row; }

// a required tensor of `rows` rows, 16-byte aligned
bool tensor_ok(const void* p, int64_t rows) { return rows == 0 || (p && aligned16(p)); }

// The calls of the split kernel, which takes 32 rows (queries times heads of a group) of a sequence
// and reads its keys for each 32: those whose sequences have up to twice that many on average.
// us of it and of the prompt kernel, 16 heads of 128 on 4: 64 sequences of 1000 keys, 32 rows 42 and 74, 64 rows 87
// and 73, 128 rows 135 and 71; of 8192 keys 202 and 509, 473 and 517, 600 and 519; 8 sequences of 4000 keys 21 and
// 79, 36 and 80, 53 and 82.  One sequence of 40000 keys does not give the prompt kernel workgroups enough, and
// would gain far beyond the border: with 2 key heads 64 rows 27 and 705, 72 rows 35 and 705, 512 rows 154 and
// 718.  Nor does the mean see a prompt of 4000 tokens with 255 single ones on 1000 keys each (279 and 360; 97 and 94
// as two calls).
bool few_rows(const flex_attn_desc* d) { return (int64_t)d->Tq * (d->Hq / d->Hkv) <= 64LL * d->B; }
int64_t row_blocks(const flex_attn_desc* d) { return (int64_t)d->Tq * (d->Hq / d->Hkv) / 32 + d->B; }

int32_t check_attn(const flex_attn_desc* d) {
  if (!d) return FLEX_ERR_INVALID_ARG;
  if (d->B <= 0 || d->Hq <= 0 || d->Hkv <= 0 || d->d <= 0 || d->Tq < 0 || d->Tk < 0) return FLEX_ERR_INVALID_ARG;
  if (d->Hq % d->Hkv != 0) return FLEX_ERR_INVALID_ARG;
  if (d->causal != 0 && d->causal != 1) return FLEX_ERR_INVALID_ARG;
  if (d->io_dtype != FLEX_F32 && d->io_dtype != FLEX_BF16) return FLEX_ERR_INVALID_ARG;
  if (!(d->scale > 0.0f) || !isfinite(d->scale)) return FLEX_ERR_INVALID_ARG;
  if (d->d != 32 && d->d != 64 && d->d != 128) return FLEX_ERR_UNSUPPORTED;
  const int64_t q = (int64_t)d->Hq * d->d, k = (int64_t)d->Hkv * d->d;
  if (q > kMaxStride) return FLEX_ERR_UNSUPPORTED;
  const int e = esize(d->io_dtype);
  if (!stride_ok(d->q_stride, q, e) || !stride_ok(d->k_stride, k, e) || !stride_ok(d->v_stride, k, e))
    return FLEX_ERR_INVALID_ARG;
  // row and head indexes fit 31 bits, and the largest launches (tiles of 128 rows with 256 threads, of keys
  // with 512, statistics with d / 8 threads a row; 32 rows of a group with 256) their threads 32
  const int64_t B = d->B, q_tiles = d->Tq / 128 + B, k_tiles = d->Tk / 128 + B;
  if ((d->Tq + B) * d->Hq >= (1LL << 31) || q_tiles * d->Hq * 256 > kMaxThreads || k_tiles * d->Hkv * 512 > kMaxThreads ||
      ((int64_t)d->Tq * d->Hq + 255) * (d->d / 8) > kMaxThreads || (few_rows(d) && row_blocks(d) * d->Hkv * 256 > kMaxThreads))
    return FLEX_ERR_INVALID_ARG;
  return FLEX_OK;
}

// Parts of each sequence's keys in the forward; 0: the kernel for prompts.
// A workgroup of it fills a CU at d = 128: one part per CU where few heads and sequences share them,
// and two where many do, whose lengths differ.  us with 256, 512 and 1024 workgroups: one
// token against 40000 rows, 4 key heads, 20.6, 24.0 and 26; 64 tokens against 253385 rows in slots
// of 8192, 2 key heads, 65.5, 63.0 and 66.  With 256 and 512, 8192 rows a sequence, 4 key heads: 4 sequences 19.3 and
// 21.9, 8 28.2 and 30.9, 12 43.9 and 43.9, 16 46.2 and 48.9, 24 95.7 and 85.7, 64 184 and 191.  The mean length decides:
// one sequence of 40000 rows among 63 of 100 gets two parts (135; alone 16).
int attn_parts(const flex_attn_desc* d) {
  if (!few_rows(d)) return 0;
  const int64_t wgs = (int64_t)d->B * d->Hkv, keys = d->Tk / d->B;
  const int64_t target = wgs < 64 ? 256 : 512;
  int64_t n = (target + wgs - 1) / wgs;
  if (n > keys / 256) n = keys / 256;
  if (n > ATTN_PARTS) n = ATTN_PARTS;
  return n < 1 ? 1 : (int)n;
}
size_t attn_part_rows(const flex_attn_desc* d) { return (size_t)d->Tq * d->Hq * (size_t)attn_parts(d); }

size_t attn_ws_bytes(const flex_attn_desc* d, int32_t pass) {
  if (pass == FLEX_PASS_BWD) return (size_t)2 * d->Tq * d->Hq * sizeof(float);
  if (attn_parts(d) <= 1) return 0;
  return align256(attn_part_rows(d) * d->d * sizeof(float)) + attn_part_rows(d) * 2 * sizeof(float);
}

AttnArgs attn_args(const flex_attn_desc* d, const void* Q, const void* K, const void* V, const int32_t* q_off,
                   const int32_t* k_off) {
  AttnArgs a;
  memset(&a, 0, sizeof(a));
  a.Q = Q; a.K = K; a.V = V; a.q_off = q_off; a.k_off = k_off;
  a.B = d->B; a.Hq = d->Hq; a.Hkv = d->Hkv; a.Tq = d->Tq; a.Tk = d->Tk; a.causal = d->causal;
  a.qs = stride_of(d->q_stride, (int64_t)d->Hq * d->d);
  a.ks = stride_of(d->k_stride, (int64_t)d->Hkv * d->d);
  a.vs = stride_of(d->v_stride, (int64_t)d->Hkv * d->d);
  a.scale = d->scale;
  return a;
}

int32_t check_delta(const flex_delta_desc* d, bool step) {
  if (!d) return FLEX_ERR_INVALID_ARG;
  if (d->B <= 0 || d->T < 0 || d->Hk <= 0 || d->H <= 0 || d->d <= 0 || d->dv <= 0) return FLEX_ERR_INVALID_ARG;
  if (d->H % d->Hk != 0) return FLEX_ERR_INVALID_ARG;
  if (d->io_dtype != FLEX_F32 && d->io_dtype != FLEX_BF16) return FLEX_ERR_INVALID_ARG;
  if (!(d->scale > 0.0f) || !isfinite(d->scale)) return FLEX_ERR_INVALID_ARG;
  if ((d->d != 64 && d->d != 128) || (d->dv != 64 && d->dv != 128)) return FLEX_ERR_UNSUPPORTED;
  const int64_t k = (int64_t)d->Hk * d->d, v = (int64_t)d->H * d->dv;
  if (k > kMaxStride || v > kMaxStride) return FLEX_ERR_UNSUPPORTED;
  const int e = esize(d->io_dtype);
  if (!stride_ok(d->q_stride, k, e) || !stride_ok(d->k_stride, k, e) || !stride_ok(d->v_stride, v, e))
    return FLEX_ERR_INVALID_ARG;
  // the threads of a launch: a state's in the step, its columns' 12 waves per 64 in the sweeps, a chunk's for
  // each key head
  const int64_t states = (int64_t)d->B * d->H, slots = step ? 0 : (int64_t)d->T / DELTA_CHUNK + d->B;
  if (states * (step ? 256 : d->dv / 32 * 384) > kMaxThreads || (slots * d->H + 3) * 64 > kMaxThreads ||
      slots * d->Hk * 256 > kMaxThreads)
    return FLEX_ERR_INVALID_ARG;
  return FLEX_OK;
}

// Chunk slots times value heads, and the bytes of what is kept per such block.
size_t delta_blocks(const flex_delta_desc* d) { return ((size_t)d->T / DELTA_CHUNK + d->B) * d->H; }
size_t delta_state_bytes(const flex_delta_desc* d) { return (size_t)d->d * d->dv * esize(d->io_dtype); }
size_t delta_rows_bytes(const flex_delta_desc* d) { return (size_t)DELTA_CHUNK * d->dv * 4; }   // hi and lo, or fp32
size_t delta_prep_bytes(const flex_delta_desc* d) { return delta_blocks(d) * DELTA_PREP_BYTES; }
size_t delta_saved_bytes(const flex_delta_desc* d) {
  return delta_blocks(d) * (DELTA_PREP_BYTES + delta_state_bytes(d) + delta_rows_bytes(d));
}
size_t delta_ws_bytes(const flex_delta_desc* d, int32_t pass) {
  if (pass == FLEX_PASS_FWD) return delta_prep_bytes(d);
  return delta_blocks(d) * (delta_state_bytes(d) + delta_rows_bytes(d));
}

DeltaArgs delta_args(const flex_delta_desc* d, const void* Q, const void* K, const void* V, const float* g,
                     const float* beta, const int32_t* off) {
  DeltaArgs a;
  memset(&a, 0, sizeof(a));
  a.Q = Q; a.K = K; a.V = V; a.g = g; a.beta = beta; a.off = off;
  a.B = d->B; a.T = d->T; a.Hk = d->Hk; a.H = d->H; a.d = d->d; a.dv = d->dv;
  a.qs = stride_of(d->q_stride, (int64_t)d->Hk * d->d);
  a.ks = stride_of(d->k_stride, (int64_t)d->Hk * d->d);
  a.vs = stride_of(d->v_stride, (int64_t)d->H * d->dv);
  a.scale = d->scale;
  return a;
}
void delta_saved(DeltaArgs& a, const flex_delta_desc* d, void* saved) {
  char* p = static_cast<char*>(saved);
  a.prep = p;
  a.st = p + delta_prep_bytes(d);
  a.ut = static_cast<char*>(a.st) + delta_blocks(d) * delta_state_bytes(d);
}

}  // namespace

extern "C" {

int32_t flex_attn_workspace_size(const flex_attn_desc* desc, int32_t pass, size_t* bytes) {
  if (!bytes) return FLEX_ERR_INVALID_ARG;
  *bytes = 0;
  if (pass != FLEX_PASS_FWD && pass != FLEX_PASS_BWD) return FLEX_ERR_INVALID_ARG;
  const int32_t st = check_attn(desc);
  if (st != FLEX_OK) return st;
  *bytes = attn_ws_bytes(desc, pass);
  return FLEX_OK;
}

int32_t flex_attn_fwd(const flex_attn_desc* desc, const void* Q, const void* K, const void* V,
                      const int32_t* q_off, const int32_t* k_off, const int32_t* k_len, void* O, float* lse,
                      void* ws, size_t ws_bytes, void* stream) {
  const int32_t st = check_attn(desc);
  if (st != FLEX_OK) return st;
  if (!q_off || !k_off) return FLEX_ERR_INVALID_ARG;
  if (!tensor_ok(Q, desc->Tq) || !tensor_ok(O, desc->Tq) || !tensor_ok(K, desc->Tk) || !tensor_ok(V, desc->Tk) ||
      (lse && !aligned16(lse)))
    return FLEX_ERR_INVALID_ARG;
  const size_t need = attn_ws_bytes(desc, FLEX_PASS_FWD);
  if (need > 0 && (!ws || ws_bytes < need || !aligned16(ws))) return FLEX_ERR_WORKSPACE;
  if (desc->Tq == 0) return FLEX_OK;
  AttnArgs a = attn_args(desc, Q, K, V, q_off, k_off);
  a.k_len = k_len; a.O = O; a.lse = lse;
  a.nsplit = attn_parts(desc);
  if (need > 0) {
    a.part_o = static_cast<float*>(ws);
    a.part_ml = reinterpret_cast<float*>(static_cast<char*>(ws) +
                                         align256(attn_part_rows(desc) * desc->d * sizeof(float)));
  }
  const hipError_t e = launch_attn_fwd(a, desc->io_dtype == FLEX_BF16, desc->d, (hipStream_t)stream);
  return e == hipSuccess ? FLEX_OK : FLEX_ERR_HIP;
}

int32_t flex_attn_bwd(const flex_attn_desc* desc, const void* Q, const void* K, const void* V,
                      const int32_t* q_off, const int32_t* k_off, const void* O, const float* lse, const void* dO,
                      void* dQ, void* dK, void* dV, void* ws, size_t ws_bytes, void* stream) {
  const int32_t st = check_attn(desc);
  if (st != FLEX_OK) return st;
  if (!q_off || !k_off) return FLEX_ERR_INVALID_ARG;
  const void* qt[] = {Q, O, lse, dO, dQ};
  for (const void* p : qt)
    if (!tensor_ok(p, desc->Tq)) return FLEX_ERR_INVALID_ARG;
  const void* kt[] = {K, V, dK, dV};
  for (const void* p : kt)
    if (!tensor_ok(p, desc->Tk)) return FLEX_ERR_INVALID_ARG;
  const size_t need = attn_ws_bytes(desc, FLEX_PASS_BWD);
  if (need > 0 && (!ws || ws_bytes < need || !aligned16(ws))) return FLEX_ERR_WORKSPACE;
  if (desc->Tq == 0 && desc->Tk == 0) return FLEX_OK;
  AttnArgs a = attn_args(desc, Q, K, V, q_off, k_off);
  a.O = const_cast<void*>(O); a.lse = const_cast<float*>(lse); a.dO = dO;
  a.dQ = dQ; a.dK = dK; a.dV = dV;
  a.delta = static_cast<float*>(ws);
  const hipError_t e = launch_attn_bwd(a, desc->io_dtype == FLEX_BF16, desc->d, (hipStream_t)stream);
  return e == hipSuccess ? FLEX_OK : FLEX_ERR_HIP;
}

int32_t flex_delta_workspace_size(const flex_delta_desc* desc, int32_t pass, size_t* bytes) {
  if (!bytes) return FLEX_ERR_INVALID_ARG;
  *bytes = 0;
  if (pass != FLEX_PASS_FWD && pass != FLEX_PASS_BWD) return FLEX_ERR_INVALID_ARG;
  const int32_t st = check_delta(desc, false);
  if (st != FLEX_OK) return st;
  *bytes = delta_ws_bytes(desc, pass);
  return FLEX_OK;
}

int32_t flex_delta_saved_size(const flex_delta_desc* desc, size_t* bytes) {
  if (!bytes) return FLEX_ERR_INVALID_ARG;
  *bytes = 0;
  const int32_t st = check_delta(desc, false);
  if (st != FLEX_OK) return st;
  *bytes = delta_saved_bytes(desc);
  return FLEX_OK;
}

int32_t flex_delta_fwd(const flex_delta_desc* desc, const void* Q, const void* K, const void* V, const float* g,
                       const float* beta, const int32_t* off, const float* state0, void* O, float* state, void* saved,
                       size_t saved_bytes, void* ws, size_t ws_bytes, void* stream) {
  const int32_t st = check_delta(desc, false);
  if (st != FLEX_OK) return st;
  if (!off) return FLEX_ERR_INVALID_ARG;
  const void* rows[] = {Q, K, V, g, beta, O};
  for (const void* p : rows)
    if (!tensor_ok(p, desc->T)) return FLEX_ERR_INVALID_ARG;
  if ((state0 && !aligned16(state0)) || (state && !aligned16(state))) return FLEX_ERR_INVALID_ARG;
  if (saved ? saved_bytes < delta_saved_bytes(desc) || !aligned16(saved)
            : !ws || ws_bytes < delta_ws_bytes(desc, FLEX_PASS_FWD) || !aligned16(ws))
    return FLEX_ERR_WORKSPACE;
  DeltaArgs a = delta_args(desc, Q, K, V, g, beta, off);
  a.state0 = state0; a.state = state; a.O = O;
  if (saved)
    delta_saved(a, desc, saved);
  else
    a.prep = static_cast<char*>(ws);
  const hipError_t e = launch_delta_fwd(a, desc->io_dtype == FLEX_BF16, (hipStream_t)stream);
  return e == hipSuccess ? FLEX_OK : FLEX_ERR_HIP;
}

int32_t flex_delta_bwd(const flex_delta_desc* desc, const void* Q, const void* K, const void* V, const float* g,
                       const float* beta, const int32_t* off, const void* saved, size_t saved_bytes, const void* dO,
                       void* dQ, void* dK, void* dV, void* dg, void* dbeta, void* ws, size_t ws_bytes, void* stream) {
  const int32_t st = check_delta(desc, false);
  if (st != FLEX_OK) return st;
  if (!off) return FLEX_ERR_INVALID_ARG;
  const void* rows[] = {Q, K, V, g, beta, dO, dQ, dK, dV, dg, dbeta};
  for (const void* p : rows)
    if (!tensor_ok(p, desc->T)) return FLEX_ERR_INVALID_ARG;
  if (!saved || saved_bytes < delta_saved_bytes(desc) || !aligned16(saved)) return FLEX_ERR_WORKSPACE;
  if (!ws || ws_bytes < delta_ws_bytes(desc, FLEX_PASS_BWD) || !aligned16(ws)) return FLEX_ERR_WORKSPACE;
  if (desc->T == 0) return FLEX_OK;
  DeltaArgs a = delta_args(desc, Q, K, V, g, beta, off);
  delta_saved(a, desc, const_cast<void*>(saved));
  a.dO = dO; a.dQ = dQ; a.dK = dK; a.dV = dV; a.dg = dg; a.dbeta = dbeta;
  a.dst = ws;
  a.drt = static_cast<char*>(ws) + delta_blocks(desc) * delta_state_bytes(desc);
  const hipError_t e = launch_delta_bwd(a, desc->io_dtype == FLEX_BF16, (hipStream_t)stream);
  return e == hipSuccess ? FLEX_OK : FLEX_ERR_HIP;
}

int32_t flex_delta_step(const flex_delta_desc* desc, const void* q, const void* k, const void* v, const float* g,
                        const float* beta, float* state, void* o, void* stream) {
  const int32_t st = check_delta(desc, true);
  if (st != FLEX_OK) return st;
  const void* rows[] = {q, k, v, g, beta, state, o};
  for (const void* p : rows)
    if (!p || !aligned16(p)) return FLEX_ERR_INVALID_ARG;
  DeltaArgs a = delta_args(desc, q, k, v, g, beta, nullptr);
  a.state = state; a.O = o;
  const hipError_t e = launch_delta_step(a, desc->io_dtype == FLEX_BF16, (hipStream_t)stream);
  return e == hipSuccess ? FLEX_OK : FLEX_ERR_HIP;
}

}  // extern "C"
