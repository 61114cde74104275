// Exact causal attention over packed sequences, backward.  The probabilities are
// formed again from the logits and the forward's lse: dQ by query tiles, dK and dV by
// key tiles over all the query heads of their group, each sum in one workgroup's
// registers and a fixed order (no atomics: results are the same from run to run).
#include "flex_seq.hpp"
#include "flex_seq_kernels.hpp"
#include "../../include/flex.h"

namespace flex {

namespace {
constexpr float LOG2E = 1.4426950408889634f;
constexpr int BM = 128;   // rows per workgroup, 32 per wave
}  // namespace

// Per row and head, transposed to [Hq][Tq] so that the sweeps read the statistics
// of consecutive rows at once: lse in units of log2, and delta = dO . O.
template <class T, int D>
__global__ __launch_bounds__(256) void k_attn_delta(AttnArgs a) {
  using S = typename Io<T>::type;
  constexpr int L = D / 8;
  const size_t row = (size_t)blockIdx.x * (256 / L) + threadIdx.x / L;
  const int e = threadIdx.x % L * 8;
  const int q = (int)(row / a.Hq), head = (int)(row % a.Hq);
  const bool in = q < a.Tq;
  const size_t at = (in ? row : 0) * D + e;
  Frag<T> o, g;
  load8(o, static_cast<const S*>(a.O) + at, in);
  load8(g, static_cast<const S*>(a.dO) + at, in);
  float sum = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) sum = __builtin_fmaf(o.get(j), g.get(j), sum);
  sum = lane_sum<L>(sum);
  if (in && e == 0) {
    a.delta[(size_t)head * a.Tq + q] = a.lse[row] * LOG2E;
    a.delta[((size_t)a.Hq + head) * a.Tq + q] = sum;
  }
}

// dQ: the forward's tiles and orientation.  Per block of 32 keys S^T = K Q^T,
// dP^T = V dO^T, dS^T = P^T (dP^T - delta), dQ^T += K^T dS^T.
template <class T, int D, int KT>
__global__ __launch_bounds__(256) void k_attn_dq(AttnArgs a) {
  using S = typename Io<T>::type;
  using RT = RowTile<T, D>;
  constexpr int KS = D / 16, NB = KT / 32, DT = D / 32;
  constexpr int TILE = KT * RT::ROW;
  __shared__ __attribute__((aligned(16))) char lds[4 * TILE];
  const int l = threadIdx.x % WAVE, c = l % 32, h = l / 32;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
  const TileCoord tc = tile_coord(seq_slots(a.Tq, a.B, BM), a.Hq, true);
  const SeqTile t = find_tile<BM>(a.q_off, a.B, a.Tq, tc.slot);
  if (t.b < 0) return;
  const SeqRange kr = seq_range(a.k_off, t.b, a.Tk);
  const int kvh = tc.head / (a.Hq / a.Hkv);
  const int rows = min(BM, t.n - t.tile * BM), first = t.tile * BM + 32 * w, shift = kr.n - t.n;
  const int qi = first + c;
  const int lim = a.causal ? min(kr.n, qi + shift + 1) : kr.n;
  const int lim_lo = a.causal ? min(kr.n, first + shift + 1) : kr.n;
  const int lim_hi = a.causal ? min(kr.n, first + 32 + shift) : kr.n;
  const int lim_wg = a.causal ? min(kr.n, t.tile * BM + rows + shift) : kr.n;
  const int ntiles = max(lim_wg + KT - 1, 0) / KT;

  Frag<T> q[KS], g[KS];
  float lse2, delta;
  {
    const int r = 32 * w + c;
    const size_t row0 = t.row0 + t.tile * BM;
    const auto rq = row_window(static_cast<const S*>(a.Q) + tc.head * D, row0, a.qs, rows, D);
    const auto rg = row_window(static_cast<const S*>(a.dO) + tc.head * D, row0, a.Hq * D, rows, D);
    const auto rl = row_window(a.delta + (size_t)tc.head * a.Tq, row0, 1, rows, 1);
    const auto rd = row_window(a.delta + ((size_t)a.Hq + tc.head) * a.Tq, row0, 1, rows, 1);
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      q[s] = window_frag<T>(rq, (r * a.qs + 16 * s + 8 * h) * (int)sizeof(S));
      g[s] = window_frag<T>(rg, (r * a.Hq * D + 16 * s + 8 * h) * (int)sizeof(S));
    }
    lse2 = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rl, r * 4, 0, 0));
    delta = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rd, r * 4, 0, 0));
  }
  f32x16 dq[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i) dq[i] = zero16();
  const float sl2 = a.scale * LOG2E;
  const S* K = static_cast<const S*>(a.K) + kvh * D;
  const S* V = static_cast<const S*>(a.V) + kvh * D;
  auto stage = [&](int i) {
    char* L = lds + (i & 1) * 2 * TILE;
    const int n = min(kr.n - i * KT, KT);
    stage_tile<T, D, KT, 4>(L, row_words(K, kr.row0 + i * KT, a.ks, n, D), a.ks * (int)sizeof(S), w);
    stage_tile<T, D, KT, 4>(L + TILE, row_words(V, kr.row0 + i * KT, a.vs, n, D), a.vs * (int)sizeof(S), w);
  };
  if (ntiles > 0) stage(0);
  wait_reg_loads();
  for (int i = 0; i < ntiles; ++i) {
    sync_tiles();   // tile i has arrived; tile i - 1 is no longer read
    if (i + 1 < ntiles) stage(i + 1);
    const char* LK = lds + (i & 1) * 2 * TILE;
    const char* LV = LK + TILE;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int j0 = i * KT + 32 * b;
      if (j0 >= lim_hi) continue;
      f32x16 s = zero16(), p = zero16();
#pragma unroll
      for (int k = 0; k < KS; ++k) mma32(s, RT::row(LK, 32 * b + c, k, h), q[k]);
#pragma unroll
      for (int k = 0; k < KS; ++k) mma32(p, RT::row(LV, 32 * b + c, k, h), g[k]);
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], sl2, -lse2)) * (p[e] - delta);
      if (j0 + 32 > lim_lo) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (j0 + res_row(e, h) >= lim) s[e] = 0.f;
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const Frag<T> ds = frag_of<T>(s, k);
#pragma unroll
        for (int d = 0; d < DT; ++d) mma32(dq[d], RT::col(LK, 32 * b + 16 * k + 4 * h, 32 * d), ds);
      }
    }
  }
  if (qi >= t.n) return;
  S* out = static_cast<S*>(a.dQ) + ((size_t)(t.row0 + qi) * a.Hq + tc.head) * D;
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int e = 0; e < 16; e += 4)
      store_io4(out + 32 * d + res_row(e, h), f32x4{dq[d][e], dq[d][e + 1], dq[d][e + 2], dq[d][e + 3]} * a.scale);
}

// dK and dV: 128 keys of one key head per workgroup, 32 per wave, their rows of K and
// V in registers; the queries of every head of the group pass by in tiles of QT
// rows.  S = Q K^T and dP = dO V^T come out with a lane per key and rows over queries,
// as dV^T += dO^T P and dK^T += Q^T dS take them.
template <class T, int D, int QT>
__global__ __launch_bounds__(256) void k_attn_dkv(AttnArgs a) {
  using S = typename Io<T>::type;
  using RT = RowTile<T, D>;
  constexpr int KS = D / 16, NB = QT / 32, DT = D / 32;
  constexpr int TILE = QT * RT::ROW;
  __shared__ __attribute__((aligned(16))) char lds[4 * TILE];
  const int l = threadIdx.x % WAVE, c = l % 32, h = l / 32;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
  const TileCoord tc = tile_coord(seq_slots(a.Tk, a.B, BM), a.Hkv, false);
  const SeqTile t = find_tile<BM>(a.k_off, a.B, a.Tk, tc.slot);
  if (t.b < 0) return;
  const SeqRange qr = seq_range(a.q_off, t.b, a.Tq);
  const int grp = a.Hq / a.Hkv, kvh = tc.head;
  const int rows = min(BM, t.n - t.tile * BM), first = t.tile * BM + 32 * w, shift = t.n - qr.n;
  const int kj = first + c;
  // the first query that sees a key of the workgroup, and of the wave
  const int q_wg = a.causal ? max(t.tile * BM - shift, 0) : 0;
  const int q_w = a.causal ? first - shift : 0;
  const int tile0 = q_wg / QT, ntiles = max((qr.n + QT - 1) / QT - tile0, 0);

  Frag<T> kf[KS], vf[KS];
  {
    const int r = 32 * w + c;
    const size_t row0 = t.row0 + t.tile * BM;
    const auto rk = row_window(static_cast<const S*>(a.K) + kvh * D, row0, a.ks, rows, D);
    const auto rv = row_window(static_cast<const S*>(a.V) + kvh * D, row0, a.vs, rows, D);
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      kf[s] = window_frag<T>(rk, (r * a.ks + 16 * s + 8 * h) * (int)sizeof(S));
      vf[s] = window_frag<T>(rv, (r * a.vs + 16 * s + 8 * h) * (int)sizeof(S));
    }
  }
  f32x16 dk[DT], dv[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i) dk[i] = dv[i] = zero16();
  const float sl2 = a.scale * LOG2E;
  const int total = grp * ntiles;
  auto stage = [&](int i) {
    char* L = lds + (i & 1) * 2 * TILE;
    const int head = kvh * grp + i / ntiles, q0 = (tile0 + i % ntiles) * QT, n = min(qr.n - q0, QT);
    stage_tile<T, D, QT, 4>(L, row_words(static_cast<const S*>(a.Q) + head * D, qr.row0 + q0, a.qs, n, D),
                            a.qs * (int)sizeof(S), w);
    stage_tile<T, D, QT, 4>(L + TILE, row_words(static_cast<const S*>(a.dO) + head * D, qr.row0 + q0, a.Hq * D, n, D),
                            a.Hq * D * (int)sizeof(S), w);
  };
  if (total > 0) stage(0);
  wait_reg_loads();
  for (int i = 0; i < total; ++i) {
    sync_tiles();   // tile i has arrived; tile i - 1 is no longer read
    if (i + 1 < total) stage(i + 1);
    const char* LQ = lds + (i & 1) * 2 * TILE;
    const char* LG = LQ + TILE;
    const int head = kvh * grp + i / ntiles, q0 = (tile0 + i % ntiles) * QT, n = min(qr.n - q0, QT);
    const auto rl = row_window(a.delta + (size_t)head * a.Tq, qr.row0 + q0, 1, n, 1);
    const auto rd = row_window(a.delta + ((size_t)a.Hq + head) * a.Tq, qr.row0 + q0, 1, n, 1);
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int i0 = q0 + 32 * b;
      if (i0 + 31 < q_w || i0 >= qr.n) continue;
      f32x4 ls[4], de[4];   // rows 8a + 4h + i
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int off = (32 * b + 8 * x + 4 * h) * 4;
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          ls[x][y] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rl, off + 4 * y, 0, 0));
          de[x][y] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rd, off + 4 * y, 0, 0));
        }
      }
      f32x16 s = zero16(), p = zero16();
#pragma unroll
      for (int k = 0; k < KS; ++k) mma32(s, RT::row(LQ, 32 * b + c, k, h), kf[k]);
#pragma unroll
      for (int k = 0; k < KS; ++k) mma32(p, RT::row(LG, 32 * b + c, k, h), vf[k]);
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        s[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], sl2, -ls[e / 4][e % 4]));
        p[e] = s[e] * (p[e] - de[e / 4][e % 4]);
      }
      if (a.causal && i0 < q_w + 31) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (i0 + res_row(e, h) + shift < kj) s[e] = p[e] = 0.f;
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const Frag<T> pf = frag_of<T>(s, k), df = frag_of<T>(p, k);
        const int kb = 32 * b + 16 * k + 4 * h;
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          mma32(dv[d], RT::col(LG, kb, 32 * d), pf);
          mma32(dk[d], RT::col(LQ, kb, 32 * d), df);
        }
      }
    }
  }
  if (kj >= t.n) return;
  const size_t at = ((size_t)(t.row0 + kj) * a.Hkv + kvh) * D;
  S* ok = static_cast<S*>(a.dK) + at;
  S* ov = static_cast<S*>(a.dV) + at;
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
      const int x = 32 * d + res_row(e, h);
      store_io4(ok + x, f32x4{dk[d][e], dk[d][e + 1], dk[d][e + 2], dk[d][e + 3]} * a.scale);
      store_io4(ov + x, f32x4{dv[d][e], dv[d][e + 1], dv[d][e + 2], dv[d][e + 3]});
    }
}

namespace {
template <class T, int D>
hipError_t run_bwd(const AttnArgs& a, hipStream_t st) {
  constexpr int R = sizeof(T) == 4 && D == 128 ? 32 : 64;   // rows of a staged tile: 64 KB of LDS at most
  timing_mark(FLEX_KERNEL_ATTN_BWD, st, true);
  if (a.Tq > 0) {
    const size_t rows = (size_t)a.Tq * a.Hq, per = 256 / (D / 8);
    k_attn_delta<T, D><<<(unsigned)((rows + per - 1) / per), 256, 0, st>>>(a);
  }
  if (a.Tk > 0) k_attn_dkv<T, D, R><<<seq_slots(a.Tk, a.B, BM) * a.Hkv, 256, 0, st>>>(a);
  if (a.Tq > 0) k_attn_dq<T, D, R><<<seq_slots(a.Tq, a.B, BM) * a.Hq, 256, 0, st>>>(a);
  timing_mark(FLEX_KERNEL_ATTN_BWD, st, false);
  return hipGetLastError();
}
}  // namespace

hipError_t launch_attn_bwd(const AttnArgs& a, bool bf16, int d, hipStream_t st) {
  if (bf16) return d == 32 ? run_bwd<__bf16, 32>(a, st) : d == 64 ? run_bwd<__bf16, 64>(a, st) : run_bwd<__bf16, 128>(a, st);
  return d == 32 ? run_bwd<float, 32>(a, st) : d == 64 ? run_bwd<float, 64>(a, st) : run_bwd<float, 128>(a, st);
}

}  // namespace flex
