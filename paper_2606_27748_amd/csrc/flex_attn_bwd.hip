// Exact causal attention over packed sequences, backward.  The probabilities are
// formed again from the logits and the forward's lse: dQ by query tiles, dK and dV by
// key tiles over all the query heads of their group, each sum in one workgroup's
// registers and a fixed order (no atomics: results are the same from run to run).  Sums under a causal mask that
// are not finite are formed again over what is seen (rare_add): a NaN in every row of dO makes 2 x 8192
// tokens, 16 heads of 128 on 4, 8.7 ms of 2.0, in one row at the end of the first sequence 5.3.
#include "flex_seq.hpp"
#include "flex_seq_kernels.hpp"
#include "../../include/flex.h"

#include <type_traits>

namespace flex {

namespace {
constexpr float LOG2E = 1.4426950408889634f;
constexpr int BM = 128;   // rows per workgroup, 32 per wave
constexpr int EXACT = 1024;   // keys of a query tile up to which delta is summed from dP
// Blocks of 32 keys whose products a wave of the dQ sweep forms together: more to work on while the
// exponentials of one are formed, and more registers.
constexpr int blocks_at_once(int d) { return d <= 64 ? 2 : 1; }
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
    // a query that sees no key: all its products are masked, exp2(-inf - 0) = 0
    a.delta[(size_t)head * a.Tq + q] = a.lse[row] == -INFINITY ? 0.f : a.lse[row] * LOG2E;
    a.delta[((size_t)a.Hq + head) * a.Tq + q] = sum;
  }
}

// dQ: the forward's tiles and orientation.  Per block of 32 keys S^T = K Q^T,
// dP^T = V dO^T, dS^T = P^T (dP^T - delta), dQ^T += K^T dS^T.
// Bound by the matrix cores (63 % busy): 756 us at 2 x 8192 tokens, 16 heads of 128 on 4 (1.09 PFLOP/s).
// delta = dO . O carries the rounding of O, which weighs in dQ and dK where a query sees few keys (its
// error against dS goes with 1 / sqrt of their number: gradients of sequences of some hundred
// rows are off by 3.2e-3 with it, against 2.4e-3 from the other roundings).  Query tiles that see
// at most EXACT keys sum delta = sum_j P_ij dP_ij in a pass of its own first, for the key sweep
// too; that is 1 % of the work of a sequence of 8192.  (Not with fp32 rows, whose O has no such rounding.)
template <class T, int D, int KT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(RowTile<T, D>::ROW > 256 ? 1 : 2))) void k_attn_dq(AttnArgs a) {
  using S = typename Io<T>::type;
  using RT = RowTile<T, D>;
  constexpr int KS = D / 16, NB = KT / 32, DT = D / 32, GB = blocks_at_once(D) < NB ? blocks_at_once(D) : NB;
  constexpr int TILE = KT * RT::ROW;
  __shared__ __attribute__((aligned(16))) char lds[4 * TILE];
  const int l = threadIdx.x % WAVE, c = l % 32, h = l / 32;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
  const TileCoord tc = tile_coord(seq_slots(a.Tq, a.B, BM), a.Hq, true);
  const SeqTile t = find_tile<BM>(a.q_off, a.B, a.Tq, tc.slot);
  if (t.b < 0) return;
  const SeqRange kr = seq_range(a.k_off, t.b, a.Tk);
  const int kvh = __builtin_amdgcn_readfirstlane(tc.head / (a.Hq / a.Hkv));   // in a scalar register, with the rows' addresses
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
  const float sl2 = a.scale * LOG2E;
  const S* K = static_cast<const S*>(a.K) + kvh * D;
  const S* V = static_cast<const S*>(a.V) + kvh * D;
  auto stage = [&](int i) {
    char* L = lds + (i & 1) * 2 * TILE;
    const int n = min(kr.n - i * KT, KT);
    stage_tile<T, D, KT, 4>(L, row_words(K, kr.row0 + i * KT, a.ks, n, D), a.ks * (int)sizeof(S), w);
    stage_tile<T, D, KT, 4>(L + TILE, row_words(V, kr.row0 + i * KT, a.vs, n, D), a.vs * (int)sizeof(S), w);
  };
  // S^T and dP^T of one block of 32 keys of tile i; a hidden key's probability is zero
  auto products = [&](f32x16& s, f32x16& p, int i, int b) {
    const char* LK = lds + (i & 1) * 2 * TILE;
    s = p = zero16();
#pragma unroll
    for (int k = 0; k < KS; ++k) mma32(s, RT::row(LK, 32 * b + c, k, h), q[k]);
#pragma unroll
    for (int k = 0; k < KS; ++k) mma32(p, RT::row(LK + TILE, 32 * b + c, k, h), g[k]);
  };
  auto mask = [&](f32x16& s, f32x16& p, int i, int b) {
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if (i * KT + 32 * b + res_row(e, h) >= lim) {
        s[e] = -INFINITY;
        p[e] = 0.f;
      }
  };
  if (IsBf16<T>::value && lim_wg <= EXACT) {
    if (ntiles > 0) stage(0);
    wait_reg_loads();
    float sum = 0.f;
    for (int i = 0; i < ntiles; ++i) {
      sync_tiles();
      if (i + 1 < ntiles) stage(i + 1);
      for (int b = 0; b < NB; ++b) {
        f32x16 s, p;
        products(s, p, i, b);
        mask(s, p, i, b);
#pragma unroll
        for (int e = 0; e < 16; ++e)
          sum = __builtin_fmaf(__builtin_amdgcn_exp2f(__builtin_fmaf(s[e], sl2, -lse2)), p[e], sum);
      }
    }
    delta = half_sum(sum);
    if (h == 0 && qi < t.n) a.delta[((size_t)a.Hq + tc.head) * a.Tq + t.row0 + qi] = delta;
    __syncthreads();
  }
  f32x16 dq[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i) dq[i] = zero16();
  if (ntiles > 0) stage(0);
  wait_reg_loads();
  for (int i = 0; i < ntiles; ++i) {
    sync_tiles();   // tile i has arrived; tile i - 1 is no longer read
    if (i + 1 < ntiles) stage(i + 1);
    const char* LK = lds + (i & 1) * 2 * TILE;
    if (i * KT >= lim_hi) continue;
#pragma unroll
    for (int b0 = 0; b0 < NB; b0 += GB) {
      f32x16 s[GB], p[GB];
#pragma unroll
      for (int b = 0; b < GB; ++b) products(s[b], p[b], i, b0 + b);
      if (i * KT + KT > lim_lo) {
#pragma unroll
        for (int b = 0; b < GB; ++b) mask(s[b], p[b], i, b0 + b);
      }
#pragma unroll
      for (int b = 0; b < GB; ++b)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
#pragma unroll
          for (int e = 8 * k; e < 8 * k + 8; ++e)
            s[b][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][e], sl2, -lse2)) * (p[b][e] - delta);
          const Frag<T> ds = frag_of<T>(s[b], k);
#pragma unroll
          for (int d = 0; d < DT; ++d) mma32(dq[d], RT::col(LK, 32 * (b0 + b) + 16 * k + 4 * h, 32 * d), ds);
        }
    }
  }
  if (a.causal && __any(qi < t.n && not_finite(dq))) {   // over what each query sees, again
    const S* Ks = K + (size_t)kr.row0 * a.ks;
    const S* Vs = V + (size_t)kr.row0 * a.vs;
    auto qs = [&](int i) { return q[i]; };
    auto gs = [&](int i) { return g[i]; };
#pragma unroll
    for (int d = 0; d < DT; ++d) dq[d] = zero16();
#pragma unroll 1
    for (int j0 = 0; j0 < lim_hi; j0 += 32) {
      if (j0 + 32 <= lim_lo) {
        const S* k = Ks + (size_t)j0 * a.ks;
        f32x16 s = rare_products<T, D>(k, a.ks, qs);
        const f32x16 p = rare_products<T, D>(Vs + (size_t)j0 * a.vs, a.vs, gs);
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], sl2, -lse2)) * (p[e] - delta);
        rare_add<T, D>(dq, k, a.ks, s);
        continue;
      }
      if (__all(qi >= t.n || none_finite(dq))) break;
#pragma unroll 1
      for (int j = j0; j < min(j0 + 32, lim_hi); ++j) {
        const S* k = Ks + (size_t)j * a.ks;
        const float s = rare_product<T, D>(k, qs), p = rare_product<T, D>(Vs + (size_t)j * a.vs, gs);
        rare_add<T, D>(dq, k, __builtin_amdgcn_exp2f(__builtin_fmaf(s, sl2, -lse2)) * (p - delta), j < lim);
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

// dK and dV: 128 keys of one key head per workgroup, 32 per wave; the queries of every head of
// the group pass by in tiles of QT rows, divided among WQ groups of four waves, whose shares of the
// sums are added up at the end.  S = Q K^T and dP = dO V^T come out with a lane per
// key and rows over queries, as dV^T += dO^T P and dK^T += Q^T dS take them.
// At d = 128 two wave groups halve the longest workgroup, that of the first keys under a causal mask (it
// meets all queries of all heads): at 2 x 8192 tokens, 4 key heads, d = 128 the grid is 520
// workgroups, all resident at once with one group, and waited for that one.  The rows of K and V
// are in registers, or with KL in LDS: at d = 128 a wave then fits half a SIMD's registers
// without spilling (a reload in the loop waits for the tile that is on its way, too).
// 1221 us there (900 TFLOP/s, matrix cores 50 % busy): the rows of K and V are read from LDS again for each
// product, and two waves per SIMD wait for a barrier every 64 rows.
template <class T, int D, int QT, int WQ, bool KL>
__global__ __launch_bounds__(256 * WQ) __attribute__((amdgpu_waves_per_eu(RowTile<T, D>::ROW > 256 ? 1 : 2))) void k_attn_dkv(
    AttnArgs a) {
  using S = typename Io<T>::type;
  using RT = RowTile<T, D>;
  constexpr int KS = D / 16, DT = D / 32, NW = 4 * WQ, WR = QT / WQ, NB = WR / 32;
  constexpr int TILE = QT * RT::ROW;
  constexpr int STAT = 64 * 4;
  constexpr int BUF = 2 * TILE + 2 * STAT;   // Q and dO, their lse and delta
  constexpr int JOIN = WQ > 1 ? BM * (D + 4) * 4 : 0;
  constexpr int LDS = 2 * BUF + (KL ? 2 * BM * RT::ROW : 0);
  __shared__ __attribute__((aligned(16))) char lds[LDS > JOIN ? LDS : JOIN];
  const char* LKeys = lds + 2 * BUF;
  const char* LVals = LKeys + BM * RT::ROW;
  const int l = threadIdx.x % WAVE, c = l % 32, h = l / 32;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE), wk = w % 4, wq = w / 4;
  const TileCoord tc = tile_coord(seq_slots(a.Tk, a.B, BM), a.Hkv, false);
  const SeqTile t = find_tile<BM>(a.k_off, a.B, a.Tk, tc.slot);
  if (t.b < 0) return;
  const SeqRange qr = seq_range(a.q_off, t.b, a.Tq);
  const int grp = a.Hq / a.Hkv, kvh = tc.head;
  const int rows = min(BM, t.n - t.tile * BM), first = t.tile * BM + 32 * wk, shift = t.n - qr.n;
  const int kj = first + c;
  // the first query that sees a key of the workgroup, and of the wave
  const int q_wg = a.causal ? max(t.tile * BM - shift, 0) : 0;
  const int q_w = a.causal ? first - shift : 0;
  // from the last query tile down, all heads of each: workgroups of different keys then read the same
  // rows at about the same time, through one L2
  const int last = (qr.n + QT - 1) / QT - 1, total = grp * max(last + 1 - q_wg / QT, 0);
  auto stage = [&](int i) {
    char* L = lds + (i & 1) * BUF;
    const int head = kvh * grp + i % grp, q0 = (last - i / grp) * QT, n = min(qr.n - q0, QT);
    stage_tile<T, D, QT, NW>(L, row_words(static_cast<const S*>(a.Q) + head * D, qr.row0 + q0, a.qs, n, D),
                             a.qs * (int)sizeof(S), w);
    stage_tile<T, D, QT, NW>(L + TILE, row_words(static_cast<const S*>(a.dO) + head * D, qr.row0 + q0, a.Hq * D, n, D),
                             a.Hq * D * (int)sizeof(S), w);
    if (w < 2)   // lse, delta
      stage_floats(L + 2 * TILE + w * STAT, row_words(a.delta + ((size_t)w * a.Hq + head) * a.Tq, qr.row0 + q0, 1, n, 1));
  };

  Frag<T> kf[KL ? 1 : KS], vf[KL ? 1 : KS];
  {
    const int r = 32 * wk + c;
    const size_t row0 = t.row0 + t.tile * BM;
    const S* K = static_cast<const S*>(a.K) + kvh * D;
    const S* V = static_cast<const S*>(a.V) + kvh * D;
    if constexpr (KL) {
      stage_tile<T, D, BM, NW>(LKeys, row_words(K, row0, a.ks, rows, D), a.ks * (int)sizeof(S), w);
      stage_tile<T, D, BM, NW>(LVals, row_words(V, row0, a.vs, rows, D), a.vs * (int)sizeof(S), w);
    } else {
      const auto rk = row_window(K, row0, a.ks, rows, D), rv = row_window(V, row0, a.vs, rows, D);
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        kf[s] = window_frag<T>(rk, (r * a.ks + 16 * s + 8 * h) * (int)sizeof(S));
        vf[s] = window_frag<T>(rv, (r * a.vs + 16 * s + 8 * h) * (int)sizeof(S));
      }
    }
  }
  f32x16 dk[DT], dv[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i) dk[i] = dv[i] = zero16();
  const float sl2 = a.scale * LOG2E;
  if (total > 0) stage(0);
  wait_reg_loads();
  for (int i = 0; i < total; ++i) {
    sync_tiles();   // tile i has arrived; tile i - 1 is no longer read
    if (i + 1 < total) stage(i + 1);
    const char* LQ = lds + (i & 1) * BUF;
    const char* LG = LQ + TILE;
    const float* Ls = reinterpret_cast<const float*>(LG + TILE) + WR * wq;
    const int q0 = (last - i / grp) * QT + WR * wq;   // this wave's rows
    if (q0 + WR <= q_w || q0 >= qr.n) continue;
    f32x16 s[NB], p[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int r = WR * wq + 32 * b + c;
      s[b] = p[b] = zero16();
#pragma unroll
      for (int k = 0; k < KS; ++k)
        mma32(s[b], RT::row(LQ, r, k, h), KL ? RT::row(LKeys, 32 * wk + c, k, h) : kf[KL ? 0 : k]);
#pragma unroll
      for (int k = 0; k < KS; ++k)
        mma32(p[b], RT::row(LG, r, k, h), KL ? RT::row(LVals, 32 * wk + c, k, h) : vf[KL ? 0 : k]);
    }
    if (a.causal && q0 < q_w + 31) {   // a hidden key's probability is zero
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (q0 + 32 * b + res_row(e, h) + shift < kj) {
            s[b][e] = -INFINITY;
            p[b][e] = 0.f;
          }
    }
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
#pragma unroll
        for (int x = 2 * k; x < 2 * k + 2; ++x) {   // rows 8x + 4h + y; those behind the sequence are zeros
          const f32x4 ls = *reinterpret_cast<const f32x4*>(Ls + 32 * b + 8 * x + 4 * h);
          const f32x4 de = *reinterpret_cast<const f32x4*>(Ls + 64 + 32 * b + 8 * x + 4 * h);
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            const int e = 4 * x + y;
            s[b][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][e], sl2, -ls[y]));
            p[b][e] = s[b][e] * (p[b][e] - de[y]);
          }
        }
        const Frag<T> pf = frag_of<T>(s[b], k), df = frag_of<T>(p[b], k);
        const int kb = WR * wq + 32 * b + 16 * k + 4 * h;
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          mma32(dv[d], RT::col(LG, kb, 32 * d), pf);
          mma32(dk[d], RT::col(LQ, kb, 32 * d), df);
        }
      }
  }
  if (a.causal && __any(kj < t.n && (not_finite(dk) || not_finite(dv)))) {   // over the queries that see each key, again
    auto ks = [&](int i) { return KL ? RT::row(LKeys, 32 * wk + RareLane().c, i, RareLane().h) : kf[KL ? 0 : i]; };
    auto vs = [&](int i) { return KL ? RT::row(LVals, 32 * wk + RareLane().c, i, RareLane().h) : vf[KL ? 0 : i]; };
    auto again = [&](f32x16 (&sum)[DT], auto is_dk) {   // one after the other: there are registers for one
#pragma unroll
      for (int d = 0; d < DT; ++d) sum[d] = zero16();
#pragma unroll 1
      for (int x = 0; x < total * NB; ++x) {   // head, tile, block of this wave's rows in it, the diagonal last
        const int head = kvh * grp + x % grp, y = x / grp, q0 = (last - y / NB) * QT + WR * wq + 32 * (NB - 1 - y % NB);
        if (q0 + 32 <= q_w || q0 >= qr.n) continue;
        const size_t at = (size_t)(qr.row0 + q0);
        const S* Q = static_cast<const S*>(a.Q) + head * D + at * a.qs;
        const S* G = static_cast<const S*>(a.dO) + (at * a.Hq + head) * D;
        const float* ls = a.delta + (size_t)head * a.Tq + at;
        const float* de = ls + (size_t)a.Hq * a.Tq;
        if (q0 >= q_w + 31 && q0 + 32 <= qr.n) {
          f32x16 s = rare_products<T, D>(Q, a.qs, ks);
          const int h = RareLane().h;
#pragma unroll
          for (int e = 0; e < 16; ++e) s[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], sl2, -ls[res_row(e, h)]));
          if (is_dk.value) {
            const f32x16 p = rare_products<T, D>(G, a.Hq * D, vs);
#pragma unroll
            for (int e = 0; e < 16; ++e) s[e] *= p[e] - de[res_row(e, h)];
          }
          rare_add<T, D>(sum, is_dk.value ? Q : G, is_dk.value ? a.qs : a.Hq * D, s);
          continue;
        }
        if (__all(kj >= t.n || none_finite(sum))) continue;
#pragma unroll 1
        for (int i = 0; i < min(32, qr.n - q0); ++i) {
          const S* qrow = Q + (size_t)i * a.qs;
          const S* grow = G + (size_t)i * a.Hq * D;
          float s = __builtin_amdgcn_exp2f(__builtin_fmaf(rare_product<T, D>(qrow, ks), sl2, -ls[i]));
          if (is_dk.value) s *= rare_product<T, D>(grow, vs) - de[i];
          rare_add<T, D>(sum, is_dk.value ? qrow : grow, s, kj <= q0 + i + shift);
        }
      }
    };
    again(dv, std::false_type{});
    again(dk, std::true_type{});
  }
  if (WQ > 1) {   // the second group's sums to the first, through LDS, dK and then dV
    float* J = reinterpret_cast<float*>(lds) + (32 * wk + c) * (D + 4);
    auto join = [&](f32x16 (&x)[DT]) {
      __syncthreads();
      if (wq == 1) {
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int e = 0; e < 16; e += 4)
            *reinterpret_cast<f32x4*>(J + 32 * d + res_row(e, h)) = f32x4{x[d][e], x[d][e + 1], x[d][e + 2], x[d][e + 3]};
      }
      __syncthreads();
      if (wq == 0) {
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int e = 0; e < 16; e += 4) {
            const f32x4 v = *reinterpret_cast<const f32x4*>(J + 32 * d + res_row(e, h));
#pragma unroll
            for (int y = 0; y < 4; ++y) x[d][e + y] += v[y];
          }
      }
    };
    join(dk);
    join(dv);
    if (wq != 0) return;
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
  if (a.Tq > 0) k_attn_dq<T, D, R><<<seq_slots(a.Tq, a.B, BM) * a.Hq, 256, 0, st>>>(a);
  constexpr bool KL = IsBf16<T>::value && D == 128;
  // us at 8279 packed tokens, 12 heads of 64: one group 84, two 105; at 16384 tokens, 16 heads of 128 on 4:
  // one 1565 (one wave per SIMD), two 1258
  if (a.Tk > 0) k_attn_dkv<T, D, R, KL ? 2 : 1, KL><<<seq_slots(a.Tk, a.B, BM) * a.Hkv, KL ? 512 : 256, 0, st>>>(a);
  timing_mark(FLEX_KERNEL_ATTN_BWD, st, false);
  return hipGetLastError();
}
}  // namespace

hipError_t launch_attn_bwd(const AttnArgs& a, bool bf16, int d, hipStream_t st) {
  if (bf16) return d == 32 ? run_bwd<__bf16, 32>(a, st) : d == 64 ? run_bwd<__bf16, 64>(a, st) : run_bwd<__bf16, 128>(a, st);
  return d == 32 ? run_bwd<float, 32>(a, st) : d == 64 ? run_bwd<float, 64>(a, st) : run_bwd<float, 128>(a, st);
}

}  // namespace flex
