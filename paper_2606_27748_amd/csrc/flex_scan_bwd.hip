// Selective scan, backward.  With dS the gradient of the state at a chunk's end, E_ij = e^{L_i - L_j} (j <= i) and
// v_j = e^{L_63 - L_j}:
//   M_ij = E_ij dy_i.x_j      W_ij = sum over a group's heads of M_ij dt_j
//   dC_i = sum_j W_ij B_j + sum_heads e^{L_i} S dy_i
//   dB_j = sum_i W_ij C_i + sum_heads dt_j v_j dS x_j
//   dxt_j = sum_i E_ij (C_i.B_j) dy_i + v_j dS^T B_j,   dx_j = dt_j dxt_j + D dy_j,   ddt_j = dxt_j.x_j,   dD = sum_t dy_t.x_t
//   dS <- e^{L_63} dS + sum_i e^{L_i} C_i dy_i^T                       (the chunk's start)
//   dg_t = sum_{i>=t} (R_i + sum_{j<i} Z_ij - sum_{j>i} Z_ji) + sum_{i<t} V_i + e^{L_63} <S, dS>
//          with Z_ij = M_ij (C_i.B_j) dt_j, R_i = e^{L_i} C_i.S dy_i, V_j = dt_j x_j.(v_j dS^T B_j)
// dg_t is what crosses t: what is read from t on of what was written before it.  Z enters as a row sum and as a
// column sum of the same fp32 numbers, so pairs on one side of t cancel to what fp32 sums of them leave; its
// diagonal crosses nothing and is left out.
// S of each chunk is the forward's, dS comes from a sweep in reverse; the rest is independent per chunk
// (k_scan_grad).
#include "flex_scan.hpp"
#include "../../include/flex.h"

namespace flex {

void launch_scan_states(const ScanArgs& a, bool bf16, hipStream_t st);

// One workgroup per chunk, group and part of its heads, over them in order and over their columns in blocks of 64; the
// next block's x, dy, S and dS on their way to LDS while one is worked on, where two fit.  Of eight waves each has
// the rows of dB and dC of 32 tokens and 32 elements n (N = 64: the upper four); the lower four form dx of 32
// tokens and columns each, three of the others the tiles of M and the sums of Z; the last one forms the
// decays of the next head and puts out dg and ddt of the one before.  A lane is a token j throughout (of M too).
// Bound by memory and by the waves in turn: with two waves a SIMD (registers and LDS hold no more) only the next block is on its
// way while one is worked on.  16384 tokens, 64 heads of 64, N = 128, bf16: 275 us (0.95 GB, S and dS more than
// half of it), where the reads alone take 196 and the work on blocks that are at hand 234.
// Fp32 rows have one block at a time, and with N = 128 S and dS one after the other, read once more for <S, dS>: 340 us over as many tokens,
// 16 heads of 64, matrix cores busy 38 % of the time.
template <class T, int N>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(1, 2))) void k_scan_grad(ScanArgs a) {
  using S = typename Io<T>::type;
  using RT = ScanTile<T, N>;
  using XT = ScanTile<T, 64>;
  using ST = StateRows<T, N>;
  constexpr bool BF = IsBf16<T>::value;
  constexpr int ROWS = SC * N * (int)sizeof(T), XROWS = SC * 64 * (int)sizeof(T);
  // fp32 states of 128 rows leave room for one of S and dS at a time
  constexpr bool ONE = 4 * ROWS + 2 * XROWS > 144 * 1024;
  constexpr int BLOCK = 2 * XROWS + (ONE ? 1 : 2) * ROWS, BUFS = 2 * ROWS + 2 * BLOCK <= 144 * 1024 ? 2 : 1;
  __shared__ __attribute__((aligned(16))) char lds[2 * ROWS + BUFS * BLOCK];
  // of a head, two in turn: decays as factors from a half's middle (or L, hi and lo), dt, e^L, v; whether they are
  // factors, that from one middle to the other, the whole decay, D
  __shared__ __attribute__((aligned(16))) float scal[2][6 * SC + 4];
  // what the waves leave for dg and ddt
  struct Dots {
    float r[4][SC], v[2][SC], i[2][SC], col[2][SC], row[2][2][SC], d[4], s[8];
  };
  __shared__ Dots dots[2];
  char* LB = lds;
  char* LC = lds + ROWS;

  const int l = threadIdx.x % WAVE, c = l % 32, h = l / 32;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE), tj = w % 2;
  const int n0 = N == 128 ? 32 * (w / 2) : 32 * (w / 2 - 2);   // the wave's rows of dB and dC
  const bool has_n = N == 128 || w >= 4;
  const int ti = w == 4 ? 0 : 1;                                // the tile of i of waves 4, 5 and 6
  // the tokens that waves 0 to 3 form dx of: those of two tiles of i are not on the SIMDs of M's tiles on the diagonal
  const int tx = w < 2 ? 1 : 0;
  const int id = blockIdx.x, sets = a.G * a.parts, k = id / NUM_XCD;
  const int slot = k / sets * NUM_XCD + id % NUM_XCD, grp = k % sets / a.parts, part = k % sets % a.parts;
  const int slots = seq_slots(a.T, a.B, SC);
  if (slot >= slots) return;
  const int hpg = a.H / a.G, hpp = hpg / a.parts, head0 = grp * hpg + part * hpp;
  const SeqTile t = find_tile<SC>(a.off, a.B, a.T, slot);
  if (t.b < 0) {
    for (int i = threadIdx.x; i < hpp; i += 512) a.part_d[(size_t)slot * a.H + head0 + i] = 0.f;
    return;
  }
  const int n = min(SC, t.n - t.tile * SC), row0 = t.row0 + t.tile * SC;
  const int tok = 32 * tj + c;   // this lane's token
  const int nb = a.P / 64, items = hpp * nb;
  // the lane, for places that are formed anew: kept over the loop they would take the registers that it is short of
  auto again = [&]() {
    int x = l;
    asm volatile("" : "+v"(x));
    return x;
  };
  auto block = [&](int it) { return lds + 2 * ROWS + (BUFS == 2 ? (it & 1) * BLOCK : 0); };
  auto state_at = [&](int it) { return (((size_t)slot * a.H + head0 + it / nb) * a.P + it % nb * 64) * N; };
  auto stage = [&](int it) {
    const size_t xcol = (size_t)(head0 + it / nb) * a.P + it % nb * 64;
    const char* L = block(it);
    if (w < 4)
      stage_rows<T, 64>(L, static_cast<const S*>(a.X) + xcol, row0, a.xs, n, w, 4);
    else
      stage_rows<T, 64>(L + XROWS, static_cast<const S*>(a.dY) + xcol, row0, a.H * a.P, n, w - 4, 4);
    stage_linear<ROWS / 1024, 8>(L + 2 * XROWS, static_cast<const S*>(a.st) + state_at(it), w);
    if (!ONE) stage_linear<ROWS / 1024, 8>(L + 2 * XROWS + ROWS, static_cast<const S*>(a.dst) + state_at(it), w);
  };
  float gn = 0.f, dn = 0.f, Dn = 0.f;   // of the next head, lane = token
  auto fetch = [&](int hd) {
    const int l = again();
    if (a.D) Dn = a.D[head0 + hd];
    if (l < n) {
      const size_t at = (size_t)(row0 + l) * a.H + head0 + hd;
      gn = a.g[at];
      dn = a.dt[at];
    }
  };
  auto decays = [&](int hd) {
    const int l = again();
    float* sc = scal[hd & 1];
    const Decay d(gn);
    const double m0 = lane_of(d.L, 15), m1 = lane_of(d.L, 47);
    const float from = (float)(d.L - (l < 32 ? m0 : m1));
    const bool product = BF && __all(fabsf(from) < 50.f);
    sc[l] = product ? __builtin_amdgcn_exp2f(from) : d.hi;
    sc[SC + l] = product ? __builtin_amdgcn_exp2f(-from) : d.lo;
    sc[2 * SC + l] = dn;
    sc[3 * SC + l] = d.from_start();
    sc[4 * SC + l] = d.to_end();
    sc[5 * SC + l] = gn < SCAN_MIN_G ? 0.f : 1.f;   // a decay of zero has no slope
    if (l == 0) {
      sc[6 * SC] = product ? 1.f : 0.f;
      sc[6 * SC + 1] = __builtin_amdgcn_exp2f((float)(m1 - m0));
      sc[6 * SC + 2] = __builtin_amdgcn_exp2f((float)d.end);
      sc[6 * SC + 3] = Dn;
    }
  };
  // dg, ddt and the chunk's part of dD of a head, by one wave; lane = token
  auto put_out = [&](int hd) {
    const int l = again();
    const float* sc = scal[hd & 1];
    const Dots& o = dots[hd & 1];
    const size_t at = (size_t)(row0 + l) * a.H + head0 + hd;
    // rows of tile 0 have the tile of j 0 alone
    const float rz = (o.row[0][0][l] + o.row[0][1][l]) + (l >= 32 ? o.row[1][0][l] + o.row[1][1][l] : 0.f);
    const float cz = l < 32 ? o.col[0][l] + o.col[1][l] : o.col[1][l];
    float x = (N == 128 ? (o.r[0][l] + o.r[1][l]) + (o.r[2][l] + o.r[3][l]) : o.r[0][l] + o.r[1][l]) * sc[3 * SC + l] + rz - cz;
    const float v = o.v[0][l] + o.v[1][l];
    if (l == SC - 1) x += sc[6 * SC + 2] * (((o.s[0] + o.s[1]) + (o.s[2] + o.s[3])) + ((o.s[4] + o.s[5]) + (o.s[6] + o.s[7])));
    // sums over i >= l, and over i < l: what is left of a whole in 64 bits
    const float z = v * sc[2 * SC + l];
    const double xs = wave_scan((double)x), zs = wave_scan((double)z);
    const float slope = (float)((lane_of(xs, WAVE - 1) - xs + (double)x) + (zs - (double)z));
    if (l < n) {
      // in the io type like every gradient of this operator, though dt and g are fp32
      static_cast<S*>(a.dg)[at] = float_to_io<S>(sc[5 * SC + l] != 0.f ? slope : 0.f);
      static_cast<S*>(a.ddt)[at] = float_to_io<S>((o.i[0][l] + o.i[1][l]) + v);
    }
    if (l == 0) a.part_d[(size_t)slot * a.H + head0 + hd] = (o.d[0] + o.d[1]) + (o.d[2] + o.d[3]);
  };

  stage_rows<T, N>(w < 4 ? LB : LC, (w < 4 ? static_cast<const S*>(a.Bt) : static_cast<const S*>(a.Ct)) + (size_t)grp * N, row0,
                   w < 4 ? a.bs : a.cs, n, w % 4, 4);
  if (w == 7) {
    fetch(0);
    decays(0);
    if (hpp > 1) fetch(1);
  }
  // ka, kb: of the lower waves C_i.B_j of the tiles 0 and 1 of i, of the upper ones that of the tile ti, and dy_i.x_j of it
  f32x16 dB = zero16(), dC = zero16(), W = zero16(), ka = zero16(), kb = zero16();
  stage(0);
  sync_tiles();
  auto products = [&](f32x16& to, int i, int j) {
#pragma unroll
    for (int s = 0; s < N / 16; ++s) mma32(to, RT::row(LC, 32 * i + c, s, h), RT::row(LB, 32 * j + c, s, h));
  };
  if (w >= 4) {
    products(ka, ti, tj);
  } else {
    if (tx == 0) products(ka, 0, tx);
    products(kb, 1, tx);
  }
  float di = 0.f, dv = 0.f, dd = 0.f, dr = 0.f, ss = 0.f;
  for (int it = 0; it < items; ++it) {
    const int hd = it / nb, head = head0 + hd, pb = it % nb;
    if (BUFS == 1 && it > 0) {
      sync_lds();   // what was staged before is no longer read
      stage(it);
    }
    // the block is in LDS; the stores of dx, behind its loads, may be on their way
    if (BUFS == 2 && w < 4)
      sync_tiles_but<BF ? 2 : 4>();
    else
      sync_tiles();
    if (BUFS == 2 && it + 1 < items) stage(it + 1);
    // fp32 rows of N = 128 have no registers for places that are kept over the loop
    const int x = BF ? l : again(), c = x % 32, h = x / 32, tok = 32 * tj + c;
    const char* LX = block(it);
    const char* LY = LX + XROWS;
    const char* LS = LY + XROWS;
    const char* LD = ONE ? LS : LS + ROWS;
    const float* sc = scal[hd & 1];
    Dots& left = dots[hd & 1];
    if (w == 7 && pb == 0) {
      if (hd > 0) put_out(hd - 1);
      if (hd + 1 < hpp) {   // its place was the head's before, which is put out
        decays(hd + 1);
        if (hd + 2 < hpp) fetch(hd + 2);
      }
    }
    if (pb == 0) {
      if (w >= 4) kb = zero16();
      di = dv = dd = dr = ss = 0.f;
    }
    if (has_n) {   // e^L S dy
      f32x16 u = zero16();
#pragma unroll
      for (int s = 0; s < 4; ++s) mma32(u, ST::steps(LS, s, n0, x), XT::row(LY, tok, s, h));
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const Frag<T> cr = RT::row(LC, tok, n0 / 16 + s, h);
#pragma unroll
        for (int j = 0; j < 8; ++j) dr = __builtin_fmaf(cr.get(j), u[8 * s + j], dr);
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) dC[e] = __builtin_fmaf(u[e], sc[3 * SC + tok], dC[e]);
    }
    if (ONE) {
      sync_lds();
      stage_linear<ROWS / 1024, 8>(LD, static_cast<const S*>(a.dst) + state_at(it), w);
      const float* s0 = reinterpret_cast<const float*>(static_cast<const S*>(a.st) + state_at(it));
      const float* d0 = reinterpret_cast<const float*>(static_cast<const S*>(a.dst) + state_at(it));
      for (int i = threadIdx.x; i < 64 * N; i += 512) ss = __builtin_fmaf(s0[i], d0[i], ss);
      sync_tiles();
    } else {
      for (int i = w * WAVE + x; i < ROWS / 16; i += 512) {   // <S, dS>: the same place in both
        if constexpr (BF) {
          const bf16x8 u = *reinterpret_cast<const bf16x8*>(LS + 16 * i), v = *reinterpret_cast<const bf16x8*>(LD + 16 * i);
#pragma unroll
          for (int j = 0; j < 8; j += 2)
            ss = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{u[j], u[j + 1]}, bf16x2{v[j], v[j + 1]}, ss, false);
        } else {
          const f32x4 u = *reinterpret_cast<const f32x4*>(LS + 16 * i), v = *reinterpret_cast<const f32x4*>(LD + 16 * i);
#pragma unroll
          for (int j = 0; j < 4; ++j) ss = __builtin_fmaf(u[j], v[j], ss);
        }
      }
    }
    if (has_n) {   // dt v dS x
      f32x16 u = zero16();
#pragma unroll
      for (int s = 0; s < 4; ++s) mma32(u, ST::steps(LD, s, n0, x), XT::row(LX, tok, s, h));
      const float dtv = sc[2 * SC + tok] * sc[4 * SC + tok];
#pragma unroll
      for (int e = 0; e < 16; ++e) dB[e] = __builtin_fmaf(u[e], dtv, dB[e]);
    }
    // use(q, f) with the decays f = e^{L_i - L_j} of the elements 4 q .. of a tile of i, from the token j = at, times by
    const bool product = sc[6 * SC] != 0.f;
    auto decays_to = [&](int tile, int at, bool next, float by, auto use) {
      const float* si = sc + 32 * tile + 4 * h;
      if (product) {
        const float bj = sc[SC + at] * by * (next ? sc[6 * SC + 1] : 1.f);
#pragma unroll
        for (int q = 0; q < 4; ++q) use(q, *reinterpret_cast<const f32x4*>(si + 8 * q) * bj);
      } else {
        const float hj = sc[at], lj = sc[SC + at];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const f32x4 hi = *reinterpret_cast<const f32x4*>(si + 8 * q), lo = *reinterpret_cast<const f32x4*>(si + SC + 8 * q);
          f32x4 f;
#pragma unroll
          for (int e = 0; e < 4; ++e) f[e] = decay<BF>(hi[e], lo[e], hj, lj) * by;
          use(q, f);
        }
      }
    };
    uint64_t whole = ~0ull;   // every lane: formed anew, so that no mask of a whole tile or the diagonal is kept over the loop
    asm volatile("" : "+s"(whole));
    if (w < 4) {   // dx of 32 of the block's columns
      const int p0 = 32 * (w % 2), tok = 32 * tx + c;
      const float dt = sc[2 * SC + tok], vj = sc[4 * SC + tok], dtv = dt * vj;
      f32x16 xa = zero16(), xv = zero16();
#pragma unroll
      for (int s = 0; s < N / 16; ++s) mma32(xv, ST::row(LD, p0, s, x), RT::row(LB, tok, s, h));
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (i >= tx) {
          f32x16 q;
          const uint64_t all = i > tx ? whole : 0;
          decays_to(i, tok, i > tx, 1.f, [&](int b, const f32x4& f) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              q[4 * b + e] = keep_lanes((i == 0 ? ka[4 * b + e] : kb[4 * b + e]) * f[e], DIAGONAL.from[4 * b + e] | all);
          });
#pragma unroll
          for (int s = 0; s < 2; ++s)
            mma32(xa, XT::colp(LY, 32 * i + 16 * s + 4 * h, 32 * i + 16 * s + 8 + 4 * h, p0, x), frag_of<T>(q, s));
        }
      const float Dh = sc[6 * SC + 3];   // not from memory: its wait would be one for the block that is on its way
      const auto rx = row_window(static_cast<S*>(a.dX) + (size_t)head * a.P + pb * 64 + p0, row0, a.dxs, n, 32);
      float o[2][8];
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const Frag<T> xr = XT::row(LX, tok, p0 / 16 + s, h), yr = XT::row(LY, tok, p0 / 16 + s, h);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float p = xa[8 * s + j], v = xv[8 * s + j];
          di = __builtin_fmaf(p, xr.get(j), di);
          dv = __builtin_fmaf(v, xr.get(j), dv);
          dd = __builtin_fmaf(yr.get(j), xr.get(j), dd);
          o[s][j] = __builtin_fmaf(dt, p, __builtin_fmaf(dtv, v, Dh * yr.get(j)));
        }
      }
      store_rows<T>(rx, 32 * tx, a.dxs, [&](int s, int j) { return o[s][j]; });
      if (pb == nb - 1) {
        di = half_sum(di);
        dv = half_sum(dv);
        if (h == 0) {
          left.i[w % 2][tok] = di;
          left.v[w % 2][tok] = dv * vj;
        }
        dd = group_sum_swap(lane_sum<16>(dd));
        if (l == 0) left.d[w] = dd;
      }
    } else if (w < 7) {   // M, and the sums of Z
#pragma unroll
      for (int s = 0; s < 4; ++s) mma32(kb, XT::row(LY, 32 * ti + c, s, h), XT::row(LX, tok, s, h));
      if (pb == nb - 1) {
        const float dt = sc[2 * SC + tok];
        const uint64_t all = ti > tj ? whole : 0;
        float cz = 0.f, z[16];
        decays_to(ti, tok, ti > tj, dt, [&](int b, const f32x4& f) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int y = 4 * b + e;
            const float m = keep_lanes(kb[y] * f[e], DIAGONAL.from[y] | all);
            W[y] += m;
            z[y] = keep_lanes(m * ka[y], DIAGONAL.behind[y] | all);
            cz += z[y];
          }
        });
        // sums over a row of 16 lanes of each element: a lane keeps the elements of its place in four, then four each
        float s8[8], s4[4];
#pragma unroll
        for (int y = 0; y < 8; ++y) s8[y] = (x & 1 ? z[2 * y + 1] : z[2 * y]) + lane_xor<1>(x & 1 ? z[2 * y] : z[2 * y + 1]);
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          s4[y] = (x & 2 ? s8[2 * y + 1] : s8[2 * y]) + lane_xor<2>(x & 2 ? s8[2 * y] : s8[2 * y + 1]);
          s4[y] = row_sum4(s4[y]);
          if (x % 16 < 4) left.row[tj][(x / 16) & 1][32 * ti + 8 * y + 4 * h + x % 4] = s4[y];
        }
        cz = half_sum(cz);
        if (h == 0) left.col[ti][tok] = cz;
      }
    }
    if (pb == nb - 1) {
      if (has_n) {
        dr = half_sum(dr);
        if (h == 0) left.r[n0 / 32][tok] = dr;
      }
      ss = group_sum_swap(lane_sum<16>(ss));
      if (l == 0) left.s[w] = ss;
    }
  }
  sync_lds();
  if (w == 7) put_out(hpp - 1);
  // dB += W^T C, dC += W B, through W as rows i in LDS, as two bf16 terms: the heads' M may cancel in it
  constexpr int TERMS = BF ? 2 : 1;
  char* LW = lds + 2 * ROWS;
  if (w >= 4) {
    const int ri = w < 7 ? ti : 0;
#pragma unroll
    for (int y = 0; y < 16; ++y) {
      const int i = 32 * ri + res_row(y, h);
      float v = w < 7 ? W[y] : 0.f;
#pragma unroll
      for (int k = 0; k < TERMS; ++k) {
        const S u = float_to_io<S>(v);
        *reinterpret_cast<S*>(LW + k * XROWS + XT::at(i, tok / XT::E) + tok % XT::E * (int)sizeof(S)) = u;
        v -= io_to_float(u);
      }
    }
  }
  sync_lds();
  if (!has_n) return;
#pragma unroll
  for (int s = 0; s < 4; ++s)
#pragma unroll
    for (int k = TERMS - 1; k >= 0; --k) {
      const char* L = LW + k * XROWS;
      if (s / 2 <= tj) mma32(dC, RT::colp(LB, 16 * s + 8 * h, 16 * s + 8 * h + 4, n0), XT::row(L, tok, s, h));
      if (s / 2 >= tj) mma32(dB, RT::colp(LC, 16 * s + 4 * h, 16 * s + 8 + 4 * h, n0), XT::col(L, 16 * s + 4 * h, 32 * tj));
    }
  auto store = [&](const f32x16& x, float* parts, void* out, int stride) {
    if (tok >= n) return;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int col = n0 + 16 * s + 8 * h;
      const f32x4 u = {x[8 * s], x[8 * s + 1], x[8 * s + 2], x[8 * s + 3]};
      const f32x4 v = {x[8 * s + 4], x[8 * s + 5], x[8 * s + 6], x[8 * s + 7]};
      if (parts) {
        float* p = parts + ((((size_t)part * slots + slot) * SC + tok) * a.G + grp) * N + col;
        *reinterpret_cast<f32x4*>(p) = u;
        *reinterpret_cast<f32x4*>(p + 4) = v;
      } else {
        S* p = static_cast<S*>(out) + (size_t)(row0 + tok) * stride + (size_t)grp * N + col;
        store_io4(p, u);
        store_io4(p + 4, v);
      }
    }
  };
  store(dB, a.part_b, a.dB, a.dbs);
  store(dC, a.part_c, a.dC, a.dcs);
}

// dB and dC from the parts of the heads, in order: a workgroup has PART_ROWS rows of a chunk, a thread four values.
constexpr int PART_ROWS = 8;
template <class S>
__global__ __launch_bounds__(256) void k_scan_parts(ScanArgs a) {
  const int slots = seq_slots(a.T, a.B, SC), slot = blockIdx.x / (SC / PART_ROWS), r0 = blockIdx.x % (SC / PART_ROWS) * PART_ROWS;
  const SeqTile t = find_tile<SC>(a.off, a.B, a.T, slot);
  if (t.b < 0) return;
  const int n = min(SC, t.n - t.tile * SC), row0 = t.row0 + t.tile * SC, width = a.G * a.N;
  for (int i = r0 * width + threadIdx.x * 4; i < min(n, r0 + PART_ROWS) * width; i += 1024) {
    const int r = i / width, col = i % width;
    f32x4 b = zero4(), c = zero4();
    for (int p = 0; p < a.parts; ++p) {
      const size_t at = (((size_t)p * slots + slot) * SC) * width + i;
      b += *reinterpret_cast<const f32x4*>(a.part_b + at);
      c += *reinterpret_cast<const f32x4*>(a.part_c + at);
    }
    store_io4(static_cast<S*>(a.dB) + (size_t)(row0 + r) * a.dbs + col, b);
    store_io4(static_cast<S*>(a.dC) + (size_t)(row0 + r) * a.dcs + col, c);
  }
}

// dD of a head: its chunks' sums, in a fixed order.
__global__ __launch_bounds__(256) void k_scan_skip(ScanArgs a) {
  __shared__ double sums[256];
  const int slots = a.T > 0 ? seq_slots(a.T, a.B, SC) : 0, head = blockIdx.x;
  double s = 0.0;
  for (int i = threadIdx.x; i < slots; i += 256) s += (double)a.part_d[(size_t)i * a.H + head];
  sums[threadIdx.x] = s;
  __syncthreads();
  for (int k = 128; k > 0; k /= 2) {
    if ((int)threadIdx.x < k) sums[threadIdx.x] += sums[threadIdx.x + k];
    __syncthreads();
  }
  if (threadIdx.x == 0) a.dD[head] = (float)sums[0];
}

namespace {
template <class T, int N>
void grad(const ScanArgs& a, hipStream_t st) {
  const int slots = seq_slots(a.T, a.B, SC);
  k_scan_grad<T, N><<<(slots + NUM_XCD - 1) / NUM_XCD * NUM_XCD * a.G * a.parts, 512, 0, st>>>(a);
  if (a.part_b) k_scan_parts<typename Io<T>::type><<<slots * (SC / PART_ROWS), 256, 0, st>>>(a);
}
}  // namespace

hipError_t launch_scan_bwd(const ScanArgs& a, bool bf16, hipStream_t st) {
  timing_mark(FLEX_KERNEL_SCAN_BWD, st, true);
  if (a.T > 0) {
    launch_scan_states(a, bf16, st);
    if (bf16)
      a.N == 64 ? grad<__bf16, 64>(a, st) : grad<__bf16, 128>(a, st);
    else
      a.N == 64 ? grad<float, 64>(a, st) : grad<float, 128>(a, st);
  }
  if (a.dD) k_scan_skip<<<a.H, 256, 0, st>>>(a);
  timing_mark(FLEX_KERNEL_SCAN_BWD, st, false);
  return hipGetLastError();
}

}  // namespace flex
