// Gated delta rule, backward.  With dO' = scale dO, dS the gradient of the state at a chunk's
// end, and the matrices of flex_delta.hpp:
//   dU = P^T dO' + w K dS         dR = T^T dU           (R = b (V - e^G K S), U = T R)
//   dS <- e^{G_63} dS + Q^T (e^G dO') - K^T (b e^G dR)                (the chunk's start)
// runs backwards over the chunks (k_delta_rsweep, the same wave per 16 columns as the forward's
// sweep), which also gives dV = b dR.  The rest is independent per chunk (k_delta_grad), from
// the states S, dS and the rows U, dR that the sweeps leave:
//   dP = low(dO' U^T), dA = -low(dR U^T), M = b dA D
//   dQ = e^G dO' S^T + (dP D) K
//   dK = (dP D)^T Q + (M + M^T) K - b F + w U dS^T,     F = e^G dR S^T
//   dbeta_i = dR_i.V_i - k_i.F_i + sum_j dA_ij D_ij k_i.k_j
//   dg_t = sum_{i>=t} (q_i.(e^G dO' S^T)_i - b_i k_i.F_i + sum_{j<i} X_ij - sum_{j>i} X_ji) + sum_{i<t} Z_i + e^{G_63} <S, dS>
//          with X = dP P + dA A (elementwise), Z_i = k_i.(w U dS^T)_i
// dg_t is what crosses t: reads from t on of states and writes before it.  X enters as a row sum and as a column
// sum of the same fp32 numbers, so pairs on one side of t cancel to what fp32 sums of them leave, some 2^-24 of
// their absolute values.  The diagonal of X and the Z from t on cross no t and are left out: they have no
// decay in them, and where a head forgets at once (e^-6 a token) that remainder of theirs was 6e-5 of its dg.
#include "flex_delta.hpp"
#include "../../include/flex.h"

namespace flex {

// As the forward's sweep: per 16 columns one wave carries dS (dS -> K dS -> dU -> dR -> dS) and a
// second forms Q^T (e^G dO'), which does not depend on it, and stores dR and dV; NL
// waves stage the chunks.
template <class T, int D, int NC>
__global__ __launch_bounds__(NC * 128 + NL * 64) __attribute__((amdgpu_waves_per_eu(1, 2))) void k_delta_rsweep(DeltaArgs a) {
  using S = typename Io<T>::type;
  using KT = Tile16<T, D>;
  using LT = LowTri<T>;
  using CL = ChunkLds<T, D, 16 * NC>;
  constexpr int KS = D / 32, DT = D / 16, TERMS = IsBf16<T>::value ? 2 : 1;
  // dR, Q^T (e^G dO'), and room to turn dV's columns into rows
  constexpr int BOX_V = (4 + DT) * WAVE * 16, BOX = BOX_V + RowBox<S>::BYTES;
  constexpr int BUFS = 2 * CL::BYTES + NC * BOX <= 160 * 1024 ? 2 : 1;
  __shared__ __attribute__((aligned(16))) char lds[BUFS * CL::BYTES + NC * BOX];
  const int l = threadIdx.x % WAVE, r16 = l % 16, g = l / 16;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE), pair = w % NC;
  const int parts = a.dv / (16 * NC);
  const SweepCoord sc = sweep_coord(a.B * a.H, parts);
  const int bh = sc.bh, b = bh / a.H, head = bh % a.H, kh = head / (a.H / a.Hk);
  const int col0 = sc.part * NC * 16, col = col0 + 16 * pair + r16;
  const SeqRange sq = seq_range(a.off, b, a.T);
  const int nchunks = (sq.n + DC - 1) / DC, slot0 = sq.row0 / DC + b;
  f32x4* box = reinterpret_cast<f32x4*>(lds + BUFS * CL::BYTES + pair * BOX) + l;   // tile i at box[i * WAVE]
  // every wave passes the same barriers in a chunk: (1) the chunk is in LDS, (2) Q^T (e^G dO') and
  // dR are, and with one buffer (3) the chunk is no longer read

  if (w >= 2 * NC) {   // staging
    const S* X = static_cast<const S*>(a.dO) + (size_t)head * a.dv + col0;
    const int xs = a.H * a.dv, lw = w - 2 * NC;
    auto stage = [&](int c) {
      CL{lds + (BUFS == 2 ? (c & 1) * CL::BYTES : 0)}.template stage<NL>(
          a, sq.row0 + c * DC, min(DC, sq.n - c * DC), kh, (size_t)(slot0 + c) * a.H + head, X, xs, lw);
    };
    constexpr int PER = (CL::LINES + 2 * NL * WAVE - 1) / (2 * NL * WAVE);   // two workgroups share a head at least
    unsigned seen[PER] = {};
    auto prefetch = [&](int c) {
      CL{nullptr}.template prefetch<NL, PER>(seen, a, sq.row0 + c * DC, min(DC, sq.n - c * DC), kh,
                                             (size_t)(slot0 + c) * a.H + head, X, xs, sc.part, parts, lw);
    };
    const int first = nchunks - 1, end = -1, step = -1;
    if (nchunks > 0) {
      stage(first);
      if (nchunks > 1) prefetch(first + step);
    }
    for (int c = first; c != end; c += step) {
      const bool more = c + step != end, far = more && c + 2 * step != end;
      // the chunk, not what was asked for after it
      if (BUFS == 2 && more)
        sync_tiles_but<PER>();
      else
        sync_tiles();
      if (BUFS == 2) {
        if (more) stage(c + step);
        if (far) prefetch(c + 2 * step);
      }
      sync_lds();
      if (BUFS == 1) {
        sync_lds();
        if (more) stage(c + step);
        if (far) prefetch(c + 2 * step);
      }
    }
#pragma unroll
    for (int u = 0; u < PER; ++u) asm volatile("" ::"v"(seen[u]));
    return;
  }

  if (w < NC) {   // dS
    f32x4 st[DT];
#pragma unroll
    for (int i = 0; i < DT; ++i) st[i] = zero4();
    Split<T> sb[KS];
    auto keep_state = [&](int c) {
      S* so = static_cast<S*>(a.dst) + ((size_t)(slot0 + c) * a.H + head) * a.dv * D;
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        sb[s] = split<T>(st[2 * s], st[2 * s + 1]);
        store_frag(so, (col0 / 16 + pair) * KS + s, 0, sb[s]);
      }
    };
    if (nchunks > 0) keep_state(nchunks - 1);
    for (int c = nchunks - 1; c >= 0; --c) {
      const CL L{lds + (BUFS == 2 ? (c & 1) * CL::BYTES : 0)};
      sync_lds();
      // dU = P^T dO' + w K dS, dR = T^T dU
      f32x4 y[4], dr[4];
      {
        Split<T> a0[2], a1[4];
        LT::transposed(a0, a1, L.p(), g);
        Frag<T> go[2];
#pragma unroll
        for (int m = 0; m < 4; ++m) {
          const auto x = L.col(m, g, 16 * pair);
#pragma unroll
          for (int e = 0; e < 4; ++e) go[m / 2].v[4 * (m % 2) + e] = x[e];
        }
#pragma unroll
        for (int m = 0; m < 4; ++m) {
          dr[m] = y[m] = zero4();
          mma_sx(y[m], a1[m], go[1]);
          if (m < 2) mma_sx(y[m], a0[m], go[0]);
        }
      }
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        Frag<T> kr[4];
#pragma unroll
        for (int m = 0; m < 4; ++m) kr[m] = KT::row8(L.k(), tile_row(m, r16), 32 * s + 8 * g);
        mma_xs4(dr, kr, sb[s]);
      }
#pragma unroll
      for (int m = 0; m < 4; ++m) dr[m] = dr[m] * L.scal(1, m, g) + y[m] * a.scale;
      LT::apply_t(dr, L.t(), g);
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        box[m * WAVE] = dr[m];
        dr[m] = -(dr[m] * L.scal(2, m, g) * L.scal(0, m, g));   // -b e^G dR
      }
      const Split<T> k0 = split<T>(dr[0], dr[1]), k1 = split<T>(dr[2], dr[3]);
      const float last = L.last();
      sync_lds();
      // dS <- e^{G_63} dS + Q^T (e^G dO') - K^T (b e^G dR)
#pragma unroll
      for (int i = 0; i < DT; i += 4) {
        Frag<T> kc[4];
#pragma unroll
        for (int m = 0; m < 4; ++m) {
          kc[m] = KT::col8(L.k(), 8 * g, i + m);
          st[i + m] = st[i + m] * last + box[(4 + i + m) * WAVE];
        }
        mma_xs4(*reinterpret_cast<f32x4(*)[4]>(&st[i]), kc, k0);
#pragma unroll
        for (int m = 0; m < 4; ++m) kc[m] = KT::col8(L.k(), 32 + 8 * g, i + m);
        mma_xs4(*reinterpret_cast<f32x4(*)[4]>(&st[i]), kc, k1);
      }
      if (c > 0) keep_state(c - 1);
      if (BUFS == 1) sync_lds();
    }
    return;
  }

  for (int c = nchunks - 1; c >= 0; --c) {
    const CL L{lds + (BUFS == 2 ? (c & 1) * CL::BYTES : 0)};
    sync_lds();
    f32x4 gf[4], be[4];
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      const auto x = L.col(m, g, 16 * pair);
      const f32x4 eg = L.scal(0, m, g) * a.scale;
      be[m] = L.scal(2, m, g);
#pragma unroll
      for (int e = 0; e < 4; ++e) gf[m][e] = (float)x[e] * eg[e];
    }
    {
      const Split<T> q0 = split<T>(gf[0], gf[1]), q1 = split<T>(gf[2], gf[3]);
#pragma unroll
      for (int i = 0; i < DT; i += 4) {
        f32x4 y[4];
        Frag<T> qc[4];
#pragma unroll
        for (int m = 0; m < 4; ++m) {
          y[m] = zero4();
          qc[m] = KT::col8(L.q(), 8 * g, i + m);
        }
        mma_xs4(y, qc, q0);
#pragma unroll
        for (int m = 0; m < 4; ++m) qc[m] = KT::col8(L.q(), 32 + 8 * g, i + m);
        mma_xs4(y, qc, q1);
#pragma unroll
        for (int m = 0; m < 4; ++m) box[(4 + i + m) * WAVE] = y[m];
      }
    }
    sync_lds();
    const size_t blk = (size_t)(slot0 + c) * a.H + head;
    S* ro = static_cast<S*>(a.drt) + blk * (size_t)(TERMS * DC) * a.dv;
    f32x4 dr[4];
#pragma unroll
    for (int m = 0; m < 4; ++m) dr[m] = box[m * WAVE];
    store_frag(ro, (col0 / 16 + pair) * 2, (size_t)DC * a.dv, split<T>(dr[0], dr[1]));
    store_frag(ro, (col0 / 16 + pair) * 2 + 1, (size_t)DC * a.dv, split<T>(dr[2], dr[3]));
#pragma unroll
    for (int m = 0; m < 4; ++m) dr[m] *= be[m];
    RowBox<S>::store(lds + BUFS * CL::BYTES + pair * BOX + BOX_V,
                     row_window(static_cast<S*>(a.dV) + (size_t)head * a.dv, sq.row0 + c * DC, a.H * a.dv,
                                min(DC, sq.n - c * DC), a.dv),
                     a.H * a.dv, col0 + 16 * pair, dr);
    if (BUFS == 1) sync_lds();
  }
}

// One workgroup per chunk and key head, over the value heads of its group in order; wave w has
// the tokens 16 w .. + 15, a lane per token, and holds the rows of dQ^T and dK^T
// ([d x 16 tokens]).  S, dS, U, dR, dO and V pass through LDS in blocks of VB value columns, the next
// block on its way while one is worked on where two fit.
// 317 us at 2 x 8192 tokens, 16 heads of 128 (the 960 MB it reads and writes take 185): one workgroup per CU, whose
// waves' registers and LDS leave no second to work while it waits.
template <class T, int D, int VB>
__global__ __launch_bounds__(256) void k_delta_grad(DeltaArgs a) {
  using S = typename Io<T>::type;
  using KT = Tile16<T, D>;
  using VT = Tile16<T, VB>;
  using MT = Tile16<T, DC>;
  using ST = Tile16<T, D, FragRows<T, D>>;
  using PT = Pair16<T, DC, FragRows<T, DC>>;
  constexpr int KS = D / 32, DT = D / 16, VS = VB / 32;
  constexpr int TERMS = IsBf16<T>::value ? 2 : 1;
  constexpr int ROWS = DC * D * (int)sizeof(T), MAT = DC * DC * (int)sizeof(T);
  constexpr int VROWS = DC * VB * (int)sizeof(T);     // a block of dO or V, or of one term of U or dR
  constexpr int SROWS = VB * D * (int)sizeof(T);      // a block of S or dS
  constexpr int STAGED = 2 * VROWS + 2 * SROWS + 2 * TERMS * VROWS;
  constexpr int BLOCK = STAGED > 2 * MAT ? STAGED : 2 * MAT;
  // rows of 256 bytes and more take a SIMD's registers per wave: one workgroup per CU, and room for two blocks
  constexpr int BUFS = D * (int)sizeof(T) >= 256 && 2 * ROWS + 2 * BLOCK <= 156 * 1024 ? 2 : 1;
  __shared__ __attribute__((aligned(16))) char lds[2 * ROWS + BUFS * BLOCK];
  __shared__ double lG[DC];
  __shared__ float col_x[4][DC], row_g[DC], row_z[DC], sum_s[4];
  const char* LK = lds;
  const char* LQ = lds + ROWS;

  const int l = threadIdx.x % WAVE, r16 = l % 16, g = l / 16;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
  const int slot = blockIdx.x / a.Hk, kh = blockIdx.x % a.Hk, grp = a.H / a.Hk;
  const SeqTile t = find_tile<DC>(a.off, a.B, a.T, slot);
  if (t.b < 0) return;
  const int n = min(DC, t.n - t.tile * DC), row0 = t.row0 + t.tile * DC;
  const int tok = 16 * w + r16;
  stage_tile<T, D, DC, 4>(LK, row_words(static_cast<const S*>(a.K) + kh * D, row0, a.ks, n, D), a.ks * (int)sizeof(S), w);
  stage_tile<T, D, DC, 4>(LQ, row_words(static_cast<const S*>(a.Q) + kh * D, row0, a.qs, n, D), a.qs * (int)sizeof(S), w);

  f32x4 dq[DT], dk[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i) dq[i] = dk[i] = zero4();

  const int nvb = a.dv / VB;
  auto stage = [&](int i) {   // block i % nvb of head i / nvb
    const int head = kh * grp + i / nvb, v0 = i % nvb * VB;
    const size_t blk = (size_t)slot * a.H + head;
    const char* L = lds + 2 * ROWS + (BUFS == 2 ? (i & 1) * BLOCK : 0);
    stage_tile<T, VB, DC, 4>(L, row_words(static_cast<const S*>(a.dO) + (size_t)head * a.dv + v0, row0, a.H * a.dv, n, VB),
                             a.H * a.dv * (int)sizeof(S), w);
    L += VROWS;
    stage_tile<T, VB, DC, 4>(L, row_words(static_cast<const S*>(a.V) + (size_t)head * a.dv + v0, row0, a.vs, n, VB),
                             a.vs * (int)sizeof(S), w);
    L += VROWS;
    stage_linear<SROWS / 1024, 4>(L, static_cast<const S*>(a.st) + (blk * a.dv + v0) * D, w);
    stage_linear<SROWS / 1024, 4>(L + SROWS, static_cast<const S*>(a.dst) + (blk * a.dv + v0) * D, w);
    L += 2 * SROWS;
#pragma unroll
    for (int k = 0; k < TERMS; ++k) {
      const size_t at = ((blk * TERMS + k) * a.dv + v0) * DC;
      stage_linear<VROWS / 1024, 4>(L + k * VROWS, static_cast<const S*>(a.ut) + at, w);
      stage_linear<VROWS / 1024, 4>(L + (TERMS + k) * VROWS, static_cast<const S*>(a.drt) + at, w);
    }
  };
  if (BUFS == 2) stage(0);
  int it = 0;
  for (int h = 0; h < grp; ++h) {
    const int head = kh * grp + h;
    const size_t blk = (size_t)slot * a.H + head;
    const char* prep = a.prep + blk * DELTA_PREP_BYTES + 2 * DELTA_MAT_BYTES;
    const float* scal = reinterpret_cast<const float*>(prep);
    const float eg = scal[tok], wt = scal[DC + tok], be = scal[2 * DC + tok], last = scal[DC - 1];
    f32x4 qi[DT], fi[DT], wi[DT];   // dO S^T, dR S^T, U dS^T, transposed
#pragma unroll
    for (int i = 0; i < DT; ++i) qi[i] = fi[i] = wi[i] = zero4();
    f32x4 dp[4], da[4];   // dO U^T and dR U^T, transposed: rows j, lane column i
#pragma unroll
    for (int i = 0; i < 4; ++i) dp[i] = da[i] = zero4();
    float rv = 0.f, ss = 0.f;
    const double Gl = threadIdx.x < DC ? reinterpret_cast<const double*>(prep + 1024)[threadIdx.x] : 0.0;
    for (int vb = 0; vb < nvb; ++vb, ++it) {
      if (BUFS == 1) {
        sync_tiles();   // what was staged or written before is no longer read
        stage(it);
      }
      sync_tiles();
      if (BUFS == 2 && it + 1 < grp * nvb) stage(it + 1);
      if (vb == 0 && threadIdx.x < DC) lG[threadIdx.x] = Gl;
      const char* LG = lds + 2 * ROWS + (BUFS == 2 ? (it & 1) * BLOCK : 0);   // dO, V, S, dS, U, dR
      const char* LV = LG + VROWS;
      const char* LS = LV + VROWS;
      const char* LD = LS + SROWS;
      const char* LU = LD + SROWS;
      const char* LR = LU + TERMS * VROWS;
#pragma unroll
      for (int s = 0; s < VS; ++s) {
        const int c0 = 32 * s + 8 * g;   // value columns c0 .. c0 + 7 in this lane's slots
        const Frag<T> go = VT::row(LG, tok, c0, c0 + 4), vv = VT::row(LV, tok, c0, c0 + 4);
        const Split<T> dr = PT::col(LR, VROWS, c0, c0 + 4, 16 * w), u = PT::col(LU, VROWS, c0, c0 + 4, 16 * w);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          float r = dr.hi.get(j);
          if constexpr (IsBf16<T>::value) r += dr.lo.get(j);
          rv = __builtin_fmaf(r, vv.get(j), rv);
        }
#pragma unroll
        for (int i = 0; i < DT; ++i) {
          const Frag<T> sf = ST::col(LS, c0, c0 + 4, 16 * i), df = ST::col(LD, c0, c0 + 4, 16 * i);
          mma(qi[i], sf, go);
          mma_xs(fi[i], sf, dr);
          mma_xs(wi[i], df, u);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (j <= w) {
            const Split<T> uj = PT::col(LU, VROWS, c0, c0 + 4, 16 * j);
            mma_sx(dp[j], uj, go);
            mma_ss(da[j], uj, dr);
          }
      }
      for (int i = threadIdx.x; i < SROWS / 16; i += 256) {   // <S, dS>: the same place in both tiles
        if constexpr (IsBf16<T>::value) {
          const bf16x8 x = *reinterpret_cast<const bf16x8*>(LS + 16 * i), y = *reinterpret_cast<const bf16x8*>(LD + 16 * i);
#pragma unroll
          for (int j = 0; j < 8; ++j) ss = __builtin_fmaf((float)x[j], (float)y[j], ss);
        } else {
          const f32x4 x = *reinterpret_cast<const f32x4*>(LS + 16 * i), y = *reinterpret_cast<const f32x4*>(LD + 16 * i);
#pragma unroll
          for (int j = 0; j < 4; ++j) ss = __builtin_fmaf(x[j], y[j], ss);
        }
      }
    }
    // the last block's place takes dP D and M, rows i
    char* LP = lds + 2 * ROWS + (BUFS == 2 ? ((it - 1) & 1) * BLOCK : 0);
    char* LM = LP + MAT;
    // the rows' parts of dg and dbeta
    float dot_q = 0.f, dot_f = 0.f, dot_z = 0.f;
    const float ge = eg * a.scale;
#pragma unroll
    for (int i = 0; i < DT; ++i) {
      const f32x4 kr = KT::quad_f(LK, tok, 16 * i + 4 * g), qr = KT::quad_f(LQ, tok, 16 * i + 4 * g);
      qi[i] *= ge;
      fi[i] *= eg;
      wi[i] *= wt;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        dot_q = __builtin_fmaf(qr[e], qi[i][e], dot_q);
        dot_f = __builtin_fmaf(kr[e], fi[i][e], dot_f);
        dot_z = __builtin_fmaf(kr[e], wi[i][e], dot_z);
      }
      dq[i] += qi[i];
      dk[i] += wi[i] - fi[i] * be;
    }
    dot_q = group_sum(dot_q);
    dot_f = group_sum(dot_f);
    dot_z = group_sum(dot_z);
    rv = group_sum(rv);
    // dP D, M, and the sums of X
    float row_x = 0.f, row_b = 0.f;
    const double Gi = lG[tok];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      f32x4 x = zero4();
      if (j <= w) {
        f32x4 kk = zero4(), qk = zero4();
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          const Frag<T> kj = KT::row(LK, 16 * j + r16, 32 * s + 8 * g, 32 * s + 8 * g + 4);
          mma(kk, kj, KT::row(LK, tok, 32 * s + 8 * g, 32 * s + 8 * g + 4));
          mma(qk, kj, KT::row(LQ, tok, 32 * s + 8 * g, 32 * s + 8 * g + 4));
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int tj = 16 * j + 4 * g + e;
          const float D_ij = tj <= tok ? expf((float)(Gi - lG[tj])) : 0.f;
          dp[j][e] *= a.scale * D_ij;
          const float dad = tj < tok ? -da[j][e] * D_ij : 0.f;
          da[j][e] = dad * be;
          row_b = __builtin_fmaf(dad, kk[e], row_b);
          x[e] = tj < tok ? dp[j][e] * qk[e] + da[j][e] * kk[e] : 0.f;
          row_x += x[e];
        }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float c = lane_sum<16>(x[e]);
        if (r16 == 0) col_x[w][16 * j + 4 * g + e] = c;
      }
    }
    row_x = group_sum(row_x);
    row_b = group_sum(row_b);
    if (g == 0) {
      row_g[tok] = dot_q - be * dot_f + row_x;
      row_z[tok] = dot_z;
    }
    if (g == 0 && tok < n) {
      const size_t at = (size_t)(row0 + tok) * a.H + head;
      // in the io type like every gradient of this operator, though beta and g are fp32
      static_cast<S*>(a.dbeta)[at] = float_to_io<S>(rv - dot_f + row_b);
    }
    ss = group_sum(lane_sum<16>(ss));
    if (l == 0) sum_s[w] = ss;
    sync_lds();   // the last block is no longer read; the next may be on its way
    if (w == 0) {
      const float gv = l < n ? a.g[(size_t)(row0 + l) * a.H + head] : 0.f;
      float x = row_g[l] - ((col_x[0][l] + col_x[1][l]) + (col_x[2][l] + col_x[3][l]));
      float z = l > 0 ? row_z[l - 1] : 0.f;
      if (l == DC - 1) x += last * ((sum_s[0] + sum_s[1]) + (sum_s[2] + sum_s[3]));
#pragma unroll
      for (int s = 1; s < WAVE; s *= 2) {   // sums over i >= l, and over i < l
        const float o = __shfl_down(x, s), p = __shfl_up(z, s);
        if (l + s < WAVE) x += o;
        if (l >= s) z += p;
      }
      x += z;
      // a decay of zero has no slope
      if (l < n) static_cast<S*>(a.dg)[(size_t)(row0 + l) * a.H + head] = float_to_io<S>(gv < -1e4f ? 0.f : x);
    }
    // (dP D) and M as rows i in LDS, with the zero blocks that share a k step with the diagonal
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j <= (w | 1)) {
        store_io4(reinterpret_cast<S*>(const_cast<char*>(MT::quad(LP, tok, 16 * j + 4 * g))), dp[j]);
        store_io4(reinterpret_cast<S*>(const_cast<char*>(MT::quad(LM, tok, 16 * j + 4 * g))), da[j]);
      }
    // dQ += (dP D) K, dK += M K over this wave's own rows
#pragma unroll
    for (int s = 0; s < 2; ++s)
      if (2 * s <= w) {
        const Split<T> pf = split<T>(dp[2 * s], dp[2 * s + 1]), mf = split<T>(da[2 * s], da[2 * s + 1]);
#pragma unroll
        for (int i = 0; i < DT; ++i) {
          const Frag<T> kc = KT::col(LK, 32 * s + 4 * g, 32 * s + 16 + 4 * g, 16 * i);
          mma_xs(dq[i], kc, pf);
          mma_xs(dk[i], kc, mf);
        }
      }
    sync_lds();
    // dK += (dP D)^T Q + M^T K over the rows that follow
#pragma unroll
    for (int s = 0; s < 2; ++s)
      if (2 * s + 1 >= w) {
        const Frag<T> pf = MT::col(LP, 32 * s + 4 * g, 32 * s + 16 + 4 * g, 16 * w);
        const Frag<T> mf = MT::col(LM, 32 * s + 4 * g, 32 * s + 16 + 4 * g, 16 * w);
#pragma unroll
        for (int i = 0; i < DT; ++i) {
          mma(dk[i], KT::col(LQ, 32 * s + 4 * g, 32 * s + 16 + 4 * g, 16 * i), pf);
          mma(dk[i], KT::col(LK, 32 * s + 4 * g, 32 * s + 16 + 4 * g, 16 * i), mf);
        }
      }
  }
  if (tok >= n) return;
  const size_t at = ((size_t)(row0 + tok) * a.Hk + kh) * D;
#pragma unroll
  for (int i = 0; i < DT; ++i) {
    store_io4(static_cast<S*>(a.dQ) + at + 16 * i + 4 * g, dq[i]);
    store_io4(static_cast<S*>(a.dK) + at + 16 * i + 4 * g, dk[i]);
  }
}

namespace {
template <class T, int D>
hipError_t run_bwd(const DeltaArgs& a, hipStream_t st) {
  timing_mark(FLEX_KERNEL_DELTA_BWD, st, true);
  const int bh = a.B * a.H;
  k_delta_rsweep<T, D, 2><<<bh * (a.dv / 32), 256 + NL * 64, 0, st>>>(a);
  k_delta_grad<T, D, 32><<<seq_slots(a.T, a.B, DC) * a.Hk, 256, 0, st>>>(a);
  timing_mark(FLEX_KERNEL_DELTA_BWD, st, false);
  return hipGetLastError();
}
}  // namespace

hipError_t launch_delta_bwd(const DeltaArgs& a, bool bf16, hipStream_t st) {
  if (bf16) return a.d == 64 ? run_bwd<__bf16, 64>(a, st) : run_bwd<__bf16, 128>(a, st);
  return a.d == 64 ? run_bwd<float, 64>(a, st) : run_bwd<float, 128>(a, st);
}

}  // namespace flex
