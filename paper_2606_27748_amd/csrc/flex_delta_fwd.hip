// Gated delta rule, forward: the chunks' matrices (k_delta_prep), the sweep over the state
// (k_delta_sweep) and the single-token step (k_delta_step).
#include "flex_delta.hpp"
#include "../../include/flex.h"

namespace flex {

namespace {
__device__ __forceinline__ void lds_fence() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// c += a b for 16 x 16 fp32 tiles: a as its transpose's result layout, b as a result
__device__ __forceinline__ void mm16(f32x4& c, const f32x4& a, const f32x4& b) {
#pragma unroll
  for (int r = 0; r < 4; ++r) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[r], b[r], c, 0, 0, 0);
}
}  // namespace

// One wave per chunk and value head; everything in fp32 from exact products.
// N = A^T is held as 16 x 16 tiles N(n, m) (rows j of block n, lane column i of block m), so
// that the tiles of X = (I + N)^-1 = T^T come out as a lane per row i of T.  The diagonal
// blocks are inverted by substitution, a lane per column, all four at once; the others
// follow from X(n,m) = -X(n,n) sum_{n<k<=m} N(n,k) X(k,m) on the fp32 matrix cores.
// Bound by the chain of substitution and block products of a wave, two waves per SIMD to cover it: 63 us
// for 2 x 8192 tokens, 16 heads of 128, where reading and writing its 250 MB takes 48.
template <class T, int D>
__global__ __launch_bounds__(256) void k_delta_prep(DeltaArgs a) {
  using S = typename Io<T>::type;
  constexpr int KS = D / 32, LD = 20;
  __shared__ __attribute__((aligned(16))) float lds_t[4][4 * 16 * LD];
  __shared__ double lds_g[4][DC];
  const int l = threadIdx.x % WAVE, r16 = l % 16, g = l / 16;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
  const int slots = seq_slots(a.T, a.B, DC);
  const int id = blockIdx.x * 4 + w, slot = id / a.H, head = id % a.H;
  if (slot >= slots) return;
  const SeqTile t = find_tile<DC>(a.off, a.B, a.T, slot);
  if (t.b < 0) return;
  const int n = min(DC, t.n - t.tile * DC), row0 = t.row0 + t.tile * DC, kh = head / (a.H / a.Hk);
  char* out = a.prep + (size_t)id * DELTA_PREP_BYTES;
  float* Lt = lds_t[w];
  double* Lg = lds_g[w];

  // the decays, lane = token.  A decay of zero (g = -inf) is kept as a finite sum whose
  // exponential is zero: differences of G stay defined.
  float gv = 0.f, bv = 0.f;
  if (l < n) {
    gv = a.g[(size_t)(row0 + l) * a.H + head];
    bv = a.beta[(size_t)(row0 + l) * a.H + head];
  }
  if (gv < -1e4f) gv = -1e4f;
  double G = gv;
#pragma unroll
  for (int s = 1; s < WAVE; s *= 2) {
    const double o = __shfl_up(G, s);
    if (l >= s) G += o;
  }
  const double Gc = __shfl(G, DC - 1);
  float* scal = reinterpret_cast<float*>(out + 2 * DELTA_MAT_BYTES);
  float eg = expf((float)G);
  scal[DC + l] = expf((float)(Gc - G));
  scal[2 * DC + l] = bv;
  reinterpret_cast<double*>(out + DELTA_SWEEP_BYTES)[l] = G;
  Lg[l] = G;
  lds_fence();

  const auto rk = row_window(static_cast<const S*>(a.K) + kh * D, row0, a.ks, n, D);
  Frag<T> kf[4][KS];
#pragma unroll
  for (int m = 0; m < 4; ++m)
#pragma unroll
    for (int s = 0; s < KS; ++s)
      kf[m][s] = window_frag<T>(rk, ((16 * m + r16) * a.ks + 32 * s + 8 * g) * (int)sizeof(S));
  double Gi[4];   // G and b of this lane's column in each block
  float bi[4];
#pragma unroll
  for (int m = 0; m < 4; ++m) {
    Gi[m] = Lg[16 * m + r16];
    bi[m] = __shfl(bv, 16 * m + r16);
  }
  auto decay = [&](double x) { return expf((float)x); };

  // N(n, m), n <= m, and for n < m also A(m, n), which is N(n, m) as a left operand
  f32x4 N[4][4], A[4][4];
  float bad = 0.f;   // NaN from the first element of A that is not finite on
#pragma unroll
  for (int m = 0; m < 4; ++m)
#pragma unroll
    for (int nn = 0; nn <= m; ++nn) {
      f32x4 c = zero4();
#pragma unroll
      for (int s = 0; s < KS; ++s) mma(c, kf[nn][s], kf[m][s]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int j = 16 * nn + 4 * g + e, i = 16 * m + r16;
        N[nn][m][e] = j < i ? c[e] * (bi[m] * decay(Gi[m] - Lg[j])) : 0.f;
      }
      if (nn == m) {
        *reinterpret_cast<f32x4*>(Lt + (m * 16 + r16) * LD + 4 * g) = N[m][m];   // A(m,m)[i][j]
#pragma unroll
        for (int e = 0; e < 4; ++e) bad = __builtin_fmaf(N[m][m][e], 0.f, bad);
      } else {
        f32x4 d = zero4();
#pragma unroll
        for (int s = 0; s < KS; ++s) mma(d, kf[m][s], kf[nn][s]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int i = 16 * m + 4 * g + e;
          A[m][nn][e] = d[e] * (__shfl(bv, i) * decay(Lg[i] - Gi[nn]));
          bad = __builtin_fmaf(A[m][nn][e], 0.f, bad);
        }
      }
    }
  lds_fence();
  // From a token on whose row of A is not finite, A is taken as zero, so that T's rows before it stay what they
  // are, and the decay as NaN, which makes the sweep's results from the token on what they then have to be.
  if (__any(bad != 0.f)) {
    int first = DC;
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      const f32x4 x = *reinterpret_cast<const f32x4*>(Lt + (m * 16 + r16) * LD + 4 * g);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (!(fabsf(x[e]) < INFINITY)) first = min(first, 16 * m + r16);
#pragma unroll
        for (int nn = 0; nn < m; ++nn)
          if (!(fabsf(A[m][nn][e]) < INFINITY)) first = min(first, 16 * m + 4 * g + e);
      }
    }
#pragma unroll
    for (int s = 1; s < WAVE; s *= 2) first = min(first, __shfl_xor(first, s));
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      if (16 * m + r16 >= first) *reinterpret_cast<f32x4*>(Lt + (m * 16 + r16) * LD + 4 * g) = zero4();
#pragma unroll
      for (int nn = 0; nn < m; ++nn)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (16 * m + 4 * g + e >= first) A[m][nn][e] = 0.f;
    }
    if (l >= first) eg = NAN;
    lds_fence();
  }
  scal[l] = eg;
  // T(g,g), lane column r16: t_i = [i == column] - sum_{k<i} A_ik t_k
  float tc[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    float x = i == r16 ? 1.f : 0.f;
#pragma unroll
    for (int k = 0; k < i; k += 4) {
      const f32x4 ar = *reinterpret_cast<const f32x4*>(Lt + (g * 16 + i) * LD + k);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (k + e < i) x = __builtin_fmaf(-ar[e], tc[k + e], x);
    }
    tc[i] = x;
  }
  lds_fence();
#pragma unroll
  for (int i = 0; i < 16; ++i) Lt[(g * 16 + i) * LD + r16] = tc[i];
  lds_fence();
  f32x4 X[4][4], Xl[4];   // X as results; the diagonal ones also as left operands
#pragma unroll
  for (int m = 0; m < 4; ++m) {
    X[m][m] = *reinterpret_cast<const f32x4*>(Lt + (m * 16 + r16) * LD + 4 * g);
#pragma unroll
    for (int e = 0; e < 4; ++e) Xl[m][e] = Lt[(m * 16 + 4 * g + e) * LD + r16];
  }
#pragma unroll
  for (int dlt = 1; dlt < 4; ++dlt)
#pragma unroll
    for (int nn = 0; nn + dlt < 4; ++nn) {
      const int m = nn + dlt;
      f32x4 y = zero4(), x = zero4();
#pragma unroll
      for (int k = nn + 1; k <= m; ++k) mm16(y, A[k][nn], X[k][m]);
      mm16(x, Xl[nn], y);
      X[nn][m] = -x;
    }
  constexpr size_t LO = LowTri<T>::TERM / sizeof(S);
#pragma unroll
  for (int m = 0; m < 4; ++m)
#pragma unroll
    for (int nn = 0; nn <= (m | 1); ++nn)   // with the zero blocks that share a k step with the diagonal
      store_split4(reinterpret_cast<S*>(out + LowTri<T>::at(16 * m + r16, 16 * nn + 4 * g)), LO,
                   nn <= m ? X[nn][m] : zero4());

  const auto rq = row_window(static_cast<const S*>(a.Q) + kh * D, row0, a.qs, n, D);
#pragma unroll
  for (int m = 0; m < 4; ++m) {
    Frag<T> qf[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s)
      qf[s] = window_frag<T>(rq, ((16 * m + r16) * a.qs + 32 * s + 8 * g) * (int)sizeof(S));
#pragma unroll
    for (int nn = 0; nn <= (m | 1); ++nn) {
      f32x4 c = zero4();
      if (nn <= m) {
#pragma unroll
        for (int s = 0; s < KS; ++s) mma(c, kf[nn][s], qf[s]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int j = 16 * nn + 4 * g + e, i = 16 * m + r16;
          c[e] = j <= i ? c[e] * decay(Gi[m] - Lg[j]) : 0.f;
        }
      }
      store_split4(reinterpret_cast<S*>(out + DELTA_MAT_BYTES + LowTri<T>::at(16 * m + r16, 16 * nn + 4 * g)), LO, c);
    }
  }
}

// The sweep: one workgroup per sequence, value head and 16 NC columns of the state.  What the
// next chunk waits for is one wave's per 16 columns (S -> K S -> U -> S, the state in its
// registers); a second forms Q S and O beside it from the operands that the first leaves in
// LDS, and writes O and what a backward needs; NL waves stage the chunks.  What bounds it is that
// chain: 82 matrix instructions of 16 clocks and the splits between them, about 4200 clocks a
// chunk at d = 128, of which the instructions fill 1300.  One wave for all of it took 4.3 us a chunk
// (256 waves for 32 heads of 128, three quarters of the SIMDs without work), two waves 2.9, these
// 2.0 (with what a backward needs kept: 12 KB of it and 4 KB of O per chunk and workgroup).
template <class T, int D, int NC, bool SAVE>
__global__ __launch_bounds__(NC * 128 + NL * 64) __attribute__((amdgpu_waves_per_eu(1, 2))) void k_delta_sweep(DeltaArgs a) {
  using S = typename Io<T>::type;
  using KT = Tile16<T, D>;
  using LT = LowTri<T>;
  using CL = ChunkLds<T, D, 16 * NC>;
  using FB = FragBox<T>;
  constexpr int KS = D / 32, DT = D / 16, TERMS = IsBf16<T>::value ? 2 : 1;
  // S as operands, U as results, and room to turn O's columns into rows
  constexpr int BOX_U = KS * FB::BYTES, BOX_O = BOX_U + 4 * WAVE * 16, BOX = BOX_O + RowBox<S>::BYTES;
  constexpr int BUFS = 2 * CL::BYTES + NC * BOX <= 160 * 1024 ? 2 : 1;
  __shared__ __attribute__((aligned(16))) char lds[BUFS * CL::BYTES + NC * BOX];
  const int l = threadIdx.x % WAVE, r16 = l % 16, g = l / 16;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE), pair = w % NC;
  const int parts = a.dv / (16 * NC);
  const SweepCoord sc = sweep_coord(a.B * a.H, parts);
  const int bh = sc.bh, b = bh / a.H, head = bh % a.H, kh = head / (a.H / a.Hk);
  const int col0 = sc.part * NC * 16, col = col0 + 16 * pair + r16;   // this lane's column of the state
  const SeqRange sq = seq_range(a.off, b, a.T);
  const int nchunks = (sq.n + DC - 1) / DC, slot0 = sq.row0 / DC + b;
  char* box = lds + BUFS * CL::BYTES + pair * BOX;
  // every wave passes the same barriers in a chunk: (1) the chunk and S are in LDS, (2) U is, and with
  // one buffer (3) the chunk is no longer read

  if (w >= 2 * NC) {   // staging
    const S* X = static_cast<const S*>(a.V) + (size_t)head * a.dv + col0;
    const int xs = a.vs, lw = w - 2 * NC;
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
    const int first = 0, end = nchunks, step = 1;
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

  if (w < NC) {   // the state
    f32x4 st[DT];
    const size_t sbase = ((size_t)bh * D) * a.dv + col;
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) st[i][e] = a.state0 ? a.state0[sbase + (size_t)tile_row(i, 4 * g + e) * a.dv] : 0.f;
    f32x4* box_u = reinterpret_cast<f32x4*>(box + BOX_U) + l;
    Split<T> sb[KS];
    auto put_state = [&]() {
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        sb[s] = split<T>(st[2 * s], st[2 * s + 1]);
        FB::put(box + s * FB::BYTES, l, sb[s]);
      }
    };
    put_state();
    for (int c = 0; c < nchunks; ++c) {
      const CL L{lds + (BUFS == 2 ? (c & 1) * CL::BYTES : 0)};
      sync_lds();
      f32x4 u[4];
#pragma unroll
      for (int m = 0; m < 4; ++m) u[m] = zero4();
      auto add_ks = [&](int s, const Split<T>& x, int r16, int g) {
        Frag<T> kr[4];
#pragma unroll
        for (int m = 0; m < 4; ++m) kr[m] = KT::row8(L.k(), tile_row(m, r16), 32 * s + 8 * g);
        mma_xs4(u, kr, x);
      };
      auto form_r = [&](int g) {   // b (V - e^G K S)
#pragma unroll
        for (int m = 0; m < 4; ++m) {
          const f32x4 eg = L.scal(0, m, g), be = L.scal(2, m, g);
          const auto vc = L.col(m, g, 16 * pair);
#pragma unroll
          for (int e = 0; e < 4; ++e) u[m][e] = be[e] * ((float)vc[e] - eg[e] * u[m][e]);
        }
      };
#pragma unroll
      for (int s = 0; s < KS; ++s) add_ks(s, sb[s], r16, g);
      form_r(g);
      const bool bad = not_finite(u);   // looked at behind the product, which hides the wait for it
      LT::apply(u, L.t(), r16, g);
      if (__any(bad)) {
        int x = l;
        asm volatile("" : "+v"(x)::"memory");   // all of it read again: no value and no address is kept for this
        const int r16 = x % 16, g = x / 16;
#pragma unroll
        for (int m = 0; m < 4; ++m) u[m] = zero4();
#pragma unroll 1
        for (int s = 0; s < KS; ++s) add_ks(s, FB::get(box + s * FB::BYTES, x), r16, g);
        form_r(g);
        const int first = first_not_finite(u, g);
        cut(u, g, first, 0.f);
        LT::apply(u, L.t(), r16, g);
        cut(u, g, first, NAN);
      }
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        box_u[m * WAVE] = u[m];
        u[m] *= L.scal(1, m, g);
      }
      const Split<T> w0 = split<T>(u[0], u[1]), w1 = split<T>(u[2], u[3]);
      const float last = L.last();
      sync_lds();
#pragma unroll
      for (int i = 0; i < DT; i += 4) {
        Frag<T> kc[4];
#pragma unroll
        for (int m = 0; m < 4; ++m) {
          kc[m] = KT::col8(L.k(), 8 * g, i + m);
          st[i + m] *= last;
        }
        mma_xs4(*reinterpret_cast<f32x4(*)[4]>(&st[i]), kc, w0);
#pragma unroll
        for (int m = 0; m < 4; ++m) kc[m] = KT::col8(L.k(), 32 + 8 * g, i + m);
        mma_xs4(*reinterpret_cast<f32x4(*)[4]>(&st[i]), kc, w1);
      }
      put_state();   // the box is free: its reader has passed the second barrier
      if (BUFS == 1) sync_lds();
    }
    if (a.state) {
#pragma unroll
      for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) a.state[sbase + (size_t)tile_row(i, 4 * g + e) * a.dv] = st[i][e];
    }
    return;
  }

  for (int c = 0; c < nchunks; ++c) {   // O
    const CL L{lds + (BUFS == 2 ? (c & 1) * CL::BYTES : 0)};
    sync_lds();
    const size_t blk = (size_t)(slot0 + c) * a.H + head;
    f32x4 o[4];
#pragma unroll
    for (int m = 0; m < 4; ++m) o[m] = zero4();
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const Split<T> sb = FB::get(box + s * FB::BYTES, l);
      Frag<T> qr[4];
#pragma unroll
      for (int m = 0; m < 4; ++m) qr[m] = KT::row8(L.q(), tile_row(m, r16), 32 * s + 8 * g);
      mma_xs4(o, qr, sb);
      if (SAVE) store_frag(static_cast<S*>(a.st) + blk * a.dv * D, (col0 / 16 + pair) * KS + s, 0, sb);
    }
#pragma unroll
    for (int m = 0; m < 4; ++m) o[m] *= L.scal(0, m, g);
    sync_lds();
    const f32x4* box_u = reinterpret_cast<const f32x4*>(box + BOX_U) + l;
    f32x4 u[4] = {box_u[0], box_u[WAVE], box_u[2 * WAVE], box_u[3 * WAVE]};
    Split<T> u0 = split<T>(u[0], u[1]), u1 = split<T>(u[2], u[3]);
    if (SAVE) {
      S* uo = static_cast<S*>(a.ut) + blk * (size_t)(TERMS * DC) * a.dv;
      store_frag(uo, (col0 / 16 + pair) * 2, (size_t)DC * a.dv, u0);
      store_frag(uo, (col0 / 16 + pair) * 2 + 1, (size_t)DC * a.dv, u1);
    }
    if (__any(not_finite(u))) {
      int x = g;
      asm volatile("" : "+v"(x));
      const int first = first_not_finite(u, x);
      cut(u, x, first, 0.f);
      cut(o, x, first, NAN);
      u0 = split<T>(u[0], u[1]);
      u1 = split<T>(u[2], u[3]);
    }
    LT::mul(o, L.p(), r16, g, u0, u1);
#pragma unroll
    for (int m = 0; m < 4; ++m) o[m] *= a.scale;
    RowBox<S>::store(box + BOX_O,
                     row_window(static_cast<S*>(a.O) + (size_t)head * a.dv, sq.row0 + c * DC, a.H * a.dv,
                                min(DC, sq.n - c * DC), a.dv),
                     a.H * a.dv, col0 + 16 * pair, o);
    if (BUFS == 1) sync_lds();
  }
}

// One token of every sequence and value head against its state, fp32 throughout.  A
// workgroup takes CW columns of one state: each thread four columns of ROWS rows, held in
// registers between the read and the write.  One pass suffices: with x = S^T k and
// y = S^T q of the old state, u = b (v - a x), S' = a S + k u^T and o = a y + (k.q) u.
// Bound by the state's read and write: 256 tokens, 16 states of 128 x 128 (537 MB), 105 us, a large copy's rate.
template <class T, int D, int CW>
__global__ __launch_bounds__(256) void k_delta_step(DeltaArgs a) {
  using S = typename Io<T>::type;
  constexpr int C4 = CW / 4, RG = 256 / C4, ROWS = D / RG;
  __shared__ float lk[D], lq[D];
  __shared__ __attribute__((aligned(16))) float px[RG][CW + 4], py[RG][CW + 4];
  const int t = threadIdx.x, c = t % C4, rg = t / C4;
  const int parts = a.dv / CW, bh = blockIdx.x / parts, c0 = blockIdx.x % parts * CW;
  const int b = bh / a.H, head = bh % a.H, kh = head / (a.H / a.Hk);
  float* sp = a.state + ((size_t)bh * D + rg * ROWS) * a.dv + c0 + 4 * c;
  f32x4 s[ROWS];
#pragma unroll
  for (int i = 0; i < ROWS; ++i) s[i] = *reinterpret_cast<const f32x4*>(sp + (size_t)i * a.dv);
  if (t < D) {
    lk[t] = io_to_float(static_cast<const S*>(a.K)[(size_t)b * a.ks + kh * D + t]);
    lq[t] = io_to_float(static_cast<const S*>(a.Q)[(size_t)b * a.qs + kh * D + t]);
  }
  const float dec = expf(a.g[bh]), be = a.beta[bh];
  f32x4 vv;
  {
    const S* vp = static_cast<const S*>(a.V) + (size_t)b * a.vs + (size_t)head * a.dv + c0 + 4 * c;
#pragma unroll
    for (int e = 0; e < 4; ++e) vv[e] = io_to_float(vp[e]);
  }
  __syncthreads();
  f32x4 x = zero4(), y = zero4();
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    s[i] *= dec;
    x += s[i] * lk[rg * ROWS + i];
    y += s[i] * lq[rg * ROWS + i];
  }
  *reinterpret_cast<f32x4*>(&px[rg][4 * c]) = x;
  *reinterpret_cast<f32x4*>(&py[rg][4 * c]) = y;
  float kq = 0.f;   // the same sum in every wave
  for (int i = t % WAVE; i < D; i += WAVE) kq = __builtin_fmaf(lk[i], lq[i], kq);
  kq = group_sum(lane_sum<16>(kq));
  __syncthreads();
  x = zero4();
  y = zero4();
#pragma unroll
  for (int i = 0; i < RG; ++i) {
    x += *reinterpret_cast<const f32x4*>(&px[i][4 * c]);
    y += *reinterpret_cast<const f32x4*>(&py[i][4 * c]);
  }
  const f32x4 u = (vv - x) * be;
#pragma unroll
  for (int i = 0; i < ROWS; ++i) *reinterpret_cast<f32x4*>(sp + (size_t)i * a.dv) = s[i] + u * lk[rg * ROWS + i];
  if (rg == 0) store_io4(static_cast<S*>(a.O) + (size_t)bh * a.dv + c0 + 4 * c, (y + u * kq) * a.scale);
}

namespace {
template <class T, int D, int NC>
void run_sweep(const DeltaArgs& a, hipStream_t st) {
  const int wgs = a.B * a.H * (a.dv / (16 * NC));
  if (a.st)
    k_delta_sweep<T, D, NC, true><<<wgs, NC * 128 + NL * 64, 0, st>>>(a);
  else
    k_delta_sweep<T, D, NC, false><<<wgs, NC * 128 + NL * 64, 0, st>>>(a);
}
template <class T, int D>
hipError_t run_fwd(const DeltaArgs& a, hipStream_t st) {
  timing_mark(FLEX_KERNEL_DELTA_FWD, st, true);
  if (a.T > 0) {
    const int64_t waves = (int64_t)seq_slots(a.T, a.B, DC) * a.H;
    k_delta_prep<T, D><<<(unsigned)((waves + 3) / 4), 256, 0, st>>>(a);
  }
  run_sweep<T, D, 2>(a, st);
  timing_mark(FLEX_KERNEL_DELTA_FWD, st, false);
  return hipGetLastError();
}
template <class T, int D>
hipError_t run_step(const DeltaArgs& a, hipStream_t st) {
  timing_mark(FLEX_KERNEL_DELTA_STEP, st, true);
  if (a.dv == 64)
    k_delta_step<T, D, 64><<<a.B * a.H, 256, 0, st>>>(a);
  else
    k_delta_step<T, D, 128><<<a.B * a.H, 256, 0, st>>>(a);
  timing_mark(FLEX_KERNEL_DELTA_STEP, st, false);
  return hipGetLastError();
}
}  // namespace

hipError_t launch_delta_fwd(const DeltaArgs& a, bool bf16, hipStream_t st) {
  if (bf16) return a.d == 64 ? run_fwd<__bf16, 64>(a, st) : run_fwd<__bf16, 128>(a, st);
  return a.d == 64 ? run_fwd<float, 64>(a, st) : run_fwd<float, 128>(a, st);
}
hipError_t launch_delta_step(const DeltaArgs& a, bool bf16, hipStream_t st) {
  if (bf16) return a.d == 64 ? run_step<__bf16, 64>(a, st) : run_step<__bf16, 128>(a, st);
  return a.d == 64 ? run_step<float, 64>(a, st) : run_step<float, 128>(a, st);
}

}  // namespace flex
