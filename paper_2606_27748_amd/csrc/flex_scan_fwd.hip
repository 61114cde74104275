// Selective scan, forward: the sweep over the chunks (k_scan_sweep), what joins the segments of a
// sequence (k_scan_join), the single-token step (k_scan_step), and the sweeps that carry a state alone,
// forwards or, for the backward, in reverse.
#include <type_traits>
#include "flex_scan.hpp"
#include "../../include/flex.h"

namespace flex {

namespace {
enum {
  SWEEP,       // y
  SWEEP_SAVE,  // y, and the state at each chunk's start
  REV_SAVE     // in reverse, the gradient of the state at each chunk's end
};

// c += a x for operands a that are exact and fp32 values x, as three bf16 terms (24 bits) or as they are.
// Two terms leave 2^-18 of each product: 1.5e-6 of a state, where fp32 sums leave 1e-7.
// By cutting bits off: each term takes the eight leading ones that are left, the third what remains.
__device__ __forceinline__ void split3(Frag<__bf16> (&t)[3], const float (&x)[8]) {
#pragma clang fp contract(off)
  u32x4 w[3];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    unsigned u = __float_as_uint(x[2 * j]), v = __float_as_uint(x[2 * j + 1]);
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      w[k][j] = __builtin_amdgcn_perm(v, u, 0x07060302);   // the upper halves
      if (k == 2) break;
      u = __float_as_uint(__uint_as_float(u) - __uint_as_float(u & 0xffff0000u));
      v = __float_as_uint(__uint_as_float(v) - __uint_as_float(v & 0xffff0000u));
    }
  }
#pragma unroll
  for (int k = 0; k < 3; ++k) t[k].v = __builtin_bit_cast(bf16x8, w[k]);
}
__device__ __forceinline__ void split3(Frag<float> (&t)[1], const float (&x)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) t[0].v[j] = x[j];
}

// u += rows^T (w x) over a chunk: x as its columns' operands, w of the tokens in LDS
template <class T, int N>
__device__ __forceinline__ void form_rows(f32x16 (&u)[N / 32], const char* rows, const Frag<T> (&xf)[4], const float* w, int l) {
  const int h = l / 32;
  constexpr int TERMS = IsBf16<T>::value ? 3 : 1;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const float* ws = w + 16 * q + 4 * h;
    const f32x4 w0 = *reinterpret_cast<const f32x4*>(ws), w1 = *reinterpret_cast<const f32x4*>(ws + 8);
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = xf[q].get(j) * (j < 4 ? w0[j % 4] : w1[j % 4]);
    Frag<T> wx[TERMS], bf[N / 32];
    split3(wx, v);
#pragma unroll
    for (int i = 0; i < N / 32; ++i) bf[i] = ScanTile<T, N>::colp(rows, 16 * q + 4 * h, 16 * q + 8 + 4 * h, 32 * i, l);
#pragma unroll
    for (int t = TERMS - 1; t >= 0; --t)
#pragma unroll
      for (int i = 0; i < N / 32; ++i) {
        mma32(u[i], bf[i], wx[t]);
      }
  }
}

// NaN from the first NaN or infinity on, else zero
__device__ __forceinline__ bool not_finite(const Frag<__bf16> (&x)[4]) {
  float s[2] = {0.f, 0.f};
#pragma unroll
  for (int q = 0; q < 4; ++q)
#pragma unroll
    for (int j = 0; j < 8; j += 2)
      s[q % 2] = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{x[q].v[j], x[q].v[j + 1]}, bf16x2{(__bf16)0.f, (__bf16)0.f}, s[q % 2], false);
  return !(s[0] + s[1] == 0.f);
}
__device__ __forceinline__ bool not_finite(const Frag<float> (&x)[4]) {
  float s = 0.f;
#pragma unroll
  for (int q = 0; q < 4; ++q)
#pragma unroll
    for (int j = 0; j < 8; ++j) s = __builtin_fmaf(x[q].get(j), 0.f, s);
  return !(s == 0.f);
}
}  // namespace

// What a segment of a sequence leaves on its own, S = sum_j e^{L_end - L_j} dt_j B_j x_j^T with L from the segment's
// start (REV: dS = sum_i e^{L_i} C_i dy_i^T), and its decay.  A workgroup has a segment and a set of heads of one group,
// a wave 32 columns of one head's state; the rows of B pass through LDS for all of them.  Forwards the chunks are
// taken from the last one, so that their weights are known and the sum has no decay in it.
// The segment that nothing starts from is left out, and of the first one state0 is a part.
// Bound by the vector instructions that form the weighted rows' terms, between the products of two waves a SIMD: 17152 tokens in 16
// prompts, 64 heads of 64, N = 128, bf16: 71 us (141 MB of x).  With one buffer and two workgroups a CU 99.
template <class T, int N, bool REV>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(1, 2))) void k_scan_carry(ScanArgs a) {
  using S = typename Io<T>::type;
  using RT = ScanTile<T, N>;
  using XT = ScanTile<T, 32>;
  constexpr int NT = N / 32;
  constexpr int ROWS = SC * N * (int)sizeof(T), XROWS = SC * 32 * (int)sizeof(T), BUF = ROWS + 8 * XROWS;
  constexpr int BUFS = 2 * BUF <= 156 * 1024 ? 2 : 1;
  __shared__ __attribute__((aligned(16))) char lds[BUFS * BUF];
  __shared__ __attribute__((aligned(16))) float scal[8][SC];
  const int l = threadIdx.x % WAVE;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE), nw = blockDim.x / WAVE;
  const SegTile sg = find_segment(a.off, a.B, a.T, a.seg, a.H / a.heads);
  if (sg.b < 0 || (REV ? sg.index == 0 : sg.index == sg.count - 1)) return;
  const int per = a.P / 32, head = sg.set * a.heads + w / per, p0 = w % per * 32, grp = head / (a.H / a.G);
  const int t0 = sg.index * a.seg, n = min(sg.n - t0, a.seg), row0 = sg.row0 + t0, nchunks = (n + SC - 1) / SC;
  const S* rb = static_cast<const S*>(REV ? a.Ct : a.Bt) + (size_t)grp * N;
  const S* rx = static_cast<const S*>(REV ? a.dY : a.X) + (size_t)head * a.P + p0;
  const int bs = REV ? a.cs : a.bs, xs = REV ? a.H * a.P : a.xs;
  auto buf = [&](int k) { return lds + (BUFS == 2 ? (k & 1) * BUF : 0); };
  auto stage = [&](int k, int chunk) {
    const int r = row0 + chunk * SC, m = min(SC, n - chunk * SC);
    stage_rows<T, N>(buf(k), rb, r, bs, m, w, nw);
    stage_tile<T, 32, SC, 1>(buf(k) + ROWS + w * XROWS, row_words(rx, r, xs, m, 32), xs * (int)sizeof(S), 0);
  };
  float gn = 0.f, dn = 0.f;   // of the next chunk, lane = token
  auto fetch = [&](int chunk) {
    const int t = chunk * SC + l;
    gn = dn = 0.f;
    if (t < n) {
      const size_t at = (size_t)(row0 + t) * a.H + head;
      gn = a.g[at];
      if (!REV) dn = a.dt[at];
    }
  };
  f32x16 st[NT];
#pragma unroll
  for (int i = 0; i < NT; ++i) st[i] = zero16();
  float* sc = scal[w];
  double total = 0.0;
  stage(0, REV ? 0 : nchunks - 1);   // a segment that another follows has chunks, and so has one behind another
  fetch(REV ? 0 : nchunks - 1);
  for (int k = 0; k < nchunks; ++k) {
    const int next = REV ? k + 1 : nchunks - 2 - k;
    const int h = l / 32;
    const char* L = buf(k);
    sync_tiles();   // the chunk is in LDS, and the buffer of the one before is free
    if (BUFS == 2 && k + 1 < nchunks) stage(k + 1, next);
    const Decay d(gn);
    sc[l] = REV ? __builtin_amdgcn_exp2f((float)(d.L + total)) : __builtin_amdgcn_exp2f((float)(d.end - d.L + total)) * dn;
    total += d.end;
    if (k + 1 < nchunks) fetch(next);
    const char* LX = L + ROWS + w * XROWS;
    Frag<T> xf[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) xf[q] = XT::colp(LX, 16 * q + 4 * h, 16 * q + 8 + 4 * h, 0, l);
    form_rows<T, N>(st, L, xf, sc, l);
    if (BUFS == 1) {
      sync_lds();
      if (k + 1 < nchunks) stage(k + 1, next);
    }
  }
  const float whole = __builtin_amdgcn_exp2f((float)total);
  if (!REV && a.state0 && sg.index == 0) {
    const float* s0 = a.state0 + ((size_t)sg.b * a.H + head) * N * a.P + p0 + perm32(l % 32);
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) st[i][e] = __builtin_fmaf(whole, s0[(size_t)(32 * i + perm_row(e, l / 32)) * a.P], st[i][e]);
  }
  float* carry = a.carry + ((size_t)sg.slot * a.H + head) * N * a.P + (size_t)p0 * N + l * 4;
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      *reinterpret_cast<f32x4*>(carry + (i * 4 + q) * WAVE * 4) =
          f32x4{st[i][4 * q], st[i][4 * q + 1], st[i][4 * q + 2], st[i][4 * q + 3]};
  if (l == 0 && p0 == 0) a.tot[(size_t)sg.slot * a.H + head] = whole;
}

// The sweep over a segment's chunks: workgroups, waves and LDS as above, with the rows of C too.  In reverse the
// state is its gradient dS, the rows are C's, x is dy and the weights are e^L:
//   dS <- e^{L_63} dS + C^T (e^L dy)
// 32 columns a wave and eight waves: two a SIMD, with S, C B^T and the terms of a chunk in 256 registers each, and the rows of B and C
// are read from memory once for eight of them.  A wave's chunk is 94 matrix instructions (N = 128; 3000 clocks of its SIMD)
// and some 950 vector instructions (4000): decays, three terms of each weighted row, roundings.  It takes some 8200: both
// waves of a SIMD are at the same place of a chunk, behind one barrier, and wait for LDS and for results at the same time.
// A wave of 64 columns by itself on a SIMD takes 3 % longer.  P of every head formed beforehand by a kernel of its own, decays
// and all, took 47 us and left 162 of the sweep's 195 then.  C B^T alone, of which a group has one where P is each head's, is 24 of the
// 94 and the same in all eight waves: sharing it has not been measured.  The prompts above: 178 us (281 MB of x and y).
// Fp32 rows: one buffer (96 KB with N = 64, 128 KB with N = 128), whose loads are waited for in full, and products at a tenth of bf16's
// rate: matrix cores busy 67 % of the time over 16384 tokens, 16 heads of 64, N = 128 (187 us).
template <class T, int N, int MODE>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(1, 2))) void k_scan_sweep(ScanArgs a) {
  using S = typename Io<T>::type;
  using RT = ScanTile<T, N>;
  using XT = ScanTile<T, 32>;
  constexpr bool REV = MODE == REV_SAVE, Y = !REV, BF = IsBf16<T>::value;
  constexpr int NS = N / 16, NT = N / 32;
  constexpr int ROWS = SC * N * (int)sizeof(T), XROWS = SC * 32 * (int)sizeof(T);
  constexpr int BUF = (Y ? 2 : 1) * ROWS + 8 * XROWS, SCAL = Y ? 5 * SC : SC;
  constexpr int BUFS = 2 * BUF + 8 * SCAL * 4 <= 160 * 1024 ? 2 : 1;
  __shared__ __attribute__((aligned(16))) char lds[BUFS * BUF];
  __shared__ __attribute__((aligned(16))) float scal[8][SCAL];
  const int l = threadIdx.x % WAVE;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE), nw = blockDim.x / WAVE;
  const SegTile sg = find_segment(a.off, a.B, a.T, a.seg, a.H / a.heads);
  if (sg.b < 0) return;
  const bool last_seg = sg.index == sg.count - 1;
  const int per = a.P / 32, head = sg.set * a.heads + w / per, p0 = w % per * 32, grp = head / (a.H / a.G);
  const int t0 = sg.index * a.seg, n = min(sg.n - t0, a.seg), row0 = sg.row0 + t0;
  const int nchunks = (n + SC - 1) / SC, slot0 = sg.row0 / SC + sg.b + t0 / SC;
  const int pc = p0 + perm32(l % 32);   // this lane's column of the state

  const S* rb = static_cast<const S*>(REV ? a.Ct : a.Bt) + (size_t)grp * N;
  const S* rc = static_cast<const S*>(a.Ct) + (size_t)grp * N;
  const S* rx = static_cast<const S*>(REV ? a.dY : a.X) + (size_t)head * a.P + p0;
  const int bs = REV ? a.cs : a.bs, xs = REV ? a.H * a.P : a.xs;
  auto buf = [&](int k) { return lds + (BUFS == 2 ? (k & 1) * BUF : 0); };
  auto stage = [&](int k, int chunk) {
    const int r = row0 + chunk * SC, m = min(SC, n - chunk * SC);
    const char* L = buf(k);
    stage_rows<T, N>(L, rb, r, bs, m, w, nw);
    if (Y) stage_rows<T, N>(L + ROWS, rc, r, a.cs, m, nw - 1 - w, nw);
    stage_tile<T, 32, SC, 1>(L + (Y ? 2 : 1) * ROWS + w * XROWS, row_words(rx, r, xs, m, 32), xs * (int)sizeof(S), 0);
  };
  float gn = 0.f, dn = 0.f;   // of the next chunk, lane = token
  auto fetch = [&](int chunk) {
    const int t = chunk * SC + l;
    gn = dn = 0.f;
    if (t < n) {
      const size_t at = (size_t)(row0 + t) * a.H + head;
      gn = a.g[at];
      if (!REV) dn = a.dt[at];
    }
  };

  f32x16 st[NT];
#pragma unroll
  for (int i = 0; i < NT; ++i) st[i] = zero16();
  // tile i's elements 4 q .. + 3 of every lane, in a row
  const float* carry = a.carry ? a.carry + ((size_t)sg.slot * a.H + head) * N * a.P + (size_t)p0 * N + l * 4 : nullptr;
  if (!REV && a.state0 && sg.count == 1) {
    const float* s0 = a.state0 + ((size_t)sg.b * a.H + head) * N * a.P + pc;
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) st[i][e] = s0[(size_t)(32 * i + perm_row(e, l / 32)) * a.P];
  } else if (carry && (REV ? !last_seg : sg.index > 0 || (a.state0 && sg.count > 1))) {
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x4 v = *reinterpret_cast<const f32x4*>(carry + (i * 4 + q) * WAVE * 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) st[i][4 * q + e] = v[e];
      }
  }
  auto keep = [&](void* base, int chunk, const Frag<T> (&f)[NS]) {
    S* p = static_cast<S*>(base) + (((size_t)(slot0 + chunk) * a.H + head) * a.P + p0) * N;
#pragma unroll
    for (int s = 0; s < NS; ++s) StateRows<T, N>::store(p, s, f[s]);
  };
  auto state_frags = [&](Frag<T> (&f)[NS]) {
#pragma unroll
    for (int s = 0; s < NS; ++s) f[s] = frag_of<T>(st[s / 2], s % 2);
  };
  // stores of a step, behind its loads
  constexpr int LATER = BUFS == 1 ? 0 : (Y ? (BF ? 4 : 8) : 0) + (MODE == SWEEP ? 0 : BF ? NS : 2 * NS);

  float* sc = scal[w];
  const float Dh = Y && a.D ? a.D[head] : 0.f;
  if (nchunks > 0) {
    const int first = REV ? nchunks - 1 : 0;
    stage(0, first);
    fetch(first);
  }
  // on every way to the loop: where a state's loads are not known to have arrived, the compiler waits for them at their first
  // use in every chunk, and so for the rows that are on their way
  wait_lds_loads();
  for (int k = 0; k < nchunks; ++k) {
    const int chunk = REV ? nchunks - 1 - k : k, next = REV ? chunk - 1 : chunk + 1;
    const char* L = buf(k);
    int x = l;
    if (Y) asm volatile("" : "+v"(x));   // places in LDS are formed anew: kept over the loop they take more registers than there are
    const int c = x % 32, h = x / 32;
    sync_tiles_but<LATER>();   // the chunk is in LDS, and the buffer of the one before is free
    if (BUFS == 2 && k + 1 < nchunks) stage(k + 1, next);
    const Decay d(gn);
    float both = 1.f;      // from the middle of the first half to that of the second
    bool product = false;
    if (Y) {
      sc[l] = d.from_start();
      sc[SC + l] = d.to_end() * dn;
      // e^{L_i - L_j} as a product of what lies between each token and its half's middle, and between the middles, where
      // the former are within 2^50: the latter then is a float's where e^{L_i - L_j} of any two tokens is above
      // 2^-26.  Fp32 rows take the exponential of each difference, whose argument has a smaller error.
      const double m0 = lane_of(d.L, 15), m1 = lane_of(d.L, 47);
      const float from = (float)(d.L - (l < 32 ? m0 : m1));
      product = BF && __all(fabsf(from) < 50.f);
      if (product) {
        both = __builtin_amdgcn_exp2f((float)(m1 - m0));
        sc[2 * SC + l] = __builtin_amdgcn_exp2f(from);
        sc[3 * SC + l] = __builtin_amdgcn_exp2f(-from) * dn;
      } else {
        sc[2 * SC + l] = d.hi;
        sc[3 * SC + l] = d.lo;
        sc[4 * SC + l] = dn;
      }
    } else {
      sc[l] = d.from_start();
    }
    const float last = __builtin_amdgcn_exp2f((float)d.end);
    if (k + 1 < nchunks) fetch(next);

    const char* LX = L + (Y ? 2 : 1) * ROWS + w * XROWS;
    // columns of x, slots the tokens 16 q + 4 h + i and 8 further
    auto columns = [&](Frag<T> (&xf)[4]) {
#pragma unroll
      for (int q = 0; q < 4; ++q) xf[q] = XT::colp(LX, 16 * q + 4 * h, 16 * q + 8 + 4 * h, 0, x);
    };
    auto advance = [&]() {   // S <- e^{L_63} S + B^T (w x)
      Frag<T> xf[4];
      columns(xf);
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) st[i][e] *= last;
      form_rows<T, N>(st, L, xf, sc + (Y ? SC : 0), x);
    };
    Frag<T> sb[NS];
    state_frags(sb);
    if constexpr (MODE == REV_SAVE) keep(a.dst, chunk, sb);
    if constexpr (MODE == SWEEP_SAVE) keep(a.st, chunk, sb);
    auto read_out = [&]() {
      const char* LC = L + ROWS;
      Frag<T> xf[4];
      columns(xf);
      // x with a value that is not finite: its column's products go over the rows before it only, and the rows from it
      // on are NaN
      int fb = SC;
      const bool any_bad = __any(not_finite(xf));
      if (any_bad) {
        auto token = [&](int q, int j) { return 16 * q + 4 * h + 8 * (j / 4) + j % 4; };
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (!(fabsf(xf[q].get(j)) < INFINITY)) fb = min(fb, token(q, j));
        fb = min(fb, __shfl_xor(fb, 32));
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (token(q, j) >= fb) xf[q].set(j, 0.f);
      }
      const int m = min(SC, n - chunk * SC), ys = a.H * a.P;
      const auto ry = row_window(static_cast<S*>(a.Y) + (size_t)head * a.P + p0, row0 + chunk * SC, ys, m, 32);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        f32x16 y = zero16(), cb[2] = {zero16(), zero16()};
#pragma unroll
        for (int s = 0; s < NS; ++s) {
          const Frag<T> cr = RT::row(LC, 32 * i + c, s, h);
          mma32(y, sb[s], cr);
#pragma unroll
          for (int j = 0; j <= i; ++j) mma32(cb[j], RT::row(L, 32 * j + c, s, h), cr);
        }
        const float eg = sc[32 * i + c];
#pragma unroll
        for (int e = 0; e < 16; ++e) y[e] *= eg;
        // P from C B^T, factor(j, q) the decays (times dt) of the elements 4 q .. of the tile of j
        auto matrix = [&](auto factor) {
#pragma unroll
          for (int j = 0; j <= i; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const f32x4 f = factor(j, q);
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float v = cb[j][4 * q + e] * f[e];
                cb[j][4 * q + e] = j < i ? v : keep_lanes(v, ~DIAGONAL.behind[4 * q + e]);   // j <= i, a lane per i
              }
            }
        };
        const float ai = sc[2 * SC + 32 * i + c];
        if (product) {
          matrix([&](int j, int q) {
            return *reinterpret_cast<const f32x4*>(sc + 3 * SC + 32 * j + 8 * q + 4 * h) * (j < i ? ai * both : ai);
          });
        } else {
          const float lo = BF ? 0.f : sc[3 * SC + 32 * i + c];
          matrix([&](int j, int q) {
            const int t = 32 * j + 8 * q + 4 * h;
            const f32x4 hj = *reinterpret_cast<const f32x4*>(sc + 2 * SC + t), dj = *reinterpret_cast<const f32x4*>(sc + 4 * SC + t);
            const f32x4 lj = BF ? zero4() : *reinterpret_cast<const f32x4*>(sc + 3 * SC + t);
            f32x4 f;
#pragma unroll
            for (int e = 0; e < 4; ++e) f[e] = decay<BF>(ai, lo, hj[e], lj[e]) * dj[e];
            return f;
          });
        }
#pragma unroll
        for (int j = 0; j <= i; ++j)
#pragma unroll
          for (int s = 0; s < 2; ++s) mma32(y, xf[2 * j + s], frag_of<T>(cb[j], s));
        if (any_bad) {
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (32 * i + c >= __shfl(fb, 8 * (e / 4) + 4 * h + e % 4)) y[e] = NAN;
        }
        const Frag<T> xr[2] = {XT::row(LX, 32 * i + c, 0, h), XT::row(LX, 32 * i + c, 1, h)};
        store_rows<T>(ry, 32 * i, ys, [&](int s, int j) { return __builtin_fmaf(Dh, xr[s].get(j), y[8 * s + j]); });
        asm volatile("" ::: "memory");   // the second half's operands are not read before the first half is done
      }
    };
    if constexpr (!Y) {
      advance();
    } else {
      read_out();
      advance();
    }
    if (BUFS == 1) {
      sync_lds();
      if (k + 1 < nchunks) stage(k + 1, next);
    }
  }
  if (Y && a.state && last_seg) {
    float* so = a.state + ((size_t)sg.b * a.H + head) * N * a.P + pc;
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) so[(size_t)(32 * i + perm_row(e, l / 32)) * a.P] = st[i][e];
  }
}

// What each segment leaves becomes what it starts from, a sequence's segments in order (in reverse: from the last
// one), a thread for four elements of a state.  The first segment left the whole state, state0 in it.
// Bound by memory, eight segments on their way at once: 22 us for the prompts above.
template <bool REV>
__global__ __launch_bounds__(256) void k_scan_join(ScanArgs a) {
  const int size = a.N * a.P / 4, blocks = (a.H * size + 255) / 256;
  const int b = blockIdx.x / blocks, id = blockIdx.x % blocks * 256 + threadIdx.x;
  if (id >= a.H * size) return;
  const int head = id / size, at = id % size;
  const SeqRange r = seq_range(a.off, b, a.T);
  const int count = (r.n + a.seg - 1) / a.seg, slot0 = r.row0 / a.seg + b;
  if (count < 2) return;
  f32x4* p = reinterpret_cast<f32x4*>(a.carry) + ((size_t)slot0 * a.H + head) * size + at;
  const float* tot = a.tot + (size_t)slot0 * a.H + head;
  const size_t step = (size_t)a.H * size;
  constexpr int U = 8;
  if (REV) {
    f32x4 s = p[(count - 1) * step];
    for (int k0 = count - 2; k0 >= 0; k0 -= U) {
      f32x4 v[U];
      float d[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int k = max(k0 - u, 1);
        v[u] = p[k * step];
        d[u] = tot[(size_t)k * a.H];
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (k0 - u >= 0) {
          p[(k0 - u) * step] = s;
#pragma unroll
          for (int e = 0; e < 4; ++e) s[e] = __builtin_fmaf(s[e], d[u], v[u][e]);
        }
    }
    return;
  }
  f32x4 s = p[0];
  if (a.state0) {   // the place of element e of lane l of tile i, 4 q + e % 4 of it
    const int l = at % WAVE, q = at / WAVE % 4, i = at / (WAVE * 4) % (a.N / 32), p0 = at / (WAVE * 4 * (a.N / 32)) * 32;
    const float* s0 = a.state0 + ((size_t)b * a.H + head) * a.N * a.P + (size_t)(32 * i + perm_row(4 * q, l / 32)) * a.P + p0 + perm32(l % 32);
    p[0] = f32x4{s0[0], s0[a.P], s0[2 * a.P], s0[3 * a.P]};
  }
  for (int k0 = 1; k0 < count; k0 += U) {
    f32x4 v[U];
    float d[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = min(k0 + u, count - 2);   // the last one's is not needed
      v[u] = p[k * step];
      d[u] = tot[(size_t)k * a.H];
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (k0 + u < count) {
        p[(k0 + u) * step] = s;
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] = __builtin_fmaf(s[e], d[u], v[u][e]);
      }
  }
}

// One token of every sequence and head, fp32 throughout.  A workgroup has a state: each thread four
// columns of N / ROWS rows, in registers between the read and the write.  Bound by the state's read and write: 256 tokens, 32
// states of 128 x 64, 537 MB in 101 us (5.3 TB/s).
template <class S, int N, int P>
__global__ __launch_bounds__(256) void k_scan_step(ScanArgs a) {
  constexpr int C4 = P / 4, RG = 256 / C4, ROWS = N / RG;
  __shared__ float lb[N], lc[N];
  __shared__ __attribute__((aligned(16))) float py[RG][P + 4];
  const int t = threadIdx.x, c = t % C4, rg = t / C4;
  const int bh = blockIdx.x, b = bh / a.H, head = bh % a.H, grp = head / (a.H / a.G);
  float* sp = a.state + ((size_t)bh * N + rg * ROWS) * P + 4 * c;
  f32x4 s[ROWS];
#pragma unroll
  for (int i = 0; i < ROWS; ++i) s[i] = *reinterpret_cast<const f32x4*>(sp + (size_t)i * P);
  if (t < N) {
    lb[t] = io_to_float(static_cast<const S*>(a.Bt)[(size_t)b * a.bs + grp * N + t]);
    lc[t] = io_to_float(static_cast<const S*>(a.Ct)[(size_t)b * a.cs + grp * N + t]);
  }
  const float dec = expf(a.g[bh]), dt = a.dt[bh], D = a.D ? a.D[head] : 0.f;
  f32x4 x;
  {
    const S* xp = static_cast<const S*>(a.X) + (size_t)b * a.xs + (size_t)head * P + 4 * c;
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = io_to_float(xp[e]);
  }
  const f32x4 u = x * dt;
  __syncthreads();
  f32x4 y = zero4();
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    s[i] = s[i] * dec + u * lb[rg * ROWS + i];
    y += s[i] * lc[rg * ROWS + i];
    *reinterpret_cast<f32x4*>(sp + (size_t)i * P) = s[i];
  }
  *reinterpret_cast<f32x4*>(&py[rg][4 * c]) = y;
  __syncthreads();
  if (rg > 0) return;
#pragma unroll
  for (int i = 1; i < RG; ++i) y += *reinterpret_cast<const f32x4*>(&py[i][4 * c]);
  store_io4(static_cast<S*>(a.Y) + (size_t)bh * P + 4 * c, y + x * D);
}

namespace {
template <class T, int N, int MODE>
void sweep(const ScanArgs& a, hipStream_t st) {
  k_scan_sweep<T, N, MODE><<<seq_slots(a.T, a.B, a.seg) * (a.H / a.heads), a.heads * a.P * 2, 0, st>>>(a);
}
template <class T, int N, bool REV>
void carry(const ScanArgs& a, hipStream_t st) {
  k_scan_carry<T, N, REV><<<seq_slots(a.T, a.B, a.seg) * (a.H / a.heads), a.heads * a.P * 2, 0, st>>>(a);
}
template <bool REV>
void join(const ScanArgs& a, hipStream_t st) {
  k_scan_join<REV><<<a.B * ((a.H * (a.N * a.P / 4) + 255) / 256), 256, 0, st>>>(a);
}
template <class T, int N>
void run_fwd(const ScanArgs& a, hipStream_t st) {
  if (a.carry) {
    carry<T, N, false>(a, st);
    join<false>(a, st);
  }
  if (a.st)
    sweep<T, N, SWEEP_SAVE>(a, st);
  else
    sweep<T, N, SWEEP>(a, st);
}
template <class T, int N>
void run_states(const ScanArgs& a, hipStream_t st) {
  if (a.carry) {
    carry<T, N, true>(a, st);
    join<true>(a, st);
  }
  sweep<T, N, REV_SAVE>(a, st);
}
template <class S>
void run_step(const ScanArgs& a, hipStream_t st) {
  const int n = a.B * a.H;
  if (a.N == 64 && a.P == 64) k_scan_step<S, 64, 64><<<n, 256, 0, st>>>(a);
  if (a.N == 64 && a.P == 128) k_scan_step<S, 64, 128><<<n, 256, 0, st>>>(a);
  if (a.N == 128 && a.P == 64) k_scan_step<S, 128, 64><<<n, 256, 0, st>>>(a);
  if (a.N == 128 && a.P == 128) k_scan_step<S, 128, 128><<<n, 256, 0, st>>>(a);
}
}  // namespace

hipError_t launch_scan_fwd(const ScanArgs& a, bool bf16, hipStream_t st) {
  timing_mark(FLEX_KERNEL_SCAN_FWD, st, true);
  if (bf16)
    a.N == 64 ? run_fwd<__bf16, 64>(a, st) : run_fwd<__bf16, 128>(a, st);
  else
    a.N == 64 ? run_fwd<float, 64>(a, st) : run_fwd<float, 128>(a, st);
  timing_mark(FLEX_KERNEL_SCAN_FWD, st, false);
  return hipGetLastError();
}
void launch_scan_states(const ScanArgs& a, bool bf16, hipStream_t st) {
  if (bf16)
    a.N == 64 ? run_states<__bf16, 64>(a, st) : run_states<__bf16, 128>(a, st);
  else
    a.N == 64 ? run_states<float, 64>(a, st) : run_states<float, 128>(a, st);
}
hipError_t launch_scan_step(const ScanArgs& a, bool bf16, hipStream_t st) {
  timing_mark(FLEX_KERNEL_SCAN_STEP, st, true);
  bf16 ? run_step<u16>(a, st) : run_step<float>(a, st);
  timing_mark(FLEX_KERNEL_SCAN_STEP, st, false);
  return hipGetLastError();
}

}  // namespace flex
