// Exact causal attention over packed sequences, forward: prompts (k_attn_fwd) and
// few rows against long key sequences (k_attn_split, k_attn_combine).
#include "flex_seq.hpp"
#include "flex_seq_kernels.hpp"
#include "../../include/flex.h"

namespace flex {

namespace {

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;
constexpr int BM = 128;   // query rows per workgroup of the prompt kernel, 32 per wave

// One query column's running softmax over a block of 32 key rows: s holds the
// products q.k (masked ones -inf) and becomes exp2(sl2 (s - max)).  Returns the
// factor for what was summed under the old maximum.
struct Soft {
  float m = -INFINITY, l = 0.f;   // running maximum of q.k, this lane half's sum
  template <class T, int NB>
  __device__ __forceinline__ float step(f32x16 (&s)[NB], float sl2) {
    float mx = s[0][0];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[b][e]);
    const float mn = fmaxf(m, half_max(mx));
    // a row that has seen no key yet: every product is -inf, exp2(-inf) = 0
    const float ref = mn == -INFINITY ? 0.f : mn;
    const float alpha = __builtin_amdgcn_exp2f((m - ref) * sl2);
    const float off = ref * sl2;
    float sum = 0.f;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        // bf16 rows: one instruction, off by half a step of the larger term (far
        // under the probability's rounding); fp32 rows: the exact difference first
        s[b][e] = __builtin_amdgcn_exp2f(IsBf16<T>::value ? __builtin_fmaf(s[b][e], sl2, -off) : (s[b][e] - ref) * sl2);
        sum += s[b][e];
      }
    l = l * alpha + sum;
    m = mn;
    return alpha;
  }
};

// The sums of a wave over the keys that each query sees, again (final maximum m, lane limits lim): blocks of 32 keys
// lo, lo + step .. below hi as products where every query sees every key (up to lim_lo), and one key at a time in the
// others, 95 keys at most, where that can change anything.  With a NaN that all its queries see, a call takes three times
// as long so (8192 tokens, 8 heads of 64: 148 and 476 us; one key at a time for all of them 4670).
template <class T, int D>
__device__ __forceinline__ void sum_seen(f32x16 (&o)[D / 32], const Frag<T> (&q)[D / 16],
                                         const typename Io<T>::type* K, const typename Io<T>::type* V, int ks, int vs,
                                         int lo, int step, int hi, int lim_lo, int lim, bool valid, float m, float sl2) {
#pragma unroll
  for (int d = 0; d < D / 32; ++d) o[d] = zero16();
  auto qs = [&](int i) { return q[i]; };
#pragma unroll 1
  for (int j0 = lo; j0 < hi; j0 += step) {
    if (j0 + 32 <= lim_lo) {
      f32x16 s = rare_products<T, D>(K + (size_t)j0 * ks, ks, qs);
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = __builtin_amdgcn_exp2f((s[e] - m) * sl2);
      rare_add<T, D>(o, V + (size_t)j0 * vs, vs, s);
      continue;
    }
    if (__all(!valid || none_finite(o))) break;
#pragma unroll 1
    for (int j = j0; j < min(j0 + 32, hi); ++j) {
      const float s = rare_product<T, D>(K + (size_t)j * ks, qs);
      rare_add<T, D>(o, V + (size_t)j * vs, __builtin_amdgcn_exp2f((s - m) * sl2), j < lim);
    }
  }
}

}  // namespace

// Prompts.  One workgroup: 128 queries of one head, 32 per wave (in registers as
// the right operand of S^T = K Q^T); K and V in tiles of KT rows, double-buffered in
// LDS.  O^T = V^T P^T accumulates in registers, one lane per query.
// Bound by the matrix cores and the exponentials beside them: at 16384 tokens, 16 heads of 128 on 2, 1061 us
// (1.04 PFLOP/s of the seen half; the matrix cores are busy 55 % of the cycles), at 17973
// ragged tokens, 16 heads of 64 on 4, 96 us (575 TFLOP/s: half the products per exponential).
// Two waves per SIMD fill each other's gaps: the next tile's S ahead of this one's P V
// measured the same at 128 and 6 % more at 64.
template <class T, int D, int KT>
__global__ __launch_bounds__(256)
    __attribute__((amdgpu_waves_per_eu(RowTile<T, D>::ROW > 256 ? 1 : RowTile<T, D>::ROW > 128 ? 2 : 4))) void k_attn_fwd(
        AttnArgs a) {
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
  const int kvh = __builtin_amdgcn_readfirstlane(tc.head / (a.Hq / a.Hkv));   // in a scalar register, with the rows' addresses
  const SeqRange kr = seq_range(a.k_off, t.b, a.Tk, a.k_len);
  const int rows = min(BM, t.n - t.tile * BM), first = t.tile * BM + 32 * w, shift = kr.n - t.n;
  const int qi = first + c;
  // keys that this lane's query, the wave's first and last, and the workgroup's last see
  const int lim = a.causal ? min(kr.n, qi + shift + 1) : kr.n;
  const int lim_lo = a.causal ? min(kr.n, first + shift + 1) : kr.n;
  const int lim_hi = a.causal ? min(kr.n, first + 32 + shift) : kr.n;
  const int lim_wg = a.causal ? min(kr.n, t.tile * BM + rows + shift) : kr.n;
  const int ntiles = max(lim_wg + KT - 1, 0) / KT;

  Frag<T> q[KS];
  {
    const auto rs = row_window(static_cast<const S*>(a.Q) + tc.head * D, t.row0 + t.tile * BM, a.qs, rows, D);
#pragma unroll
    for (int s = 0; s < KS; ++s) q[s] = window_frag<T>(rs, ((32 * w + c) * a.qs + 16 * s + 8 * h) * (int)sizeof(S));
  }
  f32x16 o[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i) o[i] = zero16();
  Soft sm;
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
    const int j0 = i * KT;
    if (j0 >= lim_hi) continue;
    f32x16 s[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      s[b] = zero16();
#pragma unroll
      for (int k = 0; k < KS; ++k) mma32(s[b], RT::row(LK, 32 * b + c, k, h), q[k]);
    }
    if (j0 + KT > lim_lo) {
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (j0 + 32 * b + res_row(e, h) >= lim) s[b][e] = -INFINITY;
    }
    const float alpha = sm.template step<T>(s, sl2);
    if (__any(alpha != 1.f)) {
#pragma unroll
      for (int d = 0; d < DT; ++d) o[d] *= alpha;
    }
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const Frag<T> p = frag_of<T>(s[b], k);
#pragma unroll
        for (int d = 0; d < DT; ++d) mma32(o[d], RT::col(LV, 32 * b + 16 * k + 4 * h, 32 * d), p);
      }
  }
  if (__builtin_expect(a.causal && __any(qi < t.n && not_finite(o)), 0))
    sum_seen<T, D>(o, q, K + (size_t)kr.row0 * a.ks, V + (size_t)kr.row0 * a.vs, a.ks, a.vs, 0, 32, lim_hi, lim_lo, lim,
                   qi < t.n, sm.m, sl2);
  if (qi >= t.n) return;
  const float l_all = half_sum(sm.l);
  const float inv = l_all > 0.f ? 1.f / l_all : (l_all == 0.f ? 0.f : l_all);   // no key: zeros; NaN stays
  const size_t row = (size_t)(t.row0 + qi) * a.Hq + tc.head;
  S* out = static_cast<S*>(a.O) + row * D;
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int e = 0; e < 16; e += 4)
      store_io4(out + 32 * d + res_row(e, h),
                f32x4{o[d][e] * inv, o[d][e + 1] * inv, o[d][e + 2] * inv, o[d][e + 3] * inv});
  if (a.lse && h == 0) a.lse[row] = l_all == 0.f ? -INFINITY : sm.m * a.scale + __logf(l_all);
}

// Blocks of 32 rows (queries times the `grp` heads that share a key head) in slots: the first B are the
// sequences' first blocks, so that single tokens need no search and what has no block comes
// last; those behind a sequence's first start at slot B + off grp / 32, which leaves room for any lengths.
// (One workgroup for all blocks of a sequence: 965 us for a prompt of 2000 among 63 single tokens with 8
// heads of 64, these 64.  A slot that may be empty next to each full one cost 18 of 55 us: a
// workgroup takes a CU's LDS, and the full one behind it waits.)
struct RowBlock {
  int b, block;
};
inline int block_slots(int T, int B, int grp) { return B + (T > 0 ? (T * grp - 1) / 32 : 0); }
__device__ __forceinline__ RowBlock find_block(const int32_t* __restrict__ off, int B, int T, int grp, int slot) {
  if (slot < B) return {slot, 0};
  const int e = slot - B;
  // sequences whose further blocks start by here
  const int cnt = leading(B, [=](int b) { return clamp_off(off[b], T) * grp / 32 <= e; });
  const int b = max(cnt - 1, 0), k = e - clamp_off(off[b], T) * grp / 32;
  return {__builtin_amdgcn_readfirstlane(b), __builtin_amdgcn_readfirstlane(k < 0 ? 1 << 25 : k + 1)};
}

// Few rows against many keys.  One workgroup: 32 rows of a sequence, one key head and one
// part of its keys; the columns are the rows of all the query heads that share it
// (row r: query r / group, head r % group).  Its waves take every fourth block of
// 32 keys, each through its own LDS, without a barrier, and join at the end.
// Bound by the reads of K and V: 64 tokens against 253385 rows in use, 2 key heads of 128 (262 MB), 45 us, 5.8
// TB/s with part of it from the last-level cache; one against 40000, 4 key heads (82 MB), 17.6.
template <class T, int D>
__global__ __launch_bounds__(256) void k_attn_split(AttnArgs a) {
  using S = typename Io<T>::type;
  using RT = RowTile<T, D>;
  constexpr int KS = D / 16, DT = D / 32;
  constexpr int TILE = 32 * RT::ROW;
  // two tiles of K and V per wave (fp32 rows of 128: one, all that fits)
  constexpr int BUFS = RT::ROW > 256 ? 1 : 2;
  __shared__ __attribute__((aligned(16))) char dyn[4 * BUFS * 2 * TILE];
  __shared__ float ml[4 * 32 * 2 + 32 * 2];   // statistics of each wave, then of the part
  static_assert(sizeof(dyn) >= 4 * 32 * (D + 4) * sizeof(float), "room to join the waves");
  const int l = threadIdx.x % WAVE, c = l % 32, h = l / 32;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
  const int grp = a.Hq / a.Hkv;
  const int part = blockIdx.x % a.nsplit, id = blockIdx.x / a.nsplit;
  const int kvh = id % a.Hkv;
  const RowBlock rb = find_block(a.q_off, a.B, a.Tq, grp, id / a.Hkv);
  const SeqRange qr = seq_range(a.q_off, rb.b, a.Tq);
  const int q0 = qr.row0, nq = qr.n, r0 = 32 * rb.block;
  if (r0 >= nq * grp) return;
  const SeqRange kr = seq_range(a.k_off, rb.b, a.Tk, a.k_len);
  const int per = ((kr.n + a.nsplit - 1) / a.nsplit + 127) / 128 * 128;
  const int shift = kr.n - nq, lo = min(part * per, kr.n);
  // the part's end: at the last key that one of the rows sees
  const int hi = min(min(lo + per, kr.n), a.causal ? min(r0 + 31, nq * grp - 1) / grp + shift + 1 : kr.n);
  const float sl2 = a.scale * LOG2E;
  const S* K = static_cast<const S*>(a.K) + kvh * D;
  const S* V = static_cast<const S*>(a.V) + kvh * D;
  char* mine = dyn + w * BUFS * 2 * TILE;

  const int r = r0 + c, qi = r / grp, head = kvh * grp + r % grp;
  const bool valid = r < nq * grp;
  const int lim = a.causal ? min(hi, qi + shift + 1) : hi;
  const int lim_lo = a.causal ? min(hi, r0 / grp + shift + 1) : hi;
  Frag<T> q[KS];
  const S* qrow = static_cast<const S*>(a.Q) + (valid ? (size_t)(q0 + qi) * a.qs + head * D : 0);
#pragma unroll
  for (int s = 0; s < KS; ++s) load8(q[s], qrow + 16 * s + 8 * h, valid);
  f32x16 o[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i) o[i] = zero16();
  Soft sm;
  auto stage = [&](int j0, int buf) {
    char* L = mine + buf * 2 * TILE;
    const int n = min(hi - j0, 32);   // of a tile: the bytes of a long sequence pass 32 bits
    stage_tile<T, D, 32, 1>(L, row_words(K, kr.row0 + j0, a.ks, n, D), a.ks * (int)sizeof(S), 0);
    stage_tile<T, D, 32, 1>(L + TILE, row_words(V, kr.row0 + j0, a.vs, n, D), a.vs * (int)sizeof(S), 0);
  };
  int buf = 0;
  const int start = lo + 32 * w;
  if (BUFS == 2 && start < hi) stage(start, 0);
  wait_reg_loads();
  for (int j0 = start; j0 < hi; j0 += 128) {
    if (BUFS == 1) {
      wait_lds_loads();
      stage(j0, 0);
    }
    wait_lds_loads();
    if (BUFS == 2 && j0 + 128 < hi) stage(j0 + 128, buf ^ 1);
    const char* LK = mine + buf * 2 * TILE;
    const char* LV = LK + TILE;
    f32x16 s[1];
    s[0] = zero16();
#pragma unroll
    for (int k = 0; k < KS; ++k) mma32(s[0], RT::row(LK, c, k, h), q[k]);
    if (j0 + 32 > lim_lo) {
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (j0 + res_row(e, h) >= lim) s[0][e] = -INFINITY;
    }
    const float alpha = sm.template step<T>(s, sl2);
    if (__any(alpha != 1.f)) {
#pragma unroll
      for (int d = 0; d < DT; ++d) o[d] *= alpha;
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const Frag<T> p = frag_of<T>(s[0], k);
#pragma unroll
      for (int d = 0; d < DT; ++d) mma32(o[d], RT::col(LV, 16 * k + 4 * h, 32 * d), p);
    }
    if (BUFS == 2) buf ^= 1;
  }
  if (__builtin_expect(a.causal && __any(valid && not_finite(o)), 0))
    sum_seen<T, D>(o, q, K + (size_t)kr.row0 * a.ks, V + (size_t)kr.row0 * a.vs, a.ks, a.vs, start, 128, hi, lim_lo, lim,
                   valid, sm.m, sl2);
  // join the four waves: statistics, then the scaled sums through LDS
  const float lw = half_sum(sm.l);
  __syncthreads();
  if (h == 0) {
    ml[(w * 32 + c) * 2] = sm.m;
    ml[(w * 32 + c) * 2 + 1] = lw;
  }
  __syncthreads();
  float m_all = -INFINITY, l_all = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) m_all = fmaxf(m_all, ml[(i * 32 + c) * 2]);
  const float ref = m_all == -INFINITY ? 0.f : m_all;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    l_all += ml[(i * 32 + c) * 2 + 1] * __builtin_amdgcn_exp2f((ml[(i * 32 + c) * 2] - ref) * sl2);
  const float f = __builtin_amdgcn_exp2f((sm.m - ref) * sl2);
  float* acc = reinterpret_cast<float*>(dyn);   // [4 waves][32 columns][D + 4]
  constexpr int LD = D + 4;
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int e = 0; e < 16; e += 4)
      *reinterpret_cast<f32x4*>(acc + (w * 32 + c) * LD + 32 * d + res_row(e, h)) =
          f32x4{o[d][e] * f, o[d][e + 1] * f, o[d][e + 2] * f, o[d][e + 3] * f};
  float* tot = ml + 256;   // [32][2]: maximum and sum of this part
  if (threadIdx.x < 32) {
    tot[2 * c] = m_all;
    tot[2 * c + 1] = l_all;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 32 * (D / 4); i += 256) {
    const int col = i / (D / 4), d = i % (D / 4) * 4, rr = r0 + col;
    if (rr >= nq * grp) break;
    f32x4 v = *reinterpret_cast<const f32x4*>(acc + col * LD + d);
#pragma unroll
    for (int k = 1; k < 4; ++k) v += *reinterpret_cast<const f32x4*>(acc + (k * 32 + col) * LD + d);
    const size_t row = (size_t)(q0 + rr / grp) * a.Hq + kvh * grp + rr % grp;
    const float m_row = tot[2 * col], l_row = tot[2 * col + 1];
    if (a.nsplit == 1) {
      const float inv = l_row == 0.f ? 0.f : 1.f / l_row;
      store_io4(static_cast<S*>(a.O) + row * D + d, v * inv);
      if (a.lse && d == 0) a.lse[row] = l_row == 0.f ? -INFINITY : m_row * a.scale + __logf(l_row);
    } else {
      *reinterpret_cast<f32x4*>(a.part_o + (row * a.nsplit + part) * D + d) = v;
      if (d == 0) {
        a.part_ml[(row * a.nsplit + part) * 2] = m_row;
        a.part_ml[(row * a.nsplit + part) * 2 + 1] = l_row;
      }
    }
  }
}

// Joins the parts of k_attn_split: one workgroup per row, D / 4 lanes across and 1024 / D
// groups of lanes that take the parts in turn, added up in a fixed order.  (One group for all parts
// of a row waited out a memory latency per part: 67 us for 156 parts, where the parts themselves
// took 20.)
template <class T, int D>
__global__ __launch_bounds__(256) void k_attn_combine(AttnArgs a) {
  using S = typename Io<T>::type;
  constexpr int L4 = D / 4, G = 256 / L4;
  __shared__ float fac[ATTN_PARTS];
  __shared__ __attribute__((aligned(16))) f32x4 acc[G][L4];
  __shared__ float red[8];
  const size_t row = blockIdx.x;
  const int t = threadIdx.x, c = t % L4, grp = t / L4;
  const int q = (int)(row / a.Hq);
  if (q < clamp_off(a.q_off[0], a.Tq) || q >= clamp_off(a.q_off[a.B], a.Tq)) return;
  const float* ml = a.part_ml + row * a.nsplit * 2;
  const float* po = a.part_o + row * a.nsplit * D + 4 * c;
  const float sl2 = a.scale * LOG2E;
  const int n = a.nsplit;   // at most ATTN_PARTS, a thread each
  const float m_t = t < n ? ml[2 * t] : -INFINITY, l_t = t < n ? ml[2 * t + 1] : 0.f;
  float m = m_t;
#pragma unroll
  for (int s = 1; s < WAVE; s *= 2) m = fmaxf(m, __shfl_xor(m, s));
  if (t % WAVE == 0) red[t / WAVE] = m;
  __syncthreads();
  m = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
  const float ref = m == -INFINITY ? 0.f : m;
  const float f_t = __builtin_amdgcn_exp2f((m_t - ref) * sl2);
  if (t < n) fac[t] = f_t;
  float sum = l_t * f_t;
  sum = group_sum(lane_sum<16>(sum));
  if (t % WAVE == 0) red[4 + t / WAVE] = sum;
  __syncthreads();
  sum = (red[4] + red[5]) + (red[6] + red[7]);
  f32x4 v = zero4();
#pragma unroll 4
  for (int i = grp; i < n; i += G) v += *reinterpret_cast<const f32x4*>(po + (size_t)i * D) * fac[i];
  acc[grp][c] = v;
  __syncthreads();
  if (grp != 0) return;
#pragma unroll
  for (int i = 1; i < G; ++i) v += acc[i][c];
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  store_io4(static_cast<S*>(a.O) + row * D + 4 * c, v * inv);
  if (a.lse && c == 0) a.lse[row] = sum == 0.f ? -INFINITY : m * a.scale + __logf(sum);
}

namespace {
template <class T, int D>
hipError_t run_fwd(const AttnArgs& a, hipStream_t st) {
  timing_mark(FLEX_KERNEL_ATTN_FWD, st, true);
  if (a.nsplit > 0) {
    k_attn_split<T, D><<<block_slots(a.Tq, a.B, a.Hq / a.Hkv) * a.Hkv * a.nsplit, 256, 0, st>>>(a);
    if (a.nsplit > 1) {
      k_attn_combine<T, D><<<(unsigned)((size_t)a.Tq * a.Hq), 256, 0, st>>>(a);
    }
  } else {
    constexpr int KT = sizeof(T) == 4 && D == 128 ? 32 : 64;
    k_attn_fwd<T, D, KT><<<seq_slots(a.Tq, a.B, BM) * a.Hq, 256, 0, st>>>(a);
  }
  timing_mark(FLEX_KERNEL_ATTN_FWD, st, false);
  return hipGetLastError();
}
}  // namespace

hipError_t launch_attn_fwd(const AttnArgs& a, bool bf16, int d, hipStream_t st) {
  if (bf16) return d == 32 ? run_fwd<__bf16, 32>(a, st) : d == 64 ? run_fwd<__bf16, 64>(a, st) : run_fwd<__bf16, 128>(a, st);
  return d == 32 ? run_fwd<float, 32>(a, st) : d == 64 ? run_fwd<float, 64>(a, st) : run_fwd<float, 128>(a, st);
}

}  // namespace flex
