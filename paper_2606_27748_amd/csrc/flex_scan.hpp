// Device building blocks of the selective scan's kernels.
//
//   S_t = e^{g_t} S_{t-1} + dt_t B_t x_t^T,   y_t = S_t^T C_t + D x_t
//
// In chunks of 64 tokens, L the inclusive sum of g within the chunk and S [N x P] the state at its start:
//   P_ij = e^{L_i - L_j} (C_i.B_j) dt_j (j <= i)     y = P x + e^L (C S) + D x
//   S <- e^{L_63} S + B^T (w x),                     w_j = e^{L_63 - L_j} dt_j
//
// A wave has 32 columns of a head's state in registers, as 32 x 32 results with the rows n and a lane per
// column.  Both matrix operands have the same layout (a row or column per lane, eight contraction indices in
// its slots), so a result whose rows are the next product's contraction is that product's operand as it is, on
// either side: S -> C S, C B^T -> P, without a pass through LDS.
// Rows of a result are dealt so that the eight a lane holds of a step of 16 are consecutive (perm32): element e
// of lane half h of a 32-row tile is row 16 (e / 8) + 8 h + e % 8.  A row operand is then read 16 bytes at once,
// and a lane's results are stored 16 bytes at once.
#pragma once
#include <type_traits>
#include "flex_seq.hpp"
#include "flex_rows.hpp"
#include "flex_layer_kernels.hpp"

namespace flex {

constexpr int SC = SCAN_CHUNK;

// the row (or column) of 32 that lane r % 32 of an operand stands for, so that results come as above
__device__ __forceinline__ constexpr int perm32(int r) { return (r & 16) | ((r >> 2) & 1) << 3 | ((r >> 3) & 1) << 2 | (r & 3); }
// row of a tile that element e of lane half h of a result of permuted rows is
__device__ __forceinline__ constexpr int perm_row(int e, int h) { return 16 * (e / 8) + 8 * h + e % 8; }

template <class T, int D>
struct ScanTile : RowTile<T, D> {
  using R = RowTile<T, D>;
  // RowTile::row: the places of the steps differ by bits that are turned over
  static __device__ __forceinline__ Frag<T> row(const char* L, int r, int s, int h) {
    Frag<T> f;
    if constexpr (IsBf16<T>::value) {
      const int lane = (h ^ R::swz(r)) << 4;
      f.v = *reinterpret_cast<const bf16x8*>(L + r * R::ROW + (lane ^ (s << 5)));
      return f;
    } else {
      return R::row(L, r, s, h);
    }
  }
  // Columns m0 + perm32(l % 32) for lane l, slots 0..3 the rows r0 .. r0+3, slots 4..7 r1 .. r1+3
  static __device__ __forceinline__ Frag<T> colp(const char* L, int r0, int r1, int m0, int l = threadIdx.x % WAVE) {
    Frag<T> f;
    if constexpr (IsBf16<T>::value) {
      // the lane's part of the read: row i / 4, of the 16 columns the quarter that place i % 4 takes
      const int i = l % 16, q = (i & 1) << 1 | (i >> 1 & 1);
      const int m = m0 + 16 * ((l / 16) & 1) + 4 * q, c = m / 8, o = (m % 8) * 2;
      const tr_v4i16 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_tr_v4i16*)(L + R::at(r0 + i / 4, c) + o));
      const tr_v4i16 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_tr_v4i16*)(L + R::at(r1 + i / 4, c) + o));
      f.v = __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
      const int m = m0 + perm32(l % 32), c = m / 4, o = (m % 4) * 4;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        f.v[j] = *reinterpret_cast<const float*>(L + R::at(r0 + j, c) + o);
        f.v[4 + j] = *reinterpret_cast<const float*>(L + R::at(r1 + j, c) + o);
      }
    }
    return f;
  }
};

// States [32 columns p][N] as the sweeps' lanes hold them: of step s the 64 lanes' eight elements, 16 bytes a lane in a
// row (fp32: twice), so that a store of them is 1 KB in a row.  Lanes of the upper half lie four places
// off, for the banks of a transposed read.
template <class T, int N>
struct StateRows {
  using S = typename Io<T>::type;
  static constexpr int E = 16 / sizeof(T), FRAG = WAVE * 8 * (int)sizeof(T), BLOCK = N / 16 * FRAG;   // bytes of 32 columns
  static __device__ __forceinline__ int place(int r, int h) { return h * 32 + (r ^ (4 * h)); }
  static __device__ __forceinline__ void store(S* base, int s, const Frag<T>& f) {
    const int l = threadIdx.x % WAVE;
    S* p = base + s * (FRAG / (int)sizeof(S)) + place(l % 32, l / 32) * E;
    if constexpr (IsBf16<T>::value) {
      *reinterpret_cast<bf16x8*>(p) = f.v;
    } else {
      *reinterpret_cast<f32x4*>(p) = f32x4{f.v[0], f.v[1], f.v[2], f.v[3]};
      *reinterpret_cast<f32x4*>(p + WAVE * E) = f32x4{f.v[4], f.v[5], f.v[6], f.v[7]};
    }
  }
  // bytes to column p of (several blocks of) 32, elements n .. of 16 bytes
  static __device__ __forceinline__ int at(int p, int n) {
    return p / 32 * BLOCK + n / 16 * FRAG + n % 8 / E * (WAVE * 16) + place(perm32(p % 32), n / 8 % 2) * 16 + n % E * (int)sizeof(T);
  }
  // the operand with lane l % 32 column p0 + perm32(l % 32) and the slots 16 s + 8 h ..
  static __device__ __forceinline__ Frag<T> row(const char* L, int p0, int s, int l) {
    const char* q = L + p0 / 32 * BLOCK + s * FRAG + place(l % 32, l / 32) * 16;
    Frag<T> f;
    if constexpr (IsBf16<T>::value) {
      f.v = *reinterpret_cast<const bf16x8*>(q);
    } else {
      const f32x4 a = *reinterpret_cast<const f32x4*>(q), b = *reinterpret_cast<const f32x4*>(q + WAVE * 16);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        f.v[j] = a[j];
        f.v[4 + j] = b[j];
      }
    }
    return f;
  }
  // the same of the slots columns 16 s + 8 h .., h = l / 32, n0 a multiple of 32: one place of the lane's for all s and n0
  static __device__ __forceinline__ Frag<T> steps(const char* L, int s, int n0, int l) {
    if constexpr (IsBf16<T>::value) {
      Frag<T> f;
      // at(16 s + 8 h + 4 k + i / 4, n0 + 16 b + 4 q), as the sum of what the lane has and what s, k and n0 have
      const int i = l % 16, b = l / 16 % 2, h = l / 32, hh = i & 1;
      const char* p = L + n0 / 16 * FRAG + s / 2 * BLOCK + s % 2 * 256 + (b * FRAG + hh * 512 + (h ^ hh) * 64 + i / 4 * 16 + (i / 2 & 1) * 8);
      const tr_v4i16 u = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_tr_v4i16*)p);
      const tr_v4i16 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_tr_v4i16*)(p + 128));
      f.v = __builtin_bit_cast(bf16x8, __builtin_shufflevector(u, v, 0, 1, 2, 3, 4, 5, 6, 7));
      return f;
    } else {
      return colp(L, 16 * s + 8 * (l / 32), n0, l);
    }
  }
  // the operand with lane l % 32 element n0 + perm32(l % 32) and the slots columns p .. p + 7
  static __device__ __forceinline__ Frag<T> colp(const char* L, int p, int n0, int l) {
    Frag<T> f;
    if constexpr (IsBf16<T>::value) {
      const int i = l % 16, q = (i & 1) << 1 | (i >> 1 & 1), n = n0 + 16 * ((l / 16) & 1) + 4 * q;
      const tr_v4i16 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_tr_v4i16*)(L + at(p + i / 4, n)));
      const tr_v4i16 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_tr_v4i16*)(L + at(p + 4 + i / 4, n)));
      f.v = __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) f.v[j] = *reinterpret_cast<const float*>(L + at(p + j, n0 + perm32(l % 32)));
    }
    return f;
  }
};

// Stages 64 rows of a window by `nw` waves of which this is w, 16 rows at a time.
template <class T, int D>
__device__ __forceinline__ void stage_rows(const char* L, const typename Io<T>::type* base, size_t row0, int stride, int n, int w,
                                           int nw) {
  for (int k = w; k < 4; k += nw)
    stage_tile<T, D, 16, 1>(L + k * 16 * D * (int)sizeof(T), row_words(base, row0 + 16 * k, stride, n - 16 * k, D),
                            stride * (int)sizeof(T), 0);
}

// Lanes (column l % 32) for which element e of a tile is a row from their column on, or behind it
struct DiagonalMasks {
  uint64_t from[16] = {}, behind[16] = {};
  constexpr DiagonalMasks() {
    for (int e = 0; e < 16; ++e)
      for (int l = 0; l < 64; ++l) {
        const int row = 8 * (e / 4) + 4 * (l / 32) + e % 4;
        from[e] |= (uint64_t)(row >= l % 32) << l;
        behind[e] |= (uint64_t)(row > l % 32) << l;
      }
  }
};
constexpr DiagonalMasks DIAGONAL;
// x in the lanes of a mask, else 0.  A mask that is a constant costs a scalar instruction: as conditions that the compiler
// keeps over a loop, 32 masks do not fit the scalar registers.
__device__ __forceinline__ float keep_lanes(float x, uint64_t lanes) { return __builtin_amdgcn_inverse_ballot_w64(lanes) ? x : 0.f; }

// the value of lane l ^ M, M 1 or 2
template <int M>
__device__ __forceinline__ float lane_xor(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), M == 1 ? 0xB1 : 0x4E, 0xF, 0xF, false));
}
// sum over the lanes of a row of 16 with the same place in four, in each of them
__device__ __forceinline__ float row_sum4(float x) {
  x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x124, 0xF, 0xF, false));   // rotated by 4
  x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x128, 0xF, 0xF, false));   // and by 8
  return x;
}

// Inclusive sum over the lanes of a wave.
__device__ __forceinline__ double wave_scan(double x) {
  auto step = [&](auto ctrl, auto rows) {
    const uint64_t v = __builtin_bit_cast(uint64_t, x);
    constexpr bool whole = decltype(rows)::value == 0xf;   // lanes without a source have a zero, without an instruction for it
    const unsigned lo = __builtin_amdgcn_update_dpp(0, (int)(unsigned)v, decltype(ctrl)::value, decltype(rows)::value, 0xf, whole);
    const unsigned hi = __builtin_amdgcn_update_dpp(0, (int)(unsigned)(v >> 32), decltype(ctrl)::value, decltype(rows)::value, 0xf, whole);
    x += __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
  };
  using std::integral_constant;
  step(integral_constant<int, 0x111>{}, integral_constant<int, 0xf>{});   // from 1, 2, 4, 8 lanes before within 16
  step(integral_constant<int, 0x112>{}, integral_constant<int, 0xf>{});
  step(integral_constant<int, 0x114>{}, integral_constant<int, 0xf>{});
  step(integral_constant<int, 0x118>{}, integral_constant<int, 0xf>{});
  step(integral_constant<int, 0x142>{}, integral_constant<int, 0xa>{});   // lane 15 of the 16 before
  step(integral_constant<int, 0x143>{}, integral_constant<int, 0xc>{});   // lane 31
  return x;
}
__device__ __forceinline__ double lane_of(double x, int lane) {
  const uint64_t v = __builtin_bit_cast(uint64_t, x);
  const unsigned lo = __builtin_amdgcn_readlane((int)(unsigned)v, lane), hi = __builtin_amdgcn_readlane((int)(unsigned)(v >> 32), lane);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// A chunk's decays, lane = token.  Sums of g in 64 bits, in units of log2 as two floats, so that differences of
// them are as exact as floats are.  Bf16 rows take the first float alone: a difference is then off by 2^-24 of the
// larger sum, e^{L_i - L_j} by less than a rounding to bf16 up to sums of 2^16.  A decay of zero (g = -inf) is kept as a
// finite sum whose exponential is zero and that no growth within a chunk makes up for, so that the differences are
// defined.
constexpr float SCAN_MIN_G = -1e3f;
struct Decay {
  double L, end;    // the token's, and the chunk's, in units of log2
  float hi, lo;     // the token's
  __device__ __forceinline__ explicit Decay(float g) {
    if (g < SCAN_MIN_G) g = SCAN_MIN_G;
    L = wave_scan((double)g * 1.4426950408889634);
    end = lane_of(L, WAVE - 1);
    hi = (float)L;
    lo = (float)(L - (double)hi);
  }
  __device__ __forceinline__ float from_start() const { return __builtin_amdgcn_exp2f(hi); }
  __device__ __forceinline__ float to_end() const { return __builtin_amdgcn_exp2f((float)(end - L)); }
};
// e^{L_i - L_j}
template <bool ONE>
__device__ __forceinline__ float decay(float hi_i, float lo_i, float hi_j, float lo_j) {
  return __builtin_amdgcn_exp2f(ONE ? hi_i - hi_j : (hi_i - hi_j) + (lo_i - lo_j));
}

// Stores 32 tokens of 32 columns from results of permuted rows (a lane per token, element e the column perm_row(e, h)):
// o(s, j) the lane's values 8 s + j.  Of bf16 rows the lanes trade places first, so that a store
// has whole rows of 64 bytes and not halves of twice as many.
template <class T, class F>
__device__ __forceinline__ void store_rows(__amdgpu_buffer_rsrc_t rs, int tok0, int stride, F o) {
  const int l = threadIdx.x % WAVE;
  if constexpr (IsBf16<T>::value) {
    u32x4 v[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      Frag<T> f;
#pragma unroll
      for (int j = 0; j < 8; ++j) f.set(j, o(s, j));
      v[s] = __builtin_bit_cast(u32x4, f.v);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {   // lanes 16 .. 31 (48 .. 63) of the first with 0 .. 15 (32 .. 47) of the second
      const auto p = __builtin_amdgcn_permlane16_swap(v[0][k], v[1][k], false, false);
      v[0][k] = p[0];
      v[1][k] = p[1];
    }
#pragma unroll
    for (int k = 0; k < 2; ++k)
      __builtin_amdgcn_raw_buffer_store_b128(v[k], rs, (tok0 + 16 * k + l % 16) * stride * 2 + (l / 16 % 2) * 32 + l / 32 * 16, 0, 0);
  } else {
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int k = 0; k < 2; ++k)
        __builtin_amdgcn_raw_buffer_store_b128(
            __builtin_bit_cast(u32x4, f32x4{o(s, 4 * k), o(s, 4 * k + 1), o(s, 4 * k + 2), o(s, 4 * k + 3)}), rs,
            (tok0 + l % 32) * stride * 4 + 64 * s + 32 * (l / 32) + 16 * k, 0, 0);
  }
}

// The work of a workgroup of a sweep: a segment of a sequence (tokens t0 .. of it) and a set of heads of one group.
// Consecutive workgroups go round-robin to the XCDs, and so do the sets of a segment: each XCD has a share of
// every segment.  (An XCD with all sets of its segments reads the rows of B and C once, but the last round of
// segments leaves some XCDs without work.)
struct SegTile {
  int b, row0, n;     // sequence (-1: none), first row and length of it
  int index, count;   // which of how many segments
  int slot, set;
};
__device__ __forceinline__ SegTile find_segment(const int32_t* __restrict__ off, int B, int T, int seg, int sets) {
  SegTile t;
  t.slot = blockIdx.x / sets;
  t.set = blockIdx.x % sets;
  t.b = -1;
  t.row0 = t.n = t.index = t.count = 0;
  const int slot = t.slot;
  const int cnt = leading(B, [=](int b) { return clamp_off(off[b], T) / seg + b <= slot; });
  if (cnt == 0) return t;
  const SeqRange r = seq_range(off, cnt - 1, T);
  t.row0 = r.row0;
  t.n = r.n;
  t.index = slot - (r.row0 / seg + cnt - 1);
  t.count = max(1, (r.n + seg - 1) / seg);   // a sequence without tokens has one, for its state
  if (t.index >= 0 && t.index < t.count) t.b = __builtin_amdgcn_readfirstlane(cnt - 1);
  t.index = __builtin_amdgcn_readfirstlane(t.index);
  t.count = __builtin_amdgcn_readfirstlane(t.count);
  return t;
}
}  // namespace flex
