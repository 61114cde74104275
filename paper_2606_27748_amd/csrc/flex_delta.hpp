// Device building blocks of the gated delta rule's kernels.
//
//   S_t = a_t S_{t-1} + b_t k_t (v_t - a_t S_{t-1}^T k_t)^T,  a_t = exp(g_t),  o_t = scale S_t^T q_t
//
// In chunks of 64 tokens, G the inclusive sum of g within the chunk, D_ij = exp(G_i - G_j) and
// S the state at the chunk's start (S [d x dv], K, Q [64 x d], V, U, O [64 x dv]):
//   A_ij = b_i D_ij k_i.k_j (j < i)    T = (I + A)^-1        P_ij = D_ij q_i.k_j (j <= i)
//   U = T b (V - e^G K S)              O = scale (e^G Q S + P U)
//   S <- e^{G_63} S + K^T (w U),       w_j = exp(G_63 - G_j)
// T, P, e^G, w and b of every chunk and value head are formed first, for all chunks at once
// (k_delta_prep); what remains in sequence is the sweep over the state.
//
// The sweeps give a wave 16 columns of the state, in registers for the whole sequence
// ([d x 16] as 16 x 16 tiles: lane l holds column l % 16 and rows 4 g + e, g = l / 16).  A
// result in that layout is the right operand of the next product as it is, so K S -> U ->
// K^T U -> S never leaves the wave.  Rows (of d, and of tokens) are dealt to the tiles so
// that the eight rows a lane holds of a pair of tiles are consecutive: row 4g + e of tile m is
// 32 (m / 2) + 8 g + 4 (m % 2) + e (tile_row).  The other operand is then read 16 bytes at once.
//
// Precision, bf16 rows: K, Q, V, dO are exact operands.  States, U, T and the like are
// fp32 and enter products as two bf16 terms (16 bits), so a carried state is right to
// about 2^-17 of its terms.  What only the gradients read is kept as one bf16 term, half the
// bytes that the sweeps write: S and dS of each chunk, and dP D and M for the rows that follow.  Those
// roundings (2^-8) come before the sums of a gradient, of which some cancel (dg, dbeta, dK): they
// scale with its terms, and in <S, dS> of dg both factors have one.
#pragma once
#include "flex_seq.hpp"
#include "flex_seq_kernels.hpp"

namespace flex {

constexpr int DC = DELTA_CHUNK;

// Waves of a sweep's workgroup that stage its chunks.  Two, although loads of one wave alone move 18 bytes a
// clock from L2, of two 27, of four 40: four hold up the carrying waves' SIMDs and the stores.  us of
// the forward and reverse sweeps at d = 128, 32 heads, 8192 tokens with one, two and four: 279, 260,
// 296 and 281, 284, 316; the forward over 9 ragged prompts 126, 127, 124.
constexpr int NL = 2;

// Workgroup of a sweep -> sequence and value head, and which of `parts` blocks of its columns: the
// workgroups of one head are a multiple of eight apart, on one XCD, where that is possible.
struct SweepCoord {
  int bh, part;
};
__device__ __forceinline__ SweepCoord sweep_coord(int BH, int parts) {
  const int per = NUM_XCD * parts, grp = blockIdx.x / per, r = blockIdx.x % per;
  const int heads = min(NUM_XCD, BH - grp * NUM_XCD);
  return {grp * NUM_XCD + r % heads, r / heads};
}

// the row that row x (0 .. 15) of tile m stands for, in the sweeps
__device__ __forceinline__ constexpr int tile_row(int m, int x) { return 32 * (m / 2) + 8 * (x / 4) + 4 * (m % 2) + x % 4; }

// fp32 values as an operand: two bf16 terms, or as they are.
template <class T> struct Split;
template <> struct Split<__bf16> {
  Frag<__bf16> hi, lo;
};
template <> struct Split<float> {
  Frag<float> hi;
};
// operand of the contraction over the rows of two result tiles
template <class T>
__device__ __forceinline__ Split<T> split(const f32x4& a, const f32x4& b);
template <>
__device__ __forceinline__ Split<__bf16> split(const f32x4& a, const f32x4& b) {
#pragma clang fp contract(off)   // the terms of the rounded value, the same wherever it comes from
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  unsigned hi[4], lo[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {   // pairs: one conversion instruction each
    const f32x2 x = j < 2 ? f32x2{a[2 * j], a[2 * j + 1]} : f32x2{b[2 * j - 4], b[2 * j - 3]};
    hi[j] = __builtin_bit_cast(unsigned, __builtin_convertvector(x, bf16x2));
    const f32x2 y = {x[0] - __uint_as_float(hi[j] << 16), x[1] - __uint_as_float(hi[j] & 0xffff0000u)};
    lo[j] = __builtin_bit_cast(unsigned, __builtin_convertvector(y, bf16x2));
  }
  Split<__bf16> s;
  s.hi.v = __builtin_bit_cast(bf16x8, make_uint4(hi[0], hi[1], hi[2], hi[3]));
  s.lo.v = __builtin_bit_cast(bf16x8, make_uint4(lo[0], lo[1], lo[2], lo[3]));
  return s;
}
template <>
__device__ __forceinline__ Split<float> split(const f32x4& a, const f32x4& b) {
  Split<float> s;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    s.hi.v[j] = a[j];
    s.hi.v[4 + j] = b[j];
  }
  return s;
}
__device__ __forceinline__ void mma_xs(f32x4& c, const Frag<__bf16>& a, const Split<__bf16>& b) {
  mma(c, a, b.lo);
  mma(c, a, b.hi);
}
__device__ __forceinline__ void mma_xs(f32x4& c, const Frag<float>& a, const Split<float>& b) { mma(c, a, b.hi); }
__device__ __forceinline__ void mma_sx(f32x4& c, const Split<__bf16>& a, const Frag<__bf16>& b) {
  mma(c, a.lo, b);
  mma(c, a.hi, b);
}
__device__ __forceinline__ void mma_sx(f32x4& c, const Split<float>& a, const Frag<float>& b) { mma(c, a.hi, b); }
__device__ __forceinline__ void mma_ss(f32x4& c, const Split<__bf16>& a, const Split<__bf16>& b) {
  mma(c, a.lo, b.hi);
  mma(c, a.hi, b.lo);
  mma(c, a.hi, b.hi);
}
__device__ __forceinline__ void mma_ss(f32x4& c, const Split<float>& a, const Split<float>& b) { mma(c, a.hi, b.hi); }

// Rows kept as the sweeps' lanes hold them: row r, columns c .. c+7 are lane (c / 8 % 4) 16 + r % 16's part
// of the operand of columns c / 32 of the rows r / 16, 16 bytes a lane (fp32: two halves).  A store of
// one is 1 KB in a row; as rows of D elements it would touch sixteen of them.
template <class T, int D>
struct FragRows {
  static constexpr int E = 16 / sizeof(T);
  static constexpr int FRAG = WAVE * 8 * (int)sizeof(T);   // bytes
  static __device__ __forceinline__ int at(int r, int ch) {
    const int c = ch * E;
    return (r / 16 * (D / 32) + c / 32) * FRAG + (c % 8) / E * (WAVE * 16) + ((c / 8 % 4) * 16 + r % 16) * 16;
  }
};

// Operand reads of a tile of rows in LDS by 16 x 16 products.
template <class T, int D, class Rows = RowTile<T, D>>
struct Tile16 : Rows {
  using R = Rows;
  // four elements of row r from column c on (c a multiple of 4)
  static __device__ __forceinline__ const char* quad(const char* L, int r, int c) {
    return L + R::at(r, c / R::E) + (c % R::E) * (int)sizeof(T);
  }
  static __device__ __forceinline__ f32x4 quad_f(const char* L, int r, int c) {
    f32x4 v;
    if constexpr (IsBf16<T>::value) {
      const bf16x4 x = *reinterpret_cast<const bf16x4*>(quad(L, r, c));
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = (float)x[j];
    } else {
      v = *reinterpret_cast<const f32x4*>(quad(L, r, c));
    }
    return v;
  }
  // row r, slots 0..3 the columns c0 .. c0+3, slots 4..7 c1 .. c1+3
  static __device__ __forceinline__ Frag<T> row(const char* L, int r, int c0, int c1) {
    Frag<T> f;
    if constexpr (IsBf16<T>::value) {
      const uint2 a = *reinterpret_cast<const uint2*>(quad(L, r, c0));
      const uint2 b = *reinterpret_cast<const uint2*>(quad(L, r, c1));
      f.v = __builtin_bit_cast(bf16x8, make_uint4(a.x, a.y, b.x, b.y));
    } else {
      const f32x4 a = *reinterpret_cast<const f32x4*>(quad(L, r, c0));
      const f32x4 b = *reinterpret_cast<const f32x4*>(quad(L, r, c1));
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        f.v[j] = a[j];
        f.v[4 + j] = b[j];
      }
    }
    return f;
  }
  // row r, the eight columns from c on (c a multiple of 8)
  static __device__ __forceinline__ Frag<T> row8(const char* L, int r, int c) {
    if constexpr (IsBf16<T>::value) {
      Frag<T> f;
      f.v = *reinterpret_cast<const bf16x8*>(L + R::at(r, c / 8));
      return f;
    } else {
      return row(L, r, c, c + 4);
    }
  }
  // column tile_row(m, l % 16), slots 0..7 the rows r0 .. r0+7
  static __device__ __forceinline__ Frag<T> col8(const char* L, int r0, int m) {
    const int i = threadIdx.x % 16;
    Frag<T> f;
    if constexpr (IsBf16<T>::value) {
      // the lane's part of the read: row i / 4, the four columns of quarter i % 4 of the tile
      const int c = tile_row(m, 4 * (i % 4));
      const tr_v4i16 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_tr_v4i16*)quad(L, r0 + i / 4, c));
      const tr_v4i16 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_tr_v4i16*)quad(L, r0 + 4 + i / 4, c));
      f.v = __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
      const int c = tile_row(m, i & ~3), o = (i & 3) * 4;
#pragma unroll
      for (int j = 0; j < 8; ++j) f.v[j] = *reinterpret_cast<const float*>(quad(L, r0 + j, c) + o);
    }
    return f;
  }
  // column m0 + l % 16 of the rows r0 .. r0+3, as they are
  typedef T quad_t __attribute__((ext_vector_type(4)));
  static __device__ __forceinline__ quad_t col4(const char* L, int r0, int m0) {
    const int i = threadIdx.x % 16;
    if constexpr (IsBf16<T>::value) {
      return __builtin_bit_cast(
          quad_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_tr_v4i16*)quad(L, r0 + i / 4, m0 + 4 * (i % 4))));
    } else {
      quad_t v;
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = *reinterpret_cast<const float*>(quad(L, r0 + j, m0 + (i & ~3)) + (i & 3) * 4);
      return v;
    }
  }
  // column m0 + l % 16, slots 0..3 the rows r0 .. r0+3, slots 4..7 r1 .. r1+3
  static __device__ __forceinline__ Frag<T> col(const char* L, int r0, int r1, int m0) {
    const int i = threadIdx.x % 16;
    Frag<T> f;
    if constexpr (IsBf16<T>::value) {
      const int c = m0 + 4 * (i % 4);
      const tr_v4i16 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_tr_v4i16*)quad(L, r0 + i / 4, c));
      const tr_v4i16 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_tr_v4i16*)quad(L, r1 + i / 4, c));
      f.v = __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
      const int m = m0 + i, c = m & ~3, o = (m & 3) * 4;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        f.v[j] = *reinterpret_cast<const float*>(quad(L, r0 + j, c) + o);
        f.v[4 + j] = *reinterpret_cast<const float*>(quad(L, r1 + j, c) + o);
      }
    }
    return f;
  }
};

// Two terms of a matrix kept as hi and lo tiles, `bytes` apart (fp32: one tile).
template <class T, int D, class Rows = RowTile<T, D>>
struct Pair16 {
  using R = Tile16<T, D, Rows>;
  template <class F>
  static __device__ __forceinline__ Split<T> both(const char* L, int bytes, F read) {
    Split<T> s;
    s.hi = read(L);
    if constexpr (IsBf16<T>::value) s.lo = read(L + bytes);
    return s;
  }
  static __device__ __forceinline__ Split<T> row8(const char* L, int bytes, int r, int c) {
    return both(L, bytes, [=](const char* p) { return R::row8(p, r, c); });
  }
  static __device__ __forceinline__ Split<T> col8(const char* L, int bytes, int r0, int m) {
    return both(L, bytes, [=](const char* p) { return R::col8(p, r0, m); });
  }
  static __device__ __forceinline__ Split<T> col(const char* L, int bytes, int r0, int r1, int m0) {
    return both(L, bytes, [=](const char* p) { return R::col(p, r0, r1, m0); });
  }
};

// Four tiles at once, term by term: no product waits for the one before it.
__device__ __forceinline__ void mma_xs4(f32x4 (&c)[4], const Frag<__bf16> (&a)[4], const Split<__bf16>& b) {
#pragma unroll
  for (int m = 0; m < 4; ++m) mma(c[m], a[m], b.lo);
#pragma unroll
  for (int m = 0; m < 4; ++m) mma(c[m], a[m], b.hi);
}
__device__ __forceinline__ void mma_xs4(f32x4 (&c)[4], const Frag<float> (&a)[4], const Split<float>& b) {
#pragma unroll
  for (int m = 0; m < 4; ++m) mma(c[m], a[m], b.hi);
}

// A lower triangular [64][64] matrix in LDS as the sweeps read it: per term the rows 0..31 of
// the columns 0..31, then the rows 32..63.
template <class T>
struct LowTri {
  using A = Pair16<T, 32>;
  using B = Pair16<T, 64>;
  static constexpr int TOP = 32 * 32 * (int)sizeof(T);           // bytes of the first part
  static constexpr int TERM = TOP + 32 * 64 * (int)sizeof(T);    // of one term
  // where row i, columns j .. j+3 of the first term lie
  static __device__ __forceinline__ int at(int i, int j) {
    return i < 32 ? (int)(A::R::quad(nullptr, i, j) - (const char*)nullptr)
                  : TOP + (int)(B::R::quad(nullptr, i - 32, j) - (const char*)nullptr);
  }
  static __device__ __forceinline__ void terms(f32x4& c, const Split<T>& a, const Split<T>& b, int k) {
    if constexpr (IsBf16<T>::value) {
      if (k == 0) mma(c, a.lo, b.hi);
      if (k == 1) mma(c, a.hi, b.lo);
      if (k == 2) mma(c, a.hi, b.hi);
    } else if (k == 2) {
      mma(c, a.hi, b.hi);
    }
  }
  // c += M b, b as two operands (rows 0..31, 32..63); term by term, so that no product
  // waits for the one before it
  static __device__ __forceinline__ void mul(f32x4 (&c)[4], const char* L, int r16, int g, const Split<T>& b0,
                                             const Split<T>& b1) {
    Split<T> a0[4], a1[2];
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      a0[m] = A::row8(L, TERM, tile_row(m, r16), 8 * g);
      a0[m + 2] = B::row8(L + TOP, TERM, tile_row(m, r16), 8 * g);
      a1[m] = B::row8(L + TOP, TERM, tile_row(m, r16), 32 + 8 * g);
    }
#pragma unroll
    for (int k = 0; k < 3; ++k) {
#pragma unroll
      for (int m = 0; m < 4; ++m) terms(c[m], a0[m], b0, k);
#pragma unroll
      for (int m = 0; m < 2; ++m) terms(c[m + 2], a1[m], b1, k);
    }
  }
  // c <- M c
  static __device__ __forceinline__ void apply(f32x4 (&c)[4], const char* L, int r16, int g) {
    const Split<T> b0 = split<T>(c[0], c[1]), b1 = split<T>(c[2], c[3]);
#pragma unroll
    for (int m = 0; m < 4; ++m) c[m] = zero4();
    mul(c, L, r16, g, b0, b1);
  }
  // the operands of M^T: contraction over the rows 0..31 (columns 0..31 only), and 32..63
  static __device__ __forceinline__ void transposed(Split<T> (&a0)[2], Split<T> (&a1)[4], const char* L, int g) {
#pragma unroll
    for (int m = 0; m < 2; ++m) a0[m] = A::col8(L, TERM, 8 * g, m);
#pragma unroll
    for (int m = 0; m < 4; ++m) a1[m] = B::col8(L + TOP, TERM, 8 * g, m);
  }
  // c <- M^T c
  static __device__ __forceinline__ void apply_t(f32x4 (&c)[4], const char* L, int g) {
    const Split<T> b0 = split<T>(c[0], c[1]), b1 = split<T>(c[2], c[3]);
    Split<T> a0[2], a1[4];
    transposed(a0, a1, L, g);
#pragma unroll
    for (int m = 0; m < 4; ++m) c[m] = zero4();
#pragma unroll
    for (int k = 0; k < 3; ++k) {
#pragma unroll
      for (int m = 0; m < 4; ++m) terms(c[m], a1[m], b1, k);
#pragma unroll
      for (int m = 0; m < 2; ++m) terms(c[m], a0[m], b0, k);
    }
  }
};

// Rows of a chunk (result tiles) that are not finite.  The products with lower triangular matrices go over whole blocks,
// and zero times NaN is not zero: a token's row would reach those before it.  Where a column has such a
// row, it and those behind it are cut out of the product (0) and are NaN in the result, as the recurrence has it.
__device__ __forceinline__ bool not_finite(const f32x4 (&u)[4]) {
  f32x4 x = zero4();   // NaN from the first NaN or infinity on
#pragma unroll
  for (int m = 0; m < 4; ++m)
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = __builtin_fmaf(u[m][e], 0.f, x[e]);
  return (x[0] + x[1]) + (x[2] + x[3]) != 0.f;
}
// of this lane's column, the first such row; DC: none
__device__ __forceinline__ int first_not_finite(const f32x4 (&u)[4], int g) {
  int first = DC;
#pragma unroll
  for (int m = 0; m < 4; ++m)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (!(fabsf(u[m][e]) < INFINITY)) first = min(first, tile_row(m, 4 * g + e));
  first = min(first, __shfl_xor(first, 16));
  return min(first, __shfl_xor(first, 32));
}
__device__ __forceinline__ void cut(f32x4 (&u)[4], int g, int first, float value) {
#pragma unroll
  for (int m = 0; m < 4; ++m)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (tile_row(m, 4 * g + e) >= first) u[m][e] = value;
}

// Operands that one wave hands to another through LDS, as the lanes hold them: 16 bytes a
// lane and instruction.
template <class T>
struct FragBox {
  static constexpr int BYTES = WAVE * 16 * 2;   // hi and lo, or eight floats
  static __device__ __forceinline__ void put(char* L, int l, const Split<__bf16>& s) {
    *reinterpret_cast<bf16x8*>(L + l * 16) = s.hi.v;
    *reinterpret_cast<bf16x8*>(L + WAVE * 16 + l * 16) = s.lo.v;
  }
  static __device__ __forceinline__ void put(char* L, int l, const Split<float>& s) {
    *reinterpret_cast<f32x4*>(L + l * 16) = f32x4{s.hi.v[0], s.hi.v[1], s.hi.v[2], s.hi.v[3]};
    *reinterpret_cast<f32x4*>(L + WAVE * 16 + l * 16) = f32x4{s.hi.v[4], s.hi.v[5], s.hi.v[6], s.hi.v[7]};
  }
  static __device__ __forceinline__ Split<T> get(const char* L, int l) {
    Split<T> s;
    if constexpr (IsBf16<T>::value) {
      s.hi.v = *reinterpret_cast<const bf16x8*>(L + l * 16);
      s.lo.v = *reinterpret_cast<const bf16x8*>(L + WAVE * 16 + l * 16);
    } else {
      const f32x4 a = *reinterpret_cast<const f32x4*>(L + l * 16), b = *reinterpret_cast<const f32x4*>(L + WAVE * 16 + l * 16);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        s.hi.v[j] = a[j];
        s.hi.v[4 + j] = b[j];
      }
    }
    return s;
  }
};
// Operand `frag` of a FragRows array, the second term `lo` elements behind the first (0: not).
__device__ __forceinline__ void store_frag(u16* base, int frag, size_t lo, const Split<__bf16>& s) {
  u16* p = base + (size_t)frag * (WAVE * 8) + threadIdx.x % WAVE * 8;
  *reinterpret_cast<bf16x8*>(p) = s.hi.v;
  if (lo) *reinterpret_cast<bf16x8*>(p + lo) = s.lo.v;
}
__device__ __forceinline__ void store_frag(float* base, int frag, size_t, const Split<float>& s) {
  float* p = base + (size_t)frag * (WAVE * 8) + threadIdx.x % WAVE * 4;
  *reinterpret_cast<f32x4*>(p) = f32x4{s.hi.v[0], s.hi.v[1], s.hi.v[2], s.hi.v[3]};
  *reinterpret_cast<f32x4*>(p + WAVE * 4) = f32x4{s.hi.v[4], s.hi.v[5], s.hi.v[6], s.hi.v[7]};
}

// A wave's 16 columns of a chunk's rows (result tiles x), rounded to the io type and written as rows of
// 32 bytes (fp32: 64) through the wave's own `box` in LDS: 16 bytes a lane in place of one element.
template <class S>
struct RowBox {
  static constexpr int LD = 16 * (int)sizeof(S) + 16;   // bytes per row
  static constexpr int BYTES = DC * LD;
  static __device__ __forceinline__ void store(char* box, __amdgpu_buffer_rsrc_t rs, int stride, int col, const f32x4 (&x)[4]) {
    const int l = threadIdx.x % WAVE, r16 = l % 16, g = l / 16;
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        *reinterpret_cast<S*>(box + tile_row(m, 4 * g + e) * LD + r16 * (int)sizeof(S)) = float_to_io<S>(x[m][e]);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
    for (int i = 0; i < (int)sizeof(S); ++i) {   // row l, its 16-byte units
      const u32x4 v = *reinterpret_cast<const u32x4*>(box + l * LD + 16 * i);
      __builtin_amdgcn_raw_buffer_store_b128(v, rs, (l * stride + col) * (int)sizeof(S) + 16 * i, 0, 0);
    }
  }
};

// four values as one or two terms, `lo` elements behind the first
__device__ __forceinline__ void store_split4(u16* p, size_t lo, const f32x4& v) {
  Split<__bf16> s = split<__bf16>(v, zero4());
  const uint4 h = __builtin_bit_cast(uint4, s.hi.v), l = __builtin_bit_cast(uint4, s.lo.v);
  *reinterpret_cast<uint2*>(p) = make_uint2(h.x, h.y);
  *reinterpret_cast<uint2*>(p + lo) = make_uint2(l.x, l.y);
}
__device__ __forceinline__ void store_split4(float* p, size_t, const f32x4& v) { *reinterpret_cast<f32x4*>(p) = v; }

// Linear copy of 1024 N bytes to LDS, one instruction per 1024 bytes, by NW waves.
template <int N, int NW>
__device__ __forceinline__ void stage_linear(const char* L, const void* src, int w) {
  u32x4 d;
  const uint64_t p = reinterpret_cast<uint64_t>(src);
  d[0] = __builtin_amdgcn_readfirstlane((unsigned)p);
  d[1] = __builtin_amdgcn_readfirstlane((unsigned)(p >> 32) & 0xffff);
  d[2] = N * 1024;
  d[3] = BUF_FLAGS;
  const unsigned base = (unsigned)(size_t)(__attribute__((address_space(3))) const char*)L;
  const int l = threadIdx.x % WAVE;
#pragma unroll
  for (int n = 0; n < (N + NW - 1) / NW; ++n) {
    const int step = n * NW + w;
    if (N % NW == 0 || step < N) {
      const unsigned to = __builtin_amdgcn_readfirstlane(base + step * 1024);
      const int off = step * 1024 + l * 16;
      asm volatile("s_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"{m0}"(to), "v"(off), "s"(d)
                   : "memory");
    }
  }
}

// What a chunk's sweep step reads, through LDS: tiles of K and Q, of VC columns of V or dO, and T,
// P, e^G, w and b.
template <class T, int D, int VC>
struct ChunkLds {
  using VT = Tile16<T, VC>;
  static constexpr int ROWS = DC * D * (int)sizeof(T);     // bytes of a K or Q tile
  static constexpr int VROWS = DC * VC * (int)sizeof(T);
  static constexpr int BYTES = 2 * ROWS + VROWS + DELTA_SWEEP_BYTES;
  const char* L;
  __device__ __forceinline__ const char* k() const { return L; }
  __device__ __forceinline__ const char* q() const { return L + ROWS; }
  __device__ __forceinline__ const char* v() const { return L + 2 * ROWS; }
  __device__ __forceinline__ const char* t() const { return L + 2 * ROWS + VROWS; }
  __device__ __forceinline__ const char* p() const { return t() + DELTA_MAT_BYTES; }
  // the lane's rows of tile m of e^G (0), w (1), b (2)
  __device__ __forceinline__ f32x4 scal(int which, int m, int g) const {
    return *reinterpret_cast<const f32x4*>(t() + 2 * DELTA_MAT_BYTES + (which * DC + tile_row(m, 4 * g)) * 4);
  }
  // exp of the chunk's whole decay
  __device__ __forceinline__ float last() const {
    return *reinterpret_cast<const float*>(t() + 2 * DELTA_MAT_BYTES + (DC - 1) * 4);
  }
  // the lane's column (of 16 from c0 on) of V or dO, its rows of tile m
  __device__ __forceinline__ typename VT::quad_t col(int m, int g, int c0) const {
    return VT::col4(v(), tile_row(m, 4 * g), c0);
  }
  // X: V or dO, from the first of the VC columns on
  template <int NW>
  __device__ __forceinline__ void stage(const DeltaArgs& a, int row0, int n, int kh, size_t blk, const void* X, int xs,
                                        int w) const {
    using S = typename Io<T>::type;
    stage_tile<T, D, DC, NW>(k(), row_words(static_cast<const S*>(a.K) + kh * D, row0, a.ks, n, D),
                             a.ks * (int)sizeof(S), w);
    stage_tile<T, VC, DC, NW>(v(), row_words(static_cast<const S*>(X), row0, xs, n, VC), xs * (int)sizeof(S), w);
    stage_tile<T, D, DC, NW>(q(), row_words(static_cast<const S*>(a.Q) + kh * D, row0, a.qs, n, D),
                             a.qs * (int)sizeof(S), w);
    stage_linear<DELTA_SWEEP_BYTES / 1024, NW>(t(), a.prep + blk * DELTA_PREP_BYTES, w);
  }
  // Brings a chunk into L2, one word per line: of its K, Q and matrices the share of `part` (the
  // workgroups of a head's other columns, on the same XCD, bring the others), and all of its V.
  // A CU has some 26 KB of loads on the way at most: straight from HBM (2000 clocks) that is
  // 13 bytes a clock, from L2 (600) 43, and a chunk is 61 KB.
  static constexpr int RL = D * (int)sizeof(T) / 128, ML = DELTA_SWEEP_BYTES / 128;   // lines of a row, of the matrices
  static constexpr int LINES = 2 * DC * RL + ML;
  template <int NW, int PER>
  __device__ __forceinline__ void prefetch(unsigned (&x)[PER], const DeltaArgs& a, int row0, int n, int kh, size_t blk,
                                           const void* X, int xs, int part, int parts, int w) const {
    using S = typename Io<T>::type;
    const int l = threadIdx.x % WAVE;
    const S* pk = static_cast<const S*>(a.K) + (size_t)row0 * a.ks + kh * D;
    const S* pq = static_cast<const S*>(a.Q) + (size_t)row0 * a.qs + kh * D;
    const S* px = static_cast<const S*>(X) + (size_t)row0 * xs;
    const char* pm = a.prep + blk * DELTA_PREP_BYTES;
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      const int i = ((u * parts + part) * NW + w) * WAVE + l, j = i - DC * RL, m = j - DC * RL;
      const S* p = px + (size_t)min(l, n - 1) * xs;   // lanes without a line of the others: a row of X
      if (i < DC * RL) p = pk + (size_t)min(i / RL, n - 1) * a.ks + i % RL * (128 / (int)sizeof(S));
      else if (m < 0) p = pq + (size_t)min(j / RL, n - 1) * a.qs + j % RL * (128 / (int)sizeof(S));
      else if (m < ML) p = reinterpret_cast<const S*>(pm + m * 128);
      x[u] = *reinterpret_cast<const unsigned*>(p);
    }
  }
};

}  // namespace flex
