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
// ([d x 16] as 16 x 16 tiles: lane l holds column l % 16 and rows 4 (l / 16) + i).  A result
// in that layout is the right operand of the next product as it is, with the contraction in
// the order 32 s + 4g + i, 32 s + 16 + 4g + i (g = l / 16), so K S -> U -> K^T U -> S
// never leaves the wave.
//
// Precision, bf16 rows: K, Q, V, dO are exact operands.  States, U, T and the like are
// fp32 and enter products as two bf16 terms (16 bits), so a carried state is right to
// about 2^-17 of its terms; a single rounding to bf16 is taken only where the result is
// rounded to bf16 itself.
#pragma once
#include "flex_seq.hpp"
#include "flex_seq_kernels.hpp"

namespace flex {

constexpr int DC = DELTA_CHUNK;

// fp32 values as an operand: two bf16 terms, or as they are.
template <class T> struct Split;
template <> struct Split<__bf16> {
  Frag<__bf16> hi, lo;
  __device__ __forceinline__ void set(int j, float x) {
    hi.v[j] = (__bf16)x;
    lo.v[j] = (__bf16)(x - (float)hi.v[j]);
  }
};
template <> struct Split<float> {
  Frag<float> hi;
  __device__ __forceinline__ void set(int j, float x) { hi.v[j] = x; }
};
// operand of the contraction over the rows of two result tiles
template <class T>
__device__ __forceinline__ Split<T> split(const f32x4& a, const f32x4& b) {
  Split<T> s;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    s.set(j, a[j]);
    s.set(4 + j, b[j]);
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

// Operand reads of a RowTile by 16 x 16 products.
template <class T, int D>
struct Tile16 : RowTile<T, D> {
  using R = RowTile<T, D>;
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

// Two terms of a matrix kept as hi and lo tiles (fp32: one tile).
template <class T, int D>
struct Pair16 {
  static constexpr int LO = IsBf16<T>::value ? 1 : 0;
  static __device__ __forceinline__ Split<T> row(const char* L, int bytes, int r, int c0, int c1) {
    Split<T> s;
    s.hi = Tile16<T, D>::row(L, r, c0, c1);
    if constexpr (IsBf16<T>::value) s.lo = Tile16<T, D>::row(L + bytes, r, c0, c1);
    return s;
  }
  static __device__ __forceinline__ Split<T> col(const char* L, int bytes, int r0, int r1, int m0) {
    Split<T> s;
    s.hi = Tile16<T, D>::col(L, r0, r1, m0);
    if constexpr (IsBf16<T>::value) s.lo = Tile16<T, D>::col(L + bytes, r0, r1, m0);
    return s;
  }
};

// one element of a window, in the io type
__device__ __forceinline__ u16 load1(__amdgpu_buffer_rsrc_t rs, int off, u16) {
  return __builtin_amdgcn_raw_buffer_load_b16(rs, off, 0, 0);
}
__device__ __forceinline__ float load1(__amdgpu_buffer_rsrc_t rs, int off, float) {
  return __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rs, off, 0, 0));
}
__device__ __forceinline__ void store1(__amdgpu_buffer_rsrc_t rs, int off, u16 v) {
  __builtin_amdgcn_raw_buffer_store_b16(v, rs, off, 0, 0);
}
__device__ __forceinline__ void store1(__amdgpu_buffer_rsrc_t rs, int off, float v) {
  __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, v), rs, off, 0, 0);
}

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
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(off), "s"(d)
                   : "memory");
    }
  }
}

// What a chunk's sweep step reads, through LDS: K and Q tiles, T and P (their terms as tiles),
// e^G, w and b.
template <class T, int D>
struct ChunkLds {
  static constexpr int ROWS = DC * D * (int)sizeof(T);     // bytes of a K or Q tile
  static constexpr int MAT = DC * DC * (int)sizeof(T);     // of one term of T or P
  static constexpr int BYTES = 2 * ROWS + 2 * DELTA_MAT_BYTES + 1024;
  static constexpr int BUFS = 2 * BYTES <= 160 * 1024 ? 2 : 1;
  const char* L;
  __device__ __forceinline__ const char* k() const { return L; }
  __device__ __forceinline__ const char* q() const { return L + ROWS; }
  __device__ __forceinline__ const char* t() const { return L + 2 * ROWS; }
  __device__ __forceinline__ const char* p() const { return L + 2 * ROWS + DELTA_MAT_BYTES; }
  // rows 16 m + 4 g .. + 3 of e^G (0), w (1), b (2)
  __device__ __forceinline__ f32x4 scal(int which, int m, int g) const {
    return *reinterpret_cast<const f32x4*>(L + 2 * ROWS + 2 * DELTA_MAT_BYTES + (which * DC + 16 * m + 4 * g) * 4);
  }
  // exp of the chunk's whole decay
  __device__ __forceinline__ float last() const {
    return *reinterpret_cast<const float*>(L + 2 * ROWS + 2 * DELTA_MAT_BYTES + (DC - 1) * 4);
  }
  template <int NW>
  __device__ __forceinline__ void stage(const DeltaArgs& a, int row0, int n, int kh, size_t blk, int w) const {
    using S = typename Io<T>::type;
    stage_tile<T, D, DC, NW>(k(), row_words(static_cast<const S*>(a.K) + kh * D, row0, a.ks, n, D),
                             a.ks * (int)sizeof(S), w);
    stage_tile<T, D, DC, NW>(q(), row_words(static_cast<const S*>(a.Q) + kh * D, row0, a.qs, n, D),
                             a.qs * (int)sizeof(S), w);
    const char* p = a.prep + blk * DELTA_PREP_BYTES;
#pragma unroll
    for (int i = 0; i < 2 * DELTA_MAT_BYTES / MAT; ++i)
      stage_tile<T, DC, DC, NW>(t() + i * MAT, row_words(reinterpret_cast<const S*>(p + i * MAT), 0, DC, DC, DC),
                                DC * (int)sizeof(S), w);
    stage_linear<1, NW>(t() + 2 * DELTA_MAT_BYTES, p + 2 * DELTA_MAT_BYTES, w);
  }
};

// A lane's column `col` of a chunk's rows (rows 16 m + 4 g + e), rows behind the sequence as zeros.
template <class S>
__device__ __forceinline__ void load_column(S (&v)[4][4], const S* base, int row0, int stride, int n, int width, int col) {
  const int g = threadIdx.x % WAVE / 16;
  const auto rs = row_window(base, row0, stride, n, width);
#pragma unroll
  for (int m = 0; m < 4; ++m)
#pragma unroll
    for (int e = 0; e < 4; ++e) v[m][e] = load1(rs, ((16 * m + 4 * g + e) * stride + col) * (int)sizeof(S), S());
}

}  // namespace flex
