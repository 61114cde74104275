// Device building blocks of the packed-sequence kernels (exact attention and the
// gated delta rule): the map from workgroups to tiles of sequences, row tiles in
// LDS, and 32 x 32 products whose result is the next product's operand.
//
// Orientation ("query-column"): with A the rows of K and B the rows of Q, the
// matrix core returns S^T with lane l holding column l % 32 (one query) and rows
// 8a + 4h + i (h = l / 32, a, i = 0..3).  A product over those rows takes them as
// they are: k slots 0..3 and 4..7 of step s are rows 16s + 4h + i and
// 16s + 8 + 4h + i, and the other operand is read from LDS in the same order.  No
// probability passes through LDS, and a query's statistics sit in its own lane.
#pragma once
#include "flex_common.hpp"
#include "flex_stage.hpp"

namespace flex {

typedef float f32x16 __attribute__((ext_vector_type(16)));

__device__ __forceinline__ f32x16 zero16() {
  f32x16 z;
#pragma unroll
  for (int i = 0; i < 16; ++i) z[i] = 0.f;
  return z;
}

// c += a b over 16 contraction indices (8 per lane half)
__device__ __forceinline__ void mma32(f32x16& c, const Frag<__bf16>& a, const Frag<__bf16>& b) {
  c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.v, b.v, c, 0, 0, 0);
}
__device__ __forceinline__ void mma32(f32x16& c, const Frag<float>& a, const Frag<float>& b) {
#pragma unroll
  for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v[j], b.v[j], c, 0, 0, 0);
}

// Operand fragment of step s (0, 1) from a 32 x 32 result: the rows it covers are
// this lane's results 8s .. 8s+7.
template <class T>
__device__ __forceinline__ Frag<T> frag_of(const f32x16& c, int s) {
  Frag<T> f;
#pragma unroll
  for (int j = 0; j < 8; ++j) f.set(j, c[8 * s + j]);
  return f;
}

// Row of the 32 x 32 result that element e (0..15) of lane half h is.
__device__ __forceinline__ constexpr int res_row(int e, int h) { return 8 * (e / 4) + 4 * h + e % 4; }

// max / sum of a value over the two lane halves (lanes l and l ^ 32)
__device__ __forceinline__ float half_max(float x) {
  const unsigned v = __float_as_uint(x);
  const auto p = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}
__device__ __forceinline__ float half_sum(float x) {
  const unsigned v = __float_as_uint(x);
  const auto p = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}

// ---------------------------------------------------------------------------
// Packed sequences.  Sequence b holds rows off[b] .. off[b+1]-1 of a tensor of T
// rows.  Tiles of M rows are numbered by slots: those of sequence b start at slot
// off[b] / M + b, which leaves every sequence room for its ragged last tile and
// needs no prefix sum over the lengths; T / M + B slots cover any lengths.
// Offsets are clamped to 0 .. T, so that no value of theirs leads outside a tensor.
// ---------------------------------------------------------------------------
__device__ __forceinline__ int clamp_off(int x, int T) { return min(max(x, 0), T); }

// How many of 0 .. B-1 hold, where those that do come first: 64 probes at once, one round for up
// to 64, two up to 4096.  0 .. B whatever holds.  (One pass over the offsets, 64 at a time, took the
// attention's backward over 4096 sequences of 20 tokens 1380 us, this 640.)
template <class P>
__device__ __forceinline__ int leading(int B, P holds) {
  const int l = threadIdx.x % WAVE;
  int lo = 0, n = B;
  while (n > 0) {
    const int step = (n + WAVE - 1) / WAVE, at = (l + 1) * step - 1;   // the last of each lane's share
    const int c = __popcll(__ballot(at < n && holds(lo + min(at, n - 1))));
    lo += c * step;
    n = step == 1 ? 0 : min(step, n - c * step);
  }
  return lo;
}

struct SeqTile {
  int b;      // sequence, or -1 for a slot without a tile
  int row0;   // its first row in the tensor
  int n;      // its length
  int tile;   // tile within it
};
template <int M>
__device__ __forceinline__ SeqTile find_tile(const int32_t* __restrict__ off, int B, int T, int slot) {
  // sequences whose first slot is not behind this one
  const int cnt = leading(B, [=](int b) { return clamp_off(off[b], T) / M + b <= slot; });
  SeqTile t{-1, 0, 0, 0};
  if (cnt == 0) return t;
  const int b = cnt - 1;
  t.row0 = clamp_off(off[b], T);
  t.n = max(clamp_off(off[b + 1], T) - t.row0, 0);
  t.tile = slot - (t.row0 / M + b);
  if (t.tile >= 0 && (long long)t.tile * M < t.n) t.b = b;   // offsets that fall may give tiles below 0
  t.b = __builtin_amdgcn_readfirstlane(t.b);
  t.row0 = __builtin_amdgcn_readfirstlane(t.row0);
  t.n = __builtin_amdgcn_readfirstlane(t.n);
  t.tile = __builtin_amdgcn_readfirstlane(t.tile);
  return t;
}
// A sequence's rows, with its used length where one is given.
struct SeqRange {
  int row0, n;
};
__device__ __forceinline__ SeqRange seq_range(const int32_t* __restrict__ off, int b, int T,
                                              const int32_t* __restrict__ len = nullptr) {
  SeqRange r;
  r.row0 = clamp_off(off[b], T);
  r.n = max(clamp_off(off[b + 1], T) - r.row0, 0);
  if (len) r.n = min(max(len[b], 0), r.n);
  r.row0 = __builtin_amdgcn_readfirstlane(r.row0);
  r.n = __builtin_amdgcn_readfirstlane(r.n);
  return r;
}
__host__ __device__ inline int seq_slots(int T, int B, int M) { return T / M + B; }

// Workgroup -> (slot, head) for a 1-D grid of slots x heads.  Consecutive workgroup
// ids go round-robin to the XCDs: where the heads divide among them, an XCD gets
// whole heads, so that the workgroups of one head read its rows through one L2.
// Within an XCD the slots come in order, or from the last one down (`down`: with a
// causal mask the later query tiles of a sequence are the longer ones, and the long ones
// first leave the least to wait for at its end).  Among sequences the order is that of
// the packing: where the longest is in front, its tiles come last.
struct TileCoord {
  int slot, head;
};
__device__ __forceinline__ TileCoord tile_coord(int slots, int heads, bool down) {
  const int id = blockIdx.x;
  TileCoord t;
  if (heads % NUM_XCD == 0) {
    const int per = heads / NUM_XCD, k = id / NUM_XCD;
    t.slot = k / per;
    t.head = id % NUM_XCD * per + k % per;
  } else {
    t.slot = id / heads;
    t.head = id % heads;
  }
  if (down) t.slot = slots - 1 - t.slot;
  return t;
}

// ---------------------------------------------------------------------------
// A tile of rows in LDS: D elements per row in 16-byte chunks, chunk c of row r at
// place c ^ swz(r).  Without the swizzle the 32 rows of an operand read lie in the
// same banks.  swz moves four consecutive rows to different groups of four chunks
// (a transposed read takes four chunks of eight rows) and sixteen rows to
// different places (an operand read takes one chunk of 32 rows).
// ---------------------------------------------------------------------------
template <class T, int D>
struct RowTile {
  static constexpr int E = 16 / sizeof(T);      // elements per chunk
  static constexpr int CH = D / E;              // chunks per row
  static constexpr int ROW = D * sizeof(T);     // bytes per row
  static __device__ __forceinline__ int swz(int r) {
    if (CH >= 16) return ((r & 3) << 2) | ((r >> 2) & 3);
    if (CH == 8) return (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
    return (r >> 2) & 3;
  }
  static __device__ __forceinline__ int at(int r, int c) { return r * ROW + ((c ^ swz(r)) << 4); }

  // operand fragment: row r, elements 16 s + 8 h .. + 7
  static __device__ __forceinline__ Frag<T> row(const char* L, int r, int s, int h) {
    Frag<T> f;
    if constexpr (IsBf16<T>::value) {
      f.v = *reinterpret_cast<const bf16x8*>(L + at(r, 2 * s + h));
    } else {
      const float4 a = *reinterpret_cast<const float4*>(L + at(r, 4 * s + 2 * h));
      const float4 b = *reinterpret_cast<const float4*>(L + at(r, 4 * s + 2 * h + 1));
      f.v[0] = a.x; f.v[1] = a.y; f.v[2] = a.z; f.v[3] = a.w;
      f.v[4] = b.x; f.v[5] = b.y; f.v[6] = b.z; f.v[7] = b.w;
    }
    return f;
  }
  // transposed: element column m0 + l % 32, k slots rows kb + i and kb + 8 + i
  // (kb = 16 s + 4 h: the order of frag_of)
  static __device__ __forceinline__ Frag<T> col(const char* L, int kb, int m0) {
    const int l = threadIdx.x % WAVE;
    Frag<T> f;
    if constexpr (IsBf16<T>::value) {
      const int i = l % 16, r = kb + i / 4, c = (m0 + 16 * ((l / 16) & 1)) / 8 + ((i & 2) >> 1), o = (i & 1) * 8;
      const tr_v4i16 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_tr_v4i16*)(L + at(r, c) + o));
      const tr_v4i16 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_tr_v4i16*)(L + at(r + 8, c) + o));
      f.v = __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
      const int m = m0 + l % 32, c = m / 4, o = (m % 4) * 4;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        f.v[j] = *reinterpret_cast<const float*>(L + at(kb + j, c) + o);
        f.v[4 + j] = *reinterpret_cast<const float*>(L + at(kb + 8 + j, c) + o);
      }
    }
    return f;
  }
};

// Rows of a strided row-major tensor as a buffer resource: rows r0 .. r0 + rows - 1
// (elements [0, D) of each, `stride` elements apart), zeros behind them.
template <class S>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t row_window(const S* base, size_t row0, int stride, int rows, int D) {
  const int bytes = rows > 0 ? ((rows - 1) * stride + D) * (int)sizeof(S) : 0;
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<S*>(base) + row0 * (size_t)stride, 0, bytes, BUF_FLAGS);
}

// The same window as the four descriptor words that stage_tile takes.
template <class S>
__device__ __forceinline__ u32x4 row_words(const S* base, size_t row0, int stride, int rows, int D) {
  const int bytes = rows > 0 ? ((rows - 1) * stride + D) * (int)sizeof(S) : 0;
  const uint64_t p = reinterpret_cast<uint64_t>(base + row0 * (size_t)stride);
  u32x4 d;
  d[0] = __builtin_amdgcn_readfirstlane((unsigned)p);
  d[1] = __builtin_amdgcn_readfirstlane((unsigned)(p >> 32) & 0xffff);
  d[2] = __builtin_amdgcn_readfirstlane(bytes);
  d[3] = BUF_FLAGS;
  return d;
}

// Operand fragment at a byte offset of a window (zeros outside it).
template <class T>
__device__ __forceinline__ Frag<T> window_frag(__amdgpu_buffer_rsrc_t rs, int off) {
  Frag<T> f;
  if constexpr (IsBf16<T>::value) {
    f.v = __builtin_bit_cast(bf16x8, __builtin_amdgcn_raw_buffer_load_b128(rs, off, 0, 0));
  } else {
    const f32x4 a = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, off, 0, 0));
    const f32x4 b = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, off + 16, 0, 0));
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      f.v[j] = a[j];
      f.v[4 + j] = b[j];
    }
  }
  return f;
}

// ---------------------------------------------------------------------------
// Sums of rows that a wave forms once more, from memory.  A hidden row has the weight zero, and zero times a row
// with NaN or infinities is NaN: where a wave's sums are not finite, they are formed again over what each of its
// columns sees, as products (blocks of 32 rows that every column sees) and a row at a time (the others).  These
// paths are rare, and nothing of them may cost the loops before them: the lane is opaque and the loads are
// kept in order, so that no address and no operand of theirs lies in a register outside them.
// ---------------------------------------------------------------------------
struct RareLane {
  int c, h;   // column, lane half
  __device__ __forceinline__ RareLane() {
    int l = threadIdx.x % WAVE;
    asm volatile("" : "+v"(l));
    c = l % 32;
    h = l / 32;
  }
};
template <int N>
__device__ __forceinline__ bool not_finite(const f32x16 (&o)[N]) {
  float x = 0.f;   // NaN from the first NaN or infinity on
#pragma unroll
  for (int d = 0; d < N; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e) x = __builtin_fmaf(o[d][e], 0.f, x);
  return x != 0.f;
}
// Whether none of a lane's results is finite: no further row changes that.
template <int N>
__device__ __forceinline__ bool none_finite(const f32x16 (&o)[N]) {
  float x = INFINITY;   // NaN is passed over
#pragma unroll
  for (int d = 0; d < N; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e) x = fminf(x, fabsf(o[d][e]));
  return !(x < INFINITY);
}
// the products of 32 rows with the wave's columns, q(i) operand i of them
template <class T, int D, class S, class Q>
__device__ __forceinline__ f32x16 rare_products(const S* rows, int stride, Q q) {
  const RareLane l;
  const S* r = rows + (unsigned)(l.c * stride + 8 * l.h);
  f32x16 s = zero16();
#pragma unroll
  for (int i = 0; i < D / 16; ++i) {
    Frag<T> f;
    load8(f, r + 16 * i, true);
    mma32(s, f, q(i));
    asm volatile("" ::: "memory");
  }
  return s;
}
// o += rows^T w over 32 rows, w as rare_products gives them, rounded to the io type
template <class T, int D, class S>
__device__ __forceinline__ void rare_add(f32x16 (&o)[D / 32], const S* rows, int stride, const f32x16& w) {
  const RareLane l;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const Frag<T> p = frag_of<T>(w, i);
#pragma unroll
    for (int d = 0; d < D / 32; ++d) {
      Frag<T> f;
#pragma unroll
      for (int e = 0; e < 8; ++e)
        f.set(e, io_to_float((rows + (16 * i + 8 * (e / 4) + e % 4) * stride + 32 * d)[(unsigned)(4 * l.h * stride + l.c)]));
      mma32(o[d], f, p);
      asm volatile("" ::: "memory");
    }
  }
}
// one row's products with the columns
template <class T, int D, class S, class Q>
__device__ __forceinline__ float rare_product(const S* row, Q q) {
  const RareLane l;
  const S* r = row + 8 * l.h;
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < D / 16; ++i) {
    Frag<T> f, x = q(i);
    load8(f, r + 16 * i, true);
    if constexpr (IsBf16<T>::value) asm volatile("" : "+v"(x.v)::"memory");   // unpacked here, not before the loops
#pragma unroll
    for (int e = 0; e < 8; ++e) s = __builtin_fmaf(f.get(e), x.get(e), s);
  }
  return half_sum(s);
}
// o += row w in the columns that see it, w rounded to the io type
template <class T, int D, class S>
__device__ __forceinline__ void rare_add(f32x16 (&o)[D / 32], const S* row, float w, bool sees) {
  const RareLane l;
  const S* r = row + 4 * l.h;
  const float p = sees ? (float)(T)w : 0.f;
#pragma unroll
  for (int d = 0; d < D / 32; ++d) {
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float x = io_to_float(r[32 * d + 8 * (e / 4) + e % 4]);
      o[d][e] = __builtin_fmaf(p, sees ? x : 0.f, o[d][e]);
      if (e % 8 == 7) asm volatile("" ::: "memory");
    }
  }
}

// four consecutive values in the io type
__device__ __forceinline__ void store_io4(u16* p, f32x4 v) {
  const bf16x4 b = {(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
  *reinterpret_cast<bf16x4*>(p) = b;
}
__device__ __forceinline__ void store_io4(float* p, f32x4 v) { *reinterpret_cast<f32x4*>(p) = v; }

// This wave's loads to LDS have arrived, and its reads of LDS are done.
__device__ __forceinline__ void wait_lds_loads() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0070);   // vmcnt(0) lgkmcnt(0); the compiler counts its own loads as arrived, too
  asm volatile("" ::: "memory");
}
// This wave's loads to registers have arrived.  Before a loop that stages tiles: the
// compiler would else wait for them at their first use, in every iteration, and so
// for the tile that is on its way.
__device__ __forceinline__ void wait_reg_loads() { __builtin_amdgcn_s_waitcnt(0x0f70); }   // vmcnt(0)
// Every wave's loads to LDS have arrived, and its reads are done; up to LATER of the wave's
// last memory instructions may be on their way.  Counted in issue order: at least LATER must
// have been issued after the loads to LDS (stores of the step, which a wait for all would
// otherwise wait out, a memory latency each time).
template <int LATER>
__device__ __forceinline__ void sync_tiles_but() {
  static_assert(LATER < 64, "six bits");
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((LATER & 15) | (LATER >> 4) << 14 | 0x0070);
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
// Every wave's reads and writes of LDS are done; loads may be on their way.
__device__ __forceinline__ void sync_lds() { sync_tiles_but<63>(); }
// Every wave's loads to LDS have arrived, and its reads are done.
__device__ __forceinline__ void sync_tiles() {
  wait_lds_loads();
  __syncthreads();
}

// Loads ROWS rows of a window into a RowTile at LDS address L, by NW waves of which
// this is wave w, straight to LDS (16 bytes a lane, no registers in between).  A
// wave writes 1024 consecutive bytes of LDS at once; the swizzle is in the rows'
// and chunks' choice by each lane.  Rows outside the window become zeros.
// The loads are assembly without outputs: the compiler, which would wait for the
// builtin's before the next transposed read of any LDS, does not count them, so
// wait_lds_loads / sync_tiles must come between them and the reads of the tile.  The LDS address is m0's, an
// operand, so that the compiler writes it and knows what it holds; one wait state lies between that and its use.
template <class T, int D, int ROWS, int NW>
__device__ __forceinline__ void stage_tile(const char* L, u32x4 rs, int stride_bytes, int w) {
  using RT = RowTile<T, D>;
  constexpr int PER = 1024 / RT::ROW;          // rows per wave and instruction
  static_assert(PER >= 1 && ROWS % PER == 0, "rows of a staged tile");
  constexpr int STEPS = ROWS / PER;
  const int l = threadIdx.x % WAVE;
  const int lr = l / RT::CH, lc = l % RT::CH;
  const unsigned base = (unsigned)(size_t)(__attribute__((address_space(3))) const char*)L;
#pragma unroll
  for (int n = 0; n < (STEPS + NW - 1) / NW; ++n) {
    const int step = n * NW + w;
    if (STEPS % NW == 0 || step < STEPS) {
      const int r = step * PER + lr;
      const int off = r * stride_bytes + ((lc ^ RT::swz(r)) << 4);
      const unsigned to = __builtin_amdgcn_readfirstlane(base + step * 1024);
      asm volatile("s_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"{m0}"(to), "v"(off), "s"(rs)
                   : "memory");
    }
  }
}

// 64 consecutive floats of a window to LDS, by one wave; zeros behind it.
__device__ __forceinline__ void stage_floats(const char* L, u32x4 rs) {
  const unsigned to = __builtin_amdgcn_readfirstlane((unsigned)(size_t)(__attribute__((address_space(3))) const char*)L);
  const int off = threadIdx.x % WAVE * 4;
  asm volatile("s_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"{m0}"(to), "v"(off), "s"(rs) : "memory");
}

}  // namespace flex
