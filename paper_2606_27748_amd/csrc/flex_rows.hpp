// Device helpers of the kernels that go over rows once: 16 bytes of a row as fp32
// values, SiLU, and which sequence a packed row belongs to.
#pragma once
#include "flex_seq.hpp"

namespace flex {

// 16 bytes of a row (or 8)
template <class S, int BYTES = 16> struct Piece {
  static constexpr int N = BYTES / sizeof(S), WORDS = BYTES / 4;
  typedef unsigned Words __attribute__((ext_vector_type(WORDS)));
  Words raw;
  __device__ __forceinline__ void load(const S* p) { raw = *reinterpret_cast<const Words*>(p); }
  __device__ __forceinline__ void save(S* p) const { *reinterpret_cast<Words*>(p) = raw; }
  // of a window of rows, at a lane's place in a row (nothing outside the window) and a row's place in it, in bytes
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t rs, int at, int row) {
    if constexpr (WORDS == 1) raw[0] = __builtin_amdgcn_raw_buffer_load_b32(rs, at, row, 0);
    if constexpr (WORDS == 2) raw = __builtin_bit_cast(Words, __builtin_amdgcn_raw_buffer_load_b64(rs, at, row, 0));
    if constexpr (WORDS == 4) raw = __builtin_bit_cast(Words, __builtin_amdgcn_raw_buffer_load_b128(rs, at, row, 0));
  }
  // A store of 16 bytes has its row in the lane's offset: with a scalar one the first word has been seen to be what the
  // next instruction put into its register (in one of 2000 lanes), and the compiler leaves no room between them.
  __device__ __forceinline__ void save(__amdgpu_buffer_rsrc_t rs, int at, int row) const {
    if constexpr (WORDS == 1) __builtin_amdgcn_raw_buffer_store_b32(raw[0], rs, at, row, 0);
    if constexpr (WORDS == 2) __builtin_amdgcn_raw_buffer_store_b64(raw, rs, at, row, 0);
    if constexpr (WORDS == 4) __builtin_amdgcn_raw_buffer_store_b128(raw, rs, (int)((unsigned)at + (unsigned)row), 0, 0);
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < WORDS; ++i) raw[i] = 0;
  }
  __device__ __forceinline__ void get(float* x) const {
#pragma unroll
    for (int i = 0; i < WORDS; ++i) {
      if constexpr (sizeof(S) == 2) {
        x[2 * i] = __uint_as_float(raw[i] << 16);
        x[2 * i + 1] = __uint_as_float(raw[i] & 0xffff0000u);
      } else {
        x[i] = __uint_as_float(raw[i]);
      }
    }
  }
  __device__ __forceinline__ static Piece of(const float* x) {
    Piece v;
#pragma unroll
    for (int i = 0; i < WORDS; ++i) {
      if constexpr (sizeof(S) == 2)
        v.raw[i] = __builtin_bit_cast(unsigned, bf16x2{(__bf16)x[2 * i], (__bf16)x[2 * i + 1]});
      else
        v.raw[i] = __float_as_uint(x[i]);
    }
    return v;
  }
  __device__ __forceinline__ static void store(S* p, const float* x) { of(x).save(p); }
};

constexpr float LOG2E = 1.4426950408889634f;

// 1 / (1 + exp(-z)): the hardware's exponential and reciprocal, an ulp each
__device__ __forceinline__ float sigmoid(float z) {
  return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-LOG2E * z));
}
// the derivative of z sigmoid(z)
__device__ __forceinline__ float dsilu(float z, float sig) { return sig * __builtin_fmaf(z, 1.f - sig, 1.f); }

// The sequence that holds row t, as its rows first .. end-1; b < 0: none does, and none of
// the rows up to end-1.
struct RowSeq {
  int b, first, end;
};
// From what a search says: `cnt` sequences start at row t or before it, the last of them from row `first` on, the next one from row
// `end`.  Where offsets fall the search may be wrong: a sequence that does not hold row t is none, for this row.
__host__ __device__ inline RowSeq row_seq(int cnt, int first, int end, int B, int T, int t) {
  const bool holds = cnt > 0 && first <= t && end > t;
  RowSeq s;
  s.b = holds ? cnt - 1 : -1;
  s.first = first;
  s.end = holds ? end : cnt == 0 ? (end > t ? end : t + 1) : cnt == B ? T : t + 1;
  return s;
}
__device__ __forceinline__ RowSeq find_row(const int32_t* __restrict__ off, int B, int T, int t) {
  const int cnt = leading(B, [=](int b) { return clamp_off(off[b], T) <= t; });
  return row_seq(cnt, __builtin_amdgcn_readfirstlane(clamp_off(off[max(cnt - 1, 0)], T)),
                 __builtin_amdgcn_readfirstlane(clamp_off(off[cnt], T)), B, T, t);
}

}  // namespace flex
