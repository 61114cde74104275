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
  __device__ __forceinline__ static void store(S* p, const float* x) {
    Piece v;
#pragma unroll
    for (int i = 0; i < WORDS; ++i) {
      if constexpr (sizeof(S) == 2)
        v.raw[i] = __builtin_bit_cast(unsigned, bf16x2{(__bf16)x[2 * i], (__bf16)x[2 * i + 1]});
      else
        v.raw[i] = __float_as_uint(x[i]);
    }
    v.save(p);
  }
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
__device__ __forceinline__ RowSeq find_row(const int32_t* __restrict__ off, int B, int T, int t) {
  const int cnt = leading(B, [=](int b) { return clamp_off(off[b], T) <= t; });
  RowSeq s;
  s.b = cnt - 1;
  s.first = __builtin_amdgcn_readfirstlane(clamp_off(off[max(cnt - 1, 0)], T));
  s.end = __builtin_amdgcn_readfirstlane(clamp_off(off[cnt], T));
  if (cnt == 0) s.end = max(s.end, t + 1);
  if (cnt > 0 && s.end <= t) {
    s.b = -1;
    s.end = cnt == B ? T : t + 1;
  }
  return s;
}

}  // namespace flex
