// Device helpers of the kernels that go over rows once: 16 bytes of a row as fp32
// values, SiLU, and which sequence a packed row belongs to.
#pragma once
#include "flex_seq.hpp"

namespace flex {

// 16 bytes of a row
template <class S> struct Piece {
  static constexpr int N = 16 / sizeof(S);
  uint4 raw;
  __device__ __forceinline__ void load(const S* p) { raw = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void zero() { raw = make_uint4(0, 0, 0, 0); }
  __device__ __forceinline__ void get(float* x) const {
    const unsigned w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(S) == 2) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      } else {
        x[i] = __uint_as_float(w[i]);
      }
    }
  }
  __device__ __forceinline__ static void store(S* p, const float* x) {
    if constexpr (sizeof(S) == 2) {
      bf16x8 b;
#pragma unroll
      for (int i = 0; i < 8; ++i) b[i] = (__bf16)x[i];
      *reinterpret_cast<bf16x8*>(p) = b;
    } else {
      *reinterpret_cast<f32x4*>(p) = f32x4{x[0], x[1], x[2], x[3]};
    }
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
