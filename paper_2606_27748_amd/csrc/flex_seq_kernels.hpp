// Host-side launch interface of the packed-sequence kernels.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace flex {

// records the events of flex_timing_enable around a launch
void timing_mark(int kernel_class, hipStream_t st, bool begin);

// Exact attention.  Strides are between consecutive rows, in elements; O, dO and
// the gradients are contiguous.
struct AttnArgs {
  const void* Q;
  const void* K;
  const void* V;
  const int32_t* q_off;
  const int32_t* k_off;
  const int32_t* k_len;   // NULL: all of the sequence's key rows
  void* O;
  float* lse;             // [Tq][Hq]; the backward reads it
  int B, Hq, Hkv, Tq, Tk, causal;
  int qs, ks, vs;
  float scale;
  // forward of few rows per sequence: keys in nsplit parts, combined from
  // part_o [Tq][Hq][nsplit][D] and part_ml [Tq][Hq][nsplit][2]
  int nsplit;
  float* part_o;
  float* part_ml;
  // backward
  const void* dO;
  float* delta;           // [Tq][Hq] workspace: rows of dO . O
  void* dQ;
  void* dK;
  void* dV;
};

hipError_t launch_attn_fwd(const AttnArgs& a, bool bf16, int d, hipStream_t st);
hipError_t launch_attn_bwd(const AttnArgs& a, bool bf16, int d, hipStream_t st);

}  // namespace flex
