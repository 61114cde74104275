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
constexpr int ATTN_PARTS = 256;   // of one sequence's keys, at most
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
  float* delta;           // [2][Hq][Tq] workspace: lse in units of log2, then rows of dO . O
  void* dQ;
  void* dK;
  void* dV;
};

hipError_t launch_attn_fwd(const AttnArgs& a, bool bf16, int d, hipStream_t st);
hipError_t launch_attn_bwd(const AttnArgs& a, bool bf16, int d, hipStream_t st);

// Gated delta rule.  What the chunks of 64 tokens need beside the rows is kept per chunk
// slot and value head (block slot * H + head):
//   prep   T, then P (lower triangular [64][64]): hi and lo bf16, or fp32, each as the rows 0..31
//          of the columns 0..31 and the rows 32..63, in the order of the sweeps' LDS tiles;
//          e^G [64], w [64], b [64] (fp32) in 1 KB; G [64] (fp64) in 1 KB
//   st     the state at the chunk's start as FragRows [dv][d], io type   (training)
//   ut     U as FragRows [dv][64], hi and lo (fp32: one)                 (training)
constexpr int DELTA_CHUNK = 64;
constexpr int DELTA_MAT_BYTES = (32 * 32 + 32 * 64) * 4;   // T or P: hi and lo, or fp32
constexpr int DELTA_SWEEP_BYTES = 2 * DELTA_MAT_BYTES + 1024;
constexpr int DELTA_PREP_BYTES = DELTA_SWEEP_BYTES + 1024;

struct DeltaArgs {
  const void* Q;
  const void* K;
  const void* V;
  const float* g;
  const float* beta;
  const int32_t* off;
  const float* state0;   // NULL: zero
  float* state;          // NULL: not wanted
  void* O;
  int B, T, Hk, H, d, dv;
  int qs, ks, vs;
  float scale;
  char* prep;
  void* st;              // NULL: not kept
  void* ut;
  // backward
  const void* dO;
  void* dst;             // gradient of the state at the chunk's end, as st
  void* drt;             // gradient of T^-1 U = b (V - e^G K S), as ut
  void* dQ;
  void* dK;
  void* dV;
  void* dg;
  void* dbeta;
};

hipError_t launch_delta_fwd(const DeltaArgs& a, bool bf16, hipStream_t st);
hipError_t launch_delta_bwd(const DeltaArgs& a, bool bf16, hipStream_t st);
hipError_t launch_delta_step(const DeltaArgs& a, bool bf16, hipStream_t st);

}  // namespace flex
