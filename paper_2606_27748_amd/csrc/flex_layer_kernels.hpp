// Host-side launch interface of the kernels of selective state-space layers: short
// convolution, selective scan, gated norm.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace flex {

// records the events of flex_timing_enable around a launch
void timing_mark(int kernel_class, hipStream_t st, bool begin);

// Short convolution.  Strides are between consecutive rows, in elements.  A wave takes
// rows of the packed ones, whatever their sequences, and a lane of it 16 bytes of channels (forward) or
// CONV_BWD_CH channels.
constexpr int CONV_ROWS = 32;        // of a wave in the forward
constexpr int CONV_BWD_ROWS = 64;    // of a wave in the backward
constexpr int CONV_BWD_WAVES = 4;    // of a workgroup, one after the other: one row of partial sums
constexpr int CONV_BWD_CH = 2;
struct ConvArgs {
  const void* X;
  const float* W;
  const float* bias;      // NULL: zero
  const int32_t* off;
  const void* state0;     // NULL: zero
  void* Y;
  void* state;            // NULL: not wanted
  int B, T, D, K, act, xs;
  // backward
  const void* dY;
  void* dX;
  float* part;            // [parts][K + 1][D] workspace
  float* dW;
  float* dbias;           // NULL: not wanted
  int dxs, parts;
};
hipError_t launch_conv_fwd(const ConvArgs& a, bool bf16, hipStream_t st);
hipError_t launch_conv_bwd(const ConvArgs& a, bool bf16, hipStream_t st);
hipError_t launch_conv_step(const ConvArgs& a, bool bf16, hipStream_t st);

// Gated norm.  A team of lanes takes a group of a row at a time.
constexpr int NORM_MAX = 8192;   // channels of a group
// lanes of a group: as many as it has pieces of 8 channels, a power of two up to a wave
inline int norm_team(int group) {
  int team = 1;
  while (team < group / 8 && team < 64) team *= 2;
  return team;
}
struct NormArgs {
  const void* X;
  const void* Z;
  const float* W;
  void* Y;
  int T, D, group, gate, xs, zs;
  float eps;
  int rows;               // that are walked at once
  // backward
  const void* dY;
  void* dX;
  void* dZ;
  float* part;            // [parts][D] workspace
  float* dW;
  int dxs, dzs, parts;
  int wg_rows;            // rows of a workgroup at a time: more than one of narrow ones
};
hipError_t launch_norm_fwd(const NormArgs& a, bool bf16, hipStream_t st);
hipError_t launch_norm_bwd(const NormArgs& a, bool bf16, hipStream_t st);

// Selective scan.
constexpr int SCAN_CHUNK = 64;
struct ScanArgs {
  const void* X;
  const void* Bt;
  const void* Ct;
  const float* dt;
  const float* g;
  const float* D;         // NULL: zero
  const int32_t* off;
  const float* state0;    // NULL: zero
  float* state;           // NULL: not wanted
  void* Y;
  int B, T, G, H, N, P, xs, bs, cs;
  int heads;              // of a workgroup's sweep, all of one group
  // Sequences go in segments of `seg` tokens (a multiple of the chunk), one after the other
  // where carry is NULL (no sequence is longer than one), else at once, from
  //   carry [segment slots][H][N * P]   what each segment leaves of its own, then the state it starts from (as the lanes
  //                                     hold it)
  //   tot   [segment slots][H]          its decay
  int seg;
  float* carry;
  float* tot;
  void* st;               // states at the chunks' starts [chunk slots][H][N * P] as the lanes hold them, io type; NULL: not kept
  // backward
  const void* dY;
  void* dst;              // gradients of the states at the chunks' ends, as st
  void* dX;
  void* dB;
  void* dC;
  void* ddt;
  void* dg;
  float* dD;              // NULL: not wanted
  int dxs, dbs, dcs;
  int parts;              // of a group's heads
  float* part_b;          // [parts][chunk slots * 64][G][N] sums of dB over a part's heads; NULL: one part
  float* part_c;
  float* part_d;          // [chunk slots][H]
};
hipError_t launch_scan_fwd(const ScanArgs& a, bool bf16, hipStream_t st);
hipError_t launch_scan_bwd(const ScanArgs& a, bool bf16, hipStream_t st);
hipError_t launch_scan_step(const ScanArgs& a, bool bf16, hipStream_t st);

}  // namespace flex
