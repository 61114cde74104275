// Gated norm of rows, forward and backward.  With gate s = silu(z), r = 1 / sqrt(mean(u^2) + eps), n = u r:
//   gate first  u = x s,  y = n w        gate last  u = x,  y = n w s        none  u = x,  y = n w
//   dn = dy w (times s, gate last),  du = r (dn - n mean(dn n)),  dW = sum_rows dy n (times s, gate last)
//   first  dx = du s, ds = du x          last  dx = du, ds = dy n w          dz = ds silu'(z)
//
// A team of lanes has a group: 8 channels a lane and piece, the pieces of a group TEAM * 8 channels
// apart.  Teams stay on their channels, with their part of W (and the sum of dW) in registers, and go
// from row to row, the next row on its way while one is worked on.  One pass over the data: bound by
// memory.  Where a mean square leaves what fp32 holds, the row's sums are formed again from scaled values.
// bf16, forward of 17973 rows of 4096 channels, one group: 79 us (442 MB, 5.6 TB/s); forward and backward of 16384 rows of
// 2048 channels in groups of 128: 34.5 us (201 MB) and 55 us (335 MB, 6.1 TB/s), and 5 for the sum of dW.
#include <type_traits>
#include "flex_rows.hpp"
#include "flex_layer_kernels.hpp"
#include "../../include/flex.h"

namespace flex {

namespace {
struct Eight {
  float v[8];
};
template <class S>
struct Raw8 {
  Piece<S> p[8 / Piece<S>::N];
  __device__ __forceinline__ void load(const S* q, bool in) {
#pragma unroll
    for (int i = 0; i < 8 / Piece<S>::N; ++i)
      if (in) p[i].load(q + i * Piece<S>::N);
      else p[i].zero();
  }
  __device__ __forceinline__ void get(Eight& x) const {
#pragma unroll
    for (int i = 0; i < 8 / Piece<S>::N; ++i) p[i].get(x.v + i * Piece<S>::N);
  }
  static __device__ __forceinline__ void store(S* q, const Eight& x) {
#pragma unroll
    for (int i = 0; i < 8 / Piece<S>::N; ++i) Piece<S>::store(q + i * Piece<S>::N, x.v + i * Piece<S>::N);
  }
};

// Sums over a team, in every lane of it: aligned lanes of a wave, `team` a power of two, or a
// workgroup of four waves (each passes through `box`, of which two are used in turn: one barrier a sum).
template <bool WG, int N>
__device__ __forceinline__ void team_sum(float (&x)[N], int team, float (*box)[4], int turn) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if (WG || team > 1) x[i] = dpp_add(x[i], 0);
    if (WG || team > 2) x[i] = dpp_add(x[i], 1);
    if (WG || team > 4) x[i] = dpp_add(x[i], 2);
    if (WG || team > 8) x[i] = dpp_add(x[i], 3);
    if (WG || team > 16) {
      const unsigned v = __float_as_uint(x[i]);
      const auto p = __builtin_amdgcn_permlane16_swap(v, v, false, false);
      x[i] = __uint_as_float(p[0]) + __uint_as_float(p[1]);
    }
    if (WG || team > 32) x[i] = half_sum(x[i]);
  }
  if (WG) {
    const int w = threadIdx.x / WAVE;
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (threadIdx.x % WAVE == 0) box[turn * N + i][w] = x[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = (box[turn * N + i][0] + box[turn * N + i][1]) + (box[turn * N + i][2] + box[turn * N + i][3]);
  }
}

// Mean squares from 2^-96 on have their squares' bits, and no sum behind infinity has.  Others (eps = 0 allows any) are formed
// again from values times 2^96 or 2^-96, in place: with a way of its own for such rows behind the sums, other rows' registers grew by
// up to half (backward of 20000 rows of 2056 channels, bf16: 154 us for 143).
constexpr float NORM_LOW = 0x1p-96f;
__device__ __forceinline__ bool norm_plain(float mean) { return mean >= NORM_LOW && mean < INFINITY; }
__device__ __forceinline__ float norm_scale(float mean) { return mean < NORM_LOW ? 1.f / NORM_LOW : NORM_LOW; }
// whether a row's team has such a mean: of a workgroup, which has one row, as a scalar
template <bool WG>
__device__ __forceinline__ bool norm_rare(float mean) {
  return WG ? !norm_plain(__uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(mean)))) : !norm_plain(mean);
}
}  // namespace

// Where a lane works: rows row0, row0 + step, ... and pieces at channels c + i * team * 8 of them
struct NormPlace {
  int row0, step, c, end, team;
  // rows of a workgroup (narrow ones) or of the launch
  template <bool WG>
  __device__ __forceinline__ static NormPlace of(const NormArgs& a, int team, bool narrow) {
    NormPlace p;
    const int groups = a.D / a.group;
    p.team = WG ? 256 : team;
    const unsigned id = narrow ? threadIdx.x : blockIdx.x * 256u + threadIdx.x, t = WG ? blockIdx.x : id / (unsigned)team;
    p.row0 = t / (unsigned)groups;
    const int base = t % (unsigned)groups * a.group;
    p.c = base + (WG ? (int)threadIdx.x : (int)(id % (unsigned)team)) * 8;
    p.end = base + a.group;
    p.step = a.rows;
    if (narrow) p.row0 = p.row0 < a.wg_rows ? (int)blockIdx.x * a.wg_rows + p.row0 : a.T;
    return p;
  }
};

template <class S, int GATE, int PIECES, bool WG>
__global__ __launch_bounds__(256) void k_norm_fwd(NormArgs a, int team, float inv) {
  __shared__ float box[3][4];
  const NormPlace p = NormPlace::of<WG>(a, team, false);
  if (p.row0 >= a.rows) return;   // never a part of a team
  Eight w[PIECES];
  Raw8<S> nx[PIECES], nz[PIECES];
  bool in[PIECES];
  auto fetch = [&](int row) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int c = p.c + i * p.team * 8;
      nx[i].load(static_cast<const S*>(a.X) + (size_t)row * a.xs + c, in[i]);
      if (GATE != FLEX_GATE_NONE) nz[i].load(static_cast<const S*>(a.Z) + (size_t)row * a.zs + c, in[i]);
    }
  };
#pragma unroll
  for (int i = 0; i < PIECES; ++i) in[i] = p.c + i * p.team * 8 < p.end;
  fetch(p.row0);
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    Raw8<float> r;
    r.load(a.W + p.c + i * p.team * 8, in[i]);
    r.get(w[i]);
  }
  int turn = 0;
  for (int row = p.row0; row < a.T; row += p.step, turn ^= 1) {
    Eight u[PIECES], s[PIECES];
    float sum[1] = {0.f};
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      nx[i].get(u[i]);
      if (GATE != FLEX_GATE_NONE) {
        nz[i].get(s[i]);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[i].v[e] *= sigmoid(s[i].v[e]);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (GATE == FLEX_GATE_FIRST) u[i].v[e] *= s[i].v[e];
        sum[0] = __builtin_fmaf(u[i].v[e], u[i].v[e], sum[0]);
      }
    }
    if (row + p.step < a.T) fetch(row + p.step);
    team_sum<WG>(sum, team, box, turn);
    const float mean = __builtin_fmaf(sum[0], inv, a.eps);
    float r = __builtin_amdgcn_rsqf(mean);
    if (norm_rare<WG>(mean)) {
      const float k = norm_scale(mean);
      sum[0] = 0.f;
#pragma unroll
      for (int i = 0; i < PIECES; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          u[i].v[e] *= k;
          sum[0] = __builtin_fmaf(u[i].v[e], u[i].v[e], sum[0]);
        }
      team_sum<WG>(sum, team, box + 2, 0);
      r = __builtin_amdgcn_rsqf(__builtin_fmaf(sum[0], inv, a.eps * k * k));
    }
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        u[i].v[e] = u[i].v[e] * r * w[i].v[e];
        if (GATE == FLEX_GATE_LAST) u[i].v[e] *= s[i].v[e];
      }
      if (in[i]) Raw8<S>::store(static_cast<S*>(a.Y) + (size_t)row * a.D + p.c + i * p.team * 8, u[i]);
    }
  }
}

// NARROW: a workgroup has wg_rows whole rows at a time, and its sums of dW are one row of partial sums; otherwise each
// row that is walked has its own.
template <class S, int GATE, int PIECES, bool WG, bool NARROW>
__global__ __launch_bounds__(256) void k_norm_bwd(NormArgs a, int team, float inv) {
  __shared__ float box[6][4];
  __shared__ float sums[NARROW ? 256 * 8 : 1];
  const NormPlace p = NormPlace::of<WG>(a, team, NARROW);
  if (!NARROW && p.row0 >= a.rows) return;
  Eight w[PIECES], dw[PIECES];
  Raw8<S> nx[PIECES], nz[PIECES], ng[PIECES];
  bool in[PIECES];
  auto fetch = [&](int row) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int c = p.c + i * p.team * 8;
      nx[i].load(static_cast<const S*>(a.X) + (size_t)row * a.xs + c, in[i]);
      if (GATE != FLEX_GATE_NONE) nz[i].load(static_cast<const S*>(a.Z) + (size_t)row * a.zs + c, in[i]);
      ng[i].load(static_cast<const S*>(a.dY) + (size_t)row * a.D + c, in[i]);
    }
  };
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    in[i] = p.c + i * p.team * 8 < p.end;
#pragma unroll
    for (int e = 0; e < 8; ++e) dw[i].v[e] = 0.f;
  }
  if (p.row0 < a.T) fetch(p.row0);
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    Raw8<float> r;
    r.load(a.W + p.c + i * p.team * 8, in[i]);
    r.get(w[i]);
  }
  int turn = 0;
  for (int row = p.row0; row < a.T; row += p.step, turn ^= 1) {
    Eight x[PIECES], z[PIECES], sig[PIECES], g[PIECES];
    float sum[2] = {0.f, 0.f};   // of u^2, of dn u
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      nx[i].get(x[i]);
      ng[i].get(g[i]);
      if (GATE != FLEX_GATE_NONE) nz[i].get(z[i]);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (GATE != FLEX_GATE_NONE) sig[i].v[e] = sigmoid(z[i].v[e]);
        const float s = GATE != FLEX_GATE_NONE ? z[i].v[e] * sig[i].v[e] : 1.f;
        const float u = GATE == FLEX_GATE_FIRST ? x[i].v[e] * s : x[i].v[e];
        float dn = g[i].v[e] * w[i].v[e];
        if (GATE == FLEX_GATE_LAST) dn *= s;
        sum[0] = __builtin_fmaf(u, u, sum[0]);
        sum[1] = __builtin_fmaf(dn, u, sum[1]);
      }
    }
    if (row + p.step < a.T) fetch(row + p.step);
    team_sum<WG>(sum, team, box, turn);
    const float mean = __builtin_fmaf(sum[0], inv, a.eps);
    float r = __builtin_amdgcn_rsqf(mean), k = 1.f;
    if (norm_rare<WG>(mean)) {   // x and r of the scaled row from here on
      k = norm_scale(mean);
      sum[0] = sum[1] = 0.f;
#pragma unroll
      for (int i = 0; i < PIECES; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          x[i].v[e] *= k;
          const float s = GATE != FLEX_GATE_NONE ? z[i].v[e] * sig[i].v[e] : 1.f;
          const float u = GATE == FLEX_GATE_FIRST ? x[i].v[e] * s : x[i].v[e];
          float dn = g[i].v[e] * w[i].v[e];
          if (GATE == FLEX_GATE_LAST) dn *= s;
          sum[0] = __builtin_fmaf(u, u, sum[0]);
          sum[1] = __builtin_fmaf(dn, u, sum[1]);
        }
      team_sum<WG>(sum, team, box + 4, 0);
      r = __builtin_amdgcn_rsqf(__builtin_fmaf(sum[0], inv, a.eps * k * k));
    }
    const float m = sum[1] * r * inv;   // mean(dn n)
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      Eight dz;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float s = GATE != FLEX_GATE_NONE ? z[i].v[e] * sig[i].v[e] : 1.f;
        const float ds = GATE != FLEX_GATE_NONE ? dsilu(z[i].v[e], sig[i].v[e]) : 0.f;
        const float n = (GATE == FLEX_GATE_FIRST ? x[i].v[e] * s : x[i].v[e]) * r;
        const float gn = g[i].v[e] * n;
        float dn = g[i].v[e] * w[i].v[e];
        if (GATE == FLEX_GATE_LAST) dn *= s;
        const float du = r * (dn - n * m);
        dw[i].v[e] += GATE == FLEX_GATE_LAST ? gn * s : gn;
        dz.v[e] = (GATE == FLEX_GATE_FIRST ? du * x[i].v[e] : gn * w[i].v[e]) * ds;
        x[i].v[e] = (GATE == FLEX_GATE_FIRST ? du * s : du) * k;
      }
      const int c = p.c + i * p.team * 8;
      if (in[i]) {
        Raw8<S>::store(static_cast<S*>(a.dX) + (size_t)row * a.dxs + c, x[i]);
        if (GATE != FLEX_GATE_NONE) Raw8<S>::store(static_cast<S*>(a.dZ) + (size_t)row * a.dzs + c, dz);
      }
    }
  }
  if constexpr (NARROW) {
    const int row = (int)threadIdx.x / team / (a.D / a.group);
    if (row < a.wg_rows && in[0]) Raw8<float>::store(sums + row * a.D + p.c, dw[0]);
    __syncthreads();
    for (int c = threadIdx.x; c < a.D; c += 256) {
      float v = sums[c];
      for (int r = 1; r < a.wg_rows; ++r) v += sums[r * a.D + c];
      a.part[(size_t)blockIdx.x * a.D + c] = v;
    }
  } else {
#pragma unroll
    for (int i = 0; i < PIECES; ++i)
      if (in[i]) Raw8<float>::store(a.part + (size_t)p.row0 * a.D + p.c + i * p.team * 8, dw[i]);
  }
}

// Sums of the parts, 64 channels to a workgroup, each of its 16 waves a sixteenth of the parts.
__global__ __launch_bounds__(1024) void k_norm_sum(NormArgs a) {
  __shared__ double sums[16][WAVE];
  const int l = threadIdx.x % WAVE, w = threadIdx.x / WAVE, c = blockIdx.x * WAVE + l;
  const float* p = a.part + (c < a.D ? c : 0);
  const int per = (a.parts + 15) / 16, p0 = w * per, p1 = min(p0 + per, a.parts);
  double s = 0.0;
#pragma unroll 8
  for (int i = p0; i < p1; ++i) s += (double)p[(size_t)i * a.D];
  sums[w][l] = s;
  __syncthreads();
  if (w > 0 || c >= a.D) return;
#pragma unroll
  for (int i = 1; i < 16; ++i) s += sums[i][l];
  a.dW[c] = (float)s;
}

namespace {
// Up to a wave a team has norm_team lanes, then a wave of up to four pieces a lane, then a workgroup.
template <bool BWD, class S, int GATE>
void run(const NormArgs& a, hipStream_t st) {
  const int units = a.group / 8, groups = a.D / a.group;
  const float inv = 1.f / (float)a.group;
  const int team = norm_team(a.group);
  const int64_t teams = (int64_t)a.rows * groups;
  const unsigned grid = (unsigned)((teams * team + 255) / 256), wide = (unsigned)teams;
  auto go = [&](auto pieces, auto wg) {
    constexpr int P = decltype(pieces)::value;
    constexpr bool W = decltype(wg)::value;
    if constexpr (!BWD) {
      k_norm_fwd<S, GATE, P, W><<<W ? wide : grid, 256, 0, st>>>(a, team, inv);
    } else {
      if constexpr (P == 1) {
        if (a.wg_rows > 1) {
          k_norm_bwd<S, GATE, P, W, true><<<a.parts, 256, 0, st>>>(a, team, inv);
          return;
        }
      }
      k_norm_bwd<S, GATE, P, W, false><<<W ? wide : grid, 256, 0, st>>>(a, team, inv);
    }
  };
  using std::integral_constant;
  if (units <= 64) go(integral_constant<int, 1>{}, integral_constant<bool, false>{});
  else if (units <= 128) go(integral_constant<int, 2>{}, integral_constant<bool, false>{});
  else if (units <= 256) go(integral_constant<int, 4>{}, integral_constant<bool, false>{});
  else if (units <= 512) go(integral_constant<int, 2>{}, integral_constant<bool, true>{});
  else go(integral_constant<int, 4>{}, integral_constant<bool, true>{});
}
template <bool BWD, class S>
void by_gate(const NormArgs& a, hipStream_t st) {
  if (a.gate == FLEX_GATE_NONE) run<BWD, S, FLEX_GATE_NONE>(a, st);
  if (a.gate == FLEX_GATE_FIRST) run<BWD, S, FLEX_GATE_FIRST>(a, st);
  if (a.gate == FLEX_GATE_LAST) run<BWD, S, FLEX_GATE_LAST>(a, st);
}
}  // namespace

hipError_t launch_norm_fwd(const NormArgs& a, bool bf16, hipStream_t st) {
  timing_mark(FLEX_KERNEL_NORM_FWD, st, true);
  bf16 ? by_gate<false, u16>(a, st) : by_gate<false, float>(a, st);
  timing_mark(FLEX_KERNEL_NORM_FWD, st, false);
  return hipGetLastError();
}
hipError_t launch_norm_bwd(const NormArgs& a, bool bf16, hipStream_t st) {
  timing_mark(FLEX_KERNEL_NORM_BWD, st, true);
  bf16 ? by_gate<true, u16>(a, st) : by_gate<true, float>(a, st);
  k_norm_sum<<<(a.D + WAVE - 1) / WAVE, 1024, 0, st>>>(a);
  timing_mark(FLEX_KERNEL_NORM_BWD, st, false);
  return hipGetLastError();
}

}  // namespace flex
