// Short causal convolution of packed rows: forward, backward, single-token step.
//
//   z_t = bias + sum_{k<K} W[:,k] x_{t-K+1+k},  y = z or z sigmoid(z)
//   dz = dy act'(z),  dx_t = sum_k W[:,k] dz_{t+K-1-k},  dW[:,k] = sum_t dz_t x_{t-K+1+k},  dbias = sum_t dz_t
//
// A lane has some of a row's channels with their taps in registers and walks down the rows, the
// K-1 rows before the present one in registers too: every row is read once, but for the K-1 that
// a tile shares with its neighbour.  Rows go through windows that hold a tile: a lane behind the last channel
// reads zeros and writes nothing, without a branch, and a row's place is a scalar.
#include "flex_rows.hpp"
#include "flex_layer_kernels.hpp"
#include "../../include/flex.h"

namespace flex {

namespace {
typedef float f32x2 __attribute__((ext_vector_type(2)));
constexpr int OUTSIDE = 0x7fffff00;   // of any window of rows: a lane there reads zeros and writes nothing

// a lane's channels' taps and bias
template <int E, int K>
struct Taps {
  float w[E * K], bias[E];
  __device__ __forceinline__ void load(const ConvArgs& a, int c) {
#pragma unroll
    for (int i = 0; i < E * K / 2; ++i) *reinterpret_cast<f32x2*>(w + 2 * i) = reinterpret_cast<const f32x2*>(a.W + (size_t)c * K)[i];
#pragma unroll
    for (int i = 0; i < E; ++i) bias[i] = a.bias ? a.bias[c + i] : 0.f;
  }
  // z of a row from the K-1 before it and itself
  __device__ __forceinline__ void conv(float (&z)[E], const float (&win)[K - 1][E], const float (&x)[E]) const {
#pragma unroll
    for (int i = 0; i < E; ++i) {
      float s = bias[i];
#pragma unroll
      for (int k = 0; k < K - 1; ++k) s = __builtin_fmaf(w[i * K + k], win[k][i], s);
      z[i] = __builtin_fmaf(w[i * K + K - 1], x[i], s);
    }
  }
};

// the K-1 rows before row t of a sequence
template <class S, int K, int E>
__device__ __forceinline__ void window(float (&win)[K - 1][E], const ConvArgs& a, const RowSeq& q, int t, int c) {
#pragma unroll
  for (int k = 0; k < K - 1; ++k) {
    const int r = t - (K - 1) + k;
    Piece<S, E * (int)sizeof(S)> p;
    p.zero();
    if (r >= q.first)
      p.load(static_cast<const S*>(a.X) + (size_t)r * a.xs + c);
    else if (a.state0)
      p.load(static_cast<const S*>(a.state0) + ((size_t)q.b * (K - 1) + (K - 1 + r - q.first)) * a.D + c);
    p.get(win[k]);
  }
}

template <int K, int E>
__device__ __forceinline__ void shift(float (&win)[K - 1][E], const float (&x)[E]) {
#pragma unroll
  for (int i = 0; i < E; ++i) {
#pragma unroll
    for (int k = 0; k + 1 < K - 1; ++k) win[k][i] = win[k + 1][i];
    win[K - 2][i] = x[i];
  }
}

// the last K-1 rows of sequence b, of state0 where it is shorter: all read before any is written
template <class S, int K>
__device__ __forceinline__ void last_rows(const ConvArgs& a, int b, int c) {
  const SeqRange r = seq_range(a.off, b, a.T);
  Piece<S> p[K - 1];
#pragma unroll
  for (int k = 0; k < K - 1; ++k) {
    const int t = r.n - (K - 1) + k;
    p[k].zero();
    if (t >= 0)
      p[k].load(static_cast<const S*>(a.X) + (size_t)(r.row0 + t) * a.xs + c);
    else if (a.state0)
      p[k].load(static_cast<const S*>(a.state0) + ((size_t)b * (K - 1) + (K - 1 + t)) * a.D + c);
  }
#pragma unroll
  for (int k = 0; k < K - 1; ++k)
    p[k].save(static_cast<S*>(a.state) + ((size_t)b * (K - 1) + k) * a.D + c);
}
}  // namespace

// Waves 0 .. tiles-1 of a span of channels have CONV_ROWS rows each, the B behind them a sequence's last rows.
// 16 bytes a lane, the next eight rows on their way.  Bound by memory: 35947 rows of 4352 channels in 16 prompts,
// bf16, 625 MB in 122 us (5.1 TB/s, a large copy's rate).
template <class S, int K, bool SILU>
__global__ __launch_bounds__(256) void k_conv_fwd(ConvArgs a, int spans, int tiles, int first_b) {
  constexpr int E = Piece<S>::N, U = 8;
  const int l = threadIdx.x % WAVE, w = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
  const int tile = blockIdx.x / spans * 4 + w, c = (blockIdx.x % spans * WAVE + l) * E;
  const bool in = c < a.D;
  const int cc = in ? c : 0;
  if (tile >= tiles) {
    const int b = tile - tiles + first_b;
    if (b < a.B && a.state && in) last_rows<S, K>(a, b, c);
    return;
  }
  const int r0 = tile * CONV_ROWS, r1 = min(r0 + CONV_ROWS, a.T);
  const int at = in ? c * (int)sizeof(S) : OUTSIDE, xb = a.xs * (int)sizeof(S), yb = a.D * (int)sizeof(S);
  const auto X = row_window(static_cast<const S*>(a.X), r0, a.xs, r1 - r0, a.D);
  const auto Y = row_window(static_cast<S*>(a.Y), r0, a.D, r1 - r0, a.D);
  Piece<S> next[U];
#pragma unroll
  for (int u = 0; u < U; ++u) next[u].load(X, at, (min(r0 + u, r1 - 1) - r0) * xb);
  Taps<E, K> taps;
  taps.load(a, cc);
  RowSeq q = find_row(a.off, a.B, a.T, r0);
  float win[K - 1][E] = {};
  if (q.b >= 0) window<S, K>(win, a, q, r0, cc);
  for (int t0 = r0; t0 < r1; t0 += U) {
    Piece<S> cur[U];
#pragma unroll
    for (int u = 0; u < U; ++u) cur[u] = next[u];
    if (t0 + U < r1) {
#pragma unroll
      for (int u = 0; u < U; ++u) next[u].load(X, at, (min(t0 + U + u, r1 - 1) - r0) * xb);
    }
    if (q.b >= 0 && t0 + U <= min(q.end, r1)) {   // rows of one sequence: no row's window is moved, but named
      float x[U][E];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float z[E], before[K - 1][E];
        cur[u].get(x[u]);
#pragma unroll
        for (int k = 0; k < K - 1; ++k)
#pragma unroll
          for (int i = 0; i < E; ++i) before[k][i] = u + k < K - 1 ? win[u + k < K - 1 ? u + k : 0][i] : x[u + k < K - 1 ? 0 : u + k - (K - 1)][i];
        taps.conv(z, before, x[u]);
        if (SILU) {
#pragma unroll
          for (int i = 0; i < E; ++i) z[i] *= sigmoid(z[i]);
        }
        Piece<S>::of(z).save(Y, at, (t0 + u - r0) * yb);
      }
#pragma unroll
      for (int k = 0; k < K - 1; ++k)
#pragma unroll
        for (int i = 0; i < E; ++i) win[k][i] = x[U - (K - 1) + k][i];
      continue;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int t = t0 + u;
      if (t < r1) {
        if (t == q.end) {
          q = find_row(a.off, a.B, a.T, t);
          if (q.b >= 0) window<S, K>(win, a, q, t, cc);
        }
        if (q.b >= 0) {
          float x[E], z[E];
          cur[u].get(x);
          taps.conv(z, win, x);
          shift<K, E>(win, x);
          if (SILU) {
#pragma unroll
            for (int i = 0; i < E; ++i) z[i] *= sigmoid(z[i]);
          }
          Piece<S>::of(z).save(Y, at, (t - r0) * yb);
        }
      }
    }
  }
}

// As the forward, over CONV_BWD_ROWS rows and the K-1 behind them, whose dz the last rows' dx take: at row
// t, dz_t is formed and dx of row t - (K-1) is complete.  A workgroup's waves have consecutive rows and
// leave one row of partial sums of dW and dbias.  Bound nearly by memory: 2 x 8192 rows of 4352 channels, bf16, 92 us (428 MB of
// x, dy and dx, and 454 MB by the counters: 4.9 TB/s, where a large copy has 5.2), with the SIMDs busy 76 % of the time by 29
// vector instructions an element, two of them exponential and reciprocal.  Two channels a lane leave five waves
// a SIMD; with four channels 106 us, with eight 143.
template <class S, int K, bool SILU>
__global__ __launch_bounds__(256) void k_conv_bwd(ConvArgs a, int spans) {
  constexpr int E = CONV_BWD_CH, U = 4;
  using P = Piece<S, E * (int)sizeof(S)>;
  __shared__ float sums[CONV_BWD_WAVES - 1][(K + 1) * E][WAVE];
  const int l = threadIdx.x % WAVE, w = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
  const int part = blockIdx.x / spans, c = (blockIdx.x % spans * WAVE + l) * E;
  const bool in = c < a.D;
  const int cc = in ? c : 0;
  const int r0 = (part * CONV_BWD_WAVES + w) * CONV_BWD_ROWS, r1 = min(r0 + CONV_BWD_ROWS, a.T);
  const int at = in ? c * (int)sizeof(S) : OUTSIDE;
  const int xb = a.xs * (int)sizeof(S), gb = a.D * (int)sizeof(S), dxb = a.dxs * (int)sizeof(S);
  const int rows = max(min(r0 + CONV_BWD_ROWS + K - 1, a.T) - r0, 0);
  const auto X = row_window(static_cast<const S*>(a.X), r0, a.xs, rows, a.D);
  const auto G = row_window(static_cast<const S*>(a.dY), r0, a.D, rows, a.D);
  const auto DX = row_window(static_cast<S*>(a.dX), r0, a.dxs, r1 - r0, a.D);
  float dw[K][E] = {}, db[E] = {};
  if (r0 < r1) {
    Taps<E, K> taps;
    taps.load(a, cc);
    for (int t0 = r0; t0 < r1;) {   // a sequence's rows at a time
      const RowSeq q = find_row(a.off, a.B, a.T, t0);
      if (q.b < 0) {
        t0 = q.end;
        continue;
      }
      const int e = min(q.end, r1), stop = e + K - 1, last = min(q.end, r0 + rows) - 1;   // dx of rows t0 .. e-1
      float win[K - 1][E], dzw[K - 1][E] = {};
      window<S, K>(win, a, q, t0, cc);
      P nx[U], ng[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int r = min(t0 + u, last) - r0;
        nx[u].load(X, at, r * xb);
        ng[u].load(G, at, r * gb);
      }
      for (int tb = t0; tb < stop; tb += U) {
        P px[U], pg[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          px[u] = nx[u];
          pg[u] = ng[u];
        }
        if (tb + U < stop) {
#pragma unroll
          for (int u = 0; u < U; ++u) {
            const int r = min(tb + U + u, last) - r0;
            nx[u].load(X, at, r * xb);
            ng[u].load(G, at, r * gb);
          }
        }
        if (tb > t0 && tb + U <= e) {   // every row's dz counts here, and every row's dx is one of the tile's
          static_assert(U >= K - 1, "dx of the rows before the batch");
          float x[U][E], dz[U][E];
#pragma unroll
          for (int u = 0; u < U; ++u) {
            px[u].get(x[u]);
            pg[u].get(dz[u]);
            float before[K - 1][E], z[E], dx[E];
#pragma unroll
            for (int k = 0; k < K - 1; ++k)
#pragma unroll
              for (int i = 0; i < E; ++i) before[k][i] = u + k < K - 1 ? win[u + k < K - 1 ? u + k : 0][i] : x[u + k < K - 1 ? 0 : u + k - (K - 1)][i];
            if (SILU) {
              taps.conv(z, before, x[u]);
#pragma unroll
              for (int i = 0; i < E; ++i) dz[u][i] *= dsilu(z[i], sigmoid(z[i]));
            }
#pragma unroll
            for (int i = 0; i < E; ++i) {
#pragma unroll
              for (int k = 0; k < K - 1; ++k) dw[k][i] = __builtin_fmaf(dz[u][i], before[k][i], dw[k][i]);
              dw[K - 1][i] = __builtin_fmaf(dz[u][i], x[u][i], dw[K - 1][i]);
              db[i] += dz[u][i];
              float v = taps.w[i * K] * dz[u][i];
#pragma unroll
              for (int k = 1; k < K; ++k) {
                const int j = u + K - 1 - k;   // of the K - 1 rows before the batch, then of it
                v = __builtin_fmaf(taps.w[i * K + k], j < K - 1 ? dzw[j < K - 1 ? j : 0][i] : dz[j < K - 1 ? 0 : j - (K - 1)][i], v);
              }
              dx[i] = v;
            }
            P::of(dx).save(DX, at, (tb + u - (K - 1) - r0) * dxb);
          }
#pragma unroll
          for (int k = 0; k < K - 1; ++k)
#pragma unroll
            for (int i = 0; i < E; ++i) {
              win[k][i] = x[U - (K - 1) + k][i];
              dzw[k][i] = dz[U - (K - 1) + k][i];
            }
          continue;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int t = tb + u;
          if (t < stop) {
            float dz[E] = {};
            if (t < q.end) {
              float x[E], z[E];
              px[u].get(x);
              pg[u].get(dz);
              if (SILU) {
                taps.conv(z, win, x);
#pragma unroll
                for (int i = 0; i < E; ++i) dz[i] *= dsilu(z[i], sigmoid(z[i]));
              }
              if (t < e) {
#pragma unroll
                for (int i = 0; i < E; ++i) {
#pragma unroll
                  for (int k = 0; k < K - 1; ++k) dw[k][i] = __builtin_fmaf(dz[i], win[k][i], dw[k][i]);
                  dw[K - 1][i] = __builtin_fmaf(dz[i], x[i], dw[K - 1][i]);
                  db[i] += dz[i];
                }
              }
              shift<K, E>(win, x);
            }
            const int s = t - (K - 1);
            if (s >= t0) {
              float dx[E];
#pragma unroll
              for (int i = 0; i < E; ++i) {
                float v = taps.w[i * K] * dz[i];
#pragma unroll
                for (int k = 1; k < K; ++k) v = __builtin_fmaf(taps.w[i * K + k], dzw[K - 1 - k][i], v);
                dx[i] = v;
              }
              P::of(dx).save(DX, at, (s - r0) * dxb);
            }
            shift<K, E>(dzw, dz);
          }
        }
      }
      t0 = e;
    }
  }
  if (w > 0) {
#pragma unroll
    for (int i = 0; i < E; ++i) {
#pragma unroll
      for (int k = 0; k < K; ++k) sums[w - 1][k * E + i][l] = dw[k][i];
      sums[w - 1][K * E + i][l] = db[i];
    }
  }
  __syncthreads();
  if (w > 0 || !in) return;
  float* out = a.part + (size_t)part * (K + 1) * a.D + c;
#pragma unroll
  for (int k = 0; k <= K; ++k)
#pragma unroll
    for (int i = 0; i < E; ++i) {
      float v = k < K ? dw[k < K ? k : 0][i] : db[i];
#pragma unroll
      for (int j = 0; j < CONV_BWD_WAVES - 1; ++j) v += sums[j][k * E + i][l];
      out[(size_t)k * a.D + i] = v;
    }
}

// Sums of the parts, 64 channels of a tap to a workgroup, each of its 16 waves a sixteenth of the parts.
__global__ __launch_bounds__(1024) void k_conv_sum(ConvArgs a, int spans) {
  __shared__ double sums[16][WAVE];
  const int l = threadIdx.x % WAVE, w = threadIdx.x / WAVE;
  const int k = blockIdx.x / spans, c = blockIdx.x % spans * WAVE + l;
  const float* p = a.part + (size_t)k * a.D + (c < a.D ? c : 0);
  const int per = (a.parts + 15) / 16, p0 = w * per, p1 = min(p0 + per, a.parts);
  double s = 0.0;
#pragma unroll 8
  for (int i = p0; i < p1; ++i) s += (double)p[(size_t)i * (a.K + 1) * a.D];
  sums[w][l] = s;
  __syncthreads();
  if (w > 0 || c >= a.D) return;
#pragma unroll
  for (int i = 1; i < 16; ++i) s += sums[i][l];
  if (k < a.K)
    a.dW[(size_t)c * a.K + k] = (float)s;
  else if (a.dbias)
    a.dbias[c] = (float)s;
}

// One token of every sequence; a thread has 16 bytes of channels of one sequence.  256 rows of 4352 channels, bf16: 8.3 us, 2.8 of
// them for the taps and the bias, 12 of a thread's 16 loads, which each sequence reads again; fp32 8.1, 0.4 of them.
template <class S, int K, bool SILU>
__global__ __launch_bounds__(256) void k_conv_step(ConvArgs a, int units) {
  constexpr int E = Piece<S>::N;
  const unsigned id = blockIdx.x * 256u + threadIdx.x;
  const int b = id / units, c = id % units * E;
  if (b >= a.B) return;
  S* st = static_cast<S*>(a.state) + (size_t)b * (K - 1) * a.D + c;
  Piece<S> px, ps[K - 1];
  px.load(static_cast<const S*>(a.X) + (size_t)b * a.xs + c);
#pragma unroll
  for (int k = 0; k < K - 1; ++k) ps[k].load(st + (size_t)k * a.D);
  Taps<E, K> taps;
  taps.load(a, c);
  float x[E], win[K - 1][E], z[E];
  px.get(x);
#pragma unroll
  for (int k = 0; k < K - 1; ++k) ps[k].get(win[k]);
  taps.conv(z, win, x);
  if (SILU) {
#pragma unroll
    for (int i = 0; i < E; ++i) z[i] *= sigmoid(z[i]);
  }
  Piece<S>::store(static_cast<S*>(a.Y) + (size_t)b * a.D + c, z);
#pragma unroll
  for (int k = 0; k < K - 1; ++k) (k + 1 < K - 1 ? ps[k + 1 < K - 1 ? k + 1 : 0] : px).save(st + (size_t)k * a.D);
}

namespace {
template <class S, int K, bool SILU>
void run_fwd(const ConvArgs& a, hipStream_t st) {
  const int units = a.D / Piece<S>::N, spans = (units + WAVE - 1) / WAVE;
  const int tiles = (a.T + CONV_ROWS - 1) / CONV_ROWS;
  // where the states are updated in place, they are written once every row has read its own
  const bool after = a.state && a.state == a.state0;
  const int now = tiles + (a.state && !after ? a.B : 0);
  if (now > 0) k_conv_fwd<S, K, SILU><<<(now + 3) / 4 * spans, 256, 0, st>>>(a, spans, tiles, after ? a.B : 0);
  if (after) k_conv_fwd<S, K, SILU><<<(a.B + 3) / 4 * spans, 256, 0, st>>>(a, spans, 0, 0);
}
template <class S, int K, bool SILU>
void run_bwd(const ConvArgs& a, hipStream_t st) {
  const int spans = (a.D / CONV_BWD_CH + WAVE - 1) / WAVE;
  if (a.parts > 0) k_conv_bwd<S, K, SILU><<<a.parts * spans, 256, 0, st>>>(a, spans);
  const int cols = (a.D + WAVE - 1) / WAVE;
  k_conv_sum<<<cols * (K + 1), 1024, 0, st>>>(a, cols);
}
template <class S, int K, bool SILU>
void run_step(const ConvArgs& a, hipStream_t st) {
  const int units = a.D / Piece<S>::N;
  k_conv_step<S, K, SILU><<<(unsigned)(((int64_t)a.B * units + 255) / 256), 256, 0, st>>>(a, units);
}
enum { FWD, BWD, STEP };
template <int PASS, class S, int K, bool SILU>
void run(const ConvArgs& a, hipStream_t st) {
  if (PASS == FWD) run_fwd<S, K, SILU>(a, st);
  if (PASS == BWD) run_bwd<S, K, SILU>(a, st);
  if (PASS == STEP) run_step<S, K, SILU>(a, st);
}
template <int PASS, class S>
void by_taps(const ConvArgs& a, hipStream_t st) {
  const bool silu = a.act == FLEX_ACT_SILU;
  if (a.K == 2) silu ? run<PASS, S, 2, true>(a, st) : run<PASS, S, 2, false>(a, st);
  if (a.K == 3) silu ? run<PASS, S, 3, true>(a, st) : run<PASS, S, 3, false>(a, st);
  if (a.K == 4) silu ? run<PASS, S, 4, true>(a, st) : run<PASS, S, 4, false>(a, st);
}
template <int PASS>
hipError_t launch(const ConvArgs& a, bool bf16, int timed, hipStream_t st) {
  timing_mark(timed, st, true);
  bf16 ? by_taps<PASS, u16>(a, st) : by_taps<PASS, float>(a, st);
  timing_mark(timed, st, false);
  return hipGetLastError();
}
}  // namespace

hipError_t launch_conv_fwd(const ConvArgs& a, bool bf16, hipStream_t st) { return launch<FWD>(a, bf16, FLEX_KERNEL_CONV_FWD, st); }
hipError_t launch_conv_bwd(const ConvArgs& a, bool bf16, hipStream_t st) { return launch<BWD>(a, bf16, FLEX_KERNEL_CONV_BWD, st); }
hipError_t launch_conv_step(const ConvArgs& a, bool bf16, hipStream_t st) { return launch<STEP>(a, bf16, FLEX_KERNEL_CONV_STEP, st); }

}  // namespace flex
