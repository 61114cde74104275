// Selective scan, backward.  With dS the gradient of the state at a chunk's end, E_ij = e^{L_i - L_j} (j <= i) and
// v_j = e^{L_63 - L_j}:
//   M_ij = E_ij dy_i.x_j      W_ij = sum over a group's heads of M_ij dt_j
//   dC_i = sum_j W_ij B_j + sum_heads e^{L_i} S dy_i
//   dB_j = sum_i W_ij C_i + sum_heads dt_j v_j dS x_j
//   dxt_j = sum_i E_ij (C_i.B_j) dy_i + v_j dS^T B_j,   dx_j = dt_j dxt_j + D dy_j,   ddt_j = dxt_j.x_j,   dD = sum_t dy_t.x_t
//   dS <- e^{L_63} dS + sum_i e^{L_i} C_i dy_i^T                       (the chunk's start)
//   dg_t = sum_{i>=t} (R_i + sum_{j<i} Z_ij - sum_{j>i} Z_ji) + sum_{i<t} V_i + e^{L_63} <S, dS>
//          with Z_ij = M_ij (C_i.B_j) dt_j, R_i = e^{L_i} C_i.S dy_i, V_j = dt_j x_j.(v_j dS^T B_j)
// dg_t is what crosses t: what is read from t on of what was written before it.  Z enters as a row sum and as a
// column sum of the same fp32 numbers, so pairs on one side of t cancel to what fp32 sums of them leave; its
// diagonal crosses nothing and is left out.
// S of each chunk is the forward's, dS comes from a sweep in reverse; the rest is independent per chunk
// (k_scan_grad).
#include "flex_scan.hpp"
#include "../../include/flex.h"

namespace flex {

void launch_scan_states(const ScanArgs& a, bool bf16, hipStream_t st);

// One workgroup per chunk, group and part of its heads, over them in order and over their columns in blocks of 64.
// Wave w has the tokens j of tile w % 2, a lane per token, and of what it forms for them the half w / 2: of the rows n
// of dB and dC, of the columns p of dx, and of M the tokens i of tile w / 2.
template <class T, int N>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1, 2))) void k_scan_grad(ScanArgs a) {
  using S = typename Io<T>::type;
  using RT = ScanTile<T, N>;
  using XT = ScanTile<T, 64>;
  using ST = StateRows<T, N>;
  constexpr bool BF = IsBf16<T>::value;
  constexpr int NT = N / 64, ROWS = SC * N * (int)sizeof(T), XROWS = SC * 64 * (int)sizeof(T);
  // fp32 states of 128 rows leave room for one of S and dS at a time
  constexpr bool ONE = 4 * ROWS + 2 * XROWS > 144 * 1024;
  __shared__ __attribute__((aligned(16))) char lds[(ONE ? 3 : 4) * ROWS + 2 * XROWS];
  __shared__ __attribute__((aligned(16))) float sc[5][SC];       // L (hi, lo), dt, e^L, v
  __shared__ float dot_r[2][SC], dot_v[2][SC], dot_i[2][SC], col_z[2][SC], row_z[2][2][SC], sums[2][4];
  char* LB = lds;
  char* LC = lds + ROWS;
  char* LX = lds + 2 * ROWS;
  char* LY = LX + XROWS;
  char* LS = LY + XROWS;
  char* LD = ONE ? LS : LS + ROWS;

  const int l = threadIdx.x % WAVE, c = l % 32, h = l / 32;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE), tj = w % 2, hf = w / 2;
  const int id = blockIdx.x, sets = a.G * a.parts, k = id / NUM_XCD;
  const int slot = k / sets * NUM_XCD + id % NUM_XCD, grp = k % sets / a.parts, part = k % sets % a.parts;
  const int slots = seq_slots(a.T, a.B, SC);
  if (slot >= slots) return;
  const int hpg = a.H / a.G, hpp = hpg / a.parts, head0 = grp * hpg + part * hpp;
  const SeqTile t = find_tile<SC>(a.off, a.B, a.T, slot);
  if (t.b < 0) {
    for (int i = threadIdx.x; i < hpp; i += 256) a.part_d[(size_t)slot * a.H + head0 + i] = 0.f;
    return;
  }
  const int n = min(SC, t.n - t.tile * SC), row0 = t.row0 + t.tile * SC;
  const int tok = 32 * tj + c;   // this lane's token
  stage_rows<T, N>(LB, static_cast<const S*>(a.Bt) + (size_t)grp * N, row0, a.bs, n, w, 4);
  stage_rows<T, N>(LC, static_cast<const S*>(a.Ct) + (size_t)grp * N, row0, a.cs, n, w, 4);

  f32x16 dB[NT], dC[NT], W = zero16(), cb[2];   // cb: C_i.B_j, tiles of i, lane j
#pragma unroll
  for (int i = 0; i < NT; ++i) dB[i] = dC[i] = zero16();
  sync_tiles();
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    cb[i] = zero16();
    if (i >= tj) {
#pragma unroll
      for (int s = 0; s < N / 16; ++s) mma32(cb[i], RT::row(LC, 32 * i + c, s, h), RT::row(LB, tok, s, h));
    }
  }
  const int nb = a.P / 64;
  for (int hd = 0; hd < hpp; ++hd) {
    const int head = head0 + hd;
    f32x16 m0 = zero16();   // dy_i.x_j of the tile hf of i
    float di = 0.f, dv = 0.f, dr = 0.f, ss = 0.f;
    const float Dh = a.D ? a.D[head] : 0.f;
    float last = 0.f;
    for (int pb = 0; pb < nb; ++pb) {
      const size_t xcol = (size_t)head * a.P + pb * 64, sat = (((size_t)slot * a.H + head) * a.P + pb * 64) * N;
      sync_lds();   // what was staged before is no longer read
      stage_rows<T, 64>(LX, static_cast<const S*>(a.X) + xcol, row0, a.xs, n, w, 4);
      stage_rows<T, 64>(LY, static_cast<const S*>(a.dY) + xcol, row0, a.H * a.P, n, w, 4);
      stage_linear<ROWS / 1024, 4>(LS, static_cast<const S*>(a.st) + sat, w);
      if (!ONE) stage_linear<ROWS / 1024, 4>(LD, static_cast<const S*>(a.dst) + sat, w);
      if (pb == 0) {   // every wave forms the decays, the first one writes them
        float g = 0.f, dt = 0.f;
        if (l < n) {
          const size_t at = (size_t)(row0 + l) * a.H + head;
          g = a.g[at];
          dt = a.dt[at];
        }
        const Decay d(g);
        last = __builtin_amdgcn_exp2f((float)d.end);
        if (w == 0) {
          sc[0][l] = d.hi;
          sc[1][l] = d.lo;
          sc[2][l] = dt;
          sc[3][l] = d.from_start();
          sc[4][l] = d.to_end();
        }
      }
      sync_tiles();
      const float hj = sc[0][tok], lj = sc[1][tok], dt = sc[2][tok], eg = sc[3][tok], vj = sc[4][tok];

      // M's products, and e^L S dy
      if (hf >= tj) {
#pragma unroll
        for (int s = 0; s < 4; ++s) mma32(m0, XT::row(LY, 32 * hf + c, s, h), XT::row(LX, tok, s, h));
      }
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        f32x16 u = zero16();
        const int n0 = hf * (N / 2) + 32 * i;
#pragma unroll
        for (int s = 0; s < 4; ++s)
          mma32(u, ST::colp(LS, 16 * s + 8 * h, n0), XT::row(LY, tok, s, h));
        float r = 0.f;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const Frag<T> cr = RT::row(LC, tok, n0 / 16 + s, h);
#pragma unroll
          for (int j = 0; j < 8; ++j) r = __builtin_fmaf(cr.get(j), u[8 * s + j], r);
        }
        dr += r;
#pragma unroll
        for (int e = 0; e < 16; ++e) dC[i][e] = __builtin_fmaf(u[e], eg, dC[i][e]);
      }
      if (ONE) {
        sync_lds();
        stage_linear<ROWS / 1024, 4>(LD, static_cast<const S*>(a.dst) + sat, w);
        const float* s0 = reinterpret_cast<const float*>(static_cast<const S*>(a.st) + sat);
        const float* d0 = reinterpret_cast<const float*>(static_cast<const S*>(a.dst) + sat);
        for (int i = threadIdx.x; i < 64 * N; i += 256) ss = __builtin_fmaf(s0[i], d0[i], ss);
        sync_tiles();
      } else {
        for (int i = threadIdx.x; i < ROWS / 16; i += 256) {   // <S, dS>: the same place in both tiles
          if constexpr (IsBf16<T>::value) {
            const bf16x8 x = *reinterpret_cast<const bf16x8*>(LS + 16 * i), y = *reinterpret_cast<const bf16x8*>(LD + 16 * i);
#pragma unroll
            for (int j = 0; j < 8; ++j) ss = __builtin_fmaf((float)x[j], (float)y[j], ss);
          } else {
            const f32x4 x = *reinterpret_cast<const f32x4*>(LS + 16 * i), y = *reinterpret_cast<const f32x4*>(LD + 16 * i);
#pragma unroll
            for (int j = 0; j < 4; ++j) ss = __builtin_fmaf(x[j], y[j], ss);
          }
        }
      }
      // dt v dS x
      const float dtv = dt * vj;
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        f32x16 u = zero16();
        const int n0 = hf * (N / 2) + 32 * i;
#pragma unroll
        for (int s = 0; s < 4; ++s)
          mma32(u, ST::colp(LD, 16 * s + 8 * h, n0), XT::row(LX, tok, s, h));
#pragma unroll
        for (int e = 0; e < 16; ++e) dB[i][e] = __builtin_fmaf(u[e], dtv, dB[i][e]);
      }
      // dx of the half hf of the block's columns
      f32x16 xa = zero16(), xv = zero16();
#pragma unroll
      for (int s = 0; s < N / 16; ++s) mma32(xv, ST::row(LD, 32 * hf, s), RT::row(LB, tok, s, h));
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (i >= tj) {
          f32x16 q;
#pragma unroll
          for (int b = 0; b < 4; ++b) {
            const int ti = 32 * i + 8 * b + 4 * h;
            const f32x4 hi = *reinterpret_cast<const f32x4*>(&sc[0][ti]), lo = *reinterpret_cast<const f32x4*>(&sc[1][ti]);
#pragma unroll
            for (int e = 0; e < 4; ++e)
              q[4 * b + e] = ti + e >= tok ? cb[i][4 * b + e] * decay<BF>(hi[e], lo[e], hj, lj) : 0.f;
          }
#pragma unroll
          for (int s = 0; s < 2; ++s)
            mma32(xa, XT::colp(LY, 32 * i + 16 * s + 4 * h, 32 * i + 16 * s + 8 + 4 * h, 32 * hf), frag_of<T>(q, s));
        }
      const auto rx = row_window(static_cast<S*>(a.dX) + xcol + 32 * hf, row0, a.dxs, n, 32);
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const Frag<T> xr = XT::row(LX, tok, 2 * hf + s, h), yr = XT::row(LY, tok, 2 * hf + s, h);
        const int at = (tok * a.dxs + 16 * s + 8 * h) * (int)sizeof(S);
        float o[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float p = xa[8 * s + j], v = vj * xv[8 * s + j];
          di = __builtin_fmaf(p, xr.get(j), di);
          dv = __builtin_fmaf(v, xr.get(j), dv);
          o[j] = __builtin_fmaf(dt, p + v, Dh * yr.get(j));
        }
        if constexpr (IsBf16<T>::value) {
          Frag<T> f;
#pragma unroll
          for (int j = 0; j < 8; ++j) f.set(j, o[j]);
          __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, f.v), rx, at, 0, 0);
        } else {
          __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, f32x4{o[0], o[1], o[2], o[3]}), rx, at, 0, 0);
          __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, f32x4{o[4], o[5], o[6], o[7]}), rx, at + 16, 0, 0);
        }
      }
    }
    // M, W and the sums of Z; the diagonal of dy x^T
    const float hj = sc[0][tok], lj = sc[1][tok], dt = sc[2][tok], eg = sc[3][tok];
    float dd = 0.f, cz = 0.f;
    if (hf >= tj) {
      f32x16 z;
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const int ti = 32 * hf + 8 * b + 4 * h;
        const f32x4 hi = *reinterpret_cast<const f32x4*>(&sc[0][ti]), lo = *reinterpret_cast<const f32x4*>(&sc[1][ti]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int x = 4 * b + e, i = ti + e;
          if (i == tok) dd = m0[x];
          const float m = i >= tok ? m0[x] * decay<BF>(hi[e], lo[e], hj, lj) * dt : 0.f;
          W[x] += m;
          z[x] = i > tok ? m * (hf == 0 ? cb[0][x] : cb[1][x]) : 0.f;
          cz += z[x];
        }
      }
#pragma unroll
      for (int x = 0; x < 16; ++x) {
        const float r = lane_sum<16>(z[x]);
        if (l % 16 == 0) row_z[tj][(l / 16) & 1][32 * hf + res_row(x, h)] = r;
      }
    }
    dd = group_sum_swap(lane_sum<16>(dd));
    ss = group_sum_swap(lane_sum<16>(ss));
    cz = half_sum(cz);
    di = half_sum(di);
    dv = half_sum(dv);
    dr = half_sum(dr);
    if (h == 0) {
      col_z[hf][tok] = hf >= tj ? cz : 0.f;
      dot_i[hf][tok] = di;
      dot_v[hf][tok] = dv;
      dot_r[hf][tok] = dr * eg;
    }
    if (l == 0) {
      sums[0][w] = dd;
      sums[1][w] = ss;
    }
    sync_lds();
    if (w == 0) {
      const float g = l < n ? a.g[(size_t)(row0 + l) * a.H + head] : 0.f, dtl = sc[2][l];
      // rows of tile 0 have the tile of j 0 alone
      const float rz = (row_z[0][0][l] + row_z[0][1][l]) + (l >= 32 ? row_z[1][0][l] + row_z[1][1][l] : 0.f);
      float x = (dot_r[0][l] + dot_r[1][l]) + rz - (col_z[0][l] + col_z[1][l]);
      const float v = dot_v[0][l] + dot_v[1][l];
      float z = __shfl_up(v * dtl, 1);
      if (l == 0) z = 0.f;
      if (l == SC - 1) x += last * ((sums[1][0] + sums[1][1]) + (sums[1][2] + sums[1][3]));
#pragma unroll
      for (int s = 1; s < WAVE; s *= 2) {   // sums over i >= l, and over i < l
        const float o = __shfl_down(x, s), p = __shfl_up(z, s);
        if (l + s < WAVE) x += o;
        if (l >= s) z += p;
      }
      if (l < n) {
        const size_t at = (size_t)(row0 + l) * a.H + head;
        // in the io type like every gradient of this operator, though dt and g are fp32; a decay of zero has no slope
        static_cast<S*>(a.dg)[at] = float_to_io<S>(g < SCAN_MIN_G ? 0.f : x + z);
        static_cast<S*>(a.ddt)[at] = float_to_io<S>((dot_i[0][l] + dot_i[1][l]) + v);
      }
      if (l == 0) a.part_d[(size_t)slot * a.H + head] = (sums[0][0] + sums[0][1]) + (sums[0][2] + sums[0][3]);
    }
  }
  // dB += W^T C, dC += W B, through W as rows i in LDS, as two bf16 terms: the heads' M may cancel in it
  sync_lds();
  constexpr int TERMS = IsBf16<T>::value ? 2 : 1;
#pragma unroll
  for (int x = 0; x < 16; ++x) {
    const int i = 32 * hf + res_row(x, h);
    float v = hf >= tj ? W[x] : 0.f;
#pragma unroll
    for (int t = 0; t < TERMS; ++t) {
      const S u = float_to_io<S>(v);
      *reinterpret_cast<S*>(LX + t * XROWS + XT::at(i, tok / XT::E) + tok % XT::E * (int)sizeof(S)) = u;
      v -= io_to_float(u);
    }
  }
  sync_lds();
#pragma unroll
  for (int s = 0; s < 4; ++s)
#pragma unroll
    for (int t = TERMS - 1; t >= 0; --t) {
      const char* LW = LX + t * XROWS;
      const Frag<T> wr = XT::row(LW, tok, s, h), wc = XT::col(LW, 16 * s + 4 * h, 32 * tj);
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        const int n0 = hf * (N / 2) + 32 * i;
        if (s / 2 <= tj) mma32(dC[i], RT::colp(LB, 16 * s + 8 * h, 16 * s + 8 * h + 4, n0), wr);
        if (s / 2 >= tj) mma32(dB[i], RT::colp(LC, 16 * s + 4 * h, 16 * s + 8 + 4 * h, n0), wc);
      }
    }
  auto store = [&](const f32x16 (&x)[NT], float* parts, void* out, int stride) {
    if (tok >= n) return;
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const int n0 = hf * (N / 2) + 32 * i + 16 * s + 8 * h;
        const f32x4 u = {x[i][8 * s], x[i][8 * s + 1], x[i][8 * s + 2], x[i][8 * s + 3]};
        const f32x4 v = {x[i][8 * s + 4], x[i][8 * s + 5], x[i][8 * s + 6], x[i][8 * s + 7]};
        if (parts) {
          float* p = parts + ((((size_t)part * slots + slot) * SC + tok) * a.G + grp) * N + n0;
          *reinterpret_cast<f32x4*>(p) = u;
          *reinterpret_cast<f32x4*>(p + 4) = v;
        } else {
          S* p = static_cast<S*>(out) + (size_t)(row0 + tok) * stride + (size_t)grp * N + n0;
          store_io4(p, u);
          store_io4(p + 4, v);
        }
      }
  };
  store(dB, a.part_b, a.dB, a.dbs);
  store(dC, a.part_c, a.dC, a.dcs);
}

// dB and dC from the parts of the heads, in order: a workgroup has rows of a chunk, a thread four values.
template <class S>
__global__ __launch_bounds__(256) void k_scan_parts(ScanArgs a) {
  const int slots = seq_slots(a.T, a.B, SC), slot = blockIdx.x;
  const SeqTile t = find_tile<SC>(a.off, a.B, a.T, slot);
  if (t.b < 0) return;
  const int n = min(SC, t.n - t.tile * SC), row0 = t.row0 + t.tile * SC, width = a.G * a.N;
  for (int i = threadIdx.x * 4; i < n * width; i += 1024) {
    const int r = i / width, col = i % width;
    f32x4 b = zero4(), c = zero4();
    for (int p = 0; p < a.parts; ++p) {
      const size_t at = (((size_t)p * slots + slot) * SC) * width + i;
      b += *reinterpret_cast<const f32x4*>(a.part_b + at);
      c += *reinterpret_cast<const f32x4*>(a.part_c + at);
    }
    store_io4(static_cast<S*>(a.dB) + (size_t)(row0 + r) * a.dbs + col, b);
    store_io4(static_cast<S*>(a.dC) + (size_t)(row0 + r) * a.dcs + col, c);
  }
}

// dD of a head: its chunks' sums, in a fixed order.
__global__ __launch_bounds__(256) void k_scan_skip(ScanArgs a) {
  __shared__ double sums[256];
  const int slots = a.T > 0 ? seq_slots(a.T, a.B, SC) : 0, head = blockIdx.x;
  double s = 0.0;
  for (int i = threadIdx.x; i < slots; i += 256) s += (double)a.part_d[(size_t)i * a.H + head];
  sums[threadIdx.x] = s;
  __syncthreads();
  for (int k = 128; k > 0; k /= 2) {
    if ((int)threadIdx.x < k) sums[threadIdx.x] += sums[threadIdx.x + k];
    __syncthreads();
  }
  if (threadIdx.x == 0) a.dD[head] = (float)sums[0];
}

namespace {
template <class T, int N>
void grad(const ScanArgs& a, hipStream_t st) {
  const int slots = seq_slots(a.T, a.B, SC);
  k_scan_grad<T, N><<<(slots + NUM_XCD - 1) / NUM_XCD * NUM_XCD * a.G * a.parts, 256, 0, st>>>(a);
  if (a.part_b) k_scan_parts<typename Io<T>::type><<<slots, 256, 0, st>>>(a);
}
}  // namespace

hipError_t launch_scan_bwd(const ScanArgs& a, bool bf16, hipStream_t st) {
  timing_mark(FLEX_KERNEL_SCAN_BWD, st, true);
  if (a.T > 0) {
    launch_scan_states(a, bf16, st);
    if (bf16)
      a.N == 64 ? grad<__bf16, 64>(a, st) : grad<__bf16, 128>(a, st);
    else
      a.N == 64 ? grad<float, 64>(a, st) : grad<float, 128>(a, st);
  }
  if (a.dD) k_scan_skip<<<a.H, 256, 0, st>>>(a);
  timing_mark(FLEX_KERNEL_SCAN_BWD, st, false);
  return hipGetLastError();
}

}  // namespace flex
