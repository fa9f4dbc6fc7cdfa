// RMS norm of each head of queries and keys, and their rotation by positions of several axes: forward and backward.
//   z = x r g, r = 1 / sqrt(mean x^2 + eps);  y = R z
//   dz = R' dy;  dg = sum dz x r;  dx = r (g dz - x r mean(g dz x r))
#include "common.h"
#include "rotary.h"

namespace ppll {

namespace {
struct RotaryArgs {
  RotaryPlan p;
  RotarySide side[2];
  const int32_t* positions;
  float* partials;         // [workgroups][2][head_dim], backward with scales
  int rows_wg;             // rows that a workgroup takes at a time
};

// cos and sin of every pair of the rows from row0 on, once for all heads: the angle in turns and its nearest whole number in 64 bits (a
// position of 2^31 leaves 22 bits of a turn's fraction in them, none in 32), the functions of what is left in 32.
__device__ __forceinline__ void fill_table(const RotaryArgs& a, int row0, int rows, float2* table) {
  const int P = a.p.pairs;
  for (int e = threadIdx.x; e < rows * P; e += 256) {
    const int r = e / P, p = e - r * P, token = (row0 + r) % a.p.tokens;
    const int axis = p < a.p.end[0] ? 0 : p < a.p.end[1] ? 1 : 2;
    const double turns = a.p.turns[p] * a.positions[(int64_t)token * a.p.axes + axis];
    float s, c;
    sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
    table[e] = make_float2(c, s);
  }
}

// Any head width, any alignment: a wave a head, element by element.
template <bool BWD> __global__ __launch_bounds__(256) void rotary_plain_kernel(RotaryArgs a, int dt) {
  extern __shared__ float2 table[];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, P = a.p.pairs, hd = a.p.hd;
  // lane: pairs lane and lane + 64, elements 2 P + lane + 64 k behind them
  float sums[2][8] = {};
  for (int64_t row0 = (int64_t)blockIdx.x * a.rows_wg; row0 < a.p.rows; row0 += (int64_t)gridDim.x * a.rows_wg) {
    const int rows = (int)min((int64_t)a.rows_wg, a.p.rows - row0);
    __syncthreads();
    fill_table(a, (int)row0, rows, table);
    __syncthreads();
#pragma unroll
    for (int side = 0; side < 2; ++side) {
      const RotarySide& s = a.side[side];
      for (int it = wave; it < rows * a.p.heads[side]; it += 4) {
        const int r = it / a.p.heads[side], h = it - r * a.p.heads[side];
        const int64_t row = row0 + r, at = row * s.x_ld + h * hd, to = row * s.y_ld + h * hd, from = row * s.dy_ld + h * hd;
        float v[8], d[8], g[8];
        int el[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const int p = lane + 64 * (k >> 1), e = 2 * P + lane + 64 * (k - 4);
          el[k] = k < 4 ? (p < P ? (a.p.neighbours ? 2 * p + (k & 1) : p + (k & 1) * P) : -1) : (e < hd ? e : -1);
          v[k] = el[k] >= 0 && s.x ? ld_f(s.x, at + el[k], dt) : 0.f;
          d[k] = BWD && el[k] >= 0 ? ld_f(s.dy, from + el[k], dt) : 0.f;
          g[k] = el[k] >= 0 && s.scale ? s.scale[el[k]] : 1.f;
        }
        if (!BWD && s.keep)
#pragma unroll
          for (int k = 0; k < 8; ++k)
            if (el[k] >= 0) st_f(s.keep, row * s.keep_ld + h * hd + el[k], v[k], dt);
        float rs = 1.f;
        if (s.scale) {
          float q = 0.f;
#pragma unroll
          for (int k = 0; k < 8; ++k) q += v[k] * v[k];
          rs = 1.f / sqrtf(wave_sum(q) / hd + a.p.eps);
        }
        float z[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) z[k] = BWD ? d[k] : v[k] * rs * g[k];
#pragma unroll
        for (int k = 0; k < 4; k += 2)
          if (el[k] >= 0) {
            const float2 cs = table[r * P + lane + 32 * k];
            const float sn = BWD ? -cs.y : cs.y, z0 = z[k], z1 = z[k + 1];
            z[k] = z0 * cs.x - z1 * sn;
            z[k + 1] = z1 * cs.x + z0 * sn;
          }
        if (BWD && s.scale) {
          float along = 0.f;
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            v[k] *= rs;
            sums[side][k] += z[k] * v[k];
            z[k] *= g[k];
            along += z[k] * v[k];
          }
          along = wave_sum(along) / hd;
#pragma unroll
          for (int k = 0; k < 8; ++k) z[k] = rs * (z[k] - v[k] * along);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (el[k] >= 0) st_f(s.y, to + el[k], z[k], dt);
      }
    }
  }
  if (!BWD || !a.partials) return;
  __shared__ float part[4][256];
#pragma unroll
  for (int side = 0; side < 2; ++side) {
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int p = lane + 64 * (k >> 1), e = 2 * P + lane + 64 * (k - 4);
      const int el = k < 4 ? (p < P ? (a.p.neighbours ? 2 * p + (k & 1) : p + (k & 1) * P) : -1) : (e < hd ? e : -1);
      if (el >= 0) part[wave][el] = sums[side][k];
    }
    __syncthreads();
    const int e = threadIdx.x;
    if (e < hd) a.partials[((int64_t)blockIdx.x * 2 + side) * hd + e] = part[0][e] + part[1][e] + part[2][e] + part[3][e];
  }
}

// d scale from the workgroups' partial sums, 16 elements a workgroup; queries first, then keys
__global__ __launch_bounds__(256) void rotary_scale_kernel(const float* partials, int chunks, int hd, float* dq, float* dk) {
  __shared__ float red[16][17];
  const int col = threadIdx.x & 15, grp = threadIdx.x >> 4, across = (hd + 15) / 16;
  const int side = blockIdx.x / across, e = blockIdx.x % across * 16 + col;
  float acc = 0.f;
  if (e < hd)
    for (int c = grp; c < chunks; c += 16) acc += partials[((int64_t)c * 2 + side) * hd + e];
  red[grp][col] = acc;
  __syncthreads();
  float* out = side ? dk : dq;
  if (grp || e >= hd || !out) return;
  float t = 0.f;
  for (int g = 0; g < 16; ++g) t += red[g][col];
  out[e] = t;
}

constexpr int ROWS_WG = 8;
int workgroups_of(const RotaryPlan& p, bool bwd) {
  const int64_t blocks = ((int64_t)p.rows + ROWS_WG - 1) / ROWS_WG, most = bwd ? ROTARY_PARTIALS : 65536;
  return (int)(blocks < most ? blocks : most);
}
int launch(hipStream_t s, RotaryArgs& a, int dt, bool bwd, int* workgroups) {
  a.rows_wg = ROWS_WG;
  const int wgs = workgroups_of(a.p, bwd);
  const size_t lds = (size_t)a.rows_wg * a.p.pairs * sizeof(float2);
  *workgroups = wgs;
  if (!wgs) return PPLL_OK;
  if (bwd) hipLaunchKernelGGL((rotary_plain_kernel<true>), dim3(wgs), dim3(256), lds, s, a, dt);
  else hipLaunchKernelGGL((rotary_plain_kernel<false>), dim3(wgs), dim3(256), lds, s, a, dt);
  PPLL_HIP(hipGetLastError());
  return PPLL_OK;
}
}  // namespace

int launch_rotary_fwd(hipStream_t s, const RotaryPlan& p, int dt, const int32_t* positions, const RotarySide& q, const RotarySide& k) {
  RotaryArgs a{p, {q, k}, positions, nullptr, 0};
  int wgs;
  return launch(s, a, dt, false, &wgs);
}
int launch_rotary_bwd(hipStream_t s, const RotaryPlan& p, int dt, const int32_t* positions, const RotarySide& q, const RotarySide& k, float* partials,
                      int* rows) {
  RotaryArgs a{p, {q, k}, positions, partials, 0};
  return launch(s, a, dt, true, rows);
}
int rotary_bwd_rows(const RotaryPlan& p) { return workgroups_of(p, true); }
int launch_rotary_scales(hipStream_t s, const float* partials, int rows, int hd, float* dq, float* dk) {
  hipLaunchKernelGGL(rotary_scale_kernel, dim3(2 * ((hd + 15) / 16)), dim3(256), 0, s, partials, rows, hd, dq, dk);
  PPLL_HIP(hipGetLastError());
  return PPLL_OK;
}

}  // namespace ppll
