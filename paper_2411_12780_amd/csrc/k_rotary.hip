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
  int lanes;               // of a head, in rotary_kernel: a power of two
};

// cos and sin of every pair of the rows from row0 on, once for all heads: the angle in turns and its nearest whole number in 64 bits (with a base from
// 1 on, position 2^31 leaves 22 bits of a turn's fraction in them, none in 32), the functions of what is left in 32, and what the rounding of their
// argument left out, up to 2^-25 half turns, by their derivatives: without it cos and sin are off by 3.3e-8 in the mean, over twice what rounding them
// leaves.
__device__ __forceinline__ void fill_table(const RotaryArgs& a, int row0, int rows, float2* table) {
  const int P = a.p.pairs;
  for (int e = threadIdx.x; e < rows * P; e += 256) {
    const int r = e / P, p = e - r * P, token = (row0 + r) % a.p.tokens;
    const int axis = p < a.p.end[0] ? 0 : p < a.p.end[1] ? 1 : 2;
    const double turns = a.p.turns[p] * a.positions[(int64_t)token * a.p.axes + axis];
    const double half_turns = 2.0 * (turns - rint(turns));
    const float near = (float)half_turns, rest = (float)(half_turns - near) * 3.14159265f;
    float s, c;
    sincospif(near, &s, &c);
    table[e] = make_float2(fmaf(-s, rest, c), fmaf(c, rest, s));
  }
}

// Any head width, any alignment: a wave a head, element by element.  What the kernel below does not take: heads that turn in part or not at all (the
// norm alone), widths and strides with less in common than 8 bytes.
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

// V elements in memory, 8 or 16 bytes, as fp32
template <class T, int V> struct Piece {
  static constexpr int WORDS = V * (int)sizeof(T) / 4;
  typedef __attribute__((ext_vector_type(WORDS))) uint32_t words;
  words w;
  __device__ __forceinline__ void load(const void* p, int64_t at) { w = *(const words*)((const T*)p + at); }
  __device__ __forceinline__ void store(void* p, int64_t at) const { *(words*)((T*)p + at) = w; }
  __device__ __forceinline__ float get(int i) const {
    if (sizeof(T) == 4) return __uint_as_float(w[i]);
    return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
  }
  __device__ __forceinline__ void set(const float* v) {
#pragma unroll
    for (int i = 0; i < WORDS; ++i) w[i] = sizeof(T) == 4 ? __float_as_uint(v[i]) : f32x2_to_bf16x2(v[2 * i], v[2 * i + 1]);
  }
};
__device__ __forceinline__ float head_sum(float v, int lanes) {
  for (int o = lanes >> 1; o; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

// Heads that turn whole, V pairs a lane in two pieces of V elements (of either half of the head, or neighbours), the head's P / V lanes
// rounded up to a power of two; queries and keys in workgroups of their own (blockIdx.y), which leaves registers for the sums of one side
// and the next head's elements on their way.  Bound by memory: each element is read and written once, cos and sin come from LDS.  664 MB of a
// clip's queries and keys (64800 rows, 16 and 4 heads of 128, bf16) in 127 us, 5.2 TB/s, a copy's rate; the gradients of 25216 rows with 12 + 12
// heads of 64 and the norm, 232 MB, in 49 to 53 us, 4.4 to 4.8 TB/s.  Small calls by the launch and the table, those of an ordinary layer by registers:
// 8320 rows with 6 + 6 heads of 64 and the norm 10.9 us forward and 18 backward, where memory would allow 5.0 and 7.4.  Forward takes 98 registers, so
// four workgroups to a unit and 2080 in 2.03 rounds; backward takes all 128 of four waves and keeps five more in scratch memory.
template <class T, int V, bool NEXT, bool NORM, bool BWD> __global__ __launch_bounds__(256, 4) void rotary_kernel(RotaryArgs a) {
  extern __shared__ float2 table[];
  const int side = a.p.heads[0] ? blockIdx.y : 1;
  const RotarySide& s = a.side[side];
  const int P = a.p.pairs, hd = a.p.hd, lanes = a.lanes, c = threadIdx.x & (lanes - 1), group = threadIdx.x / lanes, groups = 256 / lanes;
  const int heads = a.p.heads[side], dr = groups / heads, dh = groups - dr * heads;
  const bool on = c * V < P;
  const int e0 = !on ? 0 : NEXT ? 2 * V * c : V * c, e1 = !on ? 0 : NEXT ? e0 + V : P + e0;
  const float per = 1.f / hd;
  float g[2 * V], sums[2 * V] = {};
#pragma unroll
  for (int i = 0; i < V; ++i) { g[i] = NORM ? s.scale[e0 + i] : 1.f; g[V + i] = NORM ? s.scale[e1 + i] : 1.f; }
  for (int64_t row0 = (int64_t)blockIdx.x * a.rows_wg; row0 < a.p.rows; row0 += (int64_t)gridDim.x * a.rows_wg) {
    const int rows = (int)min((int64_t)a.rows_wg, a.p.rows - row0);
    int r = group / heads, h = group - r * heads;
    Piece<T, V> x0{}, x1{}, d0{}, d1{};
    auto load = [&]() {
      if (!on || r >= rows) return;
      const int64_t row = row0 + r;
      if (!BWD || NORM) { x0.load(s.x, row * s.x_ld + h * hd + e0); x1.load(s.x, row * s.x_ld + h * hd + e1); }
      if (BWD) { d0.load(s.dy, row * s.dy_ld + h * hd + e0); d1.load(s.dy, row * s.dy_ld + h * hd + e1); }
    };
    load();
    if (row0 != (int64_t)blockIdx.x * a.rows_wg) __syncthreads();
    fill_table(a, (int)row0, rows, table);
    __syncthreads();
    while (r < rows) {
      const int64_t row = row0 + r;
      const float2* cs = table + r * P + (on ? c * V : 0);
      const int at = h * hd;
      Piece<T, V> u0 = x0, u1 = x1;
      float z[2 * V], v[2 * V];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        v[i] = x0.get(i); v[V + i] = x1.get(i);
        z[i] = BWD ? d0.get(i) : v[i]; z[V + i] = BWD ? d1.get(i) : v[V + i];
      }
      r += dr; h += dh;
      if (h >= heads) { h -= heads; ++r; }
      load();
      float rs = 1.f;
      if (NORM) {
        float q = 0.f;
#pragma unroll
        for (int i = 0; i < 2 * V; ++i) q = fmaf(v[i], v[i], q);
        rs = 1.f / sqrtf(fmaf(head_sum(q, lanes), per, a.p.eps));
#pragma unroll
        for (int i = 0; i < 2 * V; ++i) {
          v[i] *= rs;
          if (!BWD) z[i] = v[i] * g[i];
        }
      }
#pragma unroll
      for (int i = 0; i < V; ++i) {
        float &u = NEXT ? z[2 * i] : z[i], &w = NEXT ? z[2 * i + 1] : z[V + i];
        const float sn = BWD ? -cs[i].y : cs[i].y, t = u;
        u = fmaf(t, cs[i].x, -w * sn);
        w = fmaf(w, cs[i].x, t * sn);
      }
      if (BWD && NORM) {
        float along = 0.f;
#pragma unroll
        for (int i = 0; i < 2 * V; ++i) {
          sums[i] = fmaf(z[i], v[i], sums[i]);
          z[i] *= g[i];
          along = fmaf(z[i], v[i], along);
        }
        along = head_sum(along, lanes) * per;
#pragma unroll
        for (int i = 0; i < 2 * V; ++i) z[i] = rs * fmaf(-v[i], along, z[i]);
      }
      if (on) {
        if (!BWD && s.keep) { u0.store(s.keep, row * s.keep_ld + at + e0); u1.store(s.keep, row * s.keep_ld + at + e1); }
        u0.set(z); u1.set(z + V);
        u0.store(s.y, row * s.y_ld + at + e0); u1.store(s.y, row * s.y_ld + at + e1);
      }
    }
  }
  if (!BWD || !NORM) return;
  // the sums of a head's lanes over the wave's groups, then over the four waves, in this order always
  __shared__ float part[4][256];
#pragma unroll
  for (int i = 0; i < 2 * V; ++i) {
    float v = sums[i];
    for (int o = 32; o >= lanes; o >>= 1) v += __shfl_xor(v, o);
    if (on && (threadIdx.x & 63) < lanes) part[threadIdx.x >> 6][(i < V ? e0 : e1 - V) + i] = v;
  }
  __syncthreads();
  const int e = threadIdx.x;
  if (e < hd) a.partials[((int64_t)blockIdx.x * 2 + side) * hd + e] = part[0][e] + part[1][e] + part[2][e] + part[3][e];
}

// d scale from the workgroups' partial sums, 16 elements a workgroup; queries first, then keys.  A launch of no size: 4.4 us for 512 rows of sums.
__global__ __launch_bounds__(1024) void rotary_scale_kernel(const float* partials, int chunks, int hd, float* dq, float* dk) {
  __shared__ float red[64][17];
  const int col = threadIdx.x & 15, grp = threadIdx.x >> 4, across = (hd + 15) / 16;
  const int side = blockIdx.x / across, e = blockIdx.x % across * 16 + col;
  float* out = side ? dk : dq;
  if (!out) return;
  float acc = 0.f;
  if (e < hd) {
#pragma unroll 8
    for (int c = grp; c < chunks; c += 64) acc += partials[((int64_t)c * 2 + side) * hd + e];
  }
  red[grp][col] = acc;
  for (int w = 32; w > 0; w >>= 1) {
    __syncthreads();
    if (grp < w) red[grp][col] += red[grp + w][col];
  }
  if (grp == 0 && e < hd) out[e] = red[0][col];
}

// Rows that a workgroup takes at a time.  Forward: as many as leave 2048 workgroups over both sides, eight a unit, up to 10240 elements of a side, of
// which each thread has two or three pieces whose reads overlap.  8320 rows with 6 + 6 heads of 64 and the norm get 8 rows (48 heads for 64 groups of
// lanes, so none has a second one): 10.9 us; with 16 rows, four workgroups a unit, 11.0; with 4 rows 14.1.  Backward: the partial sums hold 512
// workgroups a side, which share the rows evenly, also where there are no scales; the table of a turn is 32 KB at most.
int rows_wg(const RotaryPlan& p, bool bwd) {
  const int most = p.pairs > 64 ? 32 : 64;
  if (bwd) {
    const int64_t each = ((int64_t)p.rows + ROTARY_PARTIALS - 1) / ROTARY_PARTIALS, turns = (each + most - 1) / most;
    return (int)((each + turns - 1) / (turns > 0 ? turns : 1));
  }
  const int heads = p.heads[0] > p.heads[1] ? p.heads[0] : p.heads[1], sides = p.heads[0] && p.heads[1] ? 2 : 1;
  const int64_t few = (int64_t)p.rows * sides / 2048, busy = 10240 / ((int64_t)heads * p.hd) + 1;
  const int64_t r = few < busy ? few : busy;
  return (int)(r < 1 ? 1 : r > most ? most : r);
}
int workgroups_of(const RotaryPlan& p, bool bwd) {
  const int each = rows_wg(p, bwd) > 0 ? rows_wg(p, bwd) : 1;
  const int64_t blocks = ((int64_t)p.rows + each - 1) / each, most = bwd ? ROTARY_PARTIALS : (int64_t)1 << 23;      // (threads of a launch: under 2^32)
  return (int)(blocks < most ? blocks : most);
}
// Elements of a lane's piece: 16 bytes, or 8 where half a head or a buffer has no more in common with them; 0: no pieces.
int piece_of(const RotaryArgs& a, int dt) {
  const int P = a.p.pairs, esz = (int)dtype_size(dt);
  if (2 * P != a.p.hd) return 0;
  for (int v = 16 / esz; v >= 4; v /= 2) {
    bool ok = P % v == 0;
    for (const RotarySide& s : a.side)
      for (const void* p : {s.x, s.dy, (const void*)s.y, (const void*)s.keep}) ok = ok && !((uintptr_t)p & (v * esz - 1));
    for (const RotarySide& s : a.side)
      for (int64_t ld : {s.x_ld, s.dy_ld, s.y_ld, s.keep_ld}) ok = ok && ld % v == 0;
    if (ok) return v;
  }
  return 0;
}
template <class T, int V, bool BWD> void launch_pieces(hipStream_t s, const RotaryArgs& a, int wgs, size_t lds) {
  const dim3 grid(wgs, a.p.heads[0] && a.p.heads[1] ? 2 : 1);
  const bool norm = a.side[0].scale || a.side[1].scale;
  if (a.p.neighbours) {
    if (norm) hipLaunchKernelGGL((rotary_kernel<T, V, true, true, BWD>), grid, dim3(256), lds, s, a);
    else hipLaunchKernelGGL((rotary_kernel<T, V, true, false, BWD>), grid, dim3(256), lds, s, a);
  } else {
    if (norm) hipLaunchKernelGGL((rotary_kernel<T, V, false, true, BWD>), grid, dim3(256), lds, s, a);
    else hipLaunchKernelGGL((rotary_kernel<T, V, false, false, BWD>), grid, dim3(256), lds, s, a);
  }
}
template <bool BWD> int launch(hipStream_t s, RotaryArgs& a, int dt, int* workgroups) {
  a.rows_wg = rows_wg(a.p, BWD);
  const int wgs = workgroups_of(a.p, BWD);
  const size_t lds = (size_t)a.rows_wg * a.p.pairs * sizeof(float2);
  *workgroups = wgs;
  if (!wgs) return PPLL_OK;
  const int piece = piece_of(a, dt);
  if (piece)
    for (a.lanes = 1; a.lanes * piece < a.p.pairs;) a.lanes *= 2;
  if (!piece) hipLaunchKernelGGL((rotary_plain_kernel<BWD>), dim3(wgs), dim3(256), lds, s, a, dt);
  else if (dt == F32) launch_pieces<float, 4, BWD>(s, a, wgs, lds);
  else if (piece == 8) launch_pieces<uint16_t, 8, BWD>(s, a, wgs, lds);
  else launch_pieces<uint16_t, 4, BWD>(s, a, wgs, lds);
  PPLL_HIP(hipGetLastError());
  return PPLL_OK;
}
}  // namespace

int launch_rotary_fwd(hipStream_t s, const RotaryPlan& p, int dt, const int32_t* positions, const RotarySide& q, const RotarySide& k) {
  RotaryArgs a{p, {q, k}, positions, nullptr, 0, 0};
  int wgs;
  return launch<false>(s, a, dt, &wgs);
}
int launch_rotary_bwd(hipStream_t s, const RotaryPlan& p, int dt, const int32_t* positions, const RotarySide& q, const RotarySide& k, float* partials,
                      int* rows) {
  RotaryArgs a{p, {q, k}, positions, partials, 0, 0};
  return launch<true>(s, a, dt, rows);
}
int rotary_bwd_rows(const RotaryPlan& p) { return workgroups_of(p, true); }
int launch_rotary_scales(hipStream_t s, const float* partials, int rows, int hd, float* dq, float* dk) {
  hipLaunchKernelGGL(rotary_scale_kernel, dim3(2 * ((hd + 15) / 16)), dim3(1024), 0, s, partials, rows, hd, dq, dk);
  PPLL_HIP(hipGetLastError());
  return PPLL_OK;
}

}  // namespace ppll
