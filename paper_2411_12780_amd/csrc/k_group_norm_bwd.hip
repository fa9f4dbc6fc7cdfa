// Group norm with an activation over channels-last maps, backward: dz = dy act'(z), g = dz scale,
//   dx = r (g - mean(g) - xhat mean(g xhat)),  d_scale = sum dz xhat,  d_shift = sum dz,
// the means over a group of one image.  Both come from the sums of dz and dz xhat of each channel over an image.
//
// An image (or a slab of its channels, whole groups) that fits the registers of a workgroup is read once; a larger one goes in pieces of pixels, once
// for the channel sums and once for the gradient.  Channel sums of the images are added in a launch behind, in their order.  What bounds it: loads
// that wait, with SiLU and GELU also the slopes' instructions (16 x 96 x 96 x 256 bf16 with SiLU in pieces 46 + 5 + 44 us, 3.3 and 5.2 TB/s, a copy's rate in the
// second reading; waves wait in 59 % of their time in the first, vector instructions are issued in 53 % of its clocks; 1024 x 32 x 32 x 16 with ReLU in one go
// 42 us, 3.2 TB/s).
#include "group_norm.h"

namespace ppll {

namespace {
using namespace norm;

// What is read twice out of registers is worked out twice: kept from the first time, it would take more of them than there are
template <class T> __device__ __forceinline__ void again(T& v) {
  static_assert(sizeof(T) % 4 == 0, "");
  uint32_t w[sizeof(T) / 4];
  __builtin_memcpy(w, &v, sizeof(T));
#pragma unroll
  for (uint32_t& x : w) asm volatile("" : "+v"(x));
  __builtin_memcpy(&v, w, sizeof(T));
}

// x, from its type or from 8 bits
template <int DT, bool VEC, bool BYTES> struct XMap;
template <int DT, bool VEC> struct XMap<DT, VEC, false> {
  typedef Eight<DT> Piece;
  Map<DT, VEC> m;
  __device__ __forceinline__ void init(const NormArgs& p, int64_t pixel, int c0, int row, int c) { m.init(p.x, p.ldx, pixel, c0, row, c, p.slab, p.rt); }
  __device__ __forceinline__ void load(Piece& x, int i) const { m.load(x, i); }
};
struct BytePiece {
  uint2 w;
  int e;
  __device__ __forceinline__ void zero() { w = make_uint2(0, 0); e = 0; }
  __device__ __forceinline__ void get(float (&v)[8]) const { bytes_get(w, byte_step(e), v); }
};
template <int DT, bool VEC> struct XMap<DT, VEC, true> {
  typedef BytePiece Piece;
  const int8_t *base, *exps;
  int64_t step;
  uint32_t at, row_;
  int rt;
  __device__ __forceinline__ void init(const NormArgs& p, int64_t pixel, int c0, int row, int c) {
    base = p.q + pixel * p.ldq + c0;
    exps = p.qe + pixel;
    step = p.rt * p.ldq;
    at = (uint32_t)row * (uint32_t)p.ldq + c;
    row_ = row;
    rt = p.rt;
  }
  __device__ __forceinline__ void load(Piece& x, int i) const {
    x.w = *(const uint2*)(base + i * step + at);
    x.e = (exps + i * rt)[row_];
  }
};

// What a thread knows of its channels; GV: segments of its eight, each of one group
template <int GV> struct Channels {
  static constexpr int PER = 8 / GV;
  float mean[GV], rstd[GV], scale[8], shift[8];
  __device__ __forceinline__ void load(const NormArgs& p, int image, int c0, int c) {
#pragma unroll
    for (int e = 0; e < GV; ++e) {
      const float* st = p.stats_in + ((int64_t)image * p.groups + quotient(c0 + min(c + e * PER, p.slab - 1), p.over_cg)) * 2;
      mean[e] = st[0]; rstd[e] = st[1];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const bool in = c + e < p.slab;
      scale[e] = in ? p.scale[c0 + c + e] : 0.f;
      shift[e] = in ? p.shift[c0 + c + e] : 0.f;
    }
  }
  template <class X> __device__ __forceinline__ void xhat(const X& x, float (&h)[8]) const {
    x.get(h);
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] = (h[e] - mean[e / PER]) * rstd[e / PER];
  }
  // dz; side: y (ReLU) or the residual (curved activations)
  template <int DT> __device__ __forceinline__ void gradient(const Clamp&, const Eight<DT>& dy, const Eight<DT>& side, bool has_side, const float (&)[8], float (&d)[8]) const {
    dy.get(d);
    if (!has_side) return;       // no activation
    float s[8];
    side.get(s);
#pragma unroll
    for (int e = 0; e < 8; ++e) d[e] = s[e] > 0.f ? d[e] : 0.f;
  }
  template <int DT, class A>
  __device__ __forceinline__ void gradient(const A& act, const Eight<DT>& dy, const Eight<DT>& side, bool has_side, const float (&h)[8], float (&d)[8]) const {
    float z[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) z[e] = h[e] * scale[e] + shift[e];
    if (has_side) {
      float s[8];
      side.get(s);
#pragma unroll
      for (int e = 0; e < 8; ++e) z[e] += s[e];
    }
    dy.get(d);
#pragma unroll
    for (int e = 0; e < 8; ++e) d[e] *= act.slope(z[e]);
  }
  // d_residual and dx of a piece
  template <int DT, bool VEC>
  __device__ __forceinline__ void out(const Map<DT, VEC>& dx, const Map<DT, VEC>& dres, bool residual, int i, const float (&ga)[GV], const float (&gb)[GV],
                                      const float (&h)[8], float (&d)[8]) const {
    Eight<DT> o;
    if (residual) {
      o.set(d);
      dres.store(o, i);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) d[e] = rstd[e / PER] * (d[e] * scale[e] - ga[e / PER] - h[e] * gb[e / PER]);
    o.set(d);
    dx.store(o, i);
  }
};
// The maps of a unit of work
template <int DT, bool VEC, bool BYTES> struct Maps {
  XMap<DT, VEC, BYTES> x;
  Map<DT, VEC> dy, side, dx, dres;
  bool has_side;
  __device__ __forceinline__ void init(const NormArgs& p, int64_t pixel, int c0, int row, int c) {
    x.init(p, pixel, c0, row, c);
    dy.init(p.dy, p.ldd, pixel, c0, row, c, p.slab, p.rt);
    if (p.y_in) side.init(p.y_in, p.ldy, pixel, c0, row, c, p.slab, p.rt);
    else side.init(p.residual, p.ldr, pixel, c0, row, c, p.slab, p.rt);
    has_side = p.y_in || p.residual;
    dx.init(p.dx, p.lddx, pixel, c0, row, c, p.slab, p.rt);
    dres.init(p.dres, p.lddr, pixel, c0, row, c, p.slab, p.rt);
  }
};

// The groups' means of g and of g xhat from a slab's channel sums times scale, chan [2][slab] in LDS; group: room behind
template <int GV> __device__ __forceinline__ void group_means(const NormArgs& p, const float* chan, float* group, int c, float (&ga)[GV], float (&gb)[GV]) {
  const int cols = p.slab;
  const float over = 1.f / (float)((int64_t)p.pixels * p.cg);
  __syncthreads();
  runs_sums(2 * quotient(cols, p.over_cg), p.cg, [&](int k) { return chan + (k & 1) * cols + (k >> 1) * p.cg; },
            [&](int k, float s) { group[k] = s * over; });
  __syncthreads();
#pragma unroll
  for (int e = 0; e < GV; ++e) {
    const int g = quotient(min(c + e * (8 / GV), cols - 1), p.over_cg);
    ga[e] = group[2 * g]; gb[e] = group[2 * g + 1];
  }
}

// An image's slab in registers: channel sums, which are left in p.sums, and the gradient.  Straight and curved activations are kernels of their own: the
// former take 40 to 50 registers less, which gives a unit two workgroups of 512 (1024 x 32 x 32 x 16, two groups, ReLU, 41 us; 54 in one kernel).
template <int DT, bool VEC, int GV, bool BYTES, bool CURVED, int MI>
__global__ __launch_bounds__(MOST_THREADS, !CURVED && GV <= 4 && MI * (DT == BF16 ? 1 : 2) <= 4 ? 4 : 2) void group_norm_bwd_kernel(NormArgs p) {
  extern __shared__ float room[];
  const int t = threadIdx.x, row = quotient(t, p.over_npc), col = t - row * p.npc;
  const bool live = row < p.rt;
  const int units = p.units;
  for (int u = blockIdx.x; u < units; u += gridDim.x) {
    const Unit w = unit_of(p, u);
    if (w.image >= p.images) continue;
    const int c0 = w.slab * p.slab, c = col * 8, cols = p.slab, n = live ? p.pixels - row : 0;
    Maps<DT, VEC, BYTES> m;
    m.init(p, (int64_t)w.image * p.pixels, c0, row, c);
    typename XMap<DT, VEC, BYTES>::Piece x[MI];
    Eight<DT> dy[MI], side[MI];
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      if (i * p.rt < n) {       // (a piece that is not there is not looked at)
        m.x.load(x[i], i);
        m.dy.load(dy[i], i);
        if (m.has_side) m.side.load(side[i], i);
      }
    }
    Channels<GV> k;
    k.load(p, w.image, c0, c);
    // slopes of curved activations are worked out once, where there is room for what comes of them (1024 x 32 x 32 x 16 with GELU 51 us, 61 twice)
    constexpr bool HELD = CURVED && MI * (DT == BF16 ? 1 : 2) <= 4;
    with_activation<DT == F32, CURVED>(p.act, [&](auto act) {
      float sums[16], h[8], d[8], held[HELD ? MI : 1][8];
#pragma unroll
      for (int e = 0; e < 16; ++e) sums[e] = 0.f;
#pragma unroll
      for (int i = 0; i < MI; ++i) {
        if (i * p.rt >= n) continue;
        k.xhat(x[i], h);
        k.gradient(act, dy[i], side[i], m.has_side, h, d);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          sums[e] += d[e]; sums[8 + e] += d[e] * h[e];
          if (HELD) held[HELD ? i : 0][e] = d[e];
        }
      }
      column_sums<16>(sums, p, room);
      __syncthreads();
      if (row == 0) {
        float* to = p.sums + (int64_t)w.image * 2 * p.C + c0 + c;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (VEC || c + e < cols) {
            to[e] = sums[e]; to[p.C + e] = sums[8 + e];
            room[c + e] = sums[e] * k.scale[e]; room[cols + c + e] = sums[8 + e] * k.scale[e];
          }
      }
      float ga[GV], gb[GV];
      group_means<GV>(p, room, room + 2 * cols, c, ga, gb);
#pragma unroll
      for (int i = 0; i < MI; ++i) { again(x[i]); if (!HELD) again(dy[i]); }
#pragma unroll
      for (int i = 0; i < MI; ++i) {
        if (i * p.rt >= n) continue;
        k.xhat(x[i], h);
        if (HELD) {
#pragma unroll
          for (int e = 0; e < 8; ++e) d[e] = held[HELD ? i : 0][e];
        } else {
          k.gradient(act, dy[i], side[i], m.has_side, h, d);
        }
        k.out(m.dx, m.dres, p.dres, i, ga, gb, h, d);
      }
    });
    __syncthreads();
  }
}

// Sums over the first axis of [n][2 C], in its order: a workgroup 16 columns, ROWS rows (a sixteenth of its threads) at a time.  To out [2 C], or (null) the
// halves to d_shift and d_scale.  part: 17 floats a row.
template <int ROWS> __device__ __forceinline__ void axis_sums(float* part, int block, const float* in, int n, int C, float* out, float* d_scale, float* d_shift) {
  const int i = threadIdx.x & 15, c = block * 16 + i, r = threadIdx.x >> 4;
  float s = 0.f;
  if (c < 2 * C)
#pragma unroll 4
    for (int64_t k = r; k < n; k += ROWS) s += in[k * 2 * C + c];
  __syncthreads();
  part[r * 17 + i] = s;
  __syncthreads();
  if (r == 0 && c < 2 * C) {
    s = 0.f;
    for (int k = 0; k < ROWS; ++k) s += part[k * 17 + i];
    if (out) out[c] = s;
    else if (c < C) d_shift[c] = s;
    else d_scale[c - C] = s;
  }
}
constexpr int SUM_THREADS = 1024;

// Pieces of pixels: PART leaves their channel sums, [images][chunks][2][C]; APPLY takes the gradient from those of the image, p.sums.  Two batches of
// pieces in turn, one on its way while the other is worked on.  Beside APPLY the last workgroups add up the images' sums (a launch of its own took 5 us).
template <int DT, bool VEC, bool BYTES> struct Batch {
  static constexpr int N = DT == BF16 ? 1 : 2;
  typename XMap<DT, VEC, BYTES>::Piece x[N];
  Eight<DT> dy[N], side[N];
  __device__ __forceinline__ void load(const NormArgs& p, int64_t at, int row, int c, int n) {
    Maps<DT, VEC, BYTES> m;
    m.init(p, at, 0, row, c);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      x[i].zero();
      dy[i].zero();
      side[i].zero();
      if (i * p.rt < n) {
        m.x.load(x[i], i);
        m.dy.load(dy[i], i);
        if (m.has_side) m.side.load(side[i], i);
      }
    }
  }
};
template <int DT, int MODE, bool VEC, int GV, bool BYTES, bool CURVED>
__global__ __launch_bounds__(MOST_THREADS, DT == BF16 && (GV == 1 || (!CURVED && (GV < 8 || MODE == PART))) ? 4 : 2) void group_norm_bwd_piece_kernel(NormArgs p) {
  extern __shared__ float room[];
  typedef Batch<DT, VEC, BYTES> B;
  const int t = threadIdx.x, row = quotient(t, p.over_npc), col = t - row * p.npc;
  const bool live = row < p.rt;
  const int units = p.units, workers = gridDim.x - (MODE == APPLY ? p.sum_blocks : 0);
  if (MODE == APPLY && (int)blockIdx.x >= workers) {
    axis_sums<MOST_THREADS / 16>(room, blockIdx.x - workers, p.sums, p.images, p.C, nullptr, p.d_scale, p.d_shift);
    return;
  }
  for (int u = blockIdx.x; u < units; u += workers) {
    const Unit w = unit_of(p, u);
    const int c = col * 8, cols = p.slab, step = B::N * p.rt, end = live ? w.last - row : 0;      // pixel q + i rt + row is there where q + i rt < end
    const int64_t image = (int64_t)w.image * p.pixels;
    B even, odd;
    even.load(p, image + w.first, row, c, end - w.first);
    Channels<GV> k;
    k.load(p, w.image, 0, c);
    float sums[16], ga[GV], gb[GV], h[8], d[8];
    if (MODE == APPLY) {
      const float* from = p.sums + (int64_t)w.image * 2 * p.C;
      __syncthreads();
      for (int j = t; j < cols; j += blockDim.x) { room[j] = from[j] * p.scale[j]; room[cols + j] = from[cols + j] * p.scale[j]; }
      group_means<GV>(p, room, room + 2 * cols, c, ga, gb);
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) sums[e] = 0.f;
    with_activation<DT == F32, CURVED>(p.act, [&](auto act) {
      auto work = [&](const B& b, int q) {
        Maps<DT, VEC, BYTES> m;
        m.init(p, image + q, 0, row, c);
#pragma unroll
        for (int i = 0; i < B::N; ++i) {
          if (q + i * p.rt >= end) continue;
          k.xhat(b.x[i], h);
          k.gradient(act, b.dy[i], b.side[i], m.has_side, h, d);
          if (MODE == PART) {
#pragma unroll
            for (int e = 0; e < 8; ++e) { sums[e] += d[e]; sums[8 + e] += d[e] * h[e]; }
          } else {
            k.out(m.dx, m.dres, p.dres, i, ga, gb, h, d);
          }
        }
      };
      for (int q = w.first; q < w.last; q += 2 * step) {
        odd.load(p, image + q + step, row, c, end - q - step);
        work(even, q);
        even.load(p, image + q + 2 * step, row, c, end - q - 2 * step);
        work(odd, q + step);
      }
    });
    if (MODE == PART) {
      column_sums<16>(sums, p, room);
      if (row == 0) {
        float* to = p.parts + ((int64_t)w.image * p.chunks + w.part) * 2 * p.C + c;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (VEC || c + e < cols) { to[e] = sums[e]; to[p.C + e] = sums[8 + e]; }
      }
    }
  }
}

__global__ __launch_bounds__(SUM_THREADS) void group_norm_sum_kernel(const float* in, int n, int64_t set_stride, int sets, int C, float* out, float* d_scale,
                                                                     float* d_shift) {
  __shared__ float part[SUM_THREADS + SUM_THREADS / 16];
  for (int set = blockIdx.y; set < sets; set += gridDim.y)
    axis_sums<SUM_THREADS / 16>(part, blockIdx.x, in + set * set_stride, n, C, out ? out + (int64_t)set * 2 * C : nullptr, d_scale, d_shift);
}
__global__ __launch_bounds__(256) void group_norm_zero_kernel(float* a, float* b, int n) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i < n) a[i] = b[i] = 0.f;
}

static_assert(4 * 4096 * sizeof(float) <= 64 * 1024, "what a launch has without asking");
template <int DT, bool VEC, int GV, bool BYTES, bool CURVED> int launches(hipStream_t s, const GroupNorm& g, NormArgs& p, const Layout& l, float* d_scale, float* d_shift, float* ws) {
  constexpr int MOST = DT == BF16 ? 8 : 4;
  const int C = g.channels;
  // sums of the columns, or channel sums and those of their groups
  const size_t lds = (size_t)std::max(l.threads * 16, 2 * p.slab + 2 * (p.slab / p.cg)) * sizeof(float);
  const dim3 grid(grid_of(p)), block(l.threads), columns((2 * C + 15) / 16);
  p.sums = ws;
  if (l.whole) {
    if (l.mi <= MOST / 2) hipLaunchKernelGGL((group_norm_bwd_kernel<DT, VEC, GV, BYTES, CURVED, MOST / 2>), grid, block, lds, s, p);
    else hipLaunchKernelGGL((group_norm_bwd_kernel<DT, VEC, GV, BYTES, CURVED, MOST>), grid, block, lds, s, p);
    PPLL_HIP(hipGetLastError());
  } else {
    p.parts = ws + (int64_t)g.images * 2 * C;
    hipLaunchKernelGGL((group_norm_bwd_piece_kernel<DT, PART, VEC, GV, BYTES, CURVED>), grid, block, lds, s, p);
    PPLL_HIP(hipGetLastError());
    // pieces into images
    hipLaunchKernelGGL(group_norm_sum_kernel, dim3(columns.x, std::min(g.images, 65535)), dim3(SUM_THREADS), 0, s, p.parts, p.chunks, (int64_t)p.chunks * 2 * C, g.images, C,
                       p.sums, (float*)nullptr, (float*)nullptr);
    PPLL_HIP(hipGetLastError());
    p.sum_blocks = columns.x; p.d_scale = d_scale; p.d_shift = d_shift;
    hipLaunchKernelGGL((group_norm_bwd_piece_kernel<DT, APPLY, VEC, GV, BYTES, CURVED>), dim3(grid.x + columns.x), block, lds, s, p);
    PPLL_HIP(hipGetLastError());
    return PPLL_OK;
  }
  hipLaunchKernelGGL(group_norm_sum_kernel, columns, dim3(SUM_THREADS), 0, s, p.sums, g.images, (int64_t)0, 1, C, (float*)nullptr, d_scale, d_shift);
  PPLL_HIP(hipGetLastError());
  return PPLL_OK;
}
template <int DT, bool BYTES, bool CURVED> int bwd_as(hipStream_t s, const GroupNorm& g, NormArgs& p, const Layout& l, float* d_scale, float* d_shift, float* ws) {
  if (p.slab % 8) return launches<DT, false, 8, BYTES, CURVED>(s, g, p, l, d_scale, d_shift, ws);
  if (p.cg % 2) return launches<DT, true, 8, BYTES, CURVED>(s, g, p, l, d_scale, d_shift, ws);
  if (p.cg % 4) return launches<DT, true, 4, BYTES, CURVED>(s, g, p, l, d_scale, d_shift, ws);
  if (p.cg % 8) return launches<DT, true, 2, BYTES, CURVED>(s, g, p, l, d_scale, d_shift, ws);
  return launches<DT, true, 1, BYTES, CURVED>(s, g, p, l, d_scale, d_shift, ws);
}
template <int DT, bool BYTES> int bwd(hipStream_t s, const GroupNorm& g, NormArgs& p, const Layout& l, float* d_scale, float* d_shift, float* ws) {
  if (p.act == PPLL_ACT_SILU || p.act == PPLL_ACT_GELU) return bwd_as<DT, BYTES, true>(s, g, p, l, d_scale, d_shift, ws);
  return bwd_as<DT, BYTES, false>(s, g, p, l, d_scale, d_shift, ws);
}
}  // namespace

int launch_group_norm_bwd(hipStream_t s, const GroupNorm& g, const ppll_rows& x, const ppll_byte_rows& x8, const float* stats, const float* scale,
                          const float* shift, const ppll_rows& residual, const ppll_rows& y, const ppll_rows& dy, const ppll_rows& dx, const ppll_rows& dres,
                          float* d_scale, float* d_shift, char* ws) {
  if (g.images <= 0) {
    hipLaunchKernelGGL(group_norm_zero_kernel, dim3((g.channels + 255) / 256), dim3(256), 0, s, d_scale, d_shift, g.channels);
    PPLL_HIP(hipGetLastError());
    return PPLL_OK;
  }
  Layout l = layout_of(g);
  spread_over_units(g, l);
  NormArgs p = args_of(g, l, l.stretch);
  p.x = (const char*)x.p; p.ldx = x.ld; p.q = x8.q; p.qe = x8.e; p.ldq = x8.ld;
  p.residual = (const char*)residual.p; p.ldr = residual.ld; p.y_in = (const char*)y.p; p.ldy = y.ld; p.dy = (const char*)dy.p; p.ldd = dy.ld;
  p.dx = (char*)dx.p; p.lddx = dx.ld; p.dres = (char*)dres.p; p.lddr = dres.ld;
  p.stats_in = stats; p.scale = scale; p.shift = shift;
  const bool bytes = !p.x;
  if (g.dt == BF16) return bytes ? bwd<BF16, true>(s, g, p, l, d_scale, d_shift, (float*)ws) : bwd<BF16, false>(s, g, p, l, d_scale, d_shift, (float*)ws);
  return bytes ? bwd<F32, true>(s, g, p, l, d_scale, d_shift, (float*)ws) : bwd<F32, false>(s, g, p, l, d_scale, d_shift, (float*)ws);
}

}  // namespace ppll
