// Group norm with an activation over channels-last maps, forward.
//
// A thread holds pieces of 8 channels of every RT-th pixel in registers, so that an image (or a slab of its channels, whole groups) that fits the
// registers of a workgroup is read once and written once: mean, then the squares about it, then the result.  A larger image goes in pieces of pixels:
// statistics of each piece, joined exactly, then the result, the map read a second time, from the last-level cache where it fits.  What bounds it:
// loads that wait and vector instructions, neither alone (16 x 96 x 96 x 256 bf16 in pieces, kept in 8 bits, 34 + 5 + 36 us: 3.3 and 4.2 TB/s, a copy 5.2; waves
// wait in 58 and 66 % of their time, vector instructions are issued in 62 and 49 % of the clocks; 1024 x 32 x 32 x 16 in one go 24 us, 2.8 TB/s: load, two sums
// over a workgroup and store one behind the other).
#include "group_norm.h"

namespace ppll {

namespace {
using namespace norm;

// y of a piece: y = act((x - mean) a + b (+ residual))
template <int DT, bool VEC, class A> __device__ __forceinline__ void finish(const A& act, const float (&mean)[8], const float (&a)[8], const float (&b)[8],
                                                                            const Eight<DT>& x, const Eight<DT>& res, bool residual, const Map<DT, VEC>& to,
                                                                            int i) {
  float v[8];
  x.get(v);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = (v[e] - mean[e]) * a[e] + b[e];
  if (residual) {
    float f[8];
    res.get(f);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += f[e];
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = act(v[e]);
  Eight<DT> o;
  o.set(v);
  to.store(o, i);
}
__device__ __forceinline__ void affine(const NormArgs& p, int c0, int c, const float (&rstd)[8], float (&a)[8], float (&b)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const bool in = c + e < p.slab;
    a[e] = in ? p.scale[c0 + c + e] * rstd[e] : 0.f;
    b[e] = in ? p.shift[c0 + c + e] : 0.f;
  }
}
// The pixel's row in 8 bits, from the lanes that hold it (a power of two of one wave); all of them come here
template <int DT> __device__ __forceinline__ void keep_piece(const NormArgs& p, const Eight<DT>& x, int64_t pixel, int col, bool in) {
  float v[8];
  x.get(v);
  const uint32_t most = lanes_most_of(most_of(v, 0), p.npc);
  const int e = byte_exponent(most);
  if (!in) return;
  const bool nan = e == BYTE_NAN;
  if (col == 0) p.keep_e[pixel] = (int8_t)e;
  int8_t* to = p.keep + pixel * p.ldk + col * 8;
  *(uint2*)to = nan ? make_uint2(0, 0) : bytes_of(v, exp2_bits(nan ? 0 : -e));
  if (p.npc == 1) *(uint2*)(to + 8) = make_uint2(0, 0);      // the padding of an odd number of pieces
}

// An image's slab in registers (WHOLE), or a piece of an image, of which its statistics are left (PART).  GV: segments of a piece of 8 channels, each of
// one group; MI: pieces a thread holds.  Up to 4 of them within 128 registers, so that a unit has two workgroups of 512, one's memory busy during the
// other's sums (1024 x 32 x 32 x 16, groups of 2, 25 us; 33 with the 129 registers that the compiler took by itself).
template <int DT, int MODE, bool VEC, int GV, int MI>
__global__ __launch_bounds__(MOST_THREADS, MODE == PART || (MI * (DT == BF16 ? 1 : 2) <= 4 && GV <= 4) || (DT == F32 && GV == 1) ? 4 : 2) void group_norm_fwd_kernel(NormArgs p) {
  constexpr int PER = 8 / GV;
  extern __shared__ float room[];
  const int t = threadIdx.x, row = quotient(t, p.over_npc), col = t - row * p.npc;
  const bool live = row < p.rt;
  const int units = p.units;
  for (int u = blockIdx.x; u < units; u += gridDim.x) {
    const Unit w = unit_of(p, u);
    if (w.image >= p.images) continue;
    const int c0 = w.slab * p.slab, c = col * 8, cols = p.slab, g0 = c0 / p.cg;
    const int64_t at = (int64_t)w.image * p.pixels + w.first;
    const int n = live ? w.last - w.first - row : 0;         // piece i is there where i rt < n
    Eight<DT> x[MI], res[MODE == WHOLE ? MI : 1];
    Map<DT, VEC> from;
    from.init(p.x, p.ldx, at, c0, row, c, cols, p.rt);
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      x[i].zero();
      if (i * p.rt < n) from.load(x[i], i);
    }
    if constexpr (MODE == WHOLE) {      // on its way during the sums
#pragma unroll
      for (int i = 0; i < MI; ++i) res[i].zero();
      if (p.residual) {
        Map<DT, VEC> side;
        side.init(p.residual, p.ldr, at, c0, row, c, cols, p.rt);
#pragma unroll
        for (int i = 0; i < MI; ++i)
          if (i * p.rt < n) side.load(res[i], i);
      }
    }
    float mean[GV], rstd[GV];
    const float count = (float)((int64_t)(w.last - w.first) * p.cg);
#pragma unroll
    for (int i = 0; i < GV; ++i) mean[i] = 0.f;
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      float v[8];
      x[i].get(v);
#pragma unroll
      for (int e = 0; e < 8; ++e) mean[e / PER] += v[e];
    }
    column_sums<GV>(mean, p, room);
    group_sums<GV>(mean, p, room);
#pragma unroll
    for (int i = 0; i < GV; ++i) { mean[i] /= count; rstd[i] = 0.f; }
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      if (i * p.rt >= n) continue;
      float v[8];
      x[i].get(v);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float d = v[e] - mean[e / PER];
        rstd[e / PER] += VEC || c + e < cols ? d * d : 0.f;
      }
    }
    column_sums<GV>(rstd, p, room);
    group_sums<GV>(rstd, p, room);
    if (p.keep) {
#pragma unroll
      for (int i = 0; i < MI; ++i) keep_piece<DT>(p, x[i], at + row + i * p.rt, col, i * p.rt < n);
    }
#pragma unroll
    for (int i = 0; i < GV; ++i) {
      if (MODE == WHOLE) rstd[i] = rsqrtf(rstd[i] / count + p.eps);
      float* to = MODE == PART ? p.parts + ((int64_t)w.image * p.chunks + w.part) * p.groups * 2 : p.stats ? p.stats + (int64_t)w.image * p.groups * 2 : nullptr;
      // the first pixel's threads tell, of each group the one with its first channel
      if (to && row == 0 && c + i * PER < cols) {
        const int g = quotient(c + i * PER, p.over_cg);
        if (g * p.cg == c + i * PER) { to[2 * (g0 + g)] = mean[i]; to[2 * (g0 + g) + 1] = rstd[i]; }
      }
    }
    if constexpr (MODE == WHOLE) {
      float m[8], r[8], a[8], b[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) { m[e] = mean[e / PER]; r[e] = rstd[e / PER]; }
      affine(p, c0, c, r, a, b);
      Map<DT, VEC> to;
      to.init(p.y, p.ldy, at, c0, row, c, cols, p.rt);
      with_activation<DT == F32, -1>(p.act, [&](auto act) {
#pragma unroll
        for (int i = 0; i < MI; ++i)
          if (i * p.rt < n) finish<DT, VEC>(act, m, a, b, x[i], res[i], p.residual, to, i);
      });
    }
  }
}

// Statistics of an image's groups joined from those of its pieces, [images][chunks][groups][2] (mean, squares about it): the piece means' own spread
// counts as well.  A wave a group; each lane joins every 64th piece, then the lanes each other.
__global__ __launch_bounds__(256) void group_norm_join_kernel(NormArgs p, float* joined) {
  const int lane = threadIdx.x & 63;
  const int64_t n_groups = (int64_t)p.images * p.groups;
  for (int64_t j = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); j < n_groups; j += (int64_t)gridDim.x * 4) {
    const int64_t image = j / p.groups, g = j - image * p.groups;
    const float* at = p.parts + (image * p.chunks * p.groups + g) * 2;
    float n = 0.f, m = 0.f, s = 0.f;
    auto add = [&](float nk, float mk, float sk) {
      const float total = n + nk, share = total > 0.f ? nk / total : 0.f, d = mk - m;
      s += sk + d * d * share * n;
      m += d * share;
      n = total;
    };
    for (int k = lane; k < p.chunks; k += 64) {
      const float* from = at + (int64_t)k * p.groups * 2;
      add((float)((int64_t)(min(p.pixels, (k + 1) * p.chunk) - k * p.chunk) * p.cg), from[0], from[1]);
    }
#pragma unroll
    for (int h = 32; h >= 1; h >>= 1) {
      const float nk = __shfl_down(n, h), mk = __shfl_down(m, h), sk = __shfl_down(s, h);
      add(nk, mk, sk);
    }
    if (lane == 0) {
      const float r = rsqrtf(s / n + p.eps);
      joined[2 * j] = m; joined[2 * j + 1] = r;
      if (p.stats) { p.stats[2 * j] = m; p.stats[2 * j + 1] = r; }
    }
  }
}

// y of a piece of pixels, from the image's statistics.  Two batches of pieces in turn, one on its way while the other is worked on.
template <int DT, bool VEC> struct Batch {
  static constexpr int N = 2;
  Eight<DT> x[N], res[N];
  __device__ __forceinline__ void load(const NormArgs& p, int64_t at, int row, int c, int n) {
    Map<DT, VEC> from, side;
    from.init(p.x, p.ldx, at, 0, row, c, p.slab, p.rt);
    side.init(p.residual, p.ldr, at, 0, row, c, p.slab, p.rt);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      x[i].zero();
      res[i].zero();
      if (i * p.rt < n) {
        from.load(x[i], i);
        if (p.residual) side.load(res[i], i);
      }
    }
  }
};
template <int DT, bool VEC, bool CURVED> __global__ __launch_bounds__(MOST_THREADS, DT == BF16 ? 4 : 2) void group_norm_apply_kernel(NormArgs p) {
  constexpr int N = Batch<DT, VEC>::N;
  const int t = threadIdx.x, row = quotient(t, p.over_npc), col = t - row * p.npc;
  if (row >= p.rt) return;
  const int units = p.units;
  for (int u = blockIdx.x; u < units; u += gridDim.x) {
    const Unit w = unit_of(p, u);
    const int c = col * 8, cols = p.slab, step = N * p.rt;
    const int64_t image = (int64_t)w.image * p.pixels;
    Batch<DT, VEC> even, odd;
    even.load(p, image + w.first, row, c, w.last - w.first - row);
    float mean[8], rstd[8], a[8], b[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float* st = p.stats_in + ((int64_t)w.image * p.groups + quotient(min(c + e, cols - 1), p.over_cg)) * 2;
      mean[e] = st[0]; rstd[e] = st[1];
    }
    affine(p, 0, c, rstd, a, b);
    with_activation<DT == F32, CURVED>(p.act, [&](auto act) {
      auto finish_batch = [&](const Batch<DT, VEC>& d, int q) {
        Map<DT, VEC> to;
        to.init(p.y, p.ldy, image + q, 0, row, c, cols, p.rt);
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (i * p.rt < w.last - q - row) finish<DT, VEC>(act, mean, a, b, d.x[i], d.res[i], p.residual, to, i);
      };
      for (int q = w.first; q < w.last; q += 2 * step) {
        odd.load(p, image + q + step, row, c, w.last - q - step - row);
        finish_batch(even, q);
        even.load(p, image + q + 2 * step, row, c, w.last - q - 2 * step - row);
        finish_batch(odd, q + step);
      }
    });
  }
}

template <int DT, int MODE, bool VEC, int GV> int fwd_launch(hipStream_t s, const NormArgs& p, const Layout& l) {
  constexpr int MOST = DT == BF16 ? 8 : 4;
  const size_t lds = sizeof(float) * (size_t)(l.threads * GV + p.slab / p.cg);
  const dim3 grid(grid_of(p)), block(l.threads);
  if (MODE == PART) hipLaunchKernelGGL((group_norm_fwd_kernel<DT, MODE, VEC, GV, PART_MI>), grid, block, lds, s, p);
  else if (l.mi <= MOST / 2) hipLaunchKernelGGL((group_norm_fwd_kernel<DT, WHOLE, VEC, GV, MOST / 2>), grid, block, lds, s, p);
  else hipLaunchKernelGGL((group_norm_fwd_kernel<DT, WHOLE, VEC, GV, MOST>), grid, block, lds, s, p);
  PPLL_HIP(hipGetLastError());
  return PPLL_OK;
}
template <int DT, int MODE> int fwd(hipStream_t s, NormArgs& p, const Layout& l) {
  const bool vec = p.slab % 8 == 0;
  const int gv = vec ? segments_of(p.cg) : 8;
  p.spg = p.cg * gv / 8;
  p.over_spg = 1.f / (float)p.spg;
  if (!vec) return fwd_launch<DT, MODE, false, 8>(s, p, l);
  if (gv == 1) return fwd_launch<DT, MODE, true, 1>(s, p, l);
  if (gv == 2) return fwd_launch<DT, MODE, true, 2>(s, p, l);
  if (gv == 4) return fwd_launch<DT, MODE, true, 4>(s, p, l);
  return fwd_launch<DT, MODE, true, 8>(s, p, l);
}
template <int DT, bool VEC> int apply(hipStream_t s, const NormArgs& p, const Layout& l) {
  const dim3 grid(grid_of(p)), block(l.threads);
  if (p.act == PPLL_ACT_SILU || p.act == PPLL_ACT_GELU) hipLaunchKernelGGL((group_norm_apply_kernel<DT, VEC, true>), grid, block, 0, s, p);
  else hipLaunchKernelGGL((group_norm_apply_kernel<DT, VEC, false>), grid, block, 0, s, p);
  PPLL_HIP(hipGetLastError());
  return PPLL_OK;
}
template <int DT> int fwd_all(hipStream_t s, const GroupNorm& g, NormArgs& p, const Layout& l, float* ws) {
  if (l.whole) return fwd<DT, WHOLE>(s, p, l);
  p.parts = ws;
  float* joined = ws + (int64_t)p.images * p.chunks * p.groups * 2;
  PPLL_TRY((fwd<DT, PART>(s, p, l)));
  hipLaunchKernelGGL(group_norm_join_kernel, dim3((unsigned)std::min<int64_t>(((int64_t)p.images * p.groups + 3) / 4, MOST_BLOCKS)), dim3(256), 0, s, p, joined);
  PPLL_HIP(hipGetLastError());
  p.stats_in = joined;
  p.chunk = l.stretch; p.chunks = chunks_of(g, l.stretch); p.units = units_of(p);
  return p.slab % 8 == 0 ? apply<DT, true>(s, p, l) : apply<DT, false>(s, p, l);
}
}  // namespace

size_t group_norm_workspace(const GroupNorm& g) {
  if (g.images <= 0) return 0;
  const Layout l = layout_of(g);
  const int64_t sums = (int64_t)g.images * 2 * g.channels, stats = (int64_t)g.images * g.groups * 2;
  const int64_t bwd = l.whole ? sums : sums + chunks_of(g, l.stretch) * sums, fwd = l.whole ? 0 : stats + chunks_of(g, l.chunk) * stats;
  return (size_t)std::max(bwd, fwd) * sizeof(float);
}

int launch_group_norm_fwd(hipStream_t s, const GroupNorm& g, const ppll_rows& x, const float* scale, const float* shift, const ppll_rows& residual,
                          const ppll_rows& y, float* stats, const ppll_byte_rows& keep, char* ws) {
  if (g.images <= 0) return PPLL_OK;
  Layout l = layout_of(g);
  if (!keep.q) spread_over_units(g, l);        // (a row in 8 bits needs all channels of a pixel)
  NormArgs p = args_of(g, l, l.chunk);
  p.x = (const char*)x.p; p.ldx = x.ld; p.residual = (const char*)residual.p; p.ldr = residual.ld; p.y = (char*)y.p; p.ldy = y.ld;
  p.scale = scale; p.shift = shift; p.stats = stats;
  if (keep.q) {
    if (p.slabs == 1 && p.pow2) { p.keep = keep.q; p.keep_e = keep.e; p.ldk = keep.ld; }
    else PPLL_TRY(launch_byte_rows_pack(s, g.dt, g.images * g.pixels, g.channels, x, keep));      // (before y, which may be x)
  }
  return g.dt == BF16 ? fwd_all<BF16>(s, g, p, l, (float*)ws) : fwd_all<F32>(s, g, p, l, (float*)ws);
}

}  // namespace ppll
