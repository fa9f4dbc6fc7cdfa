// Group norm: what its forward and backward kernels share.
#pragma once
#include <algorithm>

#include "bytes.h"

namespace ppll {
namespace norm {

constexpr unsigned MOST_BLOCKS = 1u << 20;
enum Mode : int { WHOLE = 0, PART = 1, APPLY = 2 };      // an image in one go; what a piece of it leaves; the result of a piece

// How the threads of a workgroup lie over a slab: NPC piece columns (8 channels), RT pixels at a time
struct NormArgs {
  const char *x, *residual, *y_in, *dy;
  const int8_t *q, *qe;
  char *y, *dx, *dres;
  int8_t *keep, *keep_e;
  int64_t ldx, ldr, ldy, ldd, ldq, lddx, lddr, ldk;
  const float *scale, *shift, *stats_in;
  float *stats, *parts;            // parts: what PART leaves and APPLY joins
  float* sums;                     // backward: channel sums of each image, [images][2][C]
  float *d_scale, *d_shift;        // backward, pieces of pixels: added up by the last `sum_blocks` workgroups of the launch
  int sum_blocks;
  int images, pixels, C, groups, cg, act;
  int slab, slabs, npc, rt, pow2;  // channels of a slab; npc: piece columns, pow2: a power of two up to 64
  int chunk, chunks, units;        // pixels of a piece, pieces of an image, workgroups' work
  int spg;                         // segments of a group
  float eps, over_cg, over_npc, over_spg;    // 1 / cg, 1 / npc, 1 / spg: see quotient()
};

// v / n for 0 <= v <= 4096 and 1 <= n <= 4096, over = 1 / n: (v + 1/2) / n is at least 1 / (2 n) off every whole number, its value in fp32 less than 2^-12 of
// that (two instructions; a division of whole numbers takes some thirty)
__device__ __forceinline__ int quotient(int v, float over) { return (int)(((float)v + 0.5f) * over); }

template <bool EXACT> __device__ __forceinline__ float sigmoid(float z) {
  return __builtin_amdgcn_rcpf(1.f + (EXACT ? expf(-z) : __expf(-z)));
}
// Activations and slopes as types, so that a loop over elements holds one of them
struct Clamp {       // none (from = -infinity) and ReLU (0); a NaN stays one
  float from;
  __device__ __forceinline__ float operator()(float z) const { return z < from ? from : z; }
};
template <bool EXACT> struct Silu {
  __device__ __forceinline__ float operator()(float z) const { return z * sigmoid<EXACT>(z); }
  __device__ __forceinline__ float slope(float z) const {
    const float s = sigmoid<EXACT>(z);
    return s * (1.f + z * (1.f - s));
  }
};
struct Gelu {
  __device__ __forceinline__ float operator()(float z) const {
    float cdf, pdf;
    cdf_pdf(z, cdf, pdf);
    return z * cdf;
  }
  __device__ __forceinline__ float slope(float z) const {
    float cdf, pdf;
    cdf_pdf(z, cdf, pdf);
    return cdf + z * pdf;
  }
};
// KIND: 0 straight ones (none, ReLU), 1 curved ones (SiLU, GELU), -1 any
template <bool EXACT, int KIND, class F> __device__ __forceinline__ void with_activation(int act, F f) {
  if (KIND != 0 && act == PPLL_ACT_SILU) f(Silu<EXACT>());
  else if (KIND != 0 && (KIND == 1 || act == PPLL_ACT_GELU)) f(Gelu());
  else f(Clamp{act == PPLL_ACT_RELU ? 0.f : -INFINITY});
}

// Sums of NV values over all threads of a piece column; every thread has its column's.  room: NV floats a thread
template <int NV> __device__ __forceinline__ void column_sums(float (&v)[NV], const NormArgs& p, float* room) {
  const int t = threadIdx.x, T = blockDim.x, width = p.npc * NV;
  const bool live = t < p.rt * p.npc;
  if (p.pow2) {
    // lanes of one column lie npc apart; the far ones first, so that a rotation of 16 lanes brings what the lane across has (see lanes_reduce)
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (p.npc <= 32) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v[i]), __float_as_uint(v[i]), false, false);
        v[i] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
      }
      if (p.npc <= 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v[i]), __float_as_uint(v[i]), false, false);
        v[i] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
      }
      if (p.npc <= 8) v[i] += dpp_f<0x128>(v[i]);
      if (p.npc <= 4) v[i] += dpp_f<0x124>(v[i]);
      if (p.npc <= 2) v[i] += dpp_f<0x122>(v[i]);
      if (p.npc <= 1) v[i] += dpp_f<0x121>(v[i]);
    }
    if (T == 64) return;
    const int lane = t & 63, col = lane & (p.npc - 1);
    __syncthreads();
    if (lane < p.npc)
#pragma unroll
      for (int i = 0; i < NV; ++i) room[(t >> 6) * width + i * p.npc + lane] = v[i];
    __syncthreads();
    for (int j = t; j < width; j += T) {
      float s = room[j];
      for (int w = 1; w < T / 64; ++w) s += room[w * width + j];
      room[j] = s;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] = room[i * p.npc + col];
    return;
  }
  const int row = quotient(t, p.over_npc), col = t - row * p.npc;
  float* mine = room + row * width + col;
  __syncthreads();
  if (live)
#pragma unroll
    for (int i = 0; i < NV; ++i) mine[i * p.npc] = v[i];
  __syncthreads();
  for (int n = p.rt; n > 1;) {
    const int h = (n + 1) / 2;
    if (live && row < n - h)
#pragma unroll
      for (int i = 0; i < NV; ++i) mine[i * p.npc] += mine[h * width + i * p.npc];
    __syncthreads();
    n = h;
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) v[i] = live ? room[i * p.npc + col] : 0.f;
}
// Sums of `sets` runs of n neighbouring floats in LDS: at(k) the first of run k, put(k, sum) by one lane.  A lane a short run, 16 one of
// some length, 64 a long one.
template <class AT, class PUT> __device__ __forceinline__ void runs_sums(int sets, int n, AT at, PUT put) {
  const int log = n <= 4 ? 0 : n <= 64 ? 4 : 6, lane = threadIdx.x & ((1 << log) - 1);
#pragma unroll 1
  for (int k = threadIdx.x >> log; k < sets; k += blockDim.x >> log) {
    const float* from = at(k);
    float s = 0.f;
#pragma unroll 1
    for (int i = lane; i < n; i += 1 << log) s += from[i];
    if (log) s = log == 4 ? lanes_sum<16>(s) : lanes_sum<64>(s);
    if (lane == 0) put(k, s);
  }
}
// Of GV segments of a thread's piece (their column sums) the sums of their groups.  room: npc GV floats and one a group.  (A thread by itself, going
// through all segments of its groups, took two thirds of the time of wide groups: 20 x 165 x 317, one group, 67 us, so 29; 28 x 96 x 496, four groups, 51 and 15.)
template <int GV> __device__ __forceinline__ void group_sums(float (&v)[GV], const NormArgs& p, float* room) {
  if (p.spg == 1) return;
  const int col = (int)threadIdx.x - quotient(threadIdx.x, p.over_npc) * p.npc, groups = quotient(p.slab, p.over_cg);
  float* sums = room + p.npc * GV;
  __syncthreads();
  if ((int)threadIdx.x < p.npc)
#pragma unroll
    for (int i = 0; i < GV; ++i) room[col * GV + i] = v[i];
  __syncthreads();
  runs_sums(groups, p.spg, [&](int g) { return room + g * p.spg; }, [&](int g, float s) { sums[g] = s; });
  __syncthreads();
#pragma unroll
  for (int i = 0; i < GV; ++i) v[i] = sums[min(quotient(col * GV + i, p.over_spg), groups - 1)];      // (behind the last channel: any)
}

// A unit of work: an image's slab, or its piece of pixels
struct Unit { int image, slab, part, first, last; };
__device__ __forceinline__ Unit unit_of(const NormArgs& p, int u) {
  Unit w;
  if (p.slabs > 1) {       // an image's slabs share the lines of its pixels: to one XCD (workgroup id % 8).  (The last images may not be there.)
    const int eight = u / (8 * p.slabs), rest = u - eight * 8 * p.slabs;
    w.image = eight * 8 + (rest & 7);
    w.slab = rest >> 3;
    w.part = w.first = 0;
    w.last = p.pixels;
    return w;
  }
  w.slab = 0;
  w.image = u / p.chunks;
  w.part = u - w.image * p.chunks;
  w.first = w.part * p.chunk;
  w.last = min(p.pixels, w.first + p.chunk);
  return w;
}

// A thread's pieces of a map: piece i is pixel `first` + row + i rt of an image.  The address is a uniform one and 32 bits a thread (rows lie
// 2^20 elements apart at most, and a workgroup has 512 of them).  VEC: channels come in eights, so every piece is whole.
template <int DT, bool VEC> struct Map {
  static constexpr int ESZ = DT == BF16 ? 2 : 4;
  char* base;
  int64_t step;
  uint32_t at;
  int c, cols;
  __device__ __forceinline__ void init(const void* p, int64_t ld, int64_t pixel, int c0, int row, int c_, int cols_, int rt) {
    base = (char*)p + (pixel * ld + c0) * ESZ;
    step = rt * ld * ESZ;
    c = c_; cols = cols_;
    at = ((uint32_t)row * (uint32_t)ld + (VEC ? c : 0)) * ESZ;
  }
  __device__ __forceinline__ void load(Eight<DT>& x, int i) const {
    if (VEC) x.load_all(base + i * step + at);
    else x.load(base + i * step + at, c, cols);
  }
  __device__ __forceinline__ void store(const Eight<DT>& x, int i) const {
    if (VEC) x.store_all(base + i * step + at);
    else x.store(base + i * step + at, c, cols);
  }
};

// How the work is laid out: an image (slab) a workgroup where its pieces find room in the registers of one, else pieces of pixels: `chunk` of them
// where they are held (the forward's statistics), `stretch` where they pass by
struct Layout { int slab, threads, mi, chunk, stretch; bool whole; };
constexpr int MOST_THREADS = 512;
constexpr int PART_MI = 4;       // 80 registers a thread: three workgroups a unit (8 pieces take 130 and leave one: 16 x 96 x 96 x 256 55 us)
inline int most_mi(int dt) { return dt == BF16 ? 8 : 4; }
inline int piece_columns(int channels) { return (channels + 7) / 8; }
inline void set_slab(const GroupNorm& g, Layout& l, int slab) {
  const int npc = piece_columns(slab);
  const int64_t pieces = (int64_t)g.pixels * npc;
  l.slab = slab;
  l.threads = 64;
  while (l.threads < MOST_THREADS && (l.threads < npc || 2 * pieces > most_mi(g.dt) * (int64_t)l.threads)) l.threads *= 2;
  const int rt = l.threads / npc;
  l.mi = (int)(((int64_t)g.pixels + rt - 1) / rt);
}
inline Layout layout_of(const GroupNorm& g) {
  Layout l{};
  const int size = g.dt == BF16 ? 2 : 4;
  l.chunk = l.stretch = g.pixels;
  // slabs of whole groups whose rows of a pixel are whole pieces and 64 bytes or more, 32 in a map that stays in the L2s; the widest that fits
  // (bf16, forward and backward, in slabs of 32 bytes / in pieces of pixels: 10 x 756 x 384 16, 22 / 25, 38 us; 128 x 1600 x 256 100, 167 / 80, 173)
  const int least = (int64_t)g.images * g.pixels * g.channels * size <= 16 << 20 ? 32 : 64;
  for (int n = 1; n <= g.groups && !l.whole; ++n) {
    if (g.groups % n) continue;
    const int slab = g.channels / n;
    if (n > 1 && (slab % 8 || slab * size < least)) continue;
    if (g.pixels <= (int64_t)(MOST_THREADS / piece_columns(slab)) * most_mi(g.dt)) { l.whole = true; set_slab(g, l, slab); }
  }
  if (!l.whole) {
    l.slab = g.channels;
    l.threads = MOST_THREADS;
    const int rt = l.threads / piece_columns(l.slab);
    l.mi = PART_MI;
    l.chunk = rt * l.mi;
    // a round of workgroups, two a unit (16 x 96 x 96 x 256 backward: 97 us, 113 in some 1152 workgroups)
    const int64_t per_image = std::max<int64_t>(1, 512 / g.images), even = ((int64_t)g.pixels + per_image - 1) / per_image;
    l.stretch = (int)((even + rt - 1) / rt) * rt;
  }
  return l;
}
inline int chunks_of(const GroupNorm& g, int chunk) { return (int)(((int64_t)g.pixels + chunk - 1) / chunk); }

inline int units_of(const NormArgs& p) { return p.slabs > 1 ? (p.images + 7) / 8 * 8 * p.slabs : p.images * p.chunks; }
// Few images: narrower slabs, down to a piece a pixel, until every unit has one
inline void spread_over_units(const GroupNorm& g, Layout& l) {
  if (!l.whole) return;
  for (int n = g.channels / l.slab + 1; n <= g.groups && (int64_t)g.images * (g.channels / l.slab) < 256; ++n)
    if (g.groups % n == 0 && g.channels / n % 8 == 0) set_slab(g, l, g.channels / n);
}

inline NormArgs args_of(const GroupNorm& g, const Layout& l, int chunk) {
  NormArgs p{};
  p.images = g.images; p.pixels = g.pixels; p.C = g.channels; p.groups = g.groups; p.cg = g.channels / g.groups; p.act = g.activation; p.eps = g.eps;
  p.slab = l.slab; p.slabs = g.channels / l.slab; p.npc = piece_columns(l.slab); p.rt = l.threads / p.npc;
  p.pow2 = p.npc <= 64 && (p.npc & (p.npc - 1)) == 0;
  p.chunk = chunk; p.chunks = chunks_of(g, chunk);
  p.units = units_of(p);
  p.over_cg = 1.f / (float)p.cg; p.over_npc = 1.f / (float)p.npc;
  return p;
}
inline int segments_of(int cg) { return cg % 8 == 0 ? 1 : cg % 4 == 0 ? 2 : cg % 2 == 0 ? 4 : 8; }
inline unsigned grid_of(const NormArgs& p) { return (unsigned)std::min(p.units, (int)MOST_BLOCKS); }

}  // namespace norm
}  // namespace ppll
