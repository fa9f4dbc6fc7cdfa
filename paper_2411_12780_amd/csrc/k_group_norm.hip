// Group norm with an activation over channels-last maps, forward and backward.
//
// A thread holds pieces of 8 channels of every RT-th pixel in registers, so that an image (or a slab of its channels, whole groups) that fits the
// registers of a workgroup is read once and written once: mean, then the squares about it, then the result; backward likewise.  A larger image goes in
// pieces of pixels through two launches: statistics of each piece (mean and squares about it, joined exactly) or channel sums, then the result, the map
// read a second time, from the last-level cache where it fits.  What bounds it: memory.
#include <algorithm>

#include "bytes.h"

namespace ppll {

namespace {
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
  int images, pixels, C, groups, cg, act;
  int slab, slabs, npc, rt, pow2;  // channels of a slab; npc: piece columns, pow2: a power of two up to 64
  int chunk, chunks;               // pixels of a piece, pieces of an image
  int spg;                         // segments of a group
  float eps;
};

template <bool EXACT> __device__ __forceinline__ float sigmoid(float z) {
  return __builtin_amdgcn_rcpf(1.f + (EXACT ? expf(-z) : __expf(-z)));
}
template <bool EXACT> __device__ __forceinline__ float activated(int act, float z) {
  if (act == PPLL_ACT_RELU) return z < 0.f ? 0.f : z;       // (a NaN stays one)
  if (act == PPLL_ACT_SILU) return z * sigmoid<EXACT>(z);
  if (act == PPLL_ACT_GELU) {
    float cdf, pdf;
    cdf_pdf(z, cdf, pdf);
    return z * cdf;
  }
  return z;
}
template <bool EXACT> __device__ __forceinline__ float slope_of(int act, float z) {
  if (act == PPLL_ACT_SILU) {
    const float s = sigmoid<EXACT>(z);
    return s * (1.f + z * (1.f - s));
  }
  float cdf, pdf;
  cdf_pdf(z, cdf, pdf);
  return cdf + z * pdf;
}

// Sums of NV values over all threads of a piece column; every thread has its column's.  room: NV floats a thread
template <int NV> __device__ __forceinline__ void column_sums(float (&v)[NV], const NormArgs& p, float* room) {
  const int t = threadIdx.x, T = blockDim.x;
  const bool live = t < p.rt * p.npc;
  if (p.pow2) {       // lanes of one column lie npc apart
    for (int s = p.npc; s < 64; s <<= 1)
#pragma unroll
      for (int i = 0; i < NV; ++i) v[i] += __shfl_xor(v[i], s);
    if (T > 64) {
      const int lane = t & 63, width = p.npc * NV;
      __syncthreads();
      if (lane < p.npc)
#pragma unroll
        for (int i = 0; i < NV; ++i) room[(t >> 6) * width + lane * NV + i] = v[i];
      __syncthreads();
#pragma unroll
      for (int i = 0; i < NV; ++i) v[i] = 0.f;
      for (int w = 0; w < T / 64; ++w)
#pragma unroll
        for (int i = 0; i < NV; ++i) v[i] += room[w * width + (lane & (p.npc - 1)) * NV + i];
    }
    return;
  }
  const int row = t / p.npc, at = t * NV;     // (thread t is row t / npc, column t % npc)
  __syncthreads();
  if (live)
#pragma unroll
    for (int i = 0; i < NV; ++i) room[at + i] = v[i];
  __syncthreads();
  for (int n = p.rt; n > 1;) {
    const int h = (n + 1) / 2;
    if (live && row < n - h)
#pragma unroll
      for (int i = 0; i < NV; ++i) room[at + i] += room[at + h * p.npc * NV + i];
    __syncthreads();
    n = h;
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) v[i] = live ? room[(t % p.npc) * NV + i] : 0.f;
}
// Of GV segments of a thread's piece (their column sums) the sums of their groups.  room: npc GV floats
template <int GV> __device__ __forceinline__ void group_sums(float (&v)[GV], const NormArgs& p, float* room) {
  if (p.spg == 1) return;
  const int col = threadIdx.x % p.npc;
  __syncthreads();
  if ((int)threadIdx.x < p.npc)
#pragma unroll
    for (int i = 0; i < GV; ++i) room[col * GV + i] = v[i];
  __syncthreads();
  const int segments = p.slab / p.cg * p.spg;
#pragma unroll
  for (int i = 0; i < GV; ++i) {
    const int seg = col * GV + i, g0 = seg / p.spg * p.spg;
    float s = 0.f;
    if (seg < segments)
      for (int k = 0; k < p.spg; ++k) s += room[g0 + k];
    v[i] = s;
  }
}

// A unit of work: an image's slab, or its piece of pixels
struct Unit { int image, slab, part, first, last; };
__device__ __forceinline__ Unit unit_of(const NormArgs& p, int u) {
  Unit w;
  const int per = p.slabs * p.chunks;
  w.image = u / per;
  const int rest = u - w.image * per;
  w.slab = rest / p.chunks;
  w.part = rest - w.slab * p.chunks;
  w.first = w.part * p.chunk;
  w.last = min(p.pixels, w.first + p.chunk);
  return w;
}

// Statistics of an image's group joined from those of its pieces [images][chunks][groups][2] (mean, squares about it): the piece means' own spread
// counts as well
__device__ __forceinline__ void join_parts(const NormArgs& p, int image, int g, float& mean, float& rstd) {
  const float* at = p.parts + ((int64_t)image * p.chunks * p.groups + g) * 2;
  float n = 0.f, m = 0.f, s = 0.f;
  for (int k = 0; k < p.chunks; ++k, at += 2 * p.groups) {
    const float nk = (float)((int64_t)(min(p.pixels, (k + 1) * p.chunk) - k * p.chunk) * p.cg), d = at[0] - m;
    n += nk;
    m += d * (nk / n);
    s += at[1] + d * d * (nk / n) * (n - nk);
  }
  mean = m;
  rstd = rsqrtf(s / n + p.eps);
}

// GV: segments of a piece, each of one group (8 / GV channels); MI: pieces a thread holds
template <int DT, int MODE, int GV, int MI>
__global__ __launch_bounds__(512) void group_norm_fwd_kernel(NormArgs p) {
  constexpr int ESZ = DT == BF16 ? 2 : 4, PER = 8 / GV;
  constexpr bool EXACT = DT == F32;
  extern __shared__ float room[];
  const int t = threadIdx.x, col = t % p.npc, row = t / p.npc;
  const bool live = row < p.rt;
  const int units = p.images * p.slabs * p.chunks;
  for (int u = blockIdx.x; u < units; u += gridDim.x) {
    const Unit w = unit_of(p, u);
    const int c0 = w.slab * p.slab, c = col * 8, cols = p.slab, g0 = c0 / p.cg;
    const int64_t at = (int64_t)w.image * p.pixels;
    Eight<DT> x[MI];
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      const int px = w.first + row + i * p.rt;
      if (live && px < w.last) x[i].load(p.x + ((at + px) * p.ldx + c0) * ESZ, c, cols);
      else x[i].zero();
    }
    float mean[GV], rstd[GV];
    if (MODE == APPLY) {
      // a group each, then to all
      __syncthreads();
      for (int g = t; g < p.groups; g += blockDim.x) {
        float m, r;
        join_parts(p, w.image, g, m, r);
        room[2 * g] = m; room[2 * g + 1] = r;
        if (p.stats && w.part == 0) {
          p.stats[((int64_t)w.image * p.groups + g) * 2] = m;
          p.stats[((int64_t)w.image * p.groups + g) * 2 + 1] = r;
        }
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < GV; ++i) {
        const int g = min((c + i * PER) / p.cg, p.groups - 1);
        mean[i] = room[2 * g]; rstd[i] = room[2 * g + 1];
      }
    } else {
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
        const int px = w.first + row + i * p.rt;
        if (!live || px >= w.last) continue;
        float v[8];
        x[i].get(v);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float d = v[e] - mean[e / PER];
          rstd[e / PER] += c + e < cols ? d * d : 0.f;
        }
      }
      column_sums<GV>(rstd, p, room);
      group_sums<GV>(rstd, p, room);
      const bool first = row == 0;
#pragma unroll
      for (int i = 0; i < GV; ++i) {
        const int g = g0 + (c + i * PER) / p.cg;
        const bool tells = first && c + i * PER < cols && (c + i * PER) % p.cg == 0;
        if (MODE == PART) {
          if (tells) {
            float* to = p.parts + (((int64_t)w.image * p.chunks + w.part) * p.groups + g) * 2;
            to[0] = mean[i]; to[1] = rstd[i];
          }
        } else {
          rstd[i] = rsqrtf(rstd[i] / count + p.eps);
          if (tells && p.stats) {
            float* to = p.stats + ((int64_t)w.image * p.groups + g) * 2;
            to[0] = mean[i]; to[1] = rstd[i];
          }
        }
      }
    }
    if (MODE == PART) continue;
    float a[8], b[8];       // y = act(a x + b): a = scale rstd; written as a (x - mean) + shift
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const bool in = c + e < cols;
      a[e] = in ? p.scale[c0 + c + e] * rstd[e / PER] : 0.f;
      b[e] = in ? p.shift[c0 + c + e] : 0.f;
    }
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      const int px = w.first + row + i * p.rt;
      const bool in = live && px < w.last;
      float v[8];
      x[i].get(v);
      if (p.keep) {       // (the lanes of a pixel are a power of two of one wave)
        uint32_t most = most_of(v, 0);
        for (int s = 1; s < p.npc; s <<= 1) most = max(most, (uint32_t)__shfl_xor((int)most, s));
        const int e = byte_exponent(most);
        if (in) {
          const bool nan = e == BYTE_NAN;
          if (col == 0) p.keep_e[at + px] = (int8_t)e;
          int8_t* to = p.keep + (at + px) * p.ldk + c;
          *(uint2*)to = nan ? make_uint2(0, 0) : bytes_of(v, exp2_bits(nan ? 0 : -e));
          if (c + 8 >= cols && !(p.npc & 1)) continue;
          if (c + 8 >= cols) *(uint2*)(to + 8) = make_uint2(0, 0);      // an odd number of pieces: the padding
        }
      }
    }
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      const int px = w.first + row + i * p.rt;
      if (!live || px >= w.last) continue;
      float v[8];
      x[i].get(v);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = (v[e] - mean[e / PER]) * a[e] + b[e];
      if (p.residual) {
        Eight<DT> r;
        float f[8];
        r.load(p.residual + ((at + px) * p.ldr + c0) * ESZ, c, cols);
        r.get(f);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += f[e];
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = activated<EXACT>(p.act, v[e]);
      Eight<DT> o;
      o.set(v);
      o.store(p.y + ((at + px) * p.ldy + c0) * ESZ, c, cols);
    }
  }
}

// The backward's pieces: x (from its type or from 8 bits) and dz
template <int DT, bool BYTES> struct XPiece;
template <int DT> struct XPiece<DT, false> {
  Eight<DT> x;
  __device__ __forceinline__ void load(const NormArgs& p, int64_t pixel, int c0, int c, int cols) {
    x.load(p.x + (pixel * p.ldx + c0) * (DT == BF16 ? 2 : 4), c, cols);
  }
  __device__ __forceinline__ void zero() { x.zero(); }
  __device__ __forceinline__ void get(float (&v)[8]) const { x.get(v); }
};
template <int DT> struct XPiece<DT, true> {
  uint2 w;
  int e;
  __device__ __forceinline__ void load(const NormArgs& p, int64_t pixel, int c0, int c, int) {
    const int8_t* at = p.q + pixel * p.ldq + c0 + c;
    __builtin_memcpy(&w, at, 8);           // (a slab may begin off 8 bytes only where it is the whole row)
    e = p.qe[pixel];
  }
  __device__ __forceinline__ void zero() { w = make_uint2(0, 0); e = 0; }
  __device__ __forceinline__ void get(float (&v)[8]) const { bytes_get(w, byte_step(e), v); }
};

// PART: channel sums of a piece, [images][chunks][2][C]; APPLY: from the image's channel sums in p.sums
template <int DT, int MODE, bool BYTES, int MI>
__global__ __launch_bounds__(512) void group_norm_bwd_kernel(NormArgs p) {
  constexpr int ESZ = DT == BF16 ? 2 : 4;
  constexpr bool EXACT = DT == F32;
  extern __shared__ float room[];
  const int t = threadIdx.x, col = t % p.npc, row = t / p.npc;
  const bool live = row < p.rt;
  const int units = p.images * p.slabs * p.chunks;
  for (int u = blockIdx.x; u < units; u += gridDim.x) {
    const Unit w = unit_of(p, u);
    const int c0 = w.slab * p.slab, c = col * 8, cols = p.slab, g0 = c0 / p.cg;
    const int64_t at = (int64_t)w.image * p.pixels;
    float mean[8], rstd[8], scale[8], shift[8];
    XPiece<DT, BYTES> x[MI];
    Eight<DT> dz[MI];
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      const int px = w.first + row + i * p.rt;
      x[i].zero();
      dz[i].zero();
      if (live && px < w.last) {
        x[i].load(p, at + px, c0, c, cols);
        dz[i].load(p.dy + ((at + px) * p.ldd + c0) * ESZ, c, cols);
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const bool in = c + e < cols;
      const float* st = p.stats_in + ((int64_t)w.image * p.groups + g0 + (in ? (c + e) / p.cg : 0)) * 2;
      mean[e] = st[0]; rstd[e] = st[1];
      scale[e] = in ? p.scale[c0 + c + e] : 0.f;
      shift[e] = in ? p.shift[c0 + c + e] : 0.f;
    }
    float sums[16];       // of dz, of dz xhat, for each channel
#pragma unroll
    for (int e = 0; e < 16; ++e) sums[e] = 0.f;
    auto xhat = [&](int i, float (&v)[8]) {
      x[i].get(v);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = (v[e] - mean[e]) * rstd[e];
    };
    // dz = dy times the slope
    float z[8], h[8];
    auto gradient = [&](int i, int px, const float (&xh)[8], float (&d)[8]) {
      dz[i].get(d);
      if (p.act == PPLL_ACT_RELU) {
        Eight<DT> y;
        y.load(p.y_in + ((at + px) * p.ldy + c0) * ESZ, c, cols);
        y.get(z);
#pragma unroll
        for (int e = 0; e < 8; ++e) d[e] = z[e] > 0.f ? d[e] : 0.f;
      } else if (p.act != PPLL_ACT_NONE) {
        Eight<DT> r;
        r.zero();
        if (p.residual) r.load(p.residual + ((at + px) * p.ldr + c0) * ESZ, c, cols);
        r.get(z);
#pragma unroll
        for (int e = 0; e < 8; ++e) d[e] *= slope_of<EXACT>(p.act, xh[e] * scale[e] + shift[e] + z[e]);
      }
    };
    float d[8];
    if (MODE != APPLY) {
#pragma unroll
      for (int i = 0; i < MI; ++i) {
        const int px = w.first + row + i * p.rt;
        if (!live || px >= w.last) continue;
        xhat(i, h);
        gradient(i, px, h, d);
#pragma unroll
        for (int e = 0; e < 8; ++e) { sums[e] += d[e]; sums[8 + e] += d[e] * h[e]; }
      }
      column_sums<16>(sums, p, room);
      if (row == 0) {
        float* to = MODE == PART ? p.parts + ((int64_t)w.image * p.chunks + w.part) * 2 * p.C : p.sums + (int64_t)w.image * 2 * p.C;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (c + e < cols) { to[c0 + c + e] = sums[e]; to[p.C + c0 + c + e] = sums[8 + e]; }
      }
    }
    if (MODE == PART) continue;
    // the groups' means of g = dz scale and g xhat, from the channel sums
    float ga[8], gb[8];
    {
      float* chan = room;       // [2][slab]
      __syncthreads();
      if (MODE == WHOLE) {
        if (row == 0)
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (c + e < cols) { chan[c + e] = sums[e] * scale[e]; chan[cols + c + e] = sums[8 + e] * scale[e]; }
      } else {
        const float* from = p.sums + (int64_t)w.image * 2 * p.C;
        for (int k = t; k < p.C; k += blockDim.x) { chan[k] = from[k] * p.scale[k]; chan[cols + k] = from[p.C + k] * p.scale[k]; }
      }
      __syncthreads();
      float* group = room + 2 * cols;
      const float over = 1.f / (float)((int64_t)p.pixels * p.cg);
      for (int k = t; k < 2 * (cols / p.cg); k += blockDim.x) {
        float s = 0.f;
        const float* from = chan + (k & 1) * cols + (k >> 1) * p.cg;
        for (int j = 0; j < p.cg; ++j) s += from[j];
        group[k] = s * over;
      }
      __syncthreads();
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int g = c + e < cols ? (c + e) / p.cg : 0;
        ga[e] = group[2 * g]; gb[e] = group[2 * g + 1];
      }
      __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      const int px = w.first + row + i * p.rt;
      if (!live || px >= w.last) continue;
      xhat(i, h);
      gradient(i, px, h, d);
      Eight<DT> o;
      if (p.dres) {
        o.set(d);
        o.store(p.dres + ((at + px) * p.lddr + c0) * ESZ, c, cols);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) d[e] = rstd[e] * (d[e] * scale[e] - ga[e] - h[e] * gb[e]);
      o.set(d);
      o.store(p.dx + ((at + px) * p.lddx + c0) * ESZ, c, cols);
    }
  }
}

// Sums over the first axis of [n][outer stride], in its order: a workgroup 16 columns of one of `sets` stretches, 64 rows at a time
__global__ __launch_bounds__(1024) void group_norm_sum_kernel(const float* in, int n, int64_t stride, int64_t set_stride, int cols, float* out, int64_t out_set,
                                                              float* first, float* second, int split) {
  __shared__ float part[64][17];
  const int c = blockIdx.x * 16 + (threadIdx.x & 15), r = threadIdx.x >> 4;
  for (int64_t set = blockIdx.y; set < (first ? 1 : (int64_t)split); set += gridDim.y) {
    const float* from = in + set * set_stride;
    float s = 0.f;
    if (c < cols)
#pragma unroll 4
      for (int64_t k = r; k < n; k += 64) s += from[k * stride + c];
    __syncthreads();
    part[r][threadIdx.x & 15] = s;
    __syncthreads();
    if (r == 0 && c < cols) {
      s = 0.f;
      for (int k = 0; k < 64; ++k) s += part[k][threadIdx.x];
      if (!first) out[set * out_set + c] = s;
      else if (c < split) second[c] = s;       // sums of dz, then of dz xhat
      else first[c - split] = s;
    }
  }
}
__global__ __launch_bounds__(256) void group_norm_zero_kernel(float* a, float* b, int n) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i < n) a[i] = b[i] = 0.f;
}

// How the work is laid out: an image (slab) a workgroup where its pieces find room in the registers of one, else pieces of pixels
struct Layout { int slab, threads, mi, chunk; bool whole; };
constexpr int MOST_MI = 8, MOST_THREADS = 512;
int piece_columns(int channels) { return (channels + 7) / 8; }
bool slab_fits(int64_t pixels, int slab) {
  const int rt = MOST_THREADS / piece_columns(slab);
  return rt > 0 && pixels <= (int64_t)rt * MOST_MI;
}
Layout layout_of(const GroupNorm& g) {
  Layout l{};
  const int cg = g.channels / g.groups;
  // slabs of whole groups whose rows of a pixel are whole pieces and 64 bytes or more; the widest that fits
  for (int n = 1; n <= g.groups && !l.whole; ++n) {
    if (g.groups % n) continue;
    const int slab = g.channels / n;
    if (n > 1 && (slab % 8 || slab * (g.dt == BF16 ? 2 : 4) < 64)) break;
    if (slab_fits(g.pixels, slab)) { l.whole = true; l.slab = slab; }
  }
  (void)cg;
  if (!l.whole) l.slab = g.channels;
  const int npc = piece_columns(l.slab);
  const int64_t pieces = (int64_t)g.pixels * npc;
  l.threads = 64;
  if (l.whole) {
    while (l.threads < MOST_THREADS && (l.threads < npc || pieces > 4 * (int64_t)l.threads)) l.threads *= 2;
    const int rt = l.threads / npc;
    l.mi = (int)(((int64_t)g.pixels + rt - 1) / rt);
    l.chunk = g.pixels;
  } else {
    l.threads = npc > 256 ? 512 : 256;
    const int rt = l.threads / npc;
    l.mi = MOST_MI;
    l.chunk = rt * MOST_MI;
  }
  return l;
}
int chunks_of(const GroupNorm& g, const Layout& l) { return (int)(((int64_t)g.pixels + l.chunk - 1) / l.chunk); }

NormArgs args_of(const GroupNorm& g, const Layout& l) {
  NormArgs p{};
  p.images = g.images; p.pixels = g.pixels; p.C = g.channels; p.groups = g.groups; p.cg = g.channels / g.groups; p.act = g.activation; p.eps = g.eps;
  p.slab = l.slab; p.slabs = g.channels / l.slab; p.npc = piece_columns(l.slab); p.rt = l.threads / p.npc;
  p.pow2 = p.npc <= 64 && (p.npc & (p.npc - 1)) == 0;
  p.chunk = l.chunk; p.chunks = chunks_of(g, l);
  return p;
}
int segments_of(int cg) { return cg % 8 == 0 ? 1 : cg == 4 ? 2 : cg == 2 ? 4 : 8; }
unsigned grid_of(const NormArgs& p) { return (unsigned)std::min<int64_t>((int64_t)p.images * p.slabs * p.chunks, MOST_BLOCKS); }

template <int DT, int MODE, int GV> int fwd_launch(hipStream_t s, const NormArgs& p, const Layout& l) {
  const size_t lds = sizeof(float) * (size_t)std::max(std::max(l.threads * GV, p.npc * GV), MODE == APPLY ? 2 * p.groups : 0);
  const dim3 grid(grid_of(p)), block(l.threads);
  if (l.mi <= 1) hipLaunchKernelGGL((group_norm_fwd_kernel<DT, MODE, GV, 1>), grid, block, lds, s, p);
  else if (l.mi <= 2) hipLaunchKernelGGL((group_norm_fwd_kernel<DT, MODE, GV, 2>), grid, block, lds, s, p);
  else if (l.mi <= 4) hipLaunchKernelGGL((group_norm_fwd_kernel<DT, MODE, GV, 4>), grid, block, lds, s, p);
  else hipLaunchKernelGGL((group_norm_fwd_kernel<DT, MODE, GV, MOST_MI>), grid, block, lds, s, p);
  PPLL_HIP(hipGetLastError());
  return PPLL_OK;
}
template <int DT, int MODE> int fwd(hipStream_t s, NormArgs& p, const Layout& l) {
  const int gv = segments_of(p.cg);
  p.spg = p.cg * gv / 8;
  if (gv == 1) return fwd_launch<DT, MODE, 1>(s, p, l);
  if (gv == 2) return fwd_launch<DT, MODE, 2>(s, p, l);
  if (gv == 4) return fwd_launch<DT, MODE, 4>(s, p, l);
  return fwd_launch<DT, MODE, 8>(s, p, l);
}
template <int DT, int MODE, bool BYTES> int bwd(hipStream_t s, const NormArgs& p, const Layout& l) {
  static OncePerDevice once[4];
  const size_t need = (size_t)std::max(l.threads * 16, 2 * p.slab + 2 * (p.slab / p.cg)) * sizeof(float);
  constexpr int MOST_LDS = 4 * 4096 * (int)sizeof(float);      // 2 slab + 2 groups of up to 4096 channels
  const dim3 grid(grid_of(p)), block(l.threads);
  auto go = [&](auto kernel, OncePerDevice& o) -> int {
    if (need > 64 * 1024) PPLL_TRY(raise_lds((const void*)kernel, MOST_LDS, o));
    hipLaunchKernelGGL(kernel, grid, block, need, s, p);
    PPLL_HIP(hipGetLastError());
    return PPLL_OK;
  };
  if (l.mi <= 1) return go(group_norm_bwd_kernel<DT, MODE, BYTES, 1>, once[0]);
  if (l.mi <= 2) return go(group_norm_bwd_kernel<DT, MODE, BYTES, 2>, once[1]);
  if (l.mi <= 4) return go(group_norm_bwd_kernel<DT, MODE, BYTES, 4>, once[2]);
  return go(group_norm_bwd_kernel<DT, MODE, BYTES, MOST_MI>, once[3]);
}
template <int DT, bool BYTES> int bwd_all(hipStream_t s, const GroupNorm& g, NormArgs& p, const Layout& l, float* d_scale, float* d_shift, float* ws) {
  const int C = g.channels;
  p.sums = ws;
  if (l.whole) {
    PPLL_TRY((bwd<DT, WHOLE, BYTES>(s, p, l)));
  } else {
    p.parts = ws + (int64_t)g.images * 2 * C;
    PPLL_TRY((bwd<DT, PART, BYTES>(s, p, l)));
    // pieces into images
    hipLaunchKernelGGL(group_norm_sum_kernel, dim3((2 * C + 15) / 16, std::min(g.images, 65535)), dim3(1024), 0, s, p.parts, p.chunks, (int64_t)2 * C,
                       (int64_t)p.chunks * 2 * C, 2 * C, p.sums, (int64_t)2 * C, (float*)nullptr, (float*)nullptr, g.images);
    PPLL_HIP(hipGetLastError());
    PPLL_TRY((bwd<DT, APPLY, BYTES>(s, p, l)));
  }
  hipLaunchKernelGGL(group_norm_sum_kernel, dim3((2 * C + 15) / 16), dim3(1024), 0, s, p.sums, g.images, (int64_t)2 * C, (int64_t)0, 2 * C, (float*)nullptr,
                     (int64_t)0, d_scale, d_shift, C);
  PPLL_HIP(hipGetLastError());
  return PPLL_OK;
}
}  // namespace

size_t group_norm_workspace(const GroupNorm& g) {
  if (g.images <= 0) return 0;
  const Layout l = layout_of(g);
  const int64_t sums = (int64_t)g.images * 2 * g.channels, chunks = chunks_of(g, l);
  const int64_t bwd = l.whole ? sums : sums + chunks * sums, fwd = l.whole ? 0 : (int64_t)g.images * chunks * g.groups * 2;
  return (size_t)std::max(bwd, fwd) * sizeof(float);
}

int launch_group_norm_fwd(hipStream_t s, const GroupNorm& g, const ppll_rows& x, const float* scale, const float* shift, const ppll_rows& residual,
                          const ppll_rows& y, float* stats, const ppll_byte_rows& keep, char* ws) {
  if (g.images <= 0) return PPLL_OK;
  const Layout l = layout_of(g);
  NormArgs p = args_of(g, l);
  p.x = (const char*)x.p; p.ldx = x.ld; p.residual = (const char*)residual.p; p.ldr = residual.ld; p.y = (char*)y.p; p.ldy = y.ld;
  p.scale = scale; p.shift = shift; p.stats = stats; p.parts = (float*)ws;
  if (keep.q) {
    if (p.slabs == 1 && p.pow2) { p.keep = keep.q; p.keep_e = keep.e; p.ldk = keep.ld; }
    else PPLL_TRY(launch_byte_rows_pack(s, g.dt, g.images * g.pixels, g.channels, x, keep));      // (before y, which may be x)
  }
  if (l.whole) return g.dt == BF16 ? fwd<BF16, WHOLE>(s, p, l) : fwd<F32, WHOLE>(s, p, l);
  PPLL_TRY((g.dt == BF16 ? fwd<BF16, PART>(s, p, l) : fwd<F32, PART>(s, p, l)));
  return g.dt == BF16 ? fwd<BF16, APPLY>(s, p, l) : fwd<F32, APPLY>(s, p, l);
}

int launch_group_norm_bwd(hipStream_t s, const GroupNorm& g, const ppll_rows& x, const ppll_byte_rows& x8, const float* stats, const float* scale,
                          const float* shift, const ppll_rows& residual, const ppll_rows& y, const ppll_rows& dy, const ppll_rows& dx, const ppll_rows& dres,
                          float* d_scale, float* d_shift, char* ws) {
  if (g.images <= 0) {
    hipLaunchKernelGGL(group_norm_zero_kernel, dim3((g.channels + 255) / 256), dim3(256), 0, s, d_scale, d_shift, g.channels);
    PPLL_HIP(hipGetLastError());
    return PPLL_OK;
  }
  const Layout l = layout_of(g);
  NormArgs p = args_of(g, l);
  p.x = (const char*)x.p; p.ldx = x.ld; p.q = x8.q; p.qe = x8.e; p.ldq = x8.ld;
  p.residual = (const char*)residual.p; p.ldr = residual.ld; p.y_in = (const char*)y.p; p.ldy = y.ld; p.dy = (const char*)dy.p; p.ldd = dy.ld;
  p.dx = (char*)dx.p; p.lddx = dx.ld; p.dres = (char*)dres.p; p.lddr = dres.ld;
  p.stats_in = stats; p.scale = scale; p.shift = shift;
  const bool bytes = !p.x;
  if (g.dt == BF16) return bytes ? bwd_all<BF16, true>(s, g, p, l, d_scale, d_shift, (float*)ws) : bwd_all<BF16, false>(s, g, p, l, d_scale, d_shift, (float*)ws);
  return bytes ? bwd_all<F32, true>(s, g, p, l, d_scale, d_shift, (float*)ws) : bwd_all<F32, false>(s, g, p, l, d_scale, d_shift, (float*)ws);
}

}  // namespace ppll
