// Gradients of the linear layer on rows of 8 bits: dX = dY W and dW = X^T dY, the operand in 8 bits on its way to LDS made the bf16 values that it
// stands for (exactly: 7 significant bits and a power of two), then as a product in v_mfma_f32_32x32x16_bf16, fp32 sums.
//
// Both products run over the rows of the operand in 8 bits (output channels, tokens), whose other index is contiguous: it lies in LDS as in
// memory, [k][row], and fragments come out of transposing reads; so does dY in dW, while in dX its k is contiguous.  128 x 128 tiles of four
// waves, two stages of 64 k in LDS and two in registers.  dY in fp32 is three bf16 terms that add up to it exactly (8 bits each; under 2^-110 off by
// 2^-134 at most, half of bf16's least step), three products, stages of 32 k.  Operands of any alignment: 16-byte loads from where the elements lie;
// the last pieces of a ragged row are read ending at the row's end and shifted.
//
// What bounds it: no unit of the chip (8320 x 1536 x 384, both gradients and the sum of their parts 46 us, 426 TFLOP/s: matrix instructions run in 22 % of
// the kernel's clocks, LDS is at work in 26 %, without conflicts, vector instructions are issued in 36 %; a wave waits for data and barriers in 29 % of its time,
// for its turn in 32 %), but the order of a stage, load, conversion, LDS, barrier, fragments, products, with two waves a SIMD.
#include <algorithm>

#include "bytes.h"

namespace ppll {

namespace {
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

constexpr int BM = 128, BN = 128, THREADS = 256, PITCH = 320;      // PITCH: bytes between k rows of a [k][row] tile (free of bank conflicts)
constexpr int STAGE_LD = BN + 4;

struct GradArgs {
  const int8_t *q, *e; int64_t ldq; int qcols;       // operand in 8 bits: [K][qcols], qcols padded
  const char* d; int64_t ldd; int dcols;             // dY, elements: [M][K] (dX) or [K][N]
  char* out; int64_t ldo;                            // dX, or dW / its parts
  const char* gate; int64_t ldg;
  float* db;                                         // dW: column sums of dY (of a part), or null
  int M, N, K, tiles_m, tiles_n, per_xcd, parts, part_k;
  int64_t part_out;                                  // elements from part to part, and behind them of db
  bool sums;                                         // out takes sums in fp32: dW, parts
};

template <int DT> constexpr int terms() { return DT == F32 ? 3 : 1; }
template <int DT> constexpr int step_k() { return DT == F32 ? 32 : 64; }
// one term of the dY tile, the tile in 8 bits, a stage
template <bool DX, int DT> constexpr int d_bytes() { return DX ? BM * step_k<DT>() * 2 : step_k<DT>() * PITCH; }
template <int DT> constexpr int q_bytes() { return step_k<DT>() * PITCH; }
template <bool DX, int DT> constexpr int stage_bytes() { return q_bytes<DT>() + terms<DT>() * d_bytes<DX, DT>(); }
template <bool DX, int DT> constexpr int lds_bytes() { return std::max(2 * stage_bytes<DX, DT>(), BM * STAGE_LD * 4); }

template <int BK> __device__ __forceinline__ int row_major(int row, int granule) {
  return BK == 64 ? row * 128 + ((granule ^ ((row >> 1) & 7)) << 4) : row * 64 + ((granule ^ ((row >> 2) & 3)) << 4);
}
__device__ __forceinline__ uint2 lds_read_tr(const char* p) {
  const s16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p);
  return __builtin_bit_cast(uint2, v);
}
// The three terms of eight values, their 8 highest bits, the next 8 and the rest.  The first two are cut off, not rounded, so that no finite value
// becomes infinite; those behind an infinity are 0, behind a NaN (whose bits may be cut off in the first) NaN.
__device__ __forceinline__ void split(const Eight<F32>& x, uint4 (&t)[3]) {
  constexpr int INF = 0x204;      // of either sign
  float v[8];
  x.get(v);
  uint32_t w[3][4];
#pragma unroll
  for (int k = 0; k < 2; ++k)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t a = __float_as_uint(v[2 * i]), b = __float_as_uint(v[2 * i + 1]);
      w[k][i] = __builtin_amdgcn_perm(b, a, 0x07060302u);
      const bool a_inf = k == 0 && __builtin_amdgcn_classf(v[2 * i], INF), b_inf = k == 0 && __builtin_amdgcn_classf(v[2 * i + 1], INF);
      v[2 * i] = a_inf ? 0.f : v[2 * i] - __uint_as_float(a & 0xffff0000u);
      v[2 * i + 1] = b_inf ? 0.f : v[2 * i + 1] - __uint_as_float(b & 0xffff0000u);
    }
#pragma unroll
  for (int i = 0; i < 4; ++i) w[2][i] = f32x2_to_bf16x2(v[2 * i], v[2 * i + 1]);
#pragma unroll
  for (int k = 0; k < 3; ++k) t[k] = make_uint4(w[k][0], w[k][1], w[k][2], w[k][3]);
}
// Elements `by` .. 7 of eight to the front, zeros behind
__device__ __forceinline__ void shift_down(Eight<BF16>& x, int by) {
  const uint64_t lo = (uint64_t)x.w.x | (uint64_t)x.w.y << 32, hi = (uint64_t)x.w.z | (uint64_t)x.w.w << 32;
  const int bits = 16 * by, b = bits & 63;
  const uint64_t a = bits >= 64 ? hi : lo, c = bits >= 64 ? 0 : hi;
  const uint64_t l = b ? a >> b | c << (64 - b) : a, h = c >> b;
  x.w = make_uint4((uint32_t)l, (uint32_t)(l >> 32), (uint32_t)h, (uint32_t)(h >> 32));
}
__device__ __forceinline__ void shift_down(Eight<F32>& x, int by) {
  float v[8];
  x.get(v);
#pragma unroll
  for (int s = 4; s >= 1; s >>= 1)
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = by & s ? (i + s < 8 ? v[i + s] : 0.f) : v[i];
  x.set(v);
}
// Elements c .. c + 7 of a row of fewer than 8
template <int DT> __device__ __forceinline__ void load_few(Eight<DT>& x, const char* row, int c, int cols) {
  x.zero();
  if (c < cols) x.load(row, c, cols);
}

template <int DT> struct Regs {
  static constexpr int NP = step_k<DT>() / 16;
  uint2 q[NP];
  int e[NP];
  Eight<DT> d[NP];
};

// A tile (of a part of k): workgroup `group` of those of this product
template <bool DX, int DT, bool RAGGED> __device__ __forceinline__ void grad_tile(const GradArgs& p, int group) {
  constexpr int T = terms<DT>(), BK = step_k<DT>(), NP = BK / 16, ESZ = DT == BF16 ? 2 : 4;
  constexpr int QB = q_bytes<DT>(), DB = d_bytes<DX, DT>(), STAGE = stage_bytes<DX, DT>();
  extern __shared__ __align__(16) char smem[];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, wm = wave >> 1, wn = wave & 1;
  // XCD x (workgroup id % 8) takes a contiguous stretch: tiles of a row (of a part of k) share what they read in its L2
  const int tiles = p.tiles_m * p.tiles_n, u = (group & 7) * p.per_xcd + (group >> 3);
  if (u >= tiles * p.parts) return;
  const int part = u / tiles, t = u - part * tiles, m0 = t / p.tiles_n * BM, n0 = t % p.tiles_n * BN;
  const int kbeg = part * p.part_k, kend = min(p.K, kbeg + p.part_k), nk = (kend - kbeg + BK - 1) / BK;

  f32x16 acc[2][2];
#pragma unroll
  for (int a = 0; a < 2; ++a)
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[a][b][i] = 0.f;

  const int tk = tid >> 4, tc = (tid & 15) * 8;                                   // [k][row]: k rows tk + 16 j, columns tc ..
  const int rk = (tid & (BK / 8 - 1)) * 8, rr = tid / (BK / 8);                   // [row][k]: rows rr + 2048 / BK j, k rk ..
  constexpr int RSTEP = THREADS / (BK / 8);
  const int qc = min((DX ? n0 : m0) + tc, p.qcols - 8);
  // Stage i: k from kbeg + i BK (behind the last one: the last one again).  Addresses are a uniform one and 32 bits of the thread; in a last stage that
  // is cut short k rows stop at the last one, whose values are dropped on the way to LDS.
  const int last = nk - 1, left = kend - (kbeg + last * BK);
  const int d_col = DX ? 0 : n0 + tc, d_from = max(min(d_col, p.dcols - 8), 0);
  const bool few = RAGGED && p.dcols < 8;
  const uint32_t ldq = (uint32_t)p.ldq, ldd = (uint32_t)p.ldd * ESZ;               // below 2^24
  const char* d_base = DX ? p.d + (int64_t)m0 * p.ldd * ESZ : p.d;
  uint32_t d_row[DX ? NP : 1];
  if (DX) {
#pragma unroll
    for (int j = 0; j < NP; ++j) d_row[j] = (uint32_t)min(rr + RSTEP * j, p.M - 1 - m0) * ldd;
  }
  auto gload = [&](int i, Regs<DT>& r) {
    const int ic = min(i, last), k0 = kbeg + ic * BK, most = ic == last ? left - 1 : BK - 1;
    const int8_t *qb = p.q + (int64_t)k0 * p.ldq, *eb = p.e + k0;
    const char* db = p.d + (int64_t)k0 * p.ldd * ESZ;
    const uint32_t dk = (uint32_t)max(min(k0 + rk, p.dcols - 8), 0) * ESZ;
#pragma unroll
    for (int j = 0; j < NP; ++j) {
      const uint32_t k = (uint32_t)min(tk + 16 * j, most);
      r.q[j] = *(const uint2*)(qb + (__umul24(k, ldq) + qc));
      r.e[j] = eb[k];
      if (few) {
        if (DX) load_few<DT>(r.d[j], d_base + d_row[DX ? j : 0], k0 + rk, p.dcols);
        else load_few<DT>(r.d[j], db + __umul24(k, ldd), d_col, p.dcols);
      } else {
        r.d[j].load_all(DX ? d_base + (d_row[DX ? j : 0] + dk) : db + (__umul24(k, ldd) + d_from * ESZ));
      }
    }
  };
  // column sums of dY, by the workgroups of the first row of tiles, from the registers on their way
  const bool do_db = !DX && p.db && m0 == 0;
  float csum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  auto lstore = [&](int stage, int i, const Regs<DT>& r, int j) {
    if (j >= NP) return;
    char* st = smem + stage * STAGE;
    const int k0 = kbeg + i * BK;
    const bool cut = i == last && left < BK;
    float f[8];
    bytes_get(r.q[j], byte_step(r.e[j]), f);
    Eight<BF16> x;
    x.set(f);
    Eight<DT> d = r.d[j];
    if (cut) {
      if (k0 + tk + 16 * j >= kend) x.zero();
      if (DX ? k0 + rk >= kend : k0 + tk + 16 * j >= kend) d.zero();
    }
    // a piece that goes over its row's end was read ending there.  (One beyond the end keeps its last element, which no sum that is kept meets; in dX
    // it is zero already.)
    if (RAGGED && !few && (DX ? cut : n0 + BN > p.dcols)) {
      const int c = DX ? k0 + rk : d_col;
      shift_down(d, min(c - min(c, p.dcols - 8), 7));
    }
    *(u32x4*)(st + (tk + 16 * j) * PITCH + tc * 2) = (u32x4){x.w.x, x.w.y, x.w.z, x.w.w};
    if (do_db) {
      float v[8];
      d.get(v);
#pragma unroll
      for (int e = 0; e < 8; ++e) csum[e] += v[e];
    }
    char* to = st + QB + (DX ? row_major<BK>(rr, rk >> 3) + j * RSTEP * BK * 2 : (tk + 16 * j) * PITCH + tc * 2);
    if constexpr (DT == BF16) {
      *(u32x4*)to = (u32x4){d.w.x, d.w.y, d.w.z, d.w.w};
    } else {
      uint4 w[3];
      split(d, w);
#pragma unroll
      for (int s = 0; s < 3; ++s) *(u32x4*)(to + s * DB) = (u32x4){w[s].x, w[s].y, w[s].z, w[s].w};
    }
  };
  const int tr_lane = (8 * (lane >> 5) + ((lane & 15) >> 2)) * PITCH + (16 * ((lane >> 4) & 1) + 4 * (lane & 3)) * 2;
  auto frag_tr = [&](const char* tile, int row0, int kk) -> bf16x8 {
    const char* a = tile + tr_lane + kk * 16 * PITCH + row0 * 2;
    const uint2 lo = lds_read_tr(a), hi = lds_read_tr(a + 4 * PITCH);
    return __builtin_bit_cast(bf16x8, make_uint4(lo.x, lo.y, hi.x, hi.y));
  };
  auto frag_d = [&](const char* tile, int row0, int kk) -> bf16x8 {
    if (DX) return *reinterpret_cast<const bf16x8*>(tile + row_major<BK>(row0 + (lane & 31), kk * 2 + (lane >> 5)));
    return frag_tr(tile, row0, kk);
  };
  // wm: the wave's half of the rows of C, wn: of its columns
  const int q0 = DX ? wn * 64 : wm * 64, d0 = DX ? wm * 64 : wn * 64;
  bf16x8 fq[2][2], fd[2][2][T];
  auto load_frags = [&](int stage, int kk, int set) {
    const char* st = smem + stage * STAGE;
#pragma unroll
    for (int i = 0; i < 2; ++i) fq[set][i] = frag_tr(st, q0 + 32 * i, kk);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int s = 0; s < T; ++s) fd[set][i][s] = frag_d(st + QB + s * DB, d0 + 32 * i, kk);
  };
  auto multiply = [&](int stage, int i, const Regs<DT>& next, bool stage_next) {
#pragma unroll
    for (int kk = 0; kk < BK / 16; ++kk) {
      if (kk + 1 < BK / 16) load_frags(stage, kk + 1, (kk + 1) & 1);
#pragma unroll
      for (int s = T - 1; s >= 0; --s)       // the small terms first
#pragma unroll
        for (int jn = 0; jn < 2; ++jn)
#pragma unroll
          for (int im = 0; im < 2; ++im) {
            const bf16x8 b = DX ? fq[kk & 1][jn] : fd[kk & 1][jn][s], a = DX ? fd[kk & 1][im][s] : fq[kk & 1][im];
            acc[jn][im] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b, a, acc[jn][im], 0, 0, 0);
          }
      if (stage_next) lstore(stage ^ 1, i + 1, next, kk);
    }
  };
  Regs<DT> r[2];
  gload(0, r[0]);
  gload(1, r[1]);
#pragma unroll
  for (int j = 0; j < NP; ++j) lstore(0, 0, r[0], j);
  __syncthreads();
  gload(2, r[0]);
  load_frags(0, 0, 0);
  auto step = [&](int u, Regs<DT>& next, int i) {
    multiply(u, i, next, true);
    __syncthreads();
    load_frags(u ^ 1, 0, 0);
    gload(i + 3, next);
  };
  int i = 0;
  for (; i + 2 < nk; i += 2) {
    step(0, r[1], i);
    step(1, r[0], i + 1);
  }
  if (nk - i == 2) {
    step(0, r[1], i);
    multiply(1, i + 1, r[0], false);
  } else {
    multiply(0, i, r[1], false);
  }

  // Epilogue through LDS: a thread takes 8 consecutive columns of a row; the gate is on its way meanwhile
  float* tile = reinterpret_cast<float*>(smem);
  const int n = n0 + tc;
  const bool vec = (p.N & 7) == 0;
  Eight<DT> gate[DX ? BM / 16 : 1];
  if (DX && p.gate && !p.sums) {
#pragma unroll
    for (int j = 0; j < BM / 16; ++j) {
      const int64_t m = m0 + tk + 16 * j;
      gate[j].zero();
      if (m >= p.M || n >= p.N) continue;
      if (vec) gate[j].load_all(p.gate + (m * p.ldg + n) * ESZ);
      else gate[j].load(p.gate + m * p.ldg * ESZ, n, p.N);
    }
  }
  __syncthreads();
#pragma unroll
  for (int jn = 0; jn < 2; ++jn)
#pragma unroll
    for (int im = 0; im < 2; ++im)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<float4*>(tile + (wm * 64 + im * 32 + (lane & 31)) * STAGE_LD + wn * 64 + jn * 32 + 8 * q + 4 * (lane >> 5)) =
            make_float4(acc[jn][im][4 * q], acc[jn][im][4 * q + 1], acc[jn][im][4 * q + 2], acc[jn][im][4 * q + 3]);
  __syncthreads();
#pragma unroll
  for (int j = 0; j < BM / 16; ++j) {
    const int64_t m = m0 + tk + 16 * j;
    if (m >= p.M || n >= p.N) continue;
    const float4 lo = *reinterpret_cast<const float4*>(tile + (tk + 16 * j) * STAGE_LD + tc), hi = *reinterpret_cast<const float4*>(tile + (tk + 16 * j) * STAGE_LD + tc + 4);
    float v[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
    if (DX && !p.sums) {
      if (p.gate) {
        float f[8];
        gate[j].get(f);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= f[e];
      }
      Eight<DT> o;
      o.set(v);
      if (vec) o.store_all(p.out + (m * p.ldo + n) * ESZ);
      else o.store(p.out + m * p.ldo * ESZ, n, p.N);
    } else {
      Eight<F32> o;
      o.set(v);
      float* row = (float*)p.out + part * p.part_out + m * p.ldo;
      if (vec) o.store_all((char*)(row + n));
      else o.store(row, n, p.N);
    }
  }
  if (do_db) {
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 8; ++e) tile[tk * STAGE_LD + tc + e] = csum[e];
    __syncthreads();
    if (tid < BN && n0 + tid < p.N) {
      float s = 0.f;
#pragma unroll
      for (int j = 0; j < 16; ++j) s += tile[j * STAGE_LD + tid];
      p.db[part * p.part_out + n0 + tid] = s;
    }
  }
}

// Both products in one launch, the longer ones of dW first: they need nothing of each other, and neither fills its last round of units by itself
template <int DT, bool RAGGED> __global__ __launch_bounds__(THREADS, 2) void byte_grad_kernel(GradArgs dw, GradArgs dx) {
  const int first = 8 * dw.per_xcd;
  if ((int)blockIdx.x < first) grad_tile<false, DT, RAGGED>(dw, blockIdx.x);
  else grad_tile<true, DT, RAGGED>(dx, blockIdx.x - first);
}

// Sums of parts, in their order: `first` workgroups those of dW and db, the others those of dX, eight columns a thread
struct SumArgs {
  const float* parts; int n_parts; int64_t part_out; float* dw; int64_t n_dw; float* db; int n_db;
  unsigned first;
  const float* x_parts; int x_n; int64_t x_out; char* dx; int64_t ldx; const char* gate; int64_t ldg; int rows, cols;
};
template <int DT> __global__ __launch_bounds__(256) void byte_grad_sum_kernel(SumArgs p) {
  if (blockIdx.x >= p.first) {
    constexpr int ESZ = DT == BF16 ? 2 : 4;
    const uint32_t pieces = (uint32_t)(p.cols + 7) / 8;
    const uint32_t u = (blockIdx.x - p.first) * 256 + threadIdx.x, row = u / pieces;
    const int c = (int)(u - row * pieces) * 8;
    if (row >= (uint32_t)p.rows) return;
    float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, f[8];
    const float* from = p.x_parts + (int64_t)row * p.cols;
#pragma unroll 4
    for (int k = 0; k < p.x_n; ++k) {
      Eight<F32> v;
      v.load(from + k * p.x_out, c, p.cols);
      v.get(f);
#pragma unroll
      for (int e = 0; e < 8; ++e) s[e] += f[e];
    }
    Eight<DT> o;
    if (p.gate) {
      o.load(p.gate + row * p.ldg * ESZ, c, p.cols);
      o.get(f);
#pragma unroll
      for (int e = 0; e < 8; ++e) s[e] *= f[e];
    }
    o.set(s);
    o.store(p.dx + row * p.ldx * ESZ, c, p.cols);
    return;
  }
  const float* parts = p.parts;
  float *dw = p.dw, *db = p.db;
  const int n_parts = p.n_parts;
  const int64_t part_out = p.part_out, n_dw = p.n_dw, n_db = p.n_db;
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
  const int64_t n = n_dw + n_db;
  if (i >= n) return;
  float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int k = 0; k < n_parts; ++k) {       // (a part has room for whole pieces of four)
    const float4 v = *(const float4*)(parts + k * part_out + i);
    s[0] += v.x; s[1] += v.y; s[2] += v.z; s[3] += v.w;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (i + e < n_dw) dw[i + e] = s[e];
    else if (i + e < n) db[i + e - n_dw] = s[e];
  }
}

// Column sums alone: each workgroup 64 columns of a stretch of rows, 512 of them or what leaves 32768 stretches (a grid has no more)
constexpr int SUM_COLS = 64;
__host__ __device__ constexpr int sum_rows(int rows) { return rows <= 512 << 15 ? 512 : (rows + 32767) >> 15; }
template <int DT> __global__ __launch_bounds__(256) void byte_grad_columns_kernel(const char* d, int64_t ldd, int rows, int cols, float* out) {
  __shared__ float sums[4][SUM_COLS];
  const int c = blockIdx.x * SUM_COLS + (threadIdx.x & 63), w = threadIdx.x >> 6, each = sum_rows(rows), r1 = min(rows, (int)(blockIdx.y + 1) * each);
  float s = 0.f;
  if (c < cols)
#pragma unroll 8
    for (int r = blockIdx.y * each + w; r < r1; r += 4) s += ld_f(d, r * ldd + c, DT);
  sums[w][threadIdx.x & 63] = s;
  __syncthreads();
  if (w == 0 && c < cols) out[(int64_t)blockIdx.y * cols + c] = sums[0][c - blockIdx.x * SUM_COLS] + sums[1][c - blockIdx.x * SUM_COLS] +
                                                                sums[2][c - blockIdx.x * SUM_COLS] + sums[3][c - blockIdx.x * SUM_COLS];
}
__global__ __launch_bounds__(256) void byte_grad_zero_kernel(float* p, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) p[i] = 0.f;
}

template <int DT> int launch(hipStream_t s, GradArgs& dw, GradArgs& dx) {
  constexpr int LDS = std::max(lds_bytes<true, DT>(), lds_bytes<false, DT>());
  for (GradArgs* p : {&dw, &dx}) {
    p->tiles_m = (p->M + BM - 1) / BM; p->tiles_n = (p->N + BN - 1) / BN;
    p->per_xcd = (int)(((int64_t)p->tiles_m * p->tiles_n * p->parts + 7) / 8);
  }
  const dim3 grid(8 * (dw.per_xcd + dx.per_xcd));
  if ((dw.parts ? dw.dcols : dx.dcols) & 7) {
    static OncePerDevice once;
    PPLL_TRY(raise_lds((const void*)byte_grad_kernel<DT, true>, LDS, once));
    hipLaunchKernelGGL((byte_grad_kernel<DT, true>), grid, dim3(THREADS), LDS, s, dw, dx);
  } else {
    static OncePerDevice once;
    PPLL_TRY(raise_lds((const void*)byte_grad_kernel<DT, false>, LDS, once));
    hipLaunchKernelGGL((byte_grad_kernel<DT, false>), grid, dim3(THREADS), LDS, s, dw, dx);
  }
  PPLL_HIP(hipGetLastError());
  return PPLL_OK;
}

// Into how many parts a reduction goes: a workgroup a unit, none under four steps.  dX in one part / in parts of 12, 8, 6, 4, 3 steps at least, both
// gradients, us: 41 x 63 x 5645 102 / 25, 22, 21, 21, 22; 56 x 1483 x 2737 76 / 38, 30, 28, 27, 26; 1140 x 249 x 875 29 / 29, 29, 22, 21, 22; 4621 x 151 x
// 1795 in fp32 80 / 49, 50, 50, 49, 50.
struct Parts { int n, k; int64_t out; };
Parts parts_of(const ByteLinear& l, int64_t m, int64_t n, int64_t k, int64_t out) {
  const int bk = l.dt == F32 ? step_k<F32>() : step_k<BF16>();
  const int64_t tiles = ((m + BM - 1) / BM) * ((n + BN - 1) / BN), steps = (k + bk - 1) / bk;
  const int64_t want = std::max<int64_t>(1, std::min<int64_t>(256 / tiles, steps / 4));
  const int64_t each = (steps + want - 1) / want;
  Parts p;
  p.n = (int)std::max<int64_t>(1, (steps + each - 1) / each);
  p.k = (int)std::min<int64_t>(each * bk, 0x7fffffff);
  p.out = (out + 3) / 4 * 4;
  return p;
}
Parts dw_parts(const ByteLinear& l) { return parts_of(l, l.in, l.out, l.rows, (int64_t)l.in * l.out + l.out); }
Parts dx_parts(const ByteLinear& l) { return parts_of(l, l.rows, l.in, l.out, (int64_t)l.rows * l.in); }
int64_t part_floats(const Parts& p) { return p.n > 1 ? p.n * p.out : 0; }
int sum_chunks(int rows) { return (int)(((int64_t)rows + sum_rows(rows) - 1) / sum_rows(rows)); }

// ---- The other way: operands written out in bf16, which is what they stand for, and the products on the kernels of bf16 operands.  Those reach 1100
// TFLOP/s where the kernel above reaches 750, but X goes through memory twice more.
constexpr int64_t PRODUCT_BYTES = (1 << 30) - 64;      // that those kernels address of an operand, and of C at 4 bytes an element whatever its type
bool weight_fits(const ByteLinear& l) { return l.dt == BF16 && l.in % 8 == 0 && l.out % 8 == 0 && (int64_t)l.in * l.out * 2 <= PRODUCT_BYTES; }
bool both_fit(const ByteLinear& l) {
  return weight_fits(l) && (int64_t)l.rows * std::max(l.in, l.out) * 2 <= PRODUCT_BYTES && (int64_t)l.in * l.out * 4 <= PRODUCT_BYTES;
}
// Rows of dX that one product takes: all, or stretches of about as many each (x 4096 from 4096 channels: 65535 rows 1727 us, 65536 in two stretches 1766).
// 0: rows that lie so far apart that a stretch would be short, which the kernel above takes as they are.
constexpr int64_t LEAST_STRETCH = 4096;
int stretch_of(const ByteLinear& l, const ppll_rows& dy, const ppll_rows& gate, const ppll_rows& dx) {
  const int64_t widest = std::max(dx.ld, (std::max(dy.ld, gate.p ? gate.ld : 0) + 1) / 2), most = PRODUCT_BYTES / 4 / widest;
  if (l.rows <= most) return l.rows;
  if (most < LEAST_STRETCH) return 0;
  const int64_t n = (l.rows + most / 256 * 256 - 1) / (most / 256 * 256);
  return (int)(((l.rows + n - 1) / n + 255) / 256 * 256);
}
// Microseconds with the sum of parts, this kernel / values, both gradients, rows x in x out: 8320 x 1536 x 384 46 / 49, 25216 x 768 x 768 94 / 97,
// 4096 x 2048 x 2048 94 / 95, 8320 x 1536 x 1536 143 / 106, 25216 x 768 x 2304 243 / 193, 8192 x 4096 x 4096 730 / 517, 512 x 6144 x 6144 153 / 129; with few
// output channels X's way counts for more: 32768 x 4096 x 256 239 / 284.  From 4e10 operations on: 640 x 4096 x 4096 94 / 67, 2560 x 2048 x 2048 80 / 74, 2560 x
// 4096 x 1024 67.5 / 67.5; below: 5120 x 768 x 2304 60 / 66, 1280 x 2048 x 2048 40 / 42.  Over 114 products of 17 to 20124 rows and 64 to 5680 channels each
// way the rule costs half a per cent over the better way at each.
bool values_for_both(const ByteLinear& l) { return both_fit(l) && 4.0 * l.rows * l.in * l.out >= 4e10 && l.out >= 512; }
// dX alone: W alone is written out.  8320 x 1536 x 384 24 / 19, 25216 x 768 x 768 48 / 35, 8320 x 384 x 384 10.8 / 10.1, 640 x 768 x 768 13.8 / 8.2, 128 x 1536 x 384
// 9.7 / 6.9, 64 x 768 x 2304 11.9 / 10.2; behind where few rows meet a large weight, 256 x 4096 x 4096 26 / 41, 1 x 4096 x 4096 14 / 28, which no rule looks at yet.
// dW alone stays on this kernel, ahead at 8320 x 1536 x 384, 31 / 33, behind at 25216 x 768 x 768, 73 / 65, and 8192 x 4096 x 4096, 386 / 276.
GemmArgs dw_product(const ByteLinear& l, const uint16_t* xv, const ppll_rows& dy, float* dw, float* db) {
  GemmArgs g{};
  g.A = xv; g.a_dt = BF16; g.a_sm = 1; g.a_sk = l.in;
  g.B = dy.p; g.b_dt = BF16; g.b_sk = dy.p ? dy.ld : l.out; g.b_sn = 1;
  g.C = dw; g.c_dt = F32; g.ldc = l.out; g.M = l.in; g.N = l.out; g.K = l.rows;
  g.colsum = db;
  return g;
}
size_t dw_floats(const ByteLinear& l) {       // for the parts of its tiles
  const GemmArgs g = dw_product(l, nullptr, {nullptr, 0}, nullptr, nullptr);
  size_t floats = 0;
  gemm_big_grads_choice(&g, 1, &floats);
  return std::max(floats, gemm_mfma_balanced_floats());
}
int64_t values_bytes(const ByteLinear& l, bool x, bool w) { return (((x ? (int64_t)l.rows : 0) + (w ? l.out : 0)) * l.in * 2 + 255) / 256 * 256; }
GemmArgs dx_product(const ByteLinear& l, const uint16_t* wv, const ppll_rows& dy, const ppll_rows& gate, const ppll_rows& dx, int64_t first, int rows) {
  GemmArgs g{};
  g.A = (const uint16_t*)dy.p + first * dy.ld; g.a_dt = BF16; g.a_sm = dy.ld; g.a_sk = 1;
  g.B = wv; g.b_dt = BF16; g.b_sk = l.in; g.b_sn = 1;
  g.C = (uint16_t*)dx.p + first * dx.ld; g.c_dt = BF16; g.ldc = dx.ld; g.M = rows; g.N = l.in; g.K = l.out;
  if (gate.p) { g.epilogue = EPI_DGELU; g.aux = (const uint16_t*)gate.p + first * gate.ld; g.aux_dt = BF16; g.ldaux = gate.ld; }
  g.shared = l.shared; g.units = l.units;
  return g;
}
// Whether the kernels of bf16 operands take what is wanted; ws: room that begins with the values of X and W
uint16_t* w_values(const ByteLinear& l, const float* dw, char* ws) { return (uint16_t*)ws + (dw ? (int64_t)l.rows * l.in : 0); }
bool values_supported(const ByteLinear& l, const ppll_rows& dy, const ppll_rows& gate, const ppll_rows& dx, float* dw, float* db, char* ws) {
  if (!weight_fits(l) || (dw && (!both_fit(l) || !gemm_mfma_groupable(dw_product(l, (const uint16_t*)ws, dy, dw, db))))) return false;
  if (!dx.p) return true;
  const int rows = stretch_of(l, dy, gate, dx);
  return rows > 0 && gemm_mfma_supported(dx_product(l, w_values(l, dw, ws), dy, gate, dx, 0, rows));
}
int backward_values(hipStream_t s, const ByteLinear& l, const ppll_byte_rows& x, const ppll_byte_rows& w, const ppll_rows& dy, const ppll_rows& gate,
                    const ppll_rows& dx, float* dw, float* db, char* ws) {
  uint16_t *xv = (uint16_t*)ws, *wv = w_values(l, dw, ws);
  PPLL_TRY(launch_byte_rows_values(s, l.in, x, dw ? l.rows : 0, w, dx.p ? l.out : 0, xv));
  const int stretch = dx.p ? stretch_of(l, dy, gate, dx) : 0;
  for (int64_t first = 0; dx.p && first < l.rows; first += stretch)
    PPLL_TRY(launch_gemm(s, dx_product(l, wv, dy, gate, dx, first, (int)std::min<int64_t>(stretch, l.rows - first))));
  if (!dw) return PPLL_OK;
  const GemmArgs g = dw_product(l, xv, dy, dw, db);
  return launch_gemm_group(s, &g, 1, (float*)(ws + values_bytes(l, true, true)), dw_floats(l), true);
}

template <int DT> int backward_here(hipStream_t s, const ByteLinear& l, const ppll_byte_rows& x, const ppll_byte_rows& w, const ppll_rows& dy, const ppll_rows& gate,
                               const ppll_rows& dx, float* dw, float* db, float* ws) {
  GradArgs pw{}, px{};       // (no parts: not wanted)
  const Parts parts = dw_parts(l), x_parts = dx_parts(l);
  const bool whole = parts.n == 1, x_whole = x_parts.n == 1;
  float* x_ws = ws + part_floats(parts);
  if (dx.p) {
    px.d = (const char*)dy.p; px.ldd = dy.ld; px.dcols = l.out;
    px.q = w.q; px.e = w.e; px.ldq = w.ld; px.qcols = pad16(l.in);
    px.out = x_whole ? (char*)dx.p : (char*)x_ws; px.ldo = x_whole ? dx.ld : l.in; px.gate = (const char*)gate.p; px.ldg = gate.ld;
    px.M = l.rows; px.N = l.in; px.K = l.out; px.parts = x_parts.n; px.part_k = x_parts.k; px.part_out = x_parts.out;
    px.sums = !x_whole;
  }
  if (dw) {
    pw.d = (const char*)dy.p; pw.ldd = dy.ld; pw.dcols = l.out;
    pw.q = x.q; pw.e = x.e; pw.ldq = x.ld; pw.qcols = pad16(l.in);
    pw.out = (char*)(whole ? dw : ws); pw.ldo = l.out;
    pw.db = !db ? nullptr : whole ? db : ws + (int64_t)l.in * l.out;
    pw.M = l.in; pw.N = l.out; pw.K = l.rows; pw.parts = parts.n; pw.part_k = parts.k; pw.part_out = parts.out;
    pw.sums = true;
  }
  void* prof = nullptr;
  if (dx.p || dw) {
    PPLL_TRY(profile_begin(s, 2.0 * ((dx.p ? 1 : 0) + (dw ? 1 : 0)) * l.rows * l.in * l.out, &prof, l.rows < 256 ? 2 : 0));
    PPLL_TRY(launch<DT>(s, pw, px));
  }
  if ((dw && !whole) || (dx.p && !x_whole)) {
    SumArgs a{};
    if (dw && !whole) {
      a.parts = ws; a.n_parts = parts.n; a.part_out = parts.out; a.dw = dw; a.n_dw = (int64_t)l.in * l.out; a.db = db; a.n_db = db ? l.out : 0;
      a.first = (unsigned)((a.n_dw + a.n_db + 1023) / 1024);
    }
    unsigned more = 0;
    if (dx.p && !x_whole) {
      a.x_parts = x_ws; a.x_n = x_parts.n; a.x_out = x_parts.out; a.dx = (char*)dx.p; a.ldx = dx.ld; a.gate = (const char*)gate.p; a.ldg = gate.ld;
      a.rows = l.rows; a.cols = l.in;
      more = (unsigned)(((int64_t)l.rows * ((l.in + 7) / 8) + 255) / 256);      // (256 tiles at most)
    }
    hipLaunchKernelGGL(byte_grad_sum_kernel<DT>, dim3(a.first + more), dim3(256), 0, s, a);
    PPLL_HIP(hipGetLastError());
  }
  PPLL_TRY(profile_end(s, prof));
  if (db && !dw) {
    const int chunks = sum_chunks(l.rows);
    hipLaunchKernelGGL(byte_grad_columns_kernel<DT>, dim3((l.out + SUM_COLS - 1) / SUM_COLS, chunks), dim3(256), 0, s, (const char*)dy.p, dy.ld, l.rows, l.out,
                       chunks == 1 ? db : ws);
    PPLL_HIP(hipGetLastError());
    if (chunks > 1) PPLL_TRY(reduce_partials(s, ws, chunks, l.out, l.out, 1.f, db));
  }
  return PPLL_OK;
}
int zero(hipStream_t s, float* p, int64_t n) {
  if (!p) return PPLL_OK;
  hipLaunchKernelGGL(byte_grad_zero_kernel, dim3((unsigned)std::min<int64_t>((n + 255) / 256, 4096)), dim3(256), 0, s, p, n);
  PPLL_HIP(hipGetLastError());
  return PPLL_OK;
}
// way: 0 by the rules, 1 the kernel here, 2 values
int backward(hipStream_t s, int way, const ByteLinear& l, const ppll_byte_rows& x, const ppll_byte_rows& w, const ppll_rows& dy, const ppll_rows& gate,
             const ppll_rows& dx, float* dw, float* db, char* ws) {
  const bool values = (dx.p || dw) && (dw || !db) && (way ? way == 2 : dw ? dx.p && values_for_both(l) : true) && values_supported(l, dy, gate, dx, dw, db, ws);
  if (way == 2 && !values) { set_error("not as values"); return PPLL_ERR_CONFIG; }
  if (values) return backward_values(s, l, x, w, dy, gate, dx, dw, db, ws);
  return l.dt == BF16 ? backward_here<BF16>(s, l, x, w, dy, gate, dx, dw, db, (float*)ws) : backward_here<F32>(s, l, x, w, dy, gate, dx, dw, db, (float*)ws);
}
size_t workspace(const ByteLinear& l, bool any) {
  if (l.rows <= 0) return 0;
  const int64_t parts = part_floats(dw_parts(l)) + part_floats(dx_parts(l)), sums = sum_chunks(l.rows) > 1 ? (int64_t)sum_chunks(l.rows) * l.out : 0;
  int64_t bytes = std::max(parts, sums) * (int64_t)sizeof(float);
  if (weight_fits(l)) bytes = std::max(bytes, values_bytes(l, false, true));
  if (any ? both_fit(l) : values_for_both(l)) bytes = std::max(bytes, values_bytes(l, true, true) + (int64_t)(dw_floats(l) * sizeof(float)));
  return (size_t)bytes;
}
}  // namespace

size_t byte_linear_workspace(const ByteLinear& l) { return workspace(l, false); }

int launch_byte_linear_bwd(hipStream_t s, const ByteLinear& l, const ppll_byte_rows& x, const ppll_byte_rows& w, const ppll_rows& dy, const ppll_rows& gate,
                           const ppll_rows& dx, float* dw, float* db, char* ws) {
  if (l.rows <= 0) {
    PPLL_TRY(zero(s, dw, (int64_t)l.in * l.out));
    return zero(s, db, l.out);
  }
  return backward(s, 0, l, x, w, dy, gate, dx, dw, db, ws);
}

}  // namespace ppll

// Both gradients one way (backward() above), for tests of one against the other (no part of the public interface); ws null: its size to *bytes
extern "C" int ppll_internal_byte_linear_backward(int way, int rows, int in, int out, const ppll_byte_rows* x, const ppll_byte_rows* w, const ppll_rows* dy,
                                                  const ppll_rows* gate, const ppll_rows* dx, float* dw, float* db, char* ws, size_t* bytes, void* stream) {
  using namespace ppll;
  const ByteLinear l{BF16, rows, in, out, PPLL_ACT_NONE};
  if (!ws) { *bytes = workspace(l, true); return PPLL_OK; }
  const ppll_rows none{nullptr, 0};
  return backward((hipStream_t)stream, way, l, *x, *w, *dy, gate ? *gate : none, dx ? *dx : none, dw, db, ws);
}
