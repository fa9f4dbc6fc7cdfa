// Newton-Schulz orthogonalisation of batches of matrices and the Muon step around it.
#include "common.h"
#include "gemm_pipe.h"
#include "ortho.h"

#include <math.h>

namespace ppll {

namespace {
using pipe::barrier;
using pipe::f32x16;
using pipe::lds_char;
using pipe::u32x2;
using pipe::u32x4;
using pipe::wait_vm;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(4))) _Float16 f16x4;

constexpr float NS_A = 3.4445f, NS_B = -4.7750f, NS_C = 2.0315f;
constexpr double NORM_EPS = 1e-7;
// Operands are stored as hi + lo, two fp16 of a value times 2^14: 22 bits, and the products hi hi + hi lo + lo hi miss 2^-22 of a product,
// a rounding of fp32.  The scale keeps lo above fp16's denormals: entries are 1 / sqrt(m n) in the mean, 2^-13 for the largest matrices.
// It cannot overflow: singular values are 1.2023 at most (the polynomial's maximum on [0, 1.2023]), so entries are 1.2023 at most for X,
// 1.446 for A, and b A + c A A has eigenvalues from -2.81 to 0: 46000 times 1, of 65504.
constexpr double SCALE = 16384;
constexpr float UNSCALE = 1.f / 16384.f;

// The operands are scaled to a Frobenius norm of exactly 1 at the start, and what X is smaller by, t0 = |u| / (|u| + 1e-7), enters as a
// factor: X = t Y with t = min(1, a^k t0) in step k, so Y' = t / t' (a Y + (b t^2 Y Y' + c t^4 (Y Y')^2) Y).  Unless a matrix is as small as
// the constant this is t = 1; one of norm 1e-20, whose X is of norm 1e-13, would be lost in fp16 otherwise.
struct Shrink { float now, next, ratio; };
__device__ __forceinline__ Shrink shrink_of(float t0, int step) {
  float t = t0;
  for (int k = 0; k < step; ++k) t = fminf(1.f, NS_A * t);
  const float next = fminf(1.f, NS_A * t);
  return {t, next, t0 > 0.f ? t / next : 1.f};
}

constexpr int GRAM = ORTHO_GRAM, POLY = ORTHO_POLY, APPLY = ORTHO_APPLY, LAST = ORTHO_APPLY + 1;

// What a call works on.  in: blob of the matrices (orthogonalize), or null: u from g and the momentum (Muon step)
struct Source { const void* in; int dt; const float* g; float* m; float momentum; int nesterov; };
// Where the result goes: out (orthogonalize), or null: the parameters
struct Target { void* out; int dt; float* p; uint16_t* shadow; float lr, decay; };

// v is pinned to its fp32 value first: the compiler may fold the arithmetic that gives it into one of the two conversions (a fused operation
// that rounds to fp16 once) and not into the other, and at a tie hi and what lo is counted from are then two neighbours (one element in some
// 20000 was off by a whole step of hi, 2^-11 of it).
__device__ __forceinline__ void split(float v, _Float16& hi, _Float16& lo) {
  asm("" : "+v"(v));
  hi = (_Float16)v;
  lo = (_Float16)(v - (float)hi);
}
__device__ __forceinline__ int64_t element(const OrthoGroup& g, int matrix, int r, int c) {
  return g.offset + (int64_t)matrix * g.stride + (int64_t)r * g.ld + c;
}
// The matrix that work item `id` of a launch belongs to, `each(group)` items a matrix; id becomes the place within it.
struct Place { int group, matrix; };
template <class EACH> __device__ __forceinline__ Place place_of(const OrthoPlan& p, int& id, EACH each) {
  for (int k = 0; k < p.n; ++k) {
    const int e = each(p.g[k]), all = e * p.g[k].count;      // (none: no items of this kind)
    if (id < all) {
      const int i = id / e;
      id -= i * e;
      return {k, i};
    }
    id -= all;
  }
  return {-1, 0};
}
__device__ __forceinline__ float read_u(const Source& s, int64_t at) {
  if (s.in) return ld_f(s.in, (size_t)at, s.dt);
  const float m = s.m[at];
  return s.nesterov ? fmaf(s.momentum, m, s.g[at]) : m;
}

// The momentum, and the sums of squares of pieces of 32 x 256 (in 64 bits: gradients of 1e-25 or 1e25 have a norm as well).
__global__ __launch_bounds__(256) void squares_kernel(OrthoPlan p, Source s, char* ws) {
  int id = blockIdx.x;
  const Place at = place_of(p, id, [](const OrthoGroup& g) { return g.small ? 0 : g.pieces(); });
  const OrthoGroup& g = p.g[at.group];
  const int across = (g.cols + NORM_COLS - 1) / NORM_COLS, r0 = id / across * NORM_ROWS, c = id % across * NORM_COLS + threadIdx.x;
  double sum = 0;
  const int64_t first = element(g, at.matrix, r0, c);
  const int rows = c < g.cols ? min(NORM_ROWS, g.rows - r0) : 0;
  for (int r = 0; r < rows; r += 8) {        // eight rows on their way at a time
    float u[8], m[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int64_t e = first + (int64_t)(r + k) * g.ld;
      const bool on = r + k < rows;
      u[k] = !on ? 0.f : s.in ? ld_f(s.in, (size_t)e, s.dt) : s.g[e];
      m[k] = on && !s.in ? s.m[e] : 0.f;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if (!s.in) {
        m[k] = fmaf(s.momentum, m[k], u[k]);
        if (r + k < rows) s.m[first + (int64_t)(r + k) * g.ld] = m[k];
        u[k] = s.nesterov ? fmaf(s.momentum, m[k], u[k]) : m[k];
      }
      sum += (double)u[k] * u[k];
    }
  }
  __shared__ double sums[256];
  sums[threadIdx.x] = sum;
  __syncthreads();
  for (int w = 128; w > 0; w >>= 1) {
    if (threadIdx.x < w) sums[threadIdx.x] += sums[threadIdx.x + w];
    __syncthreads();
  }
  if (threadIdx.x == 0) ((double*)(ws + p.partials))[g.first_piece + at.matrix * g.pieces() + id] = sums[0];
}

// Y = u / |u|, in tiles of 64 x 64.
__global__ __launch_bounds__(256) void normalise_kernel(OrthoPlan p, Source s, char* ws) {
  int id = blockIdx.x;
  const Place at = place_of(p, id, [](const OrthoGroup& g) { return g.small ? 0 : (g.mp / 64) * (g.np / 64); });
  const OrthoGroup& g = p.g[at.group];
  const int t = threadIdx.x, i0 = id / (g.np / 64) * 64, j0 = id % (g.np / 64) * 64;
  __shared__ double sums[256];
  __shared__ float tile[64][65];
  const double* part = (const double*)(ws + p.partials) + g.first_piece + at.matrix * g.pieces();
  double sum = 0;
  for (int k = t; k < g.pieces(); k += 256) sum += part[k];
  sums[t] = sum;
  __syncthreads();
  for (int w = 128; w > 0; w >>= 1) {
    if (t < w) sums[t] += sums[t + w];
    __syncthreads();
  }
  const double norm = sqrt(sums[0]), inv = norm > 0 ? SCALE / norm : norm;      // NaN stays one
  if (id == 0 && t == 0) ((float*)(ws + p.shrink))[g.first + at.matrix] = (float)(norm / (norm + NORM_EPS));
  for (int k = 0; k < 16; ++k) {
    const int y = k * 4 + t / 64, x = t % 64;                  // in the caller's orientation: rows y
    const int r = (g.tall ? j0 : i0) + y, c = (g.tall ? i0 : j0) + x;
    const float v = r < g.rows && c < g.cols ? (float)(read_u(s, element(g, at.matrix, r, c)) * inv) : 0.f;
    if (g.tall) tile[x][y] = v;
    else tile[y][x] = v;
  }
  __syncthreads();
  const int64_t plane = g.plane_x();
  _Float16* x = (_Float16*)(ws + g.x[0]) + at.matrix * 2 * plane;
  const int y = t / 4, q = t % 4 * 16;
  f16x8 h[2], l[2];
  for (int k = 0; k < 16; ++k) {
    _Float16 a, b;
    split(tile[y][q + k], a, b);
    h[k / 8][k % 8] = a; l[k / 8][k % 8] = b;
  }
  _Float16* to = x + (int64_t)(i0 + y) * g.np + j0 + q;
  for (int k = 0; k < 2; ++k) { *(f16x8*)(to + 8 * k) = h[k]; *(f16x8*)(to + plane + 8 * k) = l[k]; }
}

// ------------------------------------------------------------------ products
// C[i][j] = sum over k of P[i][k] Q(k, j), a tile of TILE x TILE a workgroup of four waves:
//  GRAM   P = X, Q = X'        A = C                    symmetric: tiles on and under the diagonal, each stored twice
//  POLY   P = A, Q = A'        B = b A + c C            likewise
//  APPLY  P = B, Q = X         X = a X + C              (X in two buffers in turn: other tiles still read the old one)
//  LAST   the same, to where the result goes
// A stage of the pipeline is KT k of the four planes (hi and lo of P and of Q), 8 KB each and each copied by one wave straight from memory to
// LDS; there are two stages.  A wave multiplies 64 x 64: three products of 32 x 32 x 16 for each pair of fragments, 12 for eight fragments read.
//  TILE 128: a wave has a quarter of the tile and all k.  TILE 64: it has all of the tile and a quarter of the k, and the four sums are added up
//  at the end: fragments are read once for 12 products all the same, where quarters of 32 x 32 would read twice as much for each.
// Layouts in LDS, as in gemm_pipe.h: k contiguous (P, and Q of GRAM and POLY): rows of KT k, their 16-byte granules permuted; k rows (X of APPLY):
// rows of TILE columns whose 64-byte windows are permuted, for the transposing read.
template <int TILE> struct Tile {
  static constexpr int KT = TILE == 128 ? 32 : 64, PLANE = TILE * KT * 2, STAGE = 4 * PLANE, LDS = 2 * STAGE;
  static constexpr int PITCH = TILE * 2;                     // of a k row
  static constexpr int R32 = 32 * KT * 2;                    // 32 rows with k contiguous
};
struct Planes { u32x4 p[2], pl[2], q[2], ql[2]; };           // fragments: hi and lo of two 32-row tiles of P and of Q

#define NS_MMA(C, Q, P) "v_mfma_f32_32x32x16_f16 %[" C "], %[" Q "], %[" P "], %[" C "]\n"
#define NS_ACC [h00] "+v"(hh[0][0]), [h01] "+v"(hh[0][1]), [h10] "+v"(hh[1][0]), [h11] "+v"(hh[1][1]), [x00] "+v"(xx[0][0]), \
               [x01] "+v"(xx[0][1]), [x10] "+v"(xx[1][0]), [x11] "+v"(xx[1][1])
#define NS_CUR [p0] "v"(f.p[0]), [p1] "v"(f.p[1]), [a0] "v"(f.pl[0]), [a1] "v"(f.pl[1]), [q0] "v"(f.q[0]), [q1] "v"(f.q[1]), [b0] "v"(f.ql[0]), \
               [b1] "v"(f.ql[1])
#define NS_CROSS NS_MMA("x00", "b0", "p0") NS_MMA("x01", "b0", "p1") NS_MMA("x10", "b1", "p0") NS_MMA("x11", "b1", "p1") \
                 NS_MMA("x00", "q0", "a0") NS_MMA("x01", "q0", "a1") NS_MMA("x10", "q1", "a0") NS_MMA("x11", "q1", "a1")
// The 12 products of the fragments at hand (into hh: hi hi, into xx the cross terms: small terms summed apart keep their digits, error of
// 1536 x 6144 1.8e-6 instead of 3.2e-6), and under them the reads of the next ones, at rp and rq, which have arrived when the block ends.  One
// assembly block, as in gemm_pipe.h: the compiler would wait for all copies into LDS before a read that it knows of.
template <int TILE, bool TR>
__device__ __forceinline__ void k_step(f32x16 (&hh)[2][2], f32x16 (&xx)[2][2], const Planes& f, Planes& n, int rp, int rq) {
  using S = Tile<TILE>;
  if constexpr (!TR) {
    asm volatile("s_nop 1\n" NS_MMA("h00", "q0", "p0") "ds_read_b128 %[s0], %[rp]\n ds_read_b128 %[s1], %[rp] offset:%[r1]\n"
                 NS_MMA("h01", "q0", "p1") "ds_read_b128 %[t0], %[rq]\n ds_read_b128 %[t1], %[rq] offset:%[r1]\n"
                 NS_MMA("h10", "q1", "p0") "ds_read_b128 %[u0], %[rq] offset:%[l0]\n ds_read_b128 %[u1], %[rq] offset:%[l1]\n"
                 NS_MMA("h11", "q1", "p1") "ds_read_b128 %[v0], %[rp] offset:%[l0]\n ds_read_b128 %[v1], %[rp] offset:%[l1]\n"
                 NS_CROSS "s_waitcnt lgkmcnt(0)"
                 : NS_ACC, [s0] "=&v"(n.p[0]), [s1] "=&v"(n.p[1]), [v0] "=&v"(n.pl[0]), [v1] "=&v"(n.pl[1]), [t0] "=&v"(n.q[0]),
                   [t1] "=&v"(n.q[1]), [u0] "=&v"(n.ql[0]), [u1] "=&v"(n.ql[1])
                 : NS_CUR, [rp] "v"(rp), [rq] "v"(rq), [r1] "n"(S::R32), [l0] "n"(S::PLANE), [l1] "n"(S::PLANE + S::R32)
                 : "memory");
  } else {
    u32x2 t[2][2], u[2][2];
    asm volatile("s_nop 1\n" NS_MMA("h00", "q0", "p0") "ds_read_b128 %[s0], %[rp]\n ds_read_b128 %[s1], %[rp] offset:%[r1]\n"
                 "ds_read_b64_tr_b16 %[t00], %[rq]\n ds_read_b64_tr_b16 %[t01], %[rq] offset:%[f]\n"
                 NS_MMA("h01", "q0", "p1") "ds_read_b64_tr_b16 %[t10], %[rx]\n ds_read_b64_tr_b16 %[t11], %[rx] offset:%[f]\n"
                 "ds_read_b64_tr_b16 %[u00], %[rq] offset:%[l0]\n ds_read_b64_tr_b16 %[u01], %[rq] offset:%[lf]\n"
                 NS_MMA("h10", "q1", "p0") "ds_read_b64_tr_b16 %[u10], %[rx] offset:%[l0]\n ds_read_b64_tr_b16 %[u11], %[rx] offset:%[lf]\n"
                 NS_MMA("h11", "q1", "p1") "ds_read_b128 %[v0], %[rp] offset:%[l0]\n ds_read_b128 %[v1], %[rp] offset:%[l1]\n"
                 NS_CROSS "s_waitcnt lgkmcnt(0)"
                 : NS_ACC, [s0] "=&v"(n.p[0]), [s1] "=&v"(n.p[1]), [v0] "=&v"(n.pl[0]), [v1] "=&v"(n.pl[1]), [t00] "=&v"(t[0][0]),
                   [t01] "=&v"(t[0][1]), [t10] "=&v"(t[1][0]), [t11] "=&v"(t[1][1]), [u00] "=&v"(u[0][0]), [u01] "=&v"(u[0][1]),
                   [u10] "=&v"(u[1][0]), [u11] "=&v"(u[1][1])
                 : NS_CUR, [rp] "v"(rp), [rq] "v"(rq), [rx] "v"(rq ^ 64), [r1] "n"(S::R32), [l0] "n"(S::PLANE), [l1] "n"(S::PLANE + S::R32),
                   [f] "n"(4 * S::PITCH), [lf] "n"(S::PLANE + 4 * S::PITCH)
                 : "memory");
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      n.q[j] = (u32x4){t[j][0].x, t[j][0].y, t[j][1].x, t[j][1].y};
      n.ql[j] = (u32x4){u[j][0].x, u[j][0].y, u[j][1].x, u[j][1].y};
    }
  }
}

template <int TILE, int MODE> __global__ __launch_bounds__(256) void product_kernel(OrthoPlan p, XcdShares shares, Target t, char* ws, int step) {
  using S = Tile<TILE>;
  constexpr bool TR = MODE >= APPLY;
  extern __shared__ __align__(16) char stages[];
  const int xcd = blockIdx.x & 7;
  int id = shares.first[xcd] + (int)(blockIdx.x >> 3);
  if (id >= shares.first[xcd + 1]) return;
  const Place at = place_of(p, id, [](const OrthoGroup& g) { return tiles_of_matrix(g, TILE, MODE); });
  const OrthoGroup& g = p.g[at.group];
  int bi, bj;
  if (MODE <= POLY) {
    bi = (int)((sqrtf(8.f * id + 1.f) - 1.f) * 0.5f);
    while ((bi + 1) * (bi + 2) / 2 <= id) ++bi;
    while (bi * (bi + 1) / 2 > id) --bi;
    bj = id - bi * (bi + 1) / 2;
  } else {
    const int down = (g.mp + TILE - 1) / TILE;         // tiles that read the same columns of X follow one another
    bj = id / down; bi = id - bj * down;
  }
  const int64_t px = g.plane_x(), pa = g.plane_a();
  const int from = step & 1;
  _Float16* X = (_Float16*)(ws + g.x[from]) + at.matrix * 2 * px;
  _Float16* A = (_Float16*)(ws + g.a) + at.matrix * 2 * pa;
  _Float16* B = (_Float16*)(ws + g.b) + at.matrix * 2 * pa;
  const int K = MODE == GRAM ? g.np : g.mp, nk = K / S::KT;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

  // ---- what this wave copies: plane `wave` of P hi, P lo, Q hi, Q lo
  const bool is_q = wave >= 2;
  const int64_t plane = (MODE == GRAM || (TR && is_q)) ? px : pa;
  const _Float16* src = (MODE == GRAM ? X : MODE == POLY ? A : is_q ? X : B) + (wave & 1 ? plane : 0);
  const __amdgpu_buffer_rsrc_t rs = pipe::make_rsrc(src, (uint32_t)(plane * 2));
  lds_char* const lds = (lds_char*)stages;
  int off[2], every, step_k;         // bytes: this lane's of even and odd copies at stage 0, from copy to copy, from stage to stage
  if (TR && is_q) {
    const int ld2 = g.np * 2;
    const int kr = TILE == 128 ? lane >> 4 : lane >> 3, slot = TILE == 128 ? lane & 15 : lane & 7;
    const int win = (slot >> 2) ^ (TILE == 128 ? kr & 3 : kr >> 1 & 1);
    off[0] = off[1] = kr * ld2 + (bj * TILE + (win * 4 + (slot & 3)) * 8) * 2;
    every = (TILE == 128 ? 4 : 8) * ld2;
    step_k = S::KT * ld2;
  } else {
    const int ld2 = K * 2, row0 = (is_q ? bj : bi) * TILE;
    if (TILE == 128) {
      off[0] = off[1] = (row0 + (lane >> 2)) * ld2 + ((lane & 3) ^ (lane >> 4 & 3)) * 16;
      every = 16 * ld2;
    } else {
      for (int odd = 0; odd < 2; ++odd) off[odd] = (row0 + (lane >> 3)) * ld2 + ((lane & 7) ^ ((4 * odd + (lane >> 4)) & 7)) * 16;
      every = 8 * ld2;
    }
    step_k = S::KT * 2;
  }
  auto issue = [&](int i) {
    if (i >= nk) return;
    lds_char* to = lds + (i & 1) * S::STAGE + wave * S::PLANE;
#pragma unroll
    for (int c = 0; c < 8; ++c) pipe::load_to_lds(rs, to + c * 1024, off[c & 1] + c * every + i * step_k);
  };

  // ---- where this wave reads its fragments, in stage 0
  const int base = (int)(uintptr_t)lds, wi = TILE == 128 ? wave >> 1 : 0, wj = TILE == 128 ? wave & 1 : 0, kk = TILE == 128 ? 0 : wave;
  auto rows_at = [&](int region, int row0) {       // k contiguous
    const int r = lane & 31;
    if (TILE == 128) return region + (row0 + r) * 64 + (((lane >> 5) ^ (r >> 2 & 3)) << 4);
    return region + (row0 + r) * 128 + (((2 * kk + (lane >> 5)) ^ (r >> 1 & 7)) << 4);
  };
  const int rp = rows_at(base, wi * 64);
  int rq;
  if (TR) {
    const int kr = 8 * (lane >> 5) + ((lane & 15) >> 2), perm = TILE == 128 ? kr & 3 : kr >> 1 & 1;
    rq = base + 2 * S::PLANE + (kr + 16 * kk) * S::PITCH + (((wj * 2) ^ perm) << 6) + (16 * (lane >> 4 & 1) + 4 * (lane & 3)) * 2;
  } else {
    rq = rows_at(base + 2 * S::PLANE, wj * 64);
  }
  constexpr int NEXT_Q = TR ? 16 * S::PITCH : 0;    // the second k step of a stage (TILE 128)

  // ---- main loop: a stage is filled again from the moment that everyone has read it
  f32x16 hh[2][2] = {}, xx[2][2] = {};
  Planes f0, f1;
#pragma unroll
  for (int i = 0; i < 2; ++i) f1.p[i] = f1.pl[i] = f1.q[i] = f1.ql[i] = (u32x4){0, 0, 0, 0};
  issue(0);
  issue(1);
  if (nk > 1) wait_vm<8>();
  else wait_vm<0>();
  barrier();
  k_step<TILE, TR>(hh, xx, f1, f0, rp, rq);         // the first fragments: products with zeros under the reads
  if constexpr (TILE == 128) {
    for (int i = 0; i < nk; ++i) {
      const int st = (i & 1) * S::STAGE, nx = S::STAGE - st;
      k_step<TILE, TR>(hh, xx, f0, f1, TILE == 128 ? (rp ^ 32) + st : 0, (TR ? rq + NEXT_Q : rq ^ 32) + st);
      wait_vm<0>();         // this wave's part of stage i + 1 is in LDS
      barrier();            // and everyone's; nobody reads stage i any more
      issue(i + 2);
      k_step<TILE, TR>(hh, xx, f1, f0, rp + nx, rq + nx);
    }
  } else {
    for (int i = 0; i < nk; i += 2) {
      wait_vm<0>();
      barrier();
      issue(i + 2);
      k_step<TILE, TR>(hh, xx, f0, f1, rp + S::STAGE, rq + S::STAGE);
      if (i + 1 >= nk) break;
      wait_vm<0>();
      barrier();
      issue(i + 3);
      k_step<TILE, TR>(hh, xx, f1, f0, rp, rq);
    }
  }
  asm volatile("s_nop 15\n s_nop 3" ::: "memory");    // the last products are through before a vector instruction reads the accumulators
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int i = 0; i < 2; ++i) asm volatile("" : "+v"(hh[j][i]), "+v"(xx[j][i]));
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int i = 0; i < 2; ++i) hh[j][i] += xx[j][i];

  // ---- epilogue: through LDS, so that a wave reads and writes whole 16-byte pieces of whole cache lines
  const Shrink shrink = shrink_of(((const float*)(ws + p.shrink))[g.first + at.matrix], step);
  const float poly_b = NS_B * shrink.now * shrink.now, poly_c = NS_C * shrink.now * shrink.now * shrink.now * shrink.now;
  constexpr int PITCH = 68;                             // floats of a row of 64 and room: rows 4 banks apart
  // rows r0 .. of `sums`, which holds the products of rows i0 .. and columns j0 .. j0 + 63: finished and stored; `again`: the finished values
  // go back to `sums`, for the mirrored tile
  auto store_rows = [&](float* sums, int rows, int i0, int j0, bool again) {
    const int seg = (lane & 7) * 8;
#pragma unroll
    for (int r = lane >> 3; r < rows; r += 8) {
      float* from_lds = sums + r * PITCH + seg;
      const float4 lo4 = *(const float4*)from_lds, hi4 = *(const float4*)(from_lds + 4);
      float v[8] = {lo4.x, lo4.y, lo4.z, lo4.w, hi4.x, hi4.y, hi4.z, hi4.w};
      const int ld = MODE == APPLY ? g.np : g.mp;
      const int64_t at_e = (int64_t)(i0 + r) * ld + j0 + seg, pl = MODE == APPLY ? px : pa;
      if (MODE != GRAM) {
        const _Float16* add = (MODE == POLY ? A : X) + at_e;
        const f16x8 h = *(const f16x8*)add, l = *(const f16x8*)(add + pl);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float old = (float)h[k] + (float)l[k];
          v[k] = MODE == POLY ? fmaf(poly_b, old, poly_c * (v[k] * UNSCALE)) : fmaf(NS_A, old, v[k] * UNSCALE) * shrink.ratio;
        }
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] *= UNSCALE;
      }
      if (again) {
        *(float4*)from_lds = make_float4(v[0], v[1], v[2], v[3]);
        *(float4*)(from_lds + 4) = make_float4(v[4], v[5], v[6], v[7]);
      }
      f16x8 h, l;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        _Float16 a, b;
        split(v[k], a, b);
        h[k] = a; l[k] = b;
      }
      _Float16* to = (MODE == GRAM ? A : MODE == POLY ? B : (_Float16*)(ws + g.x[from ^ 1]) + at.matrix * 2 * px) + at_e;
      *(f16x8*)to = h;
      *(f16x8*)(to + pl) = l;
    }
  };
  // columns c0 .. c0 + cols - 1 of `rows` (a multiple of 8) finished rows, as rows of the mirrored tile
  auto store_mirrored = [&](const float* sums, int rows, int i0, int c0, int cols, int j0) {
    const int segs = rows / 8, seg = lane % segs * 8;
    _Float16* D = MODE == GRAM ? A : B;
    for (int c = c0 + lane / segs; c < c0 + cols; c += 64 / segs) {
      f16x8 h, l;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        _Float16 a, b;
        split(sums[(seg + k) * PITCH + c], a, b);
        h[k] = a; l[k] = b;
      }
      _Float16* to = D + (int64_t)(j0 + c) * g.mp + i0 + seg;
      *(f16x8*)to = h;
      *(f16x8*)(to + pa) = l;
    }
  };
  // n of eight elements side by side in the caller's blob, from element e on
  const bool quads = ((g.offset | g.stride | g.ld) & 3) == 0;
  auto store_eight = [&](int64_t e, int n, const float* v) {
    if (quads && n == 8) {
      float w[8];
      if (!t.out) {
        const float4 a = *(const float4*)(t.p + e), b = *(const float4*)(t.p + e + 4);
        const float old[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int k = 0; k < 8; ++k) w[k] = old[k] * t.decay - v[k];
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) w[k] = v[k];
      }
      if (!t.out || t.dt == F32) {
        float* to = (t.out ? (float*)t.out : t.p) + e;
        *(float4*)to = make_float4(w[0], w[1], w[2], w[3]);
        *(float4*)(to + 4) = make_float4(w[4], w[5], w[6], w[7]);
      }
      uint16_t* half = t.out ? t.dt == BF16 ? (uint16_t*)t.out : nullptr : t.shadow;
      if (half) {
        *(uint2*)(half + e) = make_uint2(f32x2_to_bf16x2(w[0], w[1]), f32x2_to_bf16x2(w[2], w[3]));
        *(uint2*)(half + e + 4) = make_uint2(f32x2_to_bf16x2(w[4], w[5]), f32x2_to_bf16x2(w[6], w[7]));
      }
      return;
    }
    float w[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) w[k] = !t.out && k < n ? t.p[e + k] : 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if (k >= n) continue;
      if (t.out) {
        st_f(t.out, (size_t)(e + k), v[k], t.dt);
      } else {
        w[k] = w[k] * t.decay - v[k];
        t.p[e + k] = w[k];
        if (t.shadow) t.shadow[e + k] = f32_to_bf16(w[k]);
      }
    }
  };
  // the result: rows r0 .. of `sums`; where the matrix is tall the caller's rows are columns of `sums`
  auto store_result = [&](float* sums, int r0, int rows, int i0, int j0) {
    const float scale = UNSCALE * shrink.next * (t.out ? 1.f : 0.2f * t.lr * sqrtf((float)g.n));
    const int seg = (lane & 7) * 8;
    for (int r = r0 + (lane >> 3); r < r0 + rows; r += 8) {
      float* from_lds = sums + r * PITCH + seg;
      const float4 lo4 = *(const float4*)from_lds, hi4 = *(const float4*)(from_lds + 4);
      float v[8] = {lo4.x, lo4.y, lo4.z, lo4.w, hi4.x, hi4.y, hi4.z, hi4.w};
      const _Float16* add = X + (int64_t)(i0 + r) * g.np + j0 + seg;
      const f16x8 h = *(const f16x8*)add, l = *(const f16x8*)(add + px);
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = fmaf(NS_A, (float)h[k] + (float)l[k], v[k] * UNSCALE) * shrink.ratio * scale;
      if (!g.tall) {
        if (i0 + r < g.m && j0 + seg < g.n) store_eight(element(g, at.matrix, i0 + r, j0 + seg), min(8, g.n - j0 - seg), v);
      } else {
        *(float4*)from_lds = make_float4(v[0], v[1], v[2], v[3]);
        *(float4*)(from_lds + 4) = make_float4(v[4], v[5], v[6], v[7]);
      }
    }
    if (!g.tall) return;
    wave_sync();
    const int segs = rows / 8, i = i0 + r0 + lane % segs * 8;
    for (int c = lane / segs; c < 64; c += 64 / segs) {
      float v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = sums[(r0 + lane % segs * 8 + k) * PITCH + c];
      if (i < g.m && j0 + c < g.n) store_eight(element(g, at.matrix, j0 + c, i), min(8, g.m - i), v);
    }
  };
  // a 32 x 32 tile of sums: lane l holds row l % 32, columns 8 q + 4 (l / 32) + e in element 4 q + e
  auto put = [&](float* sums, const f32x16& acc, int r0, int c0) {
#pragma unroll
    for (int q = 0; q < 4; ++q)
      *(float4*)(sums + (r0 + (lane & 31)) * PITCH + c0 + 8 * q + 4 * (lane >> 5)) =
          make_float4(acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]);
  };
  barrier();                                            // nobody reads a stage any more
  if constexpr (TILE == 128) {
    // 32 rows at a time, in a part of LDS of the wave's own; what lies past the padded size (a multiple of 64) is not stored
    float* sums = (float*)stages + wave * 32 * PITCH;
    const int i0 = bi * 128 + wi * 64, j0 = bj * 128 + wj * 64;
    if (i0 >= g.mp || j0 >= (MODE <= POLY ? g.mp : g.np)) return;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      wave_sync();
      put(sums, hh[0][i], 0, 0);
      put(sums, hh[1][i], 0, 32);
      wave_sync();
      if (MODE == LAST) {
        store_result(sums, 0, 32, i0 + 32 * i, j0);
      } else {
        store_rows(sums, 32, i0 + 32 * i, j0, MODE <= POLY && bi != bj);
        if (MODE <= POLY && bi != bj) {
          wave_sync();
          store_mirrored(sums, 32, i0 + 32 * i, 0, 64, j0);
        }
      }
    }
  } else {
    // the four waves' sums: each adds up the 32 x 32 tile of its number and finishes 16 rows of the whole
    float4* quarters = (float4*)stages;                 // [wave][tile][q][lane]
    float* sums = (float*)stages;
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x16& v = hh[k >> 1][k & 1];
        quarters[((wave * 4 + k) * 4 + q) * 64 + lane] = make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
      }
    __syncthreads();
    f32x16 acc;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      float4 a = quarters[(wave * 4 + q) * 64 + lane];
#pragma unroll
      for (int w = 1; w < 4; ++w) {
        const float4 b = quarters[((w * 4 + wave) * 4 + q) * 64 + lane];
        a.x += b.x; a.y += b.y; a.z += b.z; a.w += b.w;
      }
      acc[4 * q] = a.x; acc[4 * q + 1] = a.y; acc[4 * q + 2] = a.z; acc[4 * q + 3] = a.w;
    }
    __syncthreads();
    put(sums, acc, (wave & 1) * 32, (wave >> 1) * 32);
    __syncthreads();
    if (MODE == LAST) {
      store_result(sums, wave * 16, 16, bi * 64, bj * 64);
    } else {
      store_rows(sums + wave * 16 * PITCH, 16, bi * 64 + wave * 16, bj * 64, MODE <= POLY && bi != bj);
      if (MODE <= POLY && bi != bj) {
        __syncthreads();
        store_mirrored(sums, 64, bi * 64, wave * 16, 16, bj * 64);
      }
    }
  }
}
#undef NS_MMA
#undef NS_ACC
#undef NS_CUR
#undef NS_CROSS

// ------------------------------------------------------------------ small matrices
// All steps of one matrix in one workgroup of 16 waves: X and A (then B in its place) stay in LDS as planes, rows 16 bytes longer than their
// elements so that 16 rows' pieces meet no bank twice.  A wave multiplies 16 x 16 tiles (v_mfma_f32_16x16x32_f16) of up to NT turns; results
// wait in registers until everyone has read what they replace.  Bound by the chain of barriers and LDS reads: 64 x 64 takes some 2 us a step, where
// the three launches of the tiled kernels take 15.
typedef __attribute__((ext_vector_type(4))) float f32x4;
constexpr int SMALL_TURNS = (ORTHO_SMALL_ELEMENTS / 256 + 15) / 16;      // tiles of the largest X for each wave
constexpr int SMALL_THREADS = 1024, SMALL_WAVES = SMALL_THREADS / 64;
typedef __attribute__((ext_vector_type(4))) short i16x4;
// Four rows of 16 elements, an 8-byte piece from each of 16 lanes: each lane receives the four elements of its column.
__device__ __forceinline__ f16x4 read_columns(const _Float16* from) {
  return __builtin_bit_cast(f16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)from));
}
template <int NT> __global__ __launch_bounds__(SMALL_THREADS) void small_kernel(OrthoPlan p, Source src, Target t, int steps) {
  extern __shared__ __align__(16) char stages[];
  __shared__ double sums[SMALL_WAVES];
  int id = blockIdx.x;
  const Place at = place_of(p, id, [](const OrthoGroup& g) { return g.small ? 1 : 0; });
  const OrthoGroup& g = p.g[at.group];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lx = g.np + 8, la = g.mp + 8, px = g.mp * lx, pa = g.mp * la;      // row lengths and planes, in halves
  _Float16 *X = (_Float16*)stages, *A = X + 2 * px;
  for (int k = tid; k < (2 * px + 2 * pa) / 8; k += SMALL_THREADS) ((f16x8*)stages)[k] = f16x8{};
  // ---- momentum, norm, X
  const int all = g.rows * g.cols;
  const float per = 1.f / g.cols;
  auto place = [&](int e, int& r, int& c) { r = (int)(((float)e + 0.5f) * per); c = e - r * g.cols; };     // exact: e < 2^16
  double sum = 0;
  for (int e0 = tid; e0 < all; e0 += 4 * SMALL_THREADS) {
    float u[4], m[4];
    int64_t el[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int e = e0 + k * SMALL_THREADS;
      int r, c;
      place(e, r, c);
      el[k] = e < all ? element(g, at.matrix, r, c) : -1;
      u[k] = el[k] < 0 ? 0.f : src.in ? ld_f(src.in, (size_t)el[k], src.dt) : src.g[el[k]];
      m[k] = el[k] >= 0 && !src.in ? src.m[el[k]] : 0.f;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (!src.in) {
        m[k] = fmaf(src.momentum, m[k], u[k]);
        if (el[k] >= 0) src.m[el[k]] = m[k];
        u[k] = src.nesterov ? fmaf(src.momentum, m[k], u[k]) : m[k];
      }
      sum += (double)u[k] * u[k];
    }
  }
  for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
  if (lane == 0) sums[wave] = sum;
  __syncthreads();
  sum = 0;
  for (int w = 0; w < SMALL_WAVES; ++w) sum += sums[w];
  const double norm = sqrt(sum), inv = norm > 0 ? SCALE / norm : norm;
  const float t0 = (float)(norm / (norm + NORM_EPS));
  for (int e0 = tid; e0 < all; e0 += 4 * SMALL_THREADS) {
    float u[4];
    int r[4], c[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int e = e0 + k * SMALL_THREADS;
      place(e, r[k], c[k]);
      u[k] = e < all ? read_u(src, element(g, at.matrix, r[k], c[k])) : 0.f;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (e0 + k * SMALL_THREADS >= all) continue;
      _Float16* to = X + (g.tall ? c[k] * lx + r[k] : r[k] * lx + c[k]);
      split((float)(u[k] * inv), to[0], to[px]);
    }
  }
  __syncthreads();

  // ---- tile `n` of a product of `across` tiles a row: P rows i0 .., Q rows j0 .. (or columns of X) over K; lane l: row l % 16, columns
  // 4 (l / 16) + e of the tile in element e
  const int row = lane & 15, kpart = 8 * (lane >> 4);
  auto rows_product = [&](const _Float16* P, int ld, int plane, int i0, int j0, int K) {
    f32x4 hh = {}, xx = {};
    const _Float16 *pr = P + (i0 + row) * ld + kpart, *qr = P + (j0 + row) * ld + kpart;
    for (int k = 0; k < K; k += 32) {
      const f16x8 ph = *(const f16x8*)(pr + k), pl = *(const f16x8*)(pr + plane + k), qh = *(const f16x8*)(qr + k), ql = *(const f16x8*)(qr + plane + k);
      hh = __builtin_amdgcn_mfma_f32_16x16x32_f16(qh, ph, hh, 0, 0, 0);
      xx = __builtin_amdgcn_mfma_f32_16x16x32_f16(ql, ph, xx, 0, 0, 0);
      xx = __builtin_amdgcn_mfma_f32_16x16x32_f16(qh, pl, xx, 0, 0, 0);
    }
    return hh + xx;
  };
  auto columns_product = [&](const _Float16* B, int i0, int j0) {
    f32x4 hh = {}, xx = {};
    const _Float16 *pr = B + (i0 + row) * la + kpart, *qr = X + (kpart + (row >> 2)) * lx + j0 + 4 * (row & 3);
    for (int k = 0; k < g.mp; k += 32) {
      const f16x8 ph = *(const f16x8*)(pr + k), pl = *(const f16x8*)(pr + pa + k);
      f16x8 q[2];
#pragma unroll
      for (int pl2 = 0; pl2 < 2; ++pl2) {
        const _Float16* from = qr + pl2 * px + k * lx;
        const f16x4 a = read_columns(from), b = read_columns(from + 4 * lx);
        q[pl2] = f16x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
      }
      hh = __builtin_amdgcn_mfma_f32_16x16x32_f16(q[0], ph, hh, 0, 0, 0);
      xx = __builtin_amdgcn_mfma_f32_16x16x32_f16(q[1], ph, xx, 0, 0, 0);
      xx = __builtin_amdgcn_mfma_f32_16x16x32_f16(q[0], pl, xx, 0, 0, 0);
    }
    return hh + xx;
  };
  const int ta = g.mp / 16, tx = g.np / 16;
  f32x4 held[NT];
  // every tile of this wave: f(turn, i0, j0)
  auto tiles = [&](int across, auto f) {
    int first = wave;
    if (NT > 3) asm volatile("" : "+s"(first));     // addresses of all turns, kept from step to step, would not fit into the registers
#pragma unroll
    for (int k = 0; k < NT; ++k) {
      const int n = first + k * SMALL_WAVES;
      if (n < ta * across) f(k, n / across * 16, n % across * 16);
      if (NT > 3) __builtin_amdgcn_sched_barrier(0);     // the turns' fragments do not fit into the registers together
    }
  };
  auto add_old = [&](const _Float16* from, int plane, f32x4 v, float old_by, float by, float ratio) {
    const f16x4 h = *(const f16x4*)from, l = *(const f16x4*)(from + plane);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = fmaf(old_by, (float)h[e] + (float)l[e], by * (v[e] * UNSCALE)) * ratio;
    return v;
  };
  auto put = [&](_Float16* to, int plane, f32x4 v) {
    f16x4 h, l;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      _Float16 a, b;
      split(v[e], a, b);
      h[e] = a; l[e] = b;
    }
    *(f16x4*)to = h;
    *(f16x4*)(to + plane) = l;
  };
  const int col = 4 * (lane >> 4);
  for (int k = 0; k < steps; ++k) {
    const Shrink shrink = shrink_of(t0, k);
    const float t2 = shrink.now * shrink.now;
    tiles(ta, [&](int, int i0, int j0) { put(A + (i0 + row) * la + j0 + col, pa, rows_product(X, lx, px, i0, j0, g.np) * UNSCALE); });
    __syncthreads();
    tiles(ta, [&](int n, int i0, int j0) {
      held[n] = add_old(A + (i0 + row) * la + j0 + col, pa, rows_product(A, la, pa, i0, j0, g.mp), NS_B * t2, NS_C * t2 * t2, 1.f);
    });
    __syncthreads();
    tiles(ta, [&](int n, int i0, int j0) { put(A + (i0 + row) * la + j0 + col, pa, held[n]); });
    __syncthreads();
    tiles(tx, [&](int n, int i0, int j0) {
      held[n] = add_old(X + (i0 + row) * lx + j0 + col, px, columns_product(A, i0, j0), NS_A, 1.f, shrink.ratio);
    });
    if (k + 1 == steps) break;
    __syncthreads();
    tiles(tx, [&](int n, int i0, int j0) { put(X + (i0 + row) * lx + j0 + col, px, held[n]); });
    __syncthreads();
  }
  const float scale = UNSCALE * shrink_of(t0, steps - 1).next * (t.out ? 1.f : 0.2f * t.lr * sqrtf((float)g.n));
  tiles(tx, [&](int n, int i0, int j0) {
    const int i = i0 + row;
    int64_t el[4];
    float w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int j = j0 + col + e;
      el[e] = i >= g.m || j >= g.n ? -1 : g.tall ? element(g, at.matrix, j, i) : element(g, at.matrix, i, j);
      w[e] = !t.out && el[e] >= 0 ? t.p[el[e]] : 0.f;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (el[e] < 0) continue;
      if (t.out) {
        st_f(t.out, (size_t)el[e], held[n][e] * scale, t.dt);
      } else {
        w[e] = w[e] * t.decay - held[n][e] * scale;
        t.p[el[e]] = w[e];
        if (t.shadow) t.shadow[el[e]] = f32_to_bf16(w[e]);
      }
    }
  });
}
template <int NT> int launch_small(hipStream_t s, const OrthoPlan& p, const Source& src, const Target& dst, int steps, int matrices, int lds) {
  static OncePerDevice once;
  PPLL_TRY(raise_lds((const void*)small_kernel<NT>, ORTHO_SMALL_LDS, once));
  hipLaunchKernelGGL((small_kernel<NT>), dim3(matrices), dim3(SMALL_THREADS), lds, s, p, src, dst, steps);
  PPLL_HIP(hipGetLastError());
  return PPLL_OK;
}

template <int MODE> int launch_product(hipStream_t s, const OrthoPlan& p, const Target& t, char* ws, int step) {
  const int phase = MODE < APPLY ? MODE : APPLY, tile = p.tile[phase];
  const XcdShares& shares = p.shares[phase];
  int longest = 0;
  for (int x = 0; x < 8; ++x) longest = shares.first[x + 1] - shares.first[x] > longest ? shares.first[x + 1] - shares.first[x] : longest;
  const dim3 grid(8 * (unsigned)longest);
  if (tile == 128) hipLaunchKernelGGL((product_kernel<128, MODE>), grid, dim3(256), Tile<128>::LDS, s, p, shares, t, ws, step);
  else hipLaunchKernelGGL((product_kernel<64, MODE>), grid, dim3(256), Tile<64>::LDS, s, p, shares, t, ws, step);
  PPLL_HIP(hipGetLastError());
  return PPLL_OK;
}

int run(hipStream_t s, const OrthoPlan& p, const Source& src, const Target& dst, int steps, char* ws) {
  int64_t pieces = 0, squares = 0;
  int small = 0, tiles = 0, lds = 0;
  for (int k = 0; k < p.n; ++k) {
    const OrthoGroup& g = p.g[k];
    if (g.small) {
      small += g.count;
      tiles = g.mp / 16 * (g.np / 16) > tiles ? g.mp / 16 * (g.np / 16) : tiles;
      lds = (int)g.small_lds() > lds ? (int)g.small_lds() : lds;
    } else {
      pieces += (int64_t)g.count * g.pieces();
      squares += (int64_t)g.count * (g.mp / 64) * (g.np / 64);
    }
  }
  if (small) {
    const int turns = (tiles + SMALL_WAVES - 1) / SMALL_WAVES;
    if (turns <= 1) PPLL_TRY(launch_small<1>(s, p, src, dst, steps, small, lds));
    else if (turns <= 3) PPLL_TRY(launch_small<3>(s, p, src, dst, steps, small, lds));
    else PPLL_TRY(launch_small<SMALL_TURNS>(s, p, src, dst, steps, small, lds));
  }
  if (!pieces) return PPLL_OK;
  hipLaunchKernelGGL(squares_kernel, dim3((unsigned)pieces), dim3(256), 0, s, p, src, ws);
  PPLL_HIP(hipGetLastError());
  hipLaunchKernelGGL(normalise_kernel, dim3((unsigned)squares), dim3(256), 0, s, p, src, ws);
  PPLL_HIP(hipGetLastError());
  for (int k = 0; k < steps; ++k) {
    PPLL_TRY(launch_product<GRAM>(s, p, dst, ws, k));
    PPLL_TRY(launch_product<POLY>(s, p, dst, ws, k));
    if (k + 1 < steps) PPLL_TRY(launch_product<APPLY>(s, p, dst, ws, k));
    else PPLL_TRY(launch_product<LAST>(s, p, dst, ws, k));
  }
  return PPLL_OK;
}
}  // namespace

int launch_orthogonalize(hipStream_t s, const OrthoPlan& p, int dt, int steps, const void* in, void* out, char* ws) {
  return run(s, p, Source{in, dt, nullptr, nullptr, 0.f, 0}, Target{out, dt, nullptr, nullptr, 0.f, 0.f}, steps, ws);
}
int launch_muon(hipStream_t s, const OrthoPlan& p, int steps, const float* g, float* m, float* w, uint16_t* shadow, float lr, float momentum,
                int nesterov, float weight_decay, char* ws) {
  return run(s, p, Source{nullptr, F32, g, m, momentum, nesterov}, Target{nullptr, F32, w, shadow, lr, 1.f - lr * weight_decay}, steps, ws);
}

}  // namespace ppll
