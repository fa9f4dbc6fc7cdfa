// Newton-Schulz orthogonalisation of batches of matrices and the Muon step around it.
#include "common.h"
#include "ortho.h"

#include <math.h>

namespace ppll {

namespace {
typedef __attribute__((ext_vector_type(16))) float f32x16;
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

enum { GRAM = 0, POLY = 1, APPLY = 2, LAST = 3 };

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
    const int e = each(p.g[k]), all = e * p.g[k].count;
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
  const Place at = place_of(p, id, [](const OrthoGroup& g) { return g.pieces(); });
  const OrthoGroup& g = p.g[at.group];
  const int across = (g.cols + NORM_COLS - 1) / NORM_COLS, r0 = id / across * NORM_ROWS, c = id % across * NORM_COLS + threadIdx.x;
  double sum = 0;
  if (c < g.cols)
    for (int r = r0; r < min(r0 + NORM_ROWS, g.rows); ++r) {
      const int64_t e = element(g, at.matrix, r, c);
      if (!s.in) s.m[e] = fmaf(s.momentum, s.m[e], s.g[e]);
      const double u = read_u(s, e);
      sum += u * u;
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

// Y = u / |u| and its transpose, in tiles of 64 x 64.
__global__ __launch_bounds__(256) void normalise_kernel(OrthoPlan p, Source s, char* ws) {
  int id = blockIdx.x;
  const Place at = place_of(p, id, [](const OrthoGroup& g) { return (g.mp / 64) * (g.np / 64); });
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
  _Float16* x = (_Float16*)(ws + g.x) + at.matrix * 2 * plane;
  _Float16* xt = (_Float16*)(ws + g.xt[0]) + at.matrix * 2 * plane;
  const int y = t / 4, q = t % 4 * 16;
  f16x8 h[2], l[2];
  for (int k = 0; k < 16; ++k) {
    _Float16 a, b;
    split(tile[y][q + k], a, b);
    h[k / 8][k % 8] = a; l[k / 8][k % 8] = b;
  }
  _Float16* to = x + (int64_t)(i0 + y) * g.np + j0 + q;
  for (int k = 0; k < 2; ++k) { *(f16x8*)(to + 8 * k) = h[k]; *(f16x8*)(to + plane + 8 * k) = l[k]; }
  for (int k = 0; k < 16; ++k) {
    _Float16 a, b;
    split(tile[q + k][y], a, b);
    h[k / 8][k % 8] = a; l[k / 8][k % 8] = b;
  }
  to = xt + (int64_t)(j0 + y) * g.mp + i0 + q;
  for (int k = 0; k < 2; ++k) { *(f16x8*)(to + 8 * k) = h[k]; *(f16x8*)(to + plane + 8 * k) = l[k]; }
}

// C[i][j] = sum over k of P[i][k] Q[j][k]:
//  GRAM   P = Q = X        A = C                        symmetric: tiles on and under the diagonal, each stored twice
//  POLY   P = Q = A        B = b A + c C                likewise
//  APPLY  P = B, Q = X^T   X = a X + C and X^T          (X^T in two buffers in turn: other tiles still read the old one)
//  LAST   the same, to where the result goes
template <int TILE, int MODE> __global__ __launch_bounds__(256) void product_kernel(OrthoPlan p, Target t, char* ws, int step) {
  constexpr int BK = 32, IM = TILE / 64, OPERAND = TILE * BK * 2;      // bytes of a plane's rows
  __shared__ __align__(16) char lds[4 * OPERAND];
  int id = blockIdx.x;
  const Place at = place_of(p, id, [](const OrthoGroup& g) {
    const int a = g.mp / TILE;
    return MODE <= POLY ? a * (a + 1) / 2 : a * (g.np / TILE);
  });
  const OrthoGroup& g = p.g[at.group];
  int bi, bj;
  if (MODE <= POLY) {
    bi = (int)((sqrtf(8.f * id + 1.f) - 1.f) * 0.5f);
    while ((bi + 1) * (bi + 2) / 2 <= id) ++bi;
    while (bi * (bi + 1) / 2 > id) --bi;
    bj = id - bi * (bi + 1) / 2;
  } else {
    const int across = g.np / TILE;
    bi = id / across; bj = id % across;
  }
  const int64_t px = g.plane_x(), pa = g.plane_a();
  const int from = step & 1;
  const Shrink shrink = shrink_of(((const float*)(ws + p.shrink))[g.first + at.matrix], step);
  const float poly_b = NS_B * shrink.now * shrink.now, poly_c = NS_C * shrink.now * shrink.now * shrink.now * shrink.now;
  _Float16* X = (_Float16*)(ws + g.x) + at.matrix * 2 * px;
  _Float16* XT = (_Float16*)(ws + g.xt[from]) + at.matrix * 2 * px;
  _Float16* XN = (_Float16*)(ws + g.xt[from ^ 1]) + at.matrix * 2 * px;
  _Float16* A = (_Float16*)(ws + g.a) + at.matrix * 2 * pa;
  _Float16* B = (_Float16*)(ws + g.b) + at.matrix * 2 * pa;
  const _Float16* P = MODE == GRAM ? X : MODE == POLY ? A : B;
  const _Float16* Q = MODE == GRAM ? X : MODE == POLY ? A : XT;
  const int64_t plane_p = MODE == GRAM ? px : pa, plane_q = MODE == POLY ? pa : px;
  const int K = MODE == GRAM ? g.np : g.mp;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wi = wave >> 1, wj = wave & 1;
  f32x16 acc[IM][IM] = {}, cross[IM][IM] = {};
  // rows of 32 k, 64 bytes; the 16-byte granule q of row r sits at q ^ (r / 4 % 4)
  for (int k0 = 0; k0 < K; k0 += BK) {
    __syncthreads();
    for (int c = tid; c < TILE * 4; c += 256) {
      const int r = c >> 2, q = c & 3, to = r * 64 + ((q ^ (r >> 2 & 3)) << 4);
      const int64_t fp = (int64_t)(bi * TILE + r) * K + k0 + q * 8, fq = (int64_t)(bj * TILE + r) * K + k0 + q * 8;
      *(f16x8*)(lds + to) = *(const f16x8*)(P + fp);
      *(f16x8*)(lds + OPERAND + to) = *(const f16x8*)(P + plane_p + fp);
      *(f16x8*)(lds + 2 * OPERAND + to) = *(const f16x8*)(Q + fq);
      *(f16x8*)(lds + 3 * OPERAND + to) = *(const f16x8*)(Q + plane_q + fq);
    }
    __syncthreads();
    for (int kk = 0; kk < 2; ++kk) {
      f16x8 ph[IM], pl[IM], qh[IM], ql[IM];
      for (int i = 0; i < IM; ++i) {
        const int q = kk * 2 + (lane >> 5), rp = (wi * IM + i) * 32 + (lane & 31), rq = (wj * IM + i) * 32 + (lane & 31);
        const int fp = rp * 64 + ((q ^ (rp >> 2 & 3)) << 4), fq = rq * 64 + ((q ^ (rq >> 2 & 3)) << 4);
        ph[i] = *(const f16x8*)(lds + fp); pl[i] = *(const f16x8*)(lds + OPERAND + fp);
        qh[i] = *(const f16x8*)(lds + 2 * OPERAND + fq); ql[i] = *(const f16x8*)(lds + 3 * OPERAND + fq);
      }
      for (int i = 0; i < IM; ++i)
        for (int j = 0; j < IM; ++j) {
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(ph[i], qh[j], acc[i][j], 0, 0, 0);
          cross[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(ph[i], ql[j], cross[i][j], 0, 0, 0);
          cross[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(pl[i], qh[j], cross[i][j], 0, 0, 0);
        }
    }
  }
  // lane: column j, rows 8 (r / 4) + 4 (lane / 32) + r % 4 of a 32 x 32 tile
  for (int ii = 0; ii < IM; ++ii)
    for (int jj = 0; jj < IM; ++jj)
      for (int r4 = 0; r4 < 4; ++r4) {
        const int i = bi * TILE + (wi * IM + ii) * 32 + r4 * 8 + 4 * (lane >> 5), j = bj * TILE + (wj * IM + jj) * 32 + (lane & 31);
        float v[4];
        for (int k = 0; k < 4; ++k) v[k] = (acc[ii][jj][r4 * 4 + k] + cross[ii][jj][r4 * 4 + k]) * UNSCALE;
        if (MODE != GRAM) {
          // A is symmetric, X^T holds X: four neighbours of a column are four of a row there
          const _Float16* add = (MODE == POLY ? A : XT) + (int64_t)j * g.mp + i;
          const f16x4 h = *(const f16x4*)add, l = *(const f16x4*)(add + (MODE == POLY ? pa : px));
          for (int k = 0; k < 4; ++k) {
            const float old = (float)h[k] + (float)l[k];
            v[k] = MODE == POLY ? fmaf(poly_b, old, poly_c * v[k]) : fmaf(NS_A, old, v[k]) * shrink.ratio;
          }
        }
        if (MODE == LAST) {
          const float scale = UNSCALE * shrink.next * (t.out ? 1.f : 0.2f * t.lr * sqrtf((float)g.n));
          for (int k = 0; k < 4; ++k) {
            if (i + k >= g.m || j >= g.n) continue;
            const int64_t e = g.tall ? element(g, at.matrix, j, i + k) : element(g, at.matrix, i + k, j);
            if (t.out) {
              st_f(t.out, (size_t)e, v[k] * scale, t.dt);
            } else {
              const float w = t.p[e] * t.decay - v[k] * scale;
              t.p[e] = w;
              if (t.shadow) t.shadow[e] = f32_to_bf16(w);
            }
          }
          continue;
        }
        f16x4 h, l;
        for (int k = 0; k < 4; ++k) {
          _Float16 a, b;
          split(v[k], a, b);
          h[k] = a; l[k] = b;
        }
        _Float16* D = MODE == GRAM ? A : MODE == POLY ? B : X;
        _Float16* DT = MODE == GRAM ? A : MODE == POLY ? B : XN;
        const int64_t plane = MODE <= POLY ? pa : px;
        const int ld = MODE <= POLY ? g.mp : g.np;
        for (int k = 0; k < 4; ++k) {
          D[(int64_t)(i + k) * ld + j] = h[k];
          D[plane + (int64_t)(i + k) * ld + j] = l[k];
        }
        if (MODE == APPLY || bi != bj) {
          *(f16x4*)(DT + (int64_t)j * g.mp + i) = h;
          *(f16x4*)(DT + plane + (int64_t)j * g.mp + i) = l;
        }
      }
}

int64_t tiles(const OrthoPlan& p, int mode) {
  int64_t n = 0;
  for (int k = 0; k < p.n; ++k) {
    const int64_t a = p.g[k].mp / p.tile, b = p.g[k].np / p.tile;
    n += p.g[k].count * (mode <= POLY ? a * (a + 1) / 2 : a * b);
  }
  return n;
}
template <int MODE> int launch_product(hipStream_t s, const OrthoPlan& p, const Target& t, char* ws, int step) {
  const dim3 grid((unsigned)tiles(p, MODE));
  if (p.tile == 128) hipLaunchKernelGGL((product_kernel<128, MODE>), grid, dim3(256), 0, s, p, t, ws, step);
  else hipLaunchKernelGGL((product_kernel<64, MODE>), grid, dim3(256), 0, s, p, t, ws, step);
  PPLL_HIP(hipGetLastError());
  return PPLL_OK;
}

int run(hipStream_t s, const OrthoPlan& p, const Source& src, const Target& dst, int steps, char* ws) {
  if (!p.n) return PPLL_OK;
  int64_t pieces = 0, squares = 0;
  for (int k = 0; k < p.n; ++k) {
    pieces += (int64_t)p.g[k].count * p.g[k].pieces();
    squares += (int64_t)p.g[k].count * (p.g[k].mp / 64) * (p.g[k].np / 64);
  }
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
