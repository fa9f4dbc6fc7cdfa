// Newton-Schulz orthogonalisation of batches of matrices and the Muon step around it.
#include "common.h"
#include "gemm_pipe.h"
#include "ortho.h"

#include <math.h>
#include <type_traits>

namespace ppll {

namespace {
using pipe::barrier;
using pipe::f32x16;
using pipe::lds_char;
using pipe::u32x2;
using pipe::u32x4;
using pipe::wait_vm;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) _Float16 f16x4;

constexpr float NS_A = 3.4445f, NS_B = -4.7750f, NS_C = 2.0315f;
constexpr double NORM_EPS = 1e-7;
// Operands are stored as hi + lo / 2048, two fp16 of a value times 2^14: 22 bits, and the products hi hi + (hi lo + lo hi) / 2048 leave lo lo out,
// 2^-22 of a product at most.  Fewer bits than fp32's 24 at the worst, chosen because three fp16 products take 40 % of an fp32 one's time (1160 and 154
// TFLOP/s in large library products): in the mean what is stored and what is left out are each off by about a rounding of fp32 (errors beside those of
// fp32 products: 1.4 times for one step of a random matrix, level after five).  lo is kept 2^11 times as large as what it stands for, about as large as
// hi, so a value beside a norm of 1 has its 22 bits down to 2^-28 and is off by 2^-50 under that.  (With lo as it is, a row of 1e-6 beside others of 1
// came out with errors of 6e-4 of itself, now 4e-7.)  Neither can overflow: singular values are 1.2023 at most (the polynomial's maximum on [0, 1.2023]),
// so entries are 1.2023 at most for X, 1.446 for A, and b A + c A A has eigenvalues from -2.81 to 0: 46000 times 1, of 65504; lo is 2048 times half a unit
// of that hi's last place, 32768.
constexpr double SCALE = 16384;
constexpr float UNSCALE = 1.f / 16384.f;
constexpr float LOW = 2048.f, UNLOW = 1.f / 2048.f;

// The operands are scaled to a Frobenius norm of exactly 1 at the start, and what X is smaller by, t0 = |u| / (|u| + 1e-7), enters as a
// factor: X = t Y with t = min(1, a^k t0) in step k, so Y' = t / t' (a Y + (b t^2 Y Y' + c t^4 (Y Y')^2) Y).  Unless a matrix is as small as
// the constant this is t = 1; one of norm 1e-20, whose X is of norm 1e-13, would be lost in fp16 otherwise.
struct Shrink { float now, next, ratio; };
__device__ __forceinline__ Shrink shrink_from(float t) {
  Shrink s{t, fminf(1.f, NS_A * t), 1.f};
  if (t > 0.f && t < 1.f) s.ratio = t / s.next;
  return s;
}
__device__ __forceinline__ Shrink shrink_of(float t0, int step) {
  float t = t0;
  for (int k = 0; k < step; ++k) t = fminf(1.f, NS_A * t);
  return shrink_from(t);
}

constexpr int GRAM = ORTHO_GRAM, POLY = ORTHO_POLY, APPLY = ORTHO_APPLY, LAST = ORTHO_APPLY + 1;

// What a call works on.  in: blob of the matrices (orthogonalize), or null: u from g and the momentum (Muon step)
struct Source { const void* in; int dt; const float* g; float* m; float momentum; int nesterov; };
// Where the result goes: out (orthogonalize), or null: the parameters
struct Target { void* out; int dt; float* p; uint16_t* shadow; float lr, decay; };

// hi and lo of n values: two values to hi in one instruction, and each lo = 2048 value - 2048 hi, rounded once, in one mixed-precision instruction that
// reads hi as it was stored.  (Left to the compiler, the arithmetic that gives a value may be folded into one of two conversions and not into the other,
// and at a tie hi and what lo is counted from are two neighbours: one element in some 20000 was off by a whole step of hi, 2^-11 of it.)
template <int N> struct Terms { _Float16 __attribute__((ext_vector_type(N))) hi, lo; };
template <int N> __device__ __forceinline__ Terms<N> split_all(const float* v) {
  typedef __attribute__((ext_vector_type(N / 2))) uint32_t words;
  words hi, lo;
#pragma unroll
  for (int k = 0; k < N / 2; ++k) {
    uint32_t h, l;
    asm("v_cvt_pk_f16_f32 %0, %1, %2" : "=v"(h) : "v"(v[2 * k]), "v"(v[2 * k + 1]));
    asm("v_fma_mixlo_f16 %0, %1, %3, %2 op_sel_hi:[1,0,0]" : "=v"(l) : "v"(h), "v"(v[2 * k] * LOW), "s"(-LOW));
    asm("v_fma_mixhi_f16 %0, %1, %3, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "+v"(l) : "v"(h), "v"(v[2 * k + 1] * LOW), "s"(-LOW));
    hi[k] = h; lo[k] = l;
  }
  return {__builtin_bit_cast(decltype(Terms<N>::hi), hi), __builtin_bit_cast(decltype(Terms<N>::lo), lo)};
}
// v[0] and v[1] plus `by` times the two values whose terms the words hold: two mixed-precision instructions a value
__device__ __forceinline__ void add_two(float* v, uint32_t hi, uint32_t lo, float by) {
  asm("v_fma_mix_f32 %0, %1, %2, %0 op_sel_hi:[1,0,0]" : "+v"(v[0]) : "v"(lo), "v"(by * UNLOW));
  asm("v_fma_mix_f32 %0, %1, %2, %0 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "+v"(v[1]) : "v"(lo), "v"(by * UNLOW));
  asm("v_fma_mix_f32 %0, %1, %2, %0 op_sel_hi:[1,0,0]" : "+v"(v[0]) : "v"(hi), "v"(by));
  asm("v_fma_mix_f32 %0, %1, %2, %0 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "+v"(v[1]) : "v"(hi), "v"(by));
}
// a / b for a >= 0, b > 0 and a quotient under 2^21 (tiles of a side, matrices of a group): in fp32 it is off by less than one
__device__ __forceinline__ int quotient(int a, int b) {
  int q = (int)((float)a * __builtin_amdgcn_rcpf((float)b));
  const int r = a - q * b;
  return r < 0 ? q - 1 : r >= b ? q + 1 : q;
}
__device__ __forceinline__ bool in_quads(const OrthoGroup& g) { return ((g.offset | g.stride | g.ld) & 3) == 0; }   // rows' pieces of four are aligned
__device__ __forceinline__ int64_t element(const OrthoGroup& g, int matrix, int r, int c) {
  return g.offset + (int64_t)matrix * g.stride + (int64_t)r * g.ld + c;
}
// The group that work item `id` of a launch belongs to; id becomes the place within the group.  All bounds are read at once: arguments lie in
// memory, and a search that reads them group by group made each launch of a small batch half a microsecond longer (five steps of five 201 x 333
// matrices 136.7 us, 129.2 with two batches of loads, of the bounds and of the group).
__device__ __forceinline__ int group_of(const int32_t (&begin)[ORTHO_GROUPS], int& id) {
  static_assert(ORTHO_GROUPS == 16, "");
  asm volatile("" ::"s"(begin[1]), "s"(begin[2]), "s"(begin[3]), "s"(begin[4]), "s"(begin[5]), "s"(begin[6]), "s"(begin[7]), "s"(begin[8]),
               "s"(begin[9]), "s"(begin[10]), "s"(begin[11]), "s"(begin[12]), "s"(begin[13]), "s"(begin[14]), "s"(begin[15]));
  int group = 0, from = 0;
#pragma unroll
  for (int k = 1; k < ORTHO_GROUPS; ++k)
    if (id >= begin[k]) { group = k; from = begin[k]; }
  id -= from;
  return group;
}
__device__ __forceinline__ float read_u(const Source& s, int64_t at) {
  if (s.in) return ld_f(s.in, (size_t)at, s.dt);
  const float m = s.m[at];
  return s.nesterov ? fmaf(s.momentum, m, s.g[at]) : m;
}

// What the update of the first n (at most eight) parameters from element e on starts from
__device__ __forceinline__ void load_eight(const Target& t, bool quads, int64_t e, int n, float* w) {
  if (quads && n >= 8) {
    const float4 a = *(const float4*)(t.p + e), b = *(const float4*)(t.p + e + 4);
    w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w; w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) w[k] = k < n ? t.p[e + k] : 0.f;
  }
}
// ... and the values themselves: as the result, or (MUON) as the update of the w that were there
template <bool MUON> __device__ __forceinline__ void store_eight(const Target& t, bool quads, int64_t e, int n, const float* v, const float* w) {
  float x[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) x[k] = MUON ? w[k] * t.decay - v[k] : v[k];
  float* to = MUON ? t.p : t.dt == F32 ? (float*)t.out : nullptr;
  uint16_t* half = MUON ? t.shadow : t.dt == BF16 ? (uint16_t*)t.out : nullptr;
  if (quads && n >= 8) {
    if (to) {
      *(float4*)(to + e) = make_float4(x[0], x[1], x[2], x[3]);
      *(float4*)(to + e + 4) = make_float4(x[4], x[5], x[6], x[7]);
    }
    if (half) {
      *(uint2*)(half + e) = make_uint2(f32x2_to_bf16x2(x[0], x[1]), f32x2_to_bf16x2(x[2], x[3]));
      *(uint2*)(half + e + 4) = make_uint2(f32x2_to_bf16x2(x[4], x[5]), f32x2_to_bf16x2(x[6], x[7]));
    }
    return;
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    if (k >= n) continue;
    if (to) to[e + k] = x[k];
    if (half) half[e + k] = f32_to_bf16(x[k]);
  }
}

// The sum over a wave, in every lane: over 16 lanes by moves within the vector unit (a move through LDS takes ten times as long), then of four
template <int MOVE> __device__ __forceinline__ double add_moved(double v) {
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, MOVE, 0xf, 0xf, true);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(b >> 32), MOVE, 0xf, 0xf, true);
  return v + __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double sum_of_wave(double v) {
  v = add_moved<0xb1>(v);                // neighbours
  v = add_moved<0x4e>(v);                // pairs
  v = add_moved<0x141>(v);               // mirrored in eight lanes
  v = add_moved<0x140>(v);               // in sixteen
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  auto row = [&](int lane) {
    const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)b, lane), hi = __builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), lane);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
  };
  return row(0) + row(16) + (row(32) + row(48));
}
// The sum over a workgroup of four waves, in every thread
__device__ __forceinline__ double sum_of_all(double v) {
  __shared__ double waves[4];
  v = sum_of_wave(v);
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = v;
  __syncthreads();
  return waves[0] + waves[1] + waves[2] + waves[3];
}

// The momentum, and the sums of squares of pieces of 16 x 256 (in 64 bits: gradients of 1e-25 or 1e25 have a norm as well).  Bound by memory: 25 M
// gradients and momenta in 55 us, 5.5 TB/s.  Longer pieces hold fewer threads' loads in flight (32 rows: 60 us, and 13 instead of 7 for five
// matrices of 201 x 333, whose rows are no multiple of 16 bytes).
__global__ __launch_bounds__(256) void squares_kernel(OrthoPlan p, Source s, char* ws) {
  int id = blockIdx.x;
  const int group = group_of(p.pieces.begin, id);
  const OrthoGroup& g = p.g[group];
  asm volatile("" ::"s"(g.offset), "s"(g.stride), "s"(g.ld), "s"(g.rows), "s"(g.cols), "s"(g.first_piece));      // one batch of loads
  const int each = p.pieces.each[group], matrix = quotient(id, each);
  id -= matrix * each;
  const int across = (g.cols + NORM_COLS - 1) / NORM_COLS, down = quotient(id, across), r0 = down * NORM_ROWS, c0 = (id - down * across) * NORM_COLS;
  double sum = 0;
  if (in_quads(g) && r0 + NORM_ROWS <= g.rows && c0 + NORM_COLS <= g.cols && !(s.in && s.dt != F32)) {
    // a wave's rows, 16 bytes a lane, all of them on their way at once
    const int64_t first = element(g, matrix, r0 + (threadIdx.x >> 6) * (NORM_ROWS / 4), c0 + (threadIdx.x & 63) * 4);
    float4 u[NORM_ROWS / 4], m[NORM_ROWS / 4];
#pragma unroll
    for (int k = 0; k < NORM_ROWS / 4; ++k) {
      u[k] = *(const float4*)((s.in ? (const float*)s.in : s.g) + first + k * g.ld);
      if (!s.in) m[k] = *(const float4*)(s.m + first + k * g.ld);
    }
#pragma unroll
    for (int k = 0; k < NORM_ROWS / 4; ++k) {
      float v[4] = {u[k].x, u[k].y, u[k].z, u[k].w};
      if (!s.in) {
        float w[4] = {m[k].x, m[k].y, m[k].z, m[k].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          w[e] = fmaf(s.momentum, w[e], v[e]);
          v[e] = s.nesterov ? fmaf(s.momentum, w[e], v[e]) : w[e];
        }
        *(float4*)(s.m + first + k * g.ld) = make_float4(w[0], w[1], w[2], w[3]);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) sum += (double)v[e] * v[e];
    }
  } else {
    const int c = c0 + threadIdx.x, rows = c < g.cols ? min(NORM_ROWS, g.rows - r0) : 0;
    const int64_t first = element(g, matrix, r0, c);
    float u[NORM_ROWS], m[NORM_ROWS];          // all on their way at once
#pragma unroll
    for (int k = 0; k < NORM_ROWS; ++k) {
      const int64_t e = first + k * g.ld;
      u[k] = k >= rows ? 0.f : s.in ? ld_f(s.in, (size_t)e, s.dt) : s.g[e];
      m[k] = k < rows && !s.in ? s.m[e] : 0.f;
    }
#pragma unroll
    for (int k = 0; k < NORM_ROWS; ++k) {
      if (!s.in) {
        m[k] = fmaf(s.momentum, m[k], u[k]);
        if (k < rows) s.m[first + k * g.ld] = m[k];
        u[k] = s.nesterov ? fmaf(s.momentum, m[k], u[k]) : m[k];
      }
      sum += (double)u[k] * u[k];
    }
  }
  sum = sum_of_all(sum);
  if (threadIdx.x == 0) ((double*)(ws + p.partials))[g.first_piece + matrix * each + id] = sum;
}

// Y = u / |u|, in tiles of 64 x 64.  Bound by memory: 25 M momenta in 47 us, 4.3 TB/s.  A tile's elements are on their way while the workgroup
// adds up the pieces' sums; tall matrices are turned in LDS.
__global__ __launch_bounds__(256, 8) void normalise_kernel(OrthoPlan p, Source s, char* ws) {
  int id = blockIdx.x;
  const int group = group_of(p.squares.begin, id);
  const OrthoGroup& g = p.g[group];
  asm volatile("" ::"s"(g.offset), "s"(g.stride), "s"(g.ld), "s"(g.rows), "s"(g.cols), "s"(g.mp), "s"(g.np), "s"(g.tall), "s"(g.first),
               "s"(g.first_piece), "s"(g.x[0]));                                   // one batch of loads
  const int each = p.squares.each[group], matrix = quotient(id, each);
  id -= matrix * each;
  const int t = threadIdx.x, across = g.np / 64, down = quotient(id, across), i0 = down * 64, j0 = (id - down * across) * 64;
  __shared__ float tile[64][65];
  const int r0 = g.tall ? j0 : i0, c0 = g.tall ? i0 : j0;                // in the caller's orientation: rows y of the tile
  const bool whole = in_quads(g) && r0 + 64 <= g.rows && c0 + 64 <= g.cols && !(s.in && s.dt != F32);
  float4 u[4], m[4];                                                     // (on their way under the sum)
  if (whole) {
    const int64_t first = element(g, matrix, r0 + t / 16, c0 + t % 16 * 4);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      u[k] = s.in || s.nesterov ? *(const float4*)((s.in ? (const float*)s.in : s.g) + first + k * 16 * g.ld) : make_float4(0.f, 0.f, 0.f, 0.f);
      if (!s.in) m[k] = *(const float4*)(s.m + first + k * 16 * g.ld);
    }
  } else {
    const int64_t first = element(g, matrix, r0 + t / 64, c0 + t % 64);
    const int rows = c0 + t % 64 < g.cols ? g.rows - r0 - t / 64 : 0;
    auto at = [&](int k) { return 4 * k < rows ? read_u(s, first + k * 4 * g.ld) : 0.f; };
#pragma unroll
    for (int k = 0; k < 4; ++k) u[k] = make_float4(at(4 * k), at(4 * k + 1), at(4 * k + 2), at(4 * k + 3));
  }
  const int pieces = g.pieces();
  const double* part = (const double*)(ws + p.partials) + g.first_piece + matrix * pieces;
  double sum = 0;
  for (int k = t; k < pieces; k += 256) sum += part[k];
  sum = sum_of_all(sum);
  const double norm = sqrt(sum), inv = norm > 0 ? SCALE / norm : norm;      // NaN stays one
  if (id == 0 && t == 0) ((float*)(ws + p.shrink))[g.first + matrix] = (float)(norm / (norm + NORM_EPS));
  if (blockIdx.x * 256 + t < p.counters) ((int*)(ws + p.arrived))[blockIdx.x * 256 + t] = 0;     // (there are more threads than tiles)
  auto put = [&](int y, int x, float v) {
    if (g.tall) tile[x][y] = v;
    else tile[y][x] = v;
  };
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float v[4] = {u[k].x, u[k].y, u[k].z, u[k].w}, w[4] = {m[k].x, m[k].y, m[k].z, m[k].w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (whole) put(k * 16 + t / 16, t % 16 * 4 + e, (float)((s.in ? v[e] : s.nesterov ? fmaf(s.momentum, w[e], v[e]) : w[e]) * inv));
      else put((4 * k + e) * 4 + t / 64, t % 64, (float)(v[e] * inv));
    }
  }
  __syncthreads();
  const int64_t plane = g.plane_x();
  _Float16* x = (_Float16*)(ws + g.x[0]) + matrix * 2 * plane;
  const int y = t / 4, q = t % 4 * 16;
  _Float16* to = x + (int64_t)(i0 + y) * g.np + j0 + q;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const Terms<8> v = split_all<8>(&tile[y][q + 8 * k]);
    *(f16x8*)(to + 8 * k) = v.hi;
    *(f16x8*)(to + plane + 8 * k) = v.lo;
  }
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
// Bound, with many tiles, by the power that the matrix instructions draw: two of 1536 x 6144, five steps, X X' 120 us, b A + c A A 43, the
// application 185, the last 190 us: 0.94 PFLOP/s of fp16 in the application, where a large library product of fp16 runs at 1.16 and clocks are 1.7
// to 1.8 GHz.  With few, by the way of the first copies and the epilogue: 7 - 9 us a launch of 50 tiles with 4 to 6 stages.  Slower: four stages and
// one workgroup a unit (application 170 -> 199 us over wide layers), eight waves that share the k of a tile of 128 (168 -> 193), the copies
// between the products of a k step (five 201 x 333 matrices 125.6 -> 130.6).
// Layouts in LDS, as in gemm_pipe.h: k contiguous (P, and Q of GRAM and POLY): rows of KT k, their 16-byte granules permuted; k rows (X of APPLY):
// rows of TILE columns whose 64-byte windows are permuted, for the transposing read.
template <int TILE> struct Tile {
  static constexpr int KT = TILE == 128 ? 32 : 64, PLANE = TILE * KT * 2, STAGE = 4 * PLANE;
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
// The 12 products of the fragments at hand (into hh: hi hi, into xx the cross terms, 2048 times as large; summed apart they keep their
// digits as well, error of 1536 x 6144 1.8e-6 instead of 3.2e-6), and under them the reads of the next ones, at rp and rq, which have arrived when the block ends.  One
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

// The sums of a tile whose k is in `pieces` pieces: each workgroup leaves its own in `sums`, and the one that finds all the others' there adds them up,
// in the order of the pieces whichever it is.  Whether this is that one.  What goes from one workgroup to another passes the L2 caches (each XCD has its
// own) both ways, as agent-wide atomic accesses do; a store has arrived when the counter of stores in flight says so.  No workgroup waits for another.
template <int N> __device__ __forceinline__ bool join(f32x16 (&v)[N], char* sums, int piece, int pieces, int* arrived, int& before, bool live) {
  constexpr int PAST_L2 = 16, BYTES = 256 * N * 64;
  const __amdgpu_buffer_rsrc_t rs = pipe::make_rsrc(sums, (uint32_t)(pieces * BYTES));
  const int at = (threadIdx.x >> 6) * N * 4096 + (threadIdx.x & 63) * 16;
  if (live) {
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, (f32x4){v[n][4 * q], v[n][4 * q + 1], v[n][4 * q + 2], v[n][4 * q + 3]}), rs,
                                               at + (4 * n + q) * 1024, piece * BYTES, PAST_L2);
  }
  wait_vm<0>();
  __syncthreads();
  if (threadIdx.x == 0) before = __hip_atomic_fetch_add(arrived, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  if (before != pieces - 1) return false;
  if (threadIdx.x == 0) __hip_atomic_store(arrived, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);      // for the next product
  if (live) {
    for (int k = 0; k < pieces; ++k) {
      u32x4 u[N][4];
#pragma unroll
      for (int n = 0; n < N; ++n)
#pragma unroll
        for (int q = 0; q < 4; ++q) u[n][q] = __builtin_amdgcn_raw_buffer_load_b128(rs, at + (4 * n + q) * 1024, k * BYTES, PAST_L2);
#pragma unroll
      for (int n = 0; n < N; ++n)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const f32x4 w = __builtin_bit_cast(f32x4, u[n][q]);
#pragma unroll
          for (int e = 0; e < 4; ++e) v[n][4 * q + e] = k ? v[n][4 * q + e] + w[e] : w[e];
        }
    }
  }
  return true;
}

template <int TILE, int MODE, bool MUON> __global__ __launch_bounds__(256, 2) void product_kernel(OrthoPlan p, Target t, char* ws, int step) {
  using S = Tile<TILE>;
  constexpr bool TR = MODE >= APPLY;
  extern __shared__ __align__(256) char stages[];     // (behind the 256 bytes of the next line and nothing else: k_step turns bits of addresses below 256)
  PPLL_CODE_TO_L2(2);
  // ---- which tile
  const OrthoProduct& all = p.product[MODE < APPLY ? MODE : APPLY];
  const int xcd = blockIdx.x & 7;
  int id = all.first[xcd] + (int)(blockIdx.x >> 3);
  const int end = all.first[xcd + 1];
  asm volatile("" ::"s"(id), "s"(end), "s"(ws), "s"(step), "s"(p.shrink));      // loaded with the bounds, before the branch
  const bool none = id >= end;
  int group = group_of(all.begin, id);
  asm volatile("" : "+s"(group));
  if (none) return;
  const OrthoGroup& g = p.g[group];
  const OrthoProduct::Group& part = all.group[group];
  // and the next batch, of the group's
  const int64_t x0 = g.x[0], x1 = g.x[1];
  asm volatile("" ::"s"(g.m), "s"(g.n), "s"(g.mp), "s"(g.np), "s"(g.tall), "s"(g.first), "s"(x0), "s"(x1), "s"(g.a), "s"(g.b),
               "s"(part.each), "s"(part.tiles), "s"(part.split), "s"(part.tile_of), "s"(part.sums_of));
  const int matrix = quotient(id, part.each);
  id -= matrix * part.each;
  constexpr bool PIECES = MODE <= POLY;
  const int pieces = PIECES ? part.split : 1;
  const int piece = PIECES && pieces > 1 ? quotient(id, part.tiles) : 0;
  if (PIECES) id -= piece * part.tiles;
  const int tile_of_all = matrix * part.tiles + id;
  int bi, bj;
  if (MODE <= POLY) {
    bi = (int)((sqrtf(8.f * id + 1.f) - 1.f) * 0.5f);
    while ((bi + 1) * (bi + 2) / 2 <= id) ++bi;
    while (bi * (bi + 1) / 2 > id) --bi;
    bj = id - bi * (bi + 1) / 2;
  } else {
    const int down = (g.mp + TILE - 1) / TILE;         // tiles that read the same columns of X follow one another
    bj = quotient(id, down); bi = id - bj * down;
  }
  const int64_t px = g.plane_x(), pa = g.plane_a();
  const int from = step & 1;
  _Float16* X = (_Float16*)(ws + (from ? x1 : x0)) + matrix * 2 * px;
  _Float16* A = (_Float16*)(ws + g.a) + matrix * 2 * pa;
  _Float16* B = (_Float16*)(ws + g.b) + matrix * 2 * pa;
  const int K = MODE == GRAM ? g.np : g.mp, stages_of_tile = K / S::KT;
  const int first_stage = piece * stages_of_tile / pieces, nk = (piece + 1) * stages_of_tile / pieces - first_stage;
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
    for (int c = 0; c < 8; ++c) pipe::load_to_lds(rs, to + c * 1024, off[c & 1] + c * every + (i + first_stage) * step_k);
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
  auto ready = [&](int i) {                         // stage i + 1 is in LDS, stage i is filled again; where stage i + 1 begins
    wait_vm<0>();                                   // this wave's part
    barrier();                                      // and everyone's; nobody reads stage i any more
    issue(i + 2);
    return (i + 1 & 1) * S::STAGE;
  };
  if constexpr (TILE == 128) {
    int st = 0;
    for (int i = 0; i < nk; ++i) {
      k_step<TILE, TR>(hh, xx, f0, f1, (rp ^ 32) + st, (TR ? rq + NEXT_Q : rq ^ 32) + st);
      st = ready(i);
      k_step<TILE, TR>(hh, xx, f1, f0, rp + st, rq + st);
    }
  } else {
    for (int i = 0; i < nk; i += 2) {
      const int st = ready(i);
      k_step<TILE, TR>(hh, xx, f0, f1, rp + st, rq + st);
      if (i + 1 >= nk) break;
      const int nx = ready(i + 1);
      k_step<TILE, TR>(hh, xx, f1, f0, rp + nx, rq + nx);
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
    for (int i = 0; i < 2; ++i) hh[j][i] += xx[j][i] * UNLOW;

  // ---- epilogue: through LDS, so that a wave reads and writes whole 16-byte pieces of whole cache lines.  A wave finishes PASSES times ROWS rows
  // of 64 columns: lane l pieces of eight at columns 8 (l % 8) of rows l / 8 + 8 n.  What lies past the padded size (a multiple of 64) is not stored.
  constexpr int PITCH = 68;                             // floats of a row of 64 and room: rows 4 banks apart
  constexpr int ROWS = TILE == 128 ? 32 : 16, PASSES = TILE == 128 ? 2 : 1, EACH = ROWS / 8;
  const int i0 = TILE == 128 ? bi * 128 + wi * 64 : bi * 64 + wave * 16, j0 = TILE == 128 ? bj * 128 + wj * 64 : bj * 64;
  const bool live = i0 < g.mp && j0 < (MODE <= POLY ? g.mp : g.np), mirrored = MODE <= POLY && bi != bj;
  const int r8 = lane >> 3, seg = (lane & 7) * 8;
  const int64_t ld = MODE >= APPLY ? g.np : g.mp, pl = MODE >= APPLY ? px : pa;
  const bool quads = in_quads(g);
  // all that the epilogue reads is on its way before the sums go through LDS: A or X, and of the last product the parameters (of tall matrices
  // in the caller's orientation: eight of a row there, columns i of the tile, ROWS / 8 lanes a row)
  f16x8 old_h[PASSES * EACH], old_l[PASSES * EACH];
  constexpr int SEGS = ROWS / 8, TURNS = 64 * SEGS / 64;
  float w[MODE == LAST && MUON ? EACH : 1][8];
  auto place = [&](int ps, int n, int& i, int& j) { i = i0 + ps * ROWS + r8 + 8 * n; j = j0 + seg; };
  auto place_tall = [&](int ps, int n, int& i, int& j) { i = i0 + ps * ROWS + lane % SEGS * 8; j = j0 + lane / SEGS + n * (64 / SEGS); };
  static_assert(TURNS == EACH, "");
  auto parameters = [&](int ps) {
    if (MODE != LAST || !MUON) return;
#pragma unroll
    for (int n = 0; n < EACH; ++n) {
      int i, j;
      if (!g.tall) {
        place(ps, n, i, j);
        load_eight(t, quads, element(g, matrix, i, j), i < g.m ? g.n - j : 0, w[n]);
      } else {
        place_tall(ps, n, i, j);
        load_eight(t, quads, element(g, matrix, j, i), j < g.n ? g.m - i : 0, w[n]);
      }
    }
  };
  auto load_old = [&]() {
    if (!live) return;
#pragma unroll
    for (int ps = 0; ps < PASSES; ++ps)
#pragma unroll
      for (int n = 0; n < EACH; ++n) {
        int i, j;
        if (MODE != GRAM) {
          place(ps, n, i, j);
          const _Float16* add = (MODE == POLY ? A : X) + i * ld + j;
          old_h[ps * EACH + n] = *(const f16x8*)add;
          old_l[ps * EACH + n] = *(const f16x8*)(add + pl);
        }
      }
    parameters(0);
  };
  if (pieces == 1) load_old();
  char* joint = nullptr;
  int& before = *(int*)(stages + 2 * S::STAGE - 4);
  int* arrived = (int*)(ws + p.arrived) + part.tile_of + tile_of_all;
  if (PIECES && pieces > 1) joint = ws + p.sums + part.sums_of + (int64_t)tile_of_all * pieces * (TILE * TILE * 4);
  const Shrink shrink = shrink_of(((const float*)(ws + p.shrink))[g.first + matrix], step);
  const float poly_b = NS_B * shrink.now * shrink.now, poly_c = NS_C * shrink.now * shrink.now * shrink.now * shrink.now * UNSCALE;
  const float scale = MODE == LAST ? shrink.ratio * shrink.next * UNSCALE * (MUON ? 0.2f * t.lr * sqrtf((float)g.n) : 1.f) : shrink.ratio;
  // rows r0 .. of `sums`, which holds the products
  auto finish = [&](float* sums, int ps) {
#pragma unroll
    for (int n = 0; n < EACH; ++n) {
      int i, j;
      place(ps, n, i, j);
      float* from_lds = sums + (r8 + 8 * n) * PITCH + seg;
      const float4 lo4 = *(const float4*)from_lds, hi4 = *(const float4*)(from_lds + 4);
      float v[8] = {lo4.x, lo4.y, lo4.z, lo4.w, hi4.x, hi4.y, hi4.z, hi4.w};
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] *= MODE == GRAM ? UNSCALE : MODE == POLY ? poly_c : UNSCALE * scale;
      if (MODE != GRAM) {
        const u32x4 h = __builtin_bit_cast(u32x4, old_h[ps * EACH + n]), l = __builtin_bit_cast(u32x4, old_l[ps * EACH + n]);
#pragma unroll
        for (int k = 0; k < 4; ++k) add_two(v + 2 * k, h[k], l[k], MODE == POLY ? poly_b : NS_A * scale);
      }
      if (mirrored || (MODE == LAST && g.tall)) {
        *(float4*)from_lds = make_float4(v[0], v[1], v[2], v[3]);
        *(float4*)(from_lds + 4) = make_float4(v[4], v[5], v[6], v[7]);
      }
      if (MODE != LAST) {
        const Terms<8> v2 = split_all<8>(v);
        _Float16* to = (MODE == GRAM ? A : MODE == POLY ? B : (_Float16*)(ws + (from ? x0 : x1)) + matrix * 2 * px) + i * ld + j;
        *(f16x8*)to = v2.hi;
        *(f16x8*)(to + pl) = v2.lo;
      } else if (!g.tall && i < g.m && j < g.n) {
        store_eight<MUON>(t, quads, element(g, matrix, i, j), g.n - j, v, w[MUON ? n : 0]);
      }
    }
  };
  auto finish_tall = [&](const float* sums, int ps) {
#pragma unroll
    for (int n = 0; n < TURNS; ++n) {
      int i, j;
      place_tall(ps, n, i, j);
      float v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = sums[(i - i0 - ps * ROWS + k) * PITCH + j - j0];
      if (i < g.m && j < g.n) store_eight<MUON>(t, quads, element(g, matrix, j, i), g.m - i, v, w[MUON ? n : 0]);
    }
  };
  // columns c0 .. c0 + cols - 1 of `rows` (a multiple of 8) finished rows, as rows of the mirrored tile
  auto finish_mirrored = [&](const float* sums, int rows, int i0, int c0, int cols) {
    const int segs = rows / 8, seg = lane % segs * 8;
    _Float16* D = MODE == GRAM ? A : B;
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const int c = c0 + lane / segs + n * (64 / segs);
      if (c >= c0 + cols) break;
      float v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = sums[(seg + k) * PITCH + c];
      const Terms<8> v2 = split_all<8>(v);
      _Float16* to = D + (int64_t)(j0 + c) * g.mp + i0 + seg;
      *(f16x8*)to = v2.hi;
      *(f16x8*)(to + pa) = v2.lo;
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
    // 32 rows at a time, in a part of LDS of the wave's own
    float* sums = (float*)stages + wave * 32 * PITCH;
    if (PIECES && pieces > 1) {
      f32x16 v[4] = {hh[0][0], hh[0][1], hh[1][0], hh[1][1]};
      if (!join<4>(v, joint, piece, pieces, arrived, before, live)) return;
      load_old();
#pragma unroll
      for (int k = 0; k < 4; ++k) hh[k >> 1][k & 1] = v[k];
    }
    if (!live) return;
#pragma unroll
    for (int ps = 0; ps < 2; ++ps) {
      if (ps) parameters(ps);
      wave_sync();
      put(sums, hh[0][ps], 0, 0);
      put(sums, hh[1][ps], 0, 32);
      wave_sync();
      finish(sums, ps);
      if (MODE == LAST && g.tall) {
        wave_sync();
        finish_tall(sums, ps);
      }
      if (mirrored) {
        wave_sync();
        finish_mirrored(sums, 32, i0 + 32 * ps, 0, 64);
      }
    }
  } else {
    // the four waves' sums: each adds up the 32 x 32 tile of its number, which it holds a part of itself, and finishes 16 rows of the whole
    float4* quarters = (float4*)stages;                 // [wave][tile][q][lane]
    float* sums = (float*)stages;
    f32x16 acc;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const f32x16& v = hh[k >> 1][k & 1];
      if (k == wave) {
        acc = v;
        continue;
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) quarters[((wave * 4 + k) * 4 + q) * 64 + lane] = make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
    }
    __syncthreads();
#pragma unroll
    for (int w = 1; w < 4; ++w) {
      const int other = wave ^ w;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float4 b = quarters[((other * 4 + wave) * 4 + q) * 64 + lane];
        acc[4 * q] += b.x; acc[4 * q + 1] += b.y; acc[4 * q + 2] += b.z; acc[4 * q + 3] += b.w;
      }
    }
    if (PIECES && pieces > 1) {
      f32x16 v[1] = {acc};
      if (!join<1>(v, joint, piece, pieces, arrived, before, true)) return;
      load_old();
      acc = v[0];
    }
    __syncthreads();
    put(sums, acc, (wave & 1) * 32, (wave >> 1) * 32);
    __syncthreads();
    finish(sums + wave * 16 * PITCH, 0);
    if (MODE == LAST && g.tall) {
      wave_sync();
      finish_tall(sums + wave * 16 * PITCH, 0);
    }
    if (mirrored) {
      __syncthreads();
      finish_mirrored(sums, 64, bi * 64, wave * 16, 16);
    }
  }
}
#undef NS_MMA
#undef NS_ACC
#undef NS_CUR
#undef NS_CROSS

// ------------------------------------------------------------------ small matrices
// All steps of one matrix in one workgroup of 8 waves: X and the symmetric matrices stay in LDS as planes, rows 16 bytes longer than their
// elements, so that pieces of neighbouring rows meet no bank twice.  Bound by the chain of LDS reads, products, conversions and barriers: a step of
// 64 x 64 takes 2.4 us, of 288 x 32 3.8, of 128 x 128 9.0 (2.8, 4.4 and 10.0 with a conversion an instruction and sums that begin with zeros in
// registers).  Tiles of 16 x 16 on 16 waves, which read each element twice as often, were level with that at 64 x 64 and took 15.3 at 128 x 128.
//  Gram and square: tiles of 32 x 32 on and under the diagonal, dealt out to the waves; where there are fewer (one, or three of long rows) the
//  waves share the k and add up in LDS.
//  The results of a product wait in registers until everyone has read what they replace, unless there is room for a second buffer.
typedef __attribute__((ext_vector_type(4))) short i16x4;
// Four rows of 16 elements, an 8-byte piece from each of 16 lanes: each lane receives the four elements of its column.
__device__ __forceinline__ f16x4 read_columns(const _Float16* from) {
  return __builtin_bit_cast(f16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)from));
}
constexpr int SMALL_THREADS = 512, SMALL_WAVES = SMALL_THREADS / 64;
constexpr int SMALL_TURNS = (ORTHO_SMALL_LDS / 4096 + SMALL_WAVES - 1) / SMALL_WAVES;      // tiles of the largest X for each wave
// NT: tiles of X for a wave, at most; NG: of the symmetric matrices
template <int NT, int NG, bool MUON> __global__ __launch_bounds__(SMALL_THREADS) void small_kernel(OrthoPlan p, Source src, Target t, int steps) {
  extern __shared__ __align__(16) char stages[];
  __shared__ double sums[SMALL_WAVES];
  int matrix = blockIdx.x;
  const OrthoGroup& g = p.g[group_of(p.small.begin, matrix)];
  asm volatile("" ::"s"(g.offset), "s"(g.stride), "s"(g.ld), "s"(g.rows), "s"(g.cols), "s"(g.m), "s"(g.n), "s"(g.mp), "s"(g.np), "s"(g.tall));
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lx = g.np + 8, la = g.mp + 8, px = g.mp * lx, pa = g.mp * la;      // row lengths and planes, in halves
  const SmallRoom room = small_room(g);
  _Float16 *X = (_Float16*)stages, *XN = room.two_x ? X + 2 * px : X, *A = XN + 2 * px, *B = room.two_a ? A + 2 * pa : A;
  float4* parts = (float4*)(B + 2 * pa);                                       // [tile][share of k][q][lane]
  // ---- momentum, norm, X: a thread takes pieces of eight elements of a row of X (tall: of a column of the caller's matrix, neighbours in
  // neighbouring threads)
  constexpr int PIECES = 2 * NT;
  const int across = g.np / 8, all = g.mp * across;
  auto piece_at = [&](int n, int& i, int& j) {
    const int q = tid + n * SMALL_THREADS;
    if (g.tall) { j = q / g.mp; i = q - j * g.mp; }
    else { i = q / across; j = q - i * across; }
    j *= 8;
    return q < all;
  };
  const bool quads = in_quads(g);
  float u[PIECES][8];
  double sum = 0;
#pragma unroll
  for (int n = 0; n < PIECES; ++n) {
    int i, j;
    const bool on = piece_at(n, i, j) && i < g.m;
    const int count = on ? min(8, g.n - j) : 0;
    const int64_t e = g.tall ? element(g, matrix, j, i) : element(g, matrix, i, j), one = g.tall ? g.ld : 1;
    float m[8];
    auto get = [&](const float* from, float* v) {
      if (!g.tall && quads && count == 8) {
        const float4 a = *(const float4*)(from + e), b = *(const float4*)(from + e + 4);
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = k < count ? from[e + k * one] : 0.f;
      }
    };
    if (MUON) {
      get(src.g, u[n]);
      get(src.m, m);
    } else if (src.dt == F32) {
      get((const float*)src.in, u[n]);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) u[n][k] = k < count ? bf16_to_f32(((const uint16_t*)src.in)[e + k * one]) : 0.f;
    }
    if (MUON) {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        m[k] = fmaf(src.momentum, m[k], u[n][k]);
        u[n][k] = src.nesterov ? fmaf(src.momentum, m[k], u[n][k]) : m[k];
      }
      if (!g.tall && quads && count == 8) {
        *(float4*)(src.m + e) = make_float4(m[0], m[1], m[2], m[3]);
        *(float4*)(src.m + e + 4) = make_float4(m[4], m[5], m[6], m[7]);
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (k < count) src.m[e + k * one] = m[k];
      }
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) sum += (double)u[n][k] * u[n][k];
  }
  sum = sum_of_wave(sum);
  if (lane == 0) sums[wave] = sum;
  __syncthreads();
  sum = 0;
#pragma unroll
  for (int w = 0; w < SMALL_WAVES; ++w) sum += sums[w];
  const double norm = sqrt(sum), inv = norm > 0 ? SCALE / norm : norm;
  Shrink shrink = shrink_from(__uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint((float)(norm / (norm + NORM_EPS))))));
  // (a norm whose reciprocal fp32 cannot hold takes the products in 64 bits)
  const float inv32 = (float)inv;
  const bool far = !(inv32 > 1e-30f && inv32 < 1e30f);
#pragma unroll
  for (int n = 0; n < PIECES; ++n) {
    int i, j;
    if (!piece_at(n, i, j)) break;
#pragma unroll
    for (int k = 0; k < 8; ++k) u[n][k] = far ? (float)(u[n][k] * inv) : u[n][k] * inv32;
    const Terms<8> v = split_all<8>(u[n]);
    *(f16x8*)(X + i * lx + j) = v.hi;
    *(f16x8*)(X + px + i * lx + j) = v.lo;
  }
  __syncthreads();

  // ---- products of 32 x 32: lane l holds row l % 32, columns 8 q + 4 (l / 32) + e in element 4 q + e
  const int row = lane & 31, kpart = 8 * (lane >> 5);
  // 64 k at a time, 32 where that many registers are taken.  (All sixteen fragments on their way before the first product, which the compiler does not
  // do by itself: five steps of 64 x 64 19.7 -> 20.2 us.)
  struct Pair { f16x8 ph, pl, qh, ql; };
  auto sum_up = [&](int from, int to, auto load) {
    f32x16 hh, xx;
    auto piece = [&](int k, auto n, auto first) {
      Pair f[decltype(n)::value];
#pragma unroll
      for (int i = 0; i < decltype(n)::value; ++i) f[i] = load(k + 16 * i);
#pragma unroll
      for (int i = 0; i < decltype(n)::value; ++i) {
        const bool none = decltype(first)::value && i == 0;          // (the instruction takes a zero as it is)
        hh = __builtin_amdgcn_mfma_f32_32x32x16_f16(f[i].qh, f[i].ph, none ? f32x16{} : hh, 0, 0, 0);
        xx = __builtin_amdgcn_mfma_f32_32x32x16_f16(f[i].ql, f[i].ph, none ? f32x16{} : xx, 0, 0, 0);
        xx = __builtin_amdgcn_mfma_f32_32x32x16_f16(f[i].qh, f[i].pl, xx, 0, 0, 0);
      }
    };
    std::integral_constant<int, 4> four;
    std::integral_constant<int, 2> two;
    if (from >= to) return f32x16{};
    int k = from;
    if (NT <= 2 && k + 64 <= to) {
      piece(k, four, std::true_type());
      for (k += 64; k + 64 <= to; k += 64) piece(k, four, std::false_type());
      if (k < to) piece(k, two, std::false_type());
    } else {
      piece(k, two, std::true_type());
      if (NT > 2)
        for (k += 32; k < to; k += 32) piece(k, two, std::false_type());
    }
    return hh + xx * UNLOW;
  };
  auto rows_product = [&](const _Float16* P, int ld, int plane, int i0, int j0, int from, int to) {
    const _Float16 *pr = P + (i0 + row) * ld + kpart, *qr = P + (j0 + row) * ld + kpart;
    return sum_up(from, to, [&](int k) {
      return Pair{*(const f16x8*)(pr + k), *(const f16x8*)(pr + plane + k), *(const f16x8*)(qr + k), *(const f16x8*)(qr + plane + k)};
    });
  };
  auto columns_product = [&](const _Float16* from, int i0, int j0) {
    const _Float16 *pr = B + (i0 + row) * la + kpart;
    const _Float16* qr = from + (kpart + ((lane & 15) >> 2)) * lx + j0 + 16 * (lane >> 4 & 1) + 4 * (lane & 3);
    return sum_up(0, g.mp, [&](int k) {
      f16x8 q[2];
#pragma unroll
      for (int plane = 0; plane < 2; ++plane) {
        const _Float16* at_k = qr + plane * px + k * lx;
        const f16x4 a = read_columns(at_k), b = read_columns(at_k + 4 * lx);
        q[plane] = f16x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
      }
      return Pair{*(const f16x8*)(pr + k), *(const f16x8*)(pr + pa + k), q[0], q[1]};
    });
  };
  const int ta = g.mp / 32, tx = g.np / 32;
  const bool whole = NT == 1 || ta <= 2;                          // as many waves as tiles: no mirroring
  auto sym_tile = [&](int n, int& i0, int& j0) {       // of up to ten
    if (whole) { i0 = n / ta * 32; j0 = n % ta * 32; return; }
    const int i = n < 1 ? 0 : n < 3 ? 1 : n < 6 ? 2 : 3;
    i0 = 32 * i; j0 = 32 * (n - i * (i + 1) / 2);
  };
  const int ts = whole ? ta * ta : ta * (ta + 1) / 2, col = 4 * (lane >> 5);
  auto add_old = [&](const _Float16* from, int plane, f32x16 v, float old_by, float by) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const u32x2 h = *(const u32x2*)(from + 8 * q), l = *(const u32x2*)(from + plane + 8 * q);
      float four[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) four[e] = v[4 * q + e] * by;
      add_two(four, h.x, l.x, old_by);
      add_two(four + 2, h.y, l.y, old_by);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[4 * q + e] = four[e];
    }
    return v;
  };
  auto put = [&](_Float16* to, int plane, f32x16 v, _Float16* mirrored) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const float four[4] = {v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
      const Terms<4> r = split_all<4>(four);
      *(f16x4*)(to + 8 * q) = r.hi;
      *(f16x4*)(to + plane + 8 * q) = r.lo;
      if (mirrored)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          mirrored[(8 * q + e) * la] = r.hi[e];
          mirrored[(8 * q + e) * la + plane] = r.lo[e];
        }
    }
  };
  auto put_sym = [&](_Float16* D, f32x16 v, int i0, int j0) {
    put(D + (i0 + row) * la + j0 + col, pa, v, !whole && i0 != j0 ? D + (j0 + col) * la + i0 + row : nullptr);
  };
  f32x16 held[NT > NG ? NT : NG];
  // this wave's n-th tile; the addresses of several, kept from step to step, would not fit into the registers
  auto nth = [&](int n) {
    int first = wave;
    if (NT > 1) {
      __builtin_amdgcn_sched_barrier(0);
      asm volatile("" : "+s"(first));
    }
    return first + n * SMALL_WAVES;
  };
  for (int k = 0; k < steps; ++k) {
    const float t2 = shrink.now * shrink.now;
    // X X'
    if (room.shares == 1) {
#pragma unroll
      for (int n = 0; n < NG; ++n) {
        const int tile = nth(n);
        if (tile >= ts) break;
        int i0, j0;
        sym_tile(tile, i0, j0);
        put_sym(A, rows_product(X, lx, px, i0, j0, 0, g.np) * UNSCALE, i0, j0);
      }
    } else {
      const int n = wave / room.shares, share = wave % room.shares;
      int i0, j0;
      sym_tile(n, i0, j0);
      const int each = (g.np / 32 + room.shares - 1) / room.shares * 32;
      f32x16 v = {};
      if (n < ts) v = rows_product(X, lx, px, i0, j0, min(share * each, g.np), min((share + 1) * each, g.np));
      if (n < ts && share > 0)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          parts[((n * room.shares + share) * 4 + q) * 64 + lane] = make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
      __syncthreads();
      if (n < ts && share == 0) {
        for (int o = 1; o < room.shares; ++o)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const float4 b = parts[((n * room.shares + o) * 4 + q) * 64 + lane];
            v[4 * q] += b.x; v[4 * q + 1] += b.y; v[4 * q + 2] += b.z; v[4 * q + 3] += b.w;
          }
        put_sym(A, v * UNSCALE, i0, j0);
      }
    }
    __syncthreads();
    // b A + c A A
#pragma unroll
    for (int n = 0; n < NG; ++n) {
      const int tile = nth(n);
      if (tile >= ts) break;
      int i0, j0;
      sym_tile(tile, i0, j0);
      held[n] = add_old(A + (i0 + row) * la + j0 + col, pa, rows_product(A, la, pa, i0, j0, 0, g.mp), NS_B * t2, NS_C * t2 * t2 * UNSCALE);
    }
    if (!room.two_a) __syncthreads();
#pragma unroll
    for (int n = 0; n < NG; ++n) {
      const int tile = nth(n);
      if (tile >= ts) break;
      int i0, j0;
      sym_tile(tile, i0, j0);
      put_sym(B, held[n], i0, j0);
    }
    __syncthreads();
    // a X + (that) X
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int tile = nth(n), i0 = tile / tx * 32, j0 = tile % tx * 32;
      if (tile >= ta * tx) break;
      held[n] = add_old(X + (i0 + row) * lx + j0 + col, px, columns_product(X, i0, j0), NS_A * shrink.ratio, UNSCALE * shrink.ratio);
    }
    if (k + 1 == steps) break;
    shrink = shrink_from(shrink.next);
    if (!room.two_x) __syncthreads();
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int tile = nth(n), i0 = tile / tx * 32, j0 = tile % tx * 32;
      if (tile >= ta * tx) break;
      put(XN + (i0 + row) * lx + j0 + col, px, held[n], nullptr);
    }
    _Float16* const swap = X;
    X = XN; XN = swap;
    __syncthreads();
  }
  // ---- the result, from LDS in the same pieces
  float* R = (float*)XN;                               // rows of lx floats, as large as the planes
  const float scale = UNSCALE * shrink.next * (MUON ? 0.2f * t.lr * sqrtf((float)g.n) : 1.f);
  if (!room.two_x) __syncthreads();
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int tile = nth(n), i0 = tile / tx * 32, j0 = tile % tx * 32;
    if (tile >= ta * tx) break;
#pragma unroll
    for (int q = 0; q < 4; ++q)
      *(float4*)(R + (i0 + row) * lx + j0 + col + 8 * q) =
          make_float4(held[n][4 * q] * scale, held[n][4 * q + 1] * scale, held[n][4 * q + 2] * scale, held[n][4 * q + 3] * scale);
  }
  __syncthreads();
  // eight of a row of the caller's
  const int segs = g.tall ? (g.m + 7) / 8 : (g.n + 7) / 8, rows = g.tall ? g.n : g.m;
  for (int q = tid; q < rows * segs; q += SMALL_THREADS) {
    const int r = q / segs, c = (q - r * segs) * 8;
    float v[8];
    if (g.tall) {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = R[(c + k) * lx + r];
    } else {
      const float4 a = *(const float4*)(R + r * lx + c), b = *(const float4*)(R + r * lx + c + 4);
      v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    }
    const int64_t e = element(g, matrix, r, c);
    const int count = (g.tall ? g.m : g.n) - c;
    float w[8];
    if (MUON) load_eight(t, quads, e, count, w);
    store_eight<MUON>(t, quads, e, count, v, w);
  }
}
template <int NT, int NG> int launch_small(hipStream_t s, const OrthoPlan& p, const Source& src, const Target& dst, int steps, int matrices, int lds) {
  static OncePerDevice once, once_muon;
  if (src.in) {
    PPLL_TRY(raise_lds((const void*)small_kernel<NT, NG, false>, ORTHO_SMALL_LDS, once));
    hipLaunchKernelGGL((small_kernel<NT, NG, false>), dim3(matrices), dim3(SMALL_THREADS), lds, s, p, src, dst, steps);
  } else {
    PPLL_TRY(raise_lds((const void*)small_kernel<NT, NG, true>, ORTHO_SMALL_LDS, once_muon));
    hipLaunchKernelGGL((small_kernel<NT, NG, true>), dim3(matrices), dim3(SMALL_THREADS), lds, s, p, src, dst, steps);
  }
  PPLL_HIP(hipGetLastError());
  return PPLL_OK;
}

template <int TILE, int MODE> int launch_tiles(hipStream_t s, const OrthoPlan& p, const Target& t, char* ws, int step) {
  const int longest = p.product[MODE < APPLY ? MODE : APPLY].longest();
  auto launch = [&](auto muon, OncePerDevice& once) -> int {
    constexpr bool MUON = decltype(muon)::value;
    const int lds = 2 * Tile<TILE>::STAGE;
    PPLL_TRY(raise_lds((const void*)product_kernel<TILE, MODE, MUON>, lds, once));
    hipLaunchKernelGGL((product_kernel<TILE, MODE, MUON>), dim3(8 * (unsigned)longest), dim3(256), lds, s, p, t, ws, step);
    PPLL_HIP(hipGetLastError());
    return PPLL_OK;
  };
  static OncePerDevice once, once_muon;
  if constexpr (MODE == LAST)
    if (!t.out) return launch(std::true_type(), once_muon);
  return launch(std::false_type(), once);
}
template <int MODE> int launch_product(hipStream_t s, const OrthoPlan& p, const Target& t, char* ws, int step) {
  return p.product[MODE < APPLY ? MODE : APPLY].tile == 128 ? launch_tiles<128, MODE>(s, p, t, ws, step) : launch_tiles<64, MODE>(s, p, t, ws, step);
}

int run(hipStream_t s, const OrthoPlan& p, const Source& src, const Target& dst, int steps, char* ws) {
  int64_t pieces = 0, squares = 0;
  int small = 0, tiles = 0, lds = 0;
  for (int k = 0; k < p.n; ++k) {
    const OrthoGroup& g = p.g[k];
    if (g.small) {
      small += g.count;
      tiles = g.mp / 32 * (g.np / 32) > tiles ? g.mp / 32 * (g.np / 32) : tiles;
      lds = small_room(g).bytes > lds ? (int)small_room(g).bytes : lds;
    } else {
      pieces += (int64_t)g.count * g.pieces();
      squares += (int64_t)g.count * (g.mp / 64) * (g.np / 64);
    }
  }
  if (small) {
    const int turns = (tiles + SMALL_WAVES - 1) / SMALL_WAVES;      // (eight tiles of X: three of the symmetric matrices at most; 16: ten)
    if (turns <= 1) PPLL_TRY((launch_small<1, 1>(s, p, src, dst, steps, small, lds)));
    else if (turns <= 2) PPLL_TRY((launch_small<2, 2>(s, p, src, dst, steps, small, lds)));
    else PPLL_TRY((launch_small<SMALL_TURNS, 2>(s, p, src, dst, steps, small, lds)));
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
