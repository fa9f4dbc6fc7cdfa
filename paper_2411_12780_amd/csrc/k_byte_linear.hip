// Linear layer on rows of 8 bits.  Forward: y = X W^T in v_mfma_i32_*_i8, both operands with k contiguous, sums exact in 32-bit whole numbers; a
// row's exponent and a channel's enter in the epilogue.
//
// The loop is that of the bf16 products (gemm_pipe.h): a fragment of 16 bytes holds 16 k instead of 8, an instruction takes the time of a
// bf16 one, so a product costs what a bf16 one of half its k does, and the same rules choose the tiles.
#include "bytes.h"
#include "gemm_pipe.h"
#include "plan.h"

namespace ppll {

namespace {
using namespace pipe;

struct ByteArgs {
  const int8_t *x, *w, *ex, *ew;
  int64_t ldx, ldw;
  char *y, *slope;
  const char* residual;
  int64_t ldy, lds, ldr;            // elements
  const float* bias;
  int M, N, K;                      // K in pairs of bytes, padded
  bool gelu, vec;                   // vec: rows of y, slope and residual in pieces of 16 bytes
  TileMap map;
  int helpers;
};

// What eight sums of a row become, columns n .. n + 7
template <int DT, bool VEC> __device__ __forceinline__ void byte_end(const ByteArgs& p, int64_t m, int n, int row_exp, const int (&col_exp)[8], const float (&bias)[8],
                                                                     const int (&sum)[8], const Eight<DT>& res) {
  constexpr int ESZ = DT == BF16 ? 2 : 4;
  auto put = [&](char* to, int64_t ld, const float (&v)[8]) {
    Eight<DT> o;
    o.set(v);
    char* row = to + m * ld * ESZ;
    if (VEC) {
      if constexpr (DT == BF16) {
        store_through(row + n * ESZ, o.w);
      } else {
        store_through(row + n * ESZ, __builtin_bit_cast(uint4, o.a));
        store_through(row + n * ESZ + 16, __builtin_bit_cast(uint4, o.b));
      }
    } else {
      o.store(row, n, p.N);
    }
  };
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = ldexpf((float)sum[i], row_exp + col_exp[i]) + bias[i];
  if (row_exp == BYTE_NAN)
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(0x7fc00000u);
  if (p.residual) {
    float r[8];
    res.get(r);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += r[i];
  }
  if (p.gelu) {
    float dg[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float cdf, pdf;
      cdf_pdf(v[i], cdf, pdf);
      dg[i] = cdf + v[i] * pdf; v[i] *= cdf;
    }
    if (p.slope) put(p.slope, p.lds, dg);
  }
  put(p.y, p.ldy, v);
}
// Exponents and biases of columns n .. n + 7; a channel of NaN has a bias of NaN
__device__ __forceinline__ void columns_of(const ByteArgs& p, int n, int (&exps)[8], float (&bias)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const bool in = n + i < p.N;
    const int e = in ? p.ew[n + i] : 0;
    bias[i] = e == BYTE_NAN ? __uint_as_float(0x7fc00000u) : in && p.bias ? p.bias[n + i] : 0.f;
    exps[i] = e == BYTE_NAN ? 0 : e;
  }
}

template <int DT, bool VEC, int WGM, int WGN, int IM, int NS, int KT>
__global__ __launch_bounds__((Shape<false, false, WGM, WGN, IM, NS, KT>::THREADS), 2) void byte_linear_kernel(ByteArgs p) {
  using S = Shape<false, false, WGM, WGN, IM, NS, KT>;
  constexpr int JN = 2, ESZ = DT == BF16 ? 2 : 4;
  extern __shared__ __align__(1024) char smem[];
  const int slot = blockIdx.x >> 3;
  int tm, tn;
  if (S::COPY_WAVES) {
    if (!tile_at(p.map, blockIdx.x & 7, slot, tm, tn)) return;
  } else {
    const int t = (blockIdx.x & 7) * p.map.per_xcd + slot;
    tm = t / p.map.tiles_n;
    tn = t % p.map.tiles_n;
    if (slot >= p.map.per_xcd || tm >= p.map.tiles_m) return;
  }
  const int m0 = tm * S::BM, n0 = tn * S::BN, rows = min(S::BM, p.M - m0), cols = min(S::BN, p.N - n0);
  f32x16 acc[JN][IM];
  float none[JN][8];
#pragma unroll
  for (int j = 0; j < JN; ++j)
#pragma unroll
    for (int i = 0; i < IM; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[j][i][e] = 0.f;
  // the tile's rows alone: offsets stay in 32 bits however long the operands are
  multiply<S, false, false, false, true>(make_rsrc(p.x + m0 * p.ldx, (uint32_t)((rows - 1) * p.ldx + 2 * p.K)),
                                         make_rsrc(p.w + n0 * p.ldw, (uint32_t)((cols - 1) * p.ldw + 2 * p.K)), p.ldx / 2, p.ldw / 2, 0, 0, rows, cols, p.K,
                                         (lds_char*)smem, acc, none, false);
  if (S::COPY_WAVES && threadIdx.x >= 64 * S::W) return;

  // Epilogue: a wave passes its sums (lane = one row, 4 consecutive columns a group) through its own piece of LDS, 32 rows at a time, and
  // takes them out 8 consecutive columns a lane
  constexpr int COLS = JN * 32, PITCH = COLS + 4, LPR = COLS / 8, RPP = 64 / LPR, NP = 32 / RPP;
  static_assert(S::W * 32 * PITCH * 4 <= S::LDS, "");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int* st = reinterpret_cast<int*>(smem) + wave * 32 * PITCH;
  const int mw = m0 + wave / WGN * IM * 32, c8 = lane % LPR * 8, n = n0 + wave % WGN * COLS + c8, r0 = lane / LPR;
  int exps[8];
  float bias[8];
  columns_of(p, n, exps, bias);
#pragma unroll
  for (int im = 0; im < IM; ++im) {
#pragma unroll
    for (int jn = 0; jn < JN; ++jn)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<float4*>(st + (lane & 31) * PITCH + jn * 32 + 8 * q + 4 * (lane >> 5)) =
            make_float4(acc[jn][im][4 * q], acc[jn][im][4 * q + 1], acc[jn][im][4 * q + 2], acc[jn][im][4 * q + 3]);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
    int sums[NP][8];
#pragma unroll
    for (int q = 0; q < NP; ++q) {
      const int4 lo = *reinterpret_cast<const int4*>(st + (q * RPP + r0) * PITCH + c8), hi = *reinterpret_cast<const int4*>(st + (q * RPP + r0) * PITCH + c8 + 4);
      sums[q][0] = lo.x; sums[q][1] = lo.y; sums[q][2] = lo.z; sums[q][3] = lo.w; sums[q][4] = hi.x; sums[q][5] = hi.y; sums[q][6] = hi.z; sums[q][7] = hi.w;
    }
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
    Eight<DT> res[NP];
    int ex[NP];
#pragma unroll
    for (int q = 0; q < NP; ++q) {
      const int64_t m = mw + im * 32 + q * RPP + r0;
      const bool in = m < p.M && n < p.N;
      res[q].zero();
      ex[q] = in ? p.ex[m] : 0;
      if (in && p.residual) {
        if (VEC) res[q].load_all(p.residual + (m * p.ldr + n) * ESZ);
        else res[q].load(p.residual + m * p.ldr * ESZ, n, p.N);
      }
    }
#pragma unroll
    for (int q = 0; q < NP; ++q) {
      const int64_t m = mw + im * 32 + q * RPP + r0;
      if (m < p.M && n < p.N) byte_end<DT, VEC>(p, m, n, ex[q], exps, bias, sums[q], res[q]);
    }
  }
}

// Few rows (tokens one by one): bound by the weight's bytes and by latency.  A workgroup has 16 channels and 16 RT rows; its eight waves take
// every eighth step of 64 k straight from memory into fragments (k of a fragment: 16 lane / 16 of both operands) and add up in LDS.
typedef __attribute__((ext_vector_type(4))) int i32x4;
constexpr int FW = 8;
template <int DT, int RT>
__global__ __launch_bounds__(64 * FW) void byte_linear_rows_kernel(ByteArgs p) {
  constexpr int ESZ = DT == BF16 ? 2 : 4;
  __shared__ int part[FW][RT][16][16 + 1];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n0 = blockIdx.x * 16, m0 = blockIdx.y * 16 * RT;
  const int r = lane & 15, kl = (lane >> 4) * 16, bytes = 2 * p.K;
  const int8_t* wr = p.w + min(n0 + r, p.N - 1) * p.ldw;      // (rows that are not there: any, their sums are dropped)
  const int8_t* xr[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) xr[t] = p.x + (int64_t)min(m0 + 16 * t + r, p.M - 1) * p.ldx;
  i32x4 acc[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) acc[t] = (i32x4){0, 0, 0, 0};
  const i32x4 zero = {0, 0, 0, 0};
#pragma unroll 4
  for (int k = wave * 64 + kl; k - kl < bytes; k += FW * 64) {
    const bool in = k < bytes;
    const i32x4 b = in ? *(const i32x4*)(wr + k) : zero;
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const i32x4 a = in ? *(const i32x4*)(xr[t] + k) : zero;
      acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(b, a, acc[t], 0, 0, 0);
    }
  }
  // lane: row lane % 16, channels 4 (lane / 16) .. + 3
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) part[wave][t][lane & 15][4 * (lane >> 4) + i] = acc[t][i];
  __syncthreads();
  for (int i = threadIdx.x; i < 16 * RT * 2; i += 64 * FW) {
    const int row = i >> 1, n = n0 + (i & 1) * 8;
    const int64_t m = m0 + row;
    if (m >= p.M || n >= p.N) continue;
    int sum[8], exps[8];
    float bias[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      sum[e] = 0;
#pragma unroll
      for (int w = 0; w < FW; ++w) sum[e] += part[w][row >> 4][row & 15][(i & 1) * 8 + e];
    }
    columns_of(p, n, exps, bias);
    Eight<DT> res;
    res.zero();
    if (p.residual) res.load(p.residual + m * p.ldr * ESZ, n, p.N);
    byte_end<DT, false>(p, m, n, p.ex[m], exps, bias, sum, res);
  }
}

template <int DT, bool VEC, int WGM, int WGN, int IM, int NS, int KT> int byte_launch_as(hipStream_t s, ByteArgs& p, int units) {
  using S = Shape<false, false, WGM, WGN, IM, NS, KT>;
  if (S::COPY_WAVES) {
    p.map = tile_map(p.M, p.N, S::BM, S::BN, units);
  } else {
    const int tiles_m = (p.M + S::BM - 1) / S::BM, tiles_n = (p.N + S::BN - 1) / S::BN;
    p.map = TileMap{tiles_m, tiles_n, (int)(((long)tiles_m * tiles_n + 7) / 8), 0, 0, 0, false};
  }
  static OncePerDevice once;
  PPLL_TRY(raise_lds((const void*)byte_linear_kernel<DT, VEC, WGM, WGN, IM, NS, KT>, S::LDS, once));
  hipLaunchKernelGGL((byte_linear_kernel<DT, VEC, WGM, WGN, IM, NS, KT>), dim3(8 * p.map.per_xcd), dim3(S::THREADS), S::LDS, s, p);
  PPLL_HIP(hipGetLastError());
  return PPLL_OK;
}

template <int DT, int WGM, int WGN, int IM, int NS, int KT> int byte_launch(hipStream_t s, ByteArgs& p, int units) {
  return p.vec ? byte_launch_as<DT, true, WGM, WGN, IM, NS, KT>(s, p, units) : byte_launch_as<DT, false, WGM, WGN, IM, NS, KT>(s, p, units);
}

constexpr int FEW_ROWS = 64;

// Which kernel a product goes to: 1 few rows, 3 tiles of 128 x 128 with copying waves, 4 / 8 / 10 tiles of 128 / 256 / 320 rows of 256 columns
int choice(const ByteArgs& p, int units) {
  if (p.M <= FEW_ROWS) return 1;
  const ProductEnd end = p.gelu ? END_GELU : p.residual ? END_RESIDUAL : END_BIAS;
  const long tiles = (long)((p.M + 127) / 128) * ((p.N + 127) / 128);
  if (tiles <= units) return 3;
  const int wide = wide_tile_rows(p.M, p.N, p.K, end, units), alone = unit_tile_rows(p.M, p.N, p.K, end, wide, units);
  const int im = alone ? alone : wide;
  return im == 5 ? 4 : im ? im : 3;
}
template <int DT> int forward(hipStream_t s, ByteArgs& p, int kernel) {
  const int units = compute_units() > 0 ? compute_units() : 256;
  if (!kernel) kernel = choice(p, units);
  if (kernel == 1) {
    const int rt = p.M <= 16 ? 1 : 2;
    const dim3 grid((p.N + 15) / 16, (p.M + 16 * rt - 1) / (16 * rt));
    if (rt == 1) hipLaunchKernelGGL((byte_linear_rows_kernel<DT, 1>), grid, dim3(64 * FW), 0, s, p);
    else hipLaunchKernelGGL((byte_linear_rows_kernel<DT, 2>), grid, dim3(64 * FW), 0, s, p);
    PPLL_HIP(hipGetLastError());
    return PPLL_OK;
  }
  if (kernel == 4) return byte_launch<DT, 1, 4, 4, 3, 32>(s, p, units);
  if (kernel == 8) return byte_launch<DT, 2, 4, 4, 2, 64>(s, p, units);
  if (kernel == 10) return byte_launch<DT, 2, 4, 5, 2, 64>(s, p, units);
  return byte_launch<DT, 2, 2, 2, 4, 64>(s, p, units);
}
int product(hipStream_t s, int kernel, const ByteLinear& l, const ppll_byte_rows& x, const ppll_byte_rows& w, const float* bias, const ppll_rows& residual,
            const ppll_rows& y, const ppll_rows& slope) {
  if (l.rows <= 0) return PPLL_OK;
  ByteArgs p{};
  p.x = x.q; p.ex = x.e; p.ldx = x.ld; p.w = w.q; p.ew = w.e; p.ldw = w.ld;
  p.y = (char*)y.p; p.ldy = y.ld; p.slope = (char*)slope.p; p.lds = slope.ld; p.residual = (const char*)residual.p; p.ldr = residual.ld;
  p.bias = bias;
  p.M = l.rows; p.N = l.out; p.K = pad16(l.in) / 2;
  p.gelu = l.activation == PPLL_ACT_GELU;
  const int each = l.dt == BF16 ? 8 : 4;
  auto whole = [&](const ppll_rows& r) { return !r.p || (r.ld % each == 0 && ((uintptr_t)r.p & 15) == 0); };
  p.vec = l.out % 8 == 0 && whole(y) && whole(slope) && whole(residual);
  return l.dt == BF16 ? forward<BF16>(s, p, kernel) : forward<F32>(s, p, kernel);
}
}  // namespace

int launch_byte_linear_fwd(hipStream_t s, const ByteLinear& l, const ppll_byte_rows& x, const ppll_byte_rows& w, const float* bias, const ppll_rows& residual,
                           const ppll_rows& y, const ppll_rows& slope) {
  return product(s, 0, l, x, w, bias, residual, y, slope);
}

}  // namespace ppll

// One product on one kernel (choice() above), for tests of a kernel against another (no part of the public interface)
extern "C" int ppll_internal_byte_linear(int kernel, int precision, int rows, int in, int out, int gelu, const ppll_byte_rows* x, const ppll_byte_rows* w,
                                         const float* bias, const ppll_rows* residual, const ppll_rows* y, const ppll_rows* slope, void* stream) {
  using namespace ppll;
  if (kernel != 1 && kernel != 3 && kernel != 4 && kernel != 8 && kernel != 10) { set_error("there is no kernel %d", kernel); return PPLL_ERR_CONFIG; }
  const ppll_rows none{nullptr, 0};
  return product((hipStream_t)stream, kernel, {precision == PPLL_BF16 ? BF16 : F32, rows, in, out, gelu ? PPLL_ACT_GELU : PPLL_ACT_NONE}, *x, *w, bias,
                 residual ? *residual : none, *y, slope ? *slope : none);
}
