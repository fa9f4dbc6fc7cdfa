// Linear layer on rows of 8 bits.  Forward: y = X W^T in v_mfma_i32_*_i8, both operands with k contiguous, sums exact in 32-bit whole numbers; a
// row's exponent and a channel's enter in the epilogue.
//
// The loop is that of the bf16 products (gemm_pipe.h): a fragment of 16 bytes holds 16 k instead of 8 and an instruction takes the time of a
// bf16 one, so a product costs what a bf16 one of half its k does: 8192 x 8192 x 8192 476 us (2312 TOP/s), 25216 x 6144 x 1536 with a residual 222 us (2142).
// What bounds it: LDS reads and products in the loop, the epilogue where k is short (8320 x 384 x 1536 with GELU and its slope 22 us, 14 without: 24
// instructions' time for an element's two results).
#include <algorithm>

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

// Steps and biases of columns n .. n + 7; a channel of NaN has a bias of NaN
struct Columns {
  int most, least;        // the largest and smallest exponent
  float step[8], bias[8];
  __device__ __forceinline__ void load(const ByteArgs& p, int n) {
    most = -256;
    least = 256;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int at = min(n + i, p.N - 1), e = p.ew[at];
      const float b = p.bias ? p.bias[at] : 0.f;
      bias[i] = e == BYTE_NAN ? __uint_as_float(0x7fc00000u) : b;
      step[i] = exp2_bits(e == BYTE_NAN ? 0 : e);
      most = max(most, e == BYTE_NAN ? 0 : e);
      least = min(least, e == BYTE_NAN ? 0 : e);
    }
  }
};
// What eight sums of a row become, columns n .. n + 7
template <int DT, bool VEC> __device__ __forceinline__ void byte_end(const ByteArgs& p, int64_t m, int n, int row_exp, const Columns& c, const int (&sum)[8],
                                                                     const Eight<DT>& res) {
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
  // the product of two steps is a power of two, exact from 2^-149 (a subnormal one) to 2^127; outside a sum of many may be in range where the step is not
  const bool rare = row_exp == BYTE_NAN || row_exp + c.most > 127 || row_exp + c.least < -149;
  const float step = exp2_bits(rare ? 0 : row_exp);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = fmaf((float)sum[i], c.step[i] * step, c.bias[i]);
  if (rare)
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = row_exp == BYTE_NAN ? __uint_as_float(0x7fc00000u) : ldexpf((float)sum[i], row_exp + (int)(__float_as_uint(c.step[i]) >> 23) - 127) + c.bias[i];
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

template <int DT, bool VEC, int WGM, int WGN, int IM, int NS, int KT>
__global__ __launch_bounds__((Shape<false, false, WGM, WGN, IM, NS, KT>::THREADS), 2) void byte_linear_kernel(ByteArgs p) {
  PPLL_CODE_TO_L2(4);
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
  // exponents of all its rows and columns at once (asked for 32 rows at a time, each time took a way to memory: a tile of 256 x 256 by itself 14.9 us,
  // so 10.7; 25216 x 768 x 2304 85 and 68)
  Columns columns;
  columns.load(p, n);
  static_assert(NP == 4, "");
  uint32_t ex[IM];
#pragma unroll
  for (int im = 0; im < IM; ++im) {
    uint32_t e[NP];
#pragma unroll
    for (int q = 0; q < NP; ++q) e[q] = (uint8_t)p.ex[min(mw + im * 32 + q * RPP + r0, p.M - 1)];
    ex[im] = e[0] | e[1] << 8 | e[2] << 16 | e[3] << 24;
  }
  constexpr int AHEAD = DT == BF16 ? 2 : 1;      // residuals of 32 rows on their way (fp32: no registers for more)
  Eight<DT> res[AHEAD][NP];
  auto ask = [&](int im) {
#pragma unroll
    for (int q = 0; q < NP; ++q) {
      const int64_t m = mw + im * 32 + q * RPP + r0;
      if (m >= p.M || n >= p.N) continue;
      if (VEC) res[im % AHEAD][q].load_all(p.residual + (m * p.ldr + n) * ESZ);
      else res[im % AHEAD][q].load(p.residual + m * p.ldr * ESZ, n, p.N);
    }
  };
  if (p.residual && AHEAD == 2) ask(0);
#pragma unroll
  for (int im = 0; im < IM; ++im) {
    if (p.residual && im + AHEAD - 1 < IM) ask(im + AHEAD - 1);
#pragma unroll
    for (int jn = 0; jn < JN; ++jn)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<float4*>(st + (lane & 31) * PITCH + jn * 32 + 8 * q + 4 * (lane >> 5)) =
            make_float4(acc[jn][im][4 * q], acc[jn][im][4 * q + 1], acc[jn][im][4 * q + 2], acc[jn][im][4 * q + 3]);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int q = 0; q < NP; ++q) {
      const int4 lo = *reinterpret_cast<const int4*>(st + (q * RPP + r0) * PITCH + c8), hi = *reinterpret_cast<const int4*>(st + (q * RPP + r0) * PITCH + c8 + 4);
      const int sums[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
      const int64_t m = mw + im * 32 + q * RPP + r0;
      if (m < p.M && n < p.N) byte_end<DT, VEC>(p, m, n, (int8_t)(ex[im] >> (8 * q)), columns, sums, res[im % AHEAD][q]);
    }
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
  }
}

// Few rows (tokens one by one) or few channels: bound by latency, of a step of k for each 512 (one token 384 -> 1536 4.0 us, one step; 6144 -> 1536 10.5, twelve,
// which wait one for the other with four written out at once or one; its bytes alone 1.8).  A workgroup has 16 channels and 16 RT rows; its eight waves take every eighth step of 64 k straight from memory into
// fragments (k of a fragment: 16 lane / 16 of both operands) and add up in LDS.
typedef __attribute__((ext_vector_type(4))) int i32x4;
constexpr int FW = 8;
template <int DT, int RT>
__global__ __launch_bounds__(64 * FW) void byte_linear_rows_kernel(ByteArgs p) {
  constexpr int ESZ = DT == BF16 ? 2 : 4;
  __shared__ int part[FW][RT][16][16 + 1];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n0 = blockIdx.y * 16, m0 = blockIdx.x * 16 * RT;
  const int r = lane & 15, kl = (lane >> 4) * 16, bytes = 2 * p.K;
  const int8_t* wr = p.w + min(n0 + r, p.N - 1) * p.ldw;      // (rows that are not there: any, their sums are dropped)
  const int8_t* xr[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) xr[t] = p.x + (int64_t)min(m0 + 16 * t + r, p.M - 1) * p.ldx;
  i32x4 acc[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) acc[t] = (i32x4){0, 0, 0, 0};
  const i32x4 zero = {0, 0, 0, 0};
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
    int sum[8];
    Columns columns;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      sum[e] = 0;
#pragma unroll
      for (int w = 0; w < FW; ++w) sum[e] += part[w][row >> 4][row & 15][(i & 1) * 8 + e];
    }
    columns.load(p, n);
    Eight<DT> res;
    res.zero();
    if (p.residual) res.load(p.residual + m * p.ldr * ESZ, n, p.N);
    byte_end<DT, false>(p, m, n, p.ex[m], columns, sum, res);
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

constexpr int FEW_ROWS = 16;

// Which kernel a product goes to: 1 few rows, 3 tiles of 128 x 128 with copying waves, 4 / 8 / 10 tiles of 128 / 256 / 320 rows of 256 columns.
// Microseconds of a round of workgroups (a unit each, two of kernel 4): per k, and with the epilogue (plain, residual, GELU and its slope); a last round that
// fills the share f of the units counts as last + (1 - last) f.  Fits to products of 4096 to 32768 rows, 512 to 1536 channels, k of 128 to 4096, within
// 13 %; 16384 x 1024, k = 1024: 46, 26, 23, 28 us, k = 128 with GELU: 35, 19.3, 19.4, 27; 8192 x 1024, k = 4096: 43, 54, 54, 63; 20480 x 1024, k = 4096:
// 116, 130, 115, 84.
// Kernel 1 by its way through k, or by its workgroups of 16 channels and 32 rows where they are many; a tile by itself takes some 1.5 us more than the fits say.
// Few rows or channels, us, kernel 1 and the best of the tiles: 128 x 768, k = 2560: 6.3, 12.1; 400 x 300, k = 1024: 4.5, 9.0; 1000 x 64, k = 6144: 12.8, 20.2;
// 256 x 2304, k = 256: 6.5, 7.1; 200 x 2304, k = 1024: 9.1, 8.9; 400 x 768, k = 2560: 13.8, 13.4; 1000 x 768, k = 1024: 12.7, 9.0.
int choice(const ByteArgs& p, int units) {
  if (p.M <= FEW_ROWS) return 1;
  struct Cost { int kernel, rows, cols, places; double last, k, end[3]; };
  static const Cost costs[] = {{3, 128, 128, 1, 0.66, 0.0036, {6.6, 8.8, 9.0}},
                               {4, 128, 256, 2, 0.70, 0.0178, {7.4, 12.2, 16.9}},
                               {8, 256, 256, 1, 0.70, 0.0133, {9.1, 14.7, 18.9}},
                               {10, 320, 256, 1, 0.70, 0.0176, {12.0, 18.3, 22.9}}};
  int best = 0;
  double least = 0;
  for (const Cost& c : costs) {
    const int64_t tiles = ((int64_t)p.M + c.rows - 1) / c.rows * (((int64_t)p.N + c.cols - 1) / c.cols), places = (int64_t)c.places * units;
    if (tiles * (c.kernel == 4 ? 256 : 512) > (int64_t)1 << 31) continue;       // a launch has under 2^32 threads; of kernel 4 there are never more than these
    const double share = std::min(1.0, (double)(tiles % places) / units), last = tiles % places == 0 ? 0 : tiles % places > units ? 1 : c.last + (c.places == 1 ? (1 - c.last) * share : 0);
    const double time = ((double)(tiles / places) + last) * (c.k * 2 * p.K + c.end[p.gelu ? 2 : p.residual ? 1 : 0]);
    if (!best || time < least) { best = c.kernel; least = time; }
  }
  const double k = 2.0 * p.K, groups = (((int64_t)p.M + 31) / 32) * (((int64_t)p.N + 15) / 16);
  if (groups > 1 << 20) return best;       // (what a launch holds)
  return 2.6 + std::max(0.0013 * k, groups * (0.0023 + 4.7e-6 * k)) < least + 1.5 ? 1 : best;
}
template <int DT> int forward(hipStream_t s, ByteArgs& p, int kernel, int units) {
  if (!units) units = compute_units();
  if (units <= 0) units = 256;
  if (!kernel) kernel = choice(p, units);
  if (kernel == 1) {
    const int rt = p.M <= 16 ? 1 : 2;
    const dim3 grid((unsigned)(((int64_t)p.M + 16 * rt - 1) / (16 * rt)), (p.N + 15) / 16);
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
  void* prof = nullptr;
  PPLL_TRY(profile_begin(s, 2.0 * p.M * l.out * l.in, &prof, p.M < 256 ? 2 : 0));
  PPLL_TRY(l.dt == BF16 ? forward<BF16>(s, p, kernel, l.units) : forward<F32>(s, p, kernel, l.units));
  return profile_end(s, prof);
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
  if (kernel != 0 && kernel != 1 && kernel != 3 && kernel != 4 && kernel != 8 && kernel != 10) { set_error("there is no kernel %d", kernel); return PPLL_ERR_CONFIG; }
  const ppll_rows none{nullptr, 0};
  return product((hipStream_t)stream, kernel, {precision == PPLL_BF16 ? BF16 : F32, rows, in, out, gelu ? PPLL_ACT_GELU : PPLL_ACT_NONE}, *x, *w, bias,
                 residual ? *residual : none, *y, slope ? *slope : none);
}
