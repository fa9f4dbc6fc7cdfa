// Rows of 8 bits: into them, out of them, and out of the columns of a matrix.
//
// L neighbouring lanes hold a row in pieces of 8 elements, P each, read once; the largest magnitude goes round the lanes in registers and the
// bytes leave 8 a lane.  What bounds it: memory, 3 bytes an element from bf16 (25216 x 1536 20 us in, 18 out: 5.8 and 6.5 TB/s with the last-level cache; 25216 x
// 6144 97, 4.8 TB/s).
#include <algorithm>

#include "bytes.h"

namespace ppll {

namespace {
constexpr int THREADS = 256;
constexpr unsigned MOST_BLOCKS = 1u << 20;

template <int DT, int L, int P>
__global__ __launch_bounds__(THREADS) void byte_rows_pack_kernel(const char* in, int64_t in_ld, int8_t* q, int8_t* e, int64_t q_ld, int rows, int cols) {
  constexpr int R = THREADS / L, ESZ = DT == BF16 ? 2 : 4;
  const int lane = threadIdx.x % L, pieces = (cols + 15) / 16 * 2;
  for (int64_t r = (int64_t)blockIdx.x * R + threadIdx.x / L; r < rows; r += (int64_t)gridDim.x * R) {
    const char* row = in + r * in_ld * ESZ;
    Eight<DT> v[P];
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int c = (lane + i * L) * 8;
      if (c < cols) v[i].load(row, c, cols);
      else v[i].zero();
    }
    uint32_t most = 0;
    float f[8];
#pragma unroll
    for (int i = 0; i < P; ++i) { v[i].get(f); most = most_of(f, most); }
    const int x = byte_exponent(lanes_most<L>(most));
    const bool nan = x == BYTE_NAN;
    const float inv = exp2_bits(nan ? 0 : -x);
    if (lane == 0) e[r] = (int8_t)x;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int p = lane + i * L;
      v[i].get(f);
      if (p < pieces) *(uint2*)(q + r * q_ld + p * 8) = nan ? make_uint2(0, 0) : bytes_of(f, inv);
    }
  }
}

// Rows that the lanes do not hold: read twice, a wave each
template <int DT>
__global__ __launch_bounds__(THREADS) void byte_rows_pack_long_kernel(const char* in, int64_t in_ld, int8_t* q, int8_t* e, int64_t q_ld, int rows, int cols) {
  constexpr int R = THREADS / 64, ESZ = DT == BF16 ? 2 : 4;
  const int lane = threadIdx.x % 64, pieces = (cols + 15) / 16 * 2;
  for (int64_t r = (int64_t)blockIdx.x * R + threadIdx.x / 64; r < rows; r += (int64_t)gridDim.x * R) {
    const char* row = in + r * in_ld * ESZ;
    uint32_t most = 0;
    float f[8];
    for (int p = lane; p * 8 < cols; p += 64) {
      Eight<DT> v;
      v.load(row, p * 8, cols);
      v.get(f);
      most = most_of(f, most);
    }
    const int x = byte_exponent(lanes_most<64>(most));
    const bool nan = x == BYTE_NAN;
    const float inv = exp2_bits(nan ? 0 : -x);
    if (lane == 0) e[r] = (int8_t)x;
    for (int p = lane; p < pieces; p += 64) {
      Eight<DT> v;
      v.zero();
      if (p * 8 < cols) v.load(row, p * 8, cols);
      v.get(f);
      *(uint2*)(q + r * q_ld + p * 8) = nan ? make_uint2(0, 0) : bytes_of(f, inv);
    }
  }
}

template <int DT, int L>
__global__ __launch_bounds__(THREADS) void byte_rows_unpack_kernel(const int8_t* q, const int8_t* e, int64_t q_ld, char* out, int64_t out_ld, int rows, int cols) {
  constexpr int R = THREADS / L, ESZ = DT == BF16 ? 2 : 4;
  const int lane = threadIdx.x % L;
  for (int64_t r = (int64_t)blockIdx.x * R + threadIdx.x / L; r < rows; r += (int64_t)gridDim.x * R) {
    const float step = byte_step(e[r]);
    char* row = out + r * out_ld * ESZ;
#pragma unroll 4
    for (int c = lane * 8; c < cols; c += L * 8) {
      const uint2 w = *(const uint2*)(q + r * q_ld + c);
      float f[8];
      bytes_get(w, step, f);
      Eight<DT> v;
      v.set(f);
      v.store(row, c, cols);
    }
  }
}

// Two operands of as many columns, one behind the other, to bf16 rows without room between them
template <int L>
__global__ __launch_bounds__(THREADS) void byte_rows_values_kernel(ppll_byte_rows a, int a_rows, ppll_byte_rows b, int b_rows, uint16_t* out, int cols) {
  constexpr int R = THREADS / L;
  const int lane = threadIdx.x % L;
  for (int64_t r = (int64_t)blockIdx.x * R + threadIdx.x / L; r < (int64_t)a_rows + b_rows; r += (int64_t)gridDim.x * R) {
    const bool first = r < a_rows;
    const int64_t k = first ? r : r - a_rows;
    const int8_t* q = first ? a.q + k * a.ld : b.q + k * b.ld;
    const float step = byte_step(first ? a.e[k] : b.e[k]);
#pragma unroll 4
    for (int c = lane * 8; c < cols; c += L * 8) {
      float f[8];
      bytes_get(*(const uint2*)(q + c), step, f);
      Eight<BF16> v;
      v.set(f);
      *(uint4*)(out + r * cols + c) = v.w;
    }
  }
}

// 8 columns a workgroup: their largest magnitudes over all rows, then the bytes, turned in LDS.  A thread has 4 rows, one behind the other, so that
// four bytes of a column are a word; the first 4096 rows stay in registers between the two passes.  A weight is small beside the chip, so what bounds
// this is how few loads wait on each other: 32 columns a workgroup of 512, 128 rows at a time and all rows loaded twice, took 20 us a weight on average
// over the four weights of an encoder layer of width 768 (fp32), where this takes 7.  The 32-byte pieces of a line belong to neighbouring
// workgroups: those of one XCD (workgroup id % 8) are neighbours.
constexpr int TC = 8, CT = 512, UNITS = 2, CHUNK = CT * 4 * UNITS, CPITCH = CHUNK + 16;
template <int DT>
__global__ __launch_bounds__(CT) void byte_rows_pack_columns_kernel(const char* in, int64_t in_ld, int8_t* q, int8_t* e, int64_t q_ld, int rows, int cols,
                                                                    int groups) {
  constexpr int ESZ = DT == BF16 ? 2 : 4;
  __shared__ uint32_t most[CT / 64][TC];
  __shared__ __align__(16) uint32_t turned[TC][CPITCH / 4];
  const int group = (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3);
  if (group >= groups) return;
  const int c0 = group * TC, ncols = cols - c0, padded = (rows + 15) & ~15;
  const char* base = in + (int64_t)c0 * ESZ;
  Eight<DT> kept[UNITS][4];
  uint32_t m[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  auto load = [&](int k0) {
#pragma unroll
    for (int u = 0; u < UNITS; ++u)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int r = k0 + (u * CT + (int)threadIdx.x) * 4 + j;
        if (r < rows) kept[u][j].load(base + r * in_ld * ESZ, 0, ncols);
        else kept[u][j].zero();
      }
  };
  for (int k0 = (rows - 1) / CHUNK * CHUNK; k0 >= 0; k0 -= CHUNK) {     // the first rows last: they are kept
    load(k0);
#pragma unroll
    for (int u = 0; u < UNITS; ++u)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float f[8];
        kept[u][j].get(f);
#pragma unroll
        for (int i = 0; i < 8; ++i) m[i] = max(m[i], __float_as_uint(f[i]) & 0x7fffffffu);
      }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    m[i] = lanes_most<64>(m[i]);
    if ((threadIdx.x & 63) == 0) most[threadIdx.x >> 6][i] = m[i];
  }
  __syncthreads();
  float inv[8];
  uint32_t fine[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    uint32_t v = most[0][i];
#pragma unroll
    for (int w = 1; w < CT / 64; ++w) v = max(v, most[w][i]);
    const int x = byte_exponent(v);
    if (threadIdx.x == i && i < ncols) e[c0 + i] = (int8_t)x;
    inv[i] = exp2_bits(x == BYTE_NAN ? 0 : -x);
    fine[i] = x == BYTE_NAN ? 0u : ~0u;
  }
  for (int k0 = 0; k0 < padded; k0 += CHUNK) {
    if (k0) load(k0);
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
      float f[4][8];
#pragma unroll
      for (int j = 0; j < 4; ++j) kept[u][j].get(f[j]);
#pragma unroll
      for (int i = 0; i < 8; ++i) turned[i][u * CT + threadIdx.x] = byte_pack4(f[0][i], f[1][i], f[2][i], f[3][i], inv[i]) & fine[i];
    }
    __syncthreads();
    const int chunk = min(CHUNK, padded - k0), c = threadIdx.x >> 6;      // a wave a column
    if (c < ncols)
      for (int k = (threadIdx.x & 63) * 16; k < chunk; k += 64 * 16) *(uint4*)(q + (int64_t)(c0 + c) * q_ld + k0 + k) = *(const uint4*)&turned[c][k / 4];
    __syncthreads();
  }
}
static_assert(TC == CT / 64 && CPITCH % 16 == 0, "");

unsigned blocks_of(int rows, int per) {
  const unsigned n = (unsigned)(((int64_t)rows + per - 1) / per);
  return n < MOST_BLOCKS ? n : MOST_BLOCKS;
}
template <int DT, int L, int P> int pack(hipStream_t s, int rows, int cols, const ppll_rows& in, const ppll_byte_rows& out) {
  hipLaunchKernelGGL((byte_rows_pack_kernel<DT, L, P>), dim3(blocks_of(rows, THREADS / L)), dim3(THREADS), 0, s, (const char*)in.p, in.ld, out.q, out.e, out.ld,
                     rows, cols);
  PPLL_HIP(hipGetLastError());
  return PPLL_OK;
}
template <int DT> int pack_any(hipStream_t s, int rows, int cols, const ppll_rows& in, const ppll_byte_rows& out) {
  const int pieces = (cols + 15) / 16 * 2;
  if (pieces <= 4) return pack<DT, 1, 4>(s, rows, cols, in, out);
  if (pieces <= 8) return pack<DT, 2, 4>(s, rows, cols, in, out);
  if (pieces <= 16) return pack<DT, 4, 4>(s, rows, cols, in, out);
  if (pieces <= 32) return pack<DT, 8, 4>(s, rows, cols, in, out);
  if (pieces <= 64) return pack<DT, 16, 4>(s, rows, cols, in, out);
  if (pieces <= 128) return pack<DT, 32, 4>(s, rows, cols, in, out);
  if (pieces <= 256) return pack<DT, 64, 4>(s, rows, cols, in, out);
  if (pieces <= 512) return pack<DT, 64, 8>(s, rows, cols, in, out);
  if (pieces <= 1024) return pack<DT, 64, 16>(s, rows, cols, in, out);
  hipLaunchKernelGGL((byte_rows_pack_long_kernel<DT>), dim3(blocks_of(rows, THREADS / 64)), dim3(THREADS), 0, s, (const char*)in.p, in.ld, out.q, out.e, out.ld,
                     rows, cols);
  PPLL_HIP(hipGetLastError());
  return PPLL_OK;
}
template <int DT, int L> int unpack(hipStream_t s, int rows, int cols, const ppll_byte_rows& in, const ppll_rows& out) {
  hipLaunchKernelGGL((byte_rows_unpack_kernel<DT, L>), dim3(blocks_of(rows, THREADS / L)), dim3(THREADS), 0, s, in.q, in.e, in.ld, (char*)out.p, out.ld, rows,
                     cols);
  PPLL_HIP(hipGetLastError());
  return PPLL_OK;
}
template <int DT> int unpack_any(hipStream_t s, int rows, int cols, const ppll_byte_rows& in, const ppll_rows& out) {
  if (cols <= 32) return unpack<DT, 1>(s, rows, cols, in, out);
  if (cols <= 128) return unpack<DT, 4>(s, rows, cols, in, out);
  if (cols <= 512) return unpack<DT, 16>(s, rows, cols, in, out);
  return unpack<DT, 64>(s, rows, cols, in, out);
}
}  // namespace

int launch_byte_rows_pack(hipStream_t s, int dt, int rows, int cols, const ppll_rows& in, const ppll_byte_rows& out) {
  if (rows <= 0) return PPLL_OK;
  return dt == BF16 ? pack_any<BF16>(s, rows, cols, in, out) : pack_any<F32>(s, rows, cols, in, out);
}
int launch_byte_rows_unpack(hipStream_t s, int dt, int rows, int cols, const ppll_byte_rows& in, const ppll_rows& out) {
  if (rows <= 0) return PPLL_OK;
  return dt == BF16 ? unpack_any<BF16>(s, rows, cols, in, out) : unpack_any<F32>(s, rows, cols, in, out);
}
int launch_byte_rows_values(hipStream_t s, int cols, const ppll_byte_rows& a, int a_rows, const ppll_byte_rows& b, int b_rows, uint16_t* out) {
  const int64_t rows = (int64_t)a_rows + b_rows;
  auto grid = [&](int per) { return dim3((unsigned)std::min<int64_t>((rows + per - 1) / per, MOST_BLOCKS)); };
  if (cols <= 512) hipLaunchKernelGGL((byte_rows_values_kernel<16>), grid(THREADS / 16), dim3(THREADS), 0, s, a, a_rows, b, b_rows, out, cols);
  else hipLaunchKernelGGL((byte_rows_values_kernel<64>), grid(THREADS / 64), dim3(THREADS), 0, s, a, a_rows, b, b_rows, out, cols);
  PPLL_HIP(hipGetLastError());
  return PPLL_OK;
}
int launch_byte_rows_pack_columns(hipStream_t s, int dt, int rows, int cols, const ppll_rows& in, const ppll_byte_rows& out) {
  if (cols <= 0) return PPLL_OK;
  const int groups = (cols + TC - 1) / TC;
  const dim3 grid((groups + 7) / 8 * 8);
  if (dt == BF16)
    hipLaunchKernelGGL(byte_rows_pack_columns_kernel<BF16>, grid, dim3(CT), 0, s, (const char*)in.p, in.ld, out.q, out.e, out.ld, rows, cols, groups);
  else
    hipLaunchKernelGGL(byte_rows_pack_columns_kernel<F32>, grid, dim3(CT), 0, s, (const char*)in.p, in.ld, out.q, out.e, out.ld, rows, cols, groups);
  PPLL_HIP(hipGetLastError());
  return PPLL_OK;
}

}  // namespace ppll
