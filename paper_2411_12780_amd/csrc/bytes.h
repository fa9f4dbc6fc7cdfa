// Rows of 8 bits (int8 q and an exponent e a row, q 2^e), the linear layer on them and group norm: what their kernels share and their launchers.
#pragma once
#include <type_traits>

#include "common.h"

namespace ppll {

constexpr int BYTE_NAN = -128;            // exponent of a row that stands for NaN
constexpr int BYTE_LEAST = -126, BYTE_MOST = 121;
constexpr int BYTE_COLS = 65536;          // columns at most: 127 * 127 * 65536 < 2^31
constexpr int64_t BYTE_LD = 1 << 20;      // bytes between rows at most: the rows of a tile stay under 2^31 bytes
constexpr int64_t ROW_LD = (int64_t)1 << 31, MAP_LD = 1 << 20;      // elements between rows, and between those of a linear layer or a map

inline int pad16(int v) { return (v + 15) & ~15; }

int launch_byte_rows_pack(hipStream_t s, int dt, int rows, int cols, const ppll_rows& in, const ppll_byte_rows& out);
int launch_byte_rows_unpack(hipStream_t s, int dt, int rows, int cols, const ppll_byte_rows& in, const ppll_rows& out);
int launch_byte_rows_pack_columns(hipStream_t s, int dt, int rows, int cols, const ppll_rows& in, const ppll_byte_rows& out);
// What rows a, and behind them rows b, stand for, in bf16, row by row; cols a multiple of 8, out 16-byte aligned
int launch_byte_rows_values(hipStream_t s, int cols, const ppll_byte_rows& a, int a_rows, const ppll_byte_rows& b, int b_rows, uint16_t* out);

// The linear layer.  residual, slope, bias may have null pointers.
struct ByteLinear {
  int dt, rows, in, out, activation;
  bool shared = false;      // as in GemmArgs
  int units = 0;
};
int launch_byte_linear_fwd(hipStream_t s, const ByteLinear& l, const ppll_byte_rows& x, const ppll_byte_rows& w, const float* bias, const ppll_rows& residual,
                           const ppll_rows& y, const ppll_rows& slope);
size_t byte_linear_workspace(const ByteLinear& l);
int launch_byte_linear_bwd(hipStream_t s, const ByteLinear& l, const ppll_byte_rows& x, const ppll_byte_rows& w, const ppll_rows& dy, const ppll_rows& gate,
                           const ppll_rows& dx, float* dw, float* db, char* ws);

struct GroupNorm {
  int dt, images, pixels, channels, groups, activation;
  float eps;
};
size_t group_norm_workspace(const GroupNorm& g);
int launch_group_norm_fwd(hipStream_t s, const GroupNorm& g, const ppll_rows& x, const float* scale, const float* shift, const ppll_rows& residual,
                          const ppll_rows& y, float* stats, const ppll_byte_rows& keep, char* ws);
// x.p null: from x8
int launch_group_norm_bwd(hipStream_t s, const GroupNorm& g, const ppll_rows& x, const ppll_byte_rows& x8, const float* stats, const float* scale,
                          const float* shift, const ppll_rows& residual, const ppll_rows& y, const ppll_rows& dy, const ppll_rows& dx, const ppll_rows& dres,
                          float* d_scale, float* d_shift, char* ws);

#ifdef __HIPCC__
// 2^e for e of -126 .. 127
__device__ __forceinline__ float exp2_bits(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
// What a row's values are multiplied by: 2^e, or NaN
__device__ __forceinline__ float byte_step(int e) { return e == BYTE_NAN ? __uint_as_float(0x7fc00000u) : exp2_bits(e); }
// Exponent of a row from the bits of its largest magnitude (those of a NaN are the largest of all): 127 2^e >= m 2^E, 1 <= m < 2, with
// e = E - 6 where m <= 127 / 64
__device__ __forceinline__ int byte_exponent(uint32_t most) {
  if (most >= 0x7f800000u) return BYTE_NAN;
  const int e = (int)(most >> 23) - 127 - 6 + ((most & 0x7fffffu) > 0x7e0000u);
  return min(max(e, BYTE_LEAST), BYTE_MOST);
}
// Four values times `inv` (2^-e) as bytes.  Adding 1.5 2^23 rounds to the nearest whole number, ties to even, which then lies in the low bits;
// the bound is met by rows over 127 2^121 only.
__device__ __forceinline__ uint32_t byte_pack4(float a, float b, float c, float d, float inv) {
  auto q = [&](float v) { return __float_as_uint(__builtin_amdgcn_fmed3f(v * inv, -127.f, 127.f) + 12582912.f); };
  const uint32_t lo = __builtin_amdgcn_perm(q(b), q(a), 0x0c0c0400u), hi = __builtin_amdgcn_perm(q(d), q(c), 0x04000c0cu);
  return lo | hi;
}

// Eight neighbouring elements of a row, c .. c + 7, whatever their alignment; those at `cols` and behind read as 0.  (load_all, store_all: all
// eight are there.)
template <int DT> struct Eight;
template <> struct Eight<F32> {
  float4 a, b;
  __device__ __forceinline__ void load(const void* row, int c, int cols) {
    const float* p = (const float*)row + c;
    if (c + 8 <= cols) {
      __builtin_memcpy(&a, p, 16);
      __builtin_memcpy(&b, p + 4, 16);
    } else {
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = c + i < cols ? p[i] : 0.f;
      a = make_float4(v[0], v[1], v[2], v[3]); b = make_float4(v[4], v[5], v[6], v[7]);
    }
  }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  }
  __device__ __forceinline__ void set(const float (&v)[8]) { a = make_float4(v[0], v[1], v[2], v[3]); b = make_float4(v[4], v[5], v[6], v[7]); }
  __device__ __forceinline__ void zero() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ __forceinline__ void load_all(const char* p) { __builtin_memcpy(&a, p, 16); __builtin_memcpy(&b, p + 16, 16); }
  __device__ __forceinline__ void store_all(char* p) const { __builtin_memcpy(p, &a, 16); __builtin_memcpy(p + 16, &b, 16); }
  __device__ __forceinline__ void store(void* row, int c, int cols) const {
    float* p = (float*)row + c;
    if (c + 8 <= cols) {
      __builtin_memcpy(p, &a, 16);
      __builtin_memcpy(p + 4, &b, 16);
    } else {
      float v[8];
      get(v);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (c + i < cols) p[i] = v[i];
    }
  }
};
template <> struct Eight<BF16> {
  uint4 w;
  __device__ __forceinline__ void load(const void* row, int c, int cols) {
    const uint16_t* p = (const uint16_t*)row + c;
    if (c + 8 <= cols) {
      __builtin_memcpy(&w, p, 16);
    } else {
      uint32_t v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = c + i < cols ? p[i] : 0;
      w = make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
    }
  }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(u[i] << 16); v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u); }
  }
  __device__ __forceinline__ void set(const float (&v)[8]) {
    w = make_uint4(f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3]), f32x2_to_bf16x2(v[4], v[5]), f32x2_to_bf16x2(v[6], v[7]));
  }
  __device__ __forceinline__ void zero() { w = make_uint4(0, 0, 0, 0); }
  __device__ __forceinline__ void load_all(const char* p) { __builtin_memcpy(&w, p, 16); }
  __device__ __forceinline__ void store_all(char* p) const { __builtin_memcpy(p, &w, 16); }
  __device__ __forceinline__ void store(void* row, int c, int cols) const {
    uint16_t* p = (uint16_t*)row + c;
    if (c + 8 <= cols) {
      __builtin_memcpy(p, &w, 16);
    } else {
      const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (c + i < cols) p[i] = (uint16_t)(u[i >> 1] >> (16 * (i & 1)));
    }
  }
};
// Eight bytes of a row times the row's step
__device__ __forceinline__ void bytes_get(uint2 w, float step, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) { v[i] = (float)(int8_t)(w.x >> (8 * i)) * step; v[4 + i] = (float)(int8_t)(w.y >> (8 * i)) * step; }
}
__device__ __forceinline__ uint2 bytes_of(const float (&v)[8], float inv) {
  return make_uint2(byte_pack4(v[0], v[1], v[2], v[3], inv), byte_pack4(v[4], v[5], v[6], v[7], inv));
}
// The largest of a value over `lanes` neighbouring lanes (a power of two, 1 to 64), every lane receiving it.  Within 8 lanes by exchanges of
// pairs, of pairs of pairs and the mirror of 8; above as lanes_reduce.
__device__ __forceinline__ uint32_t lanes_most_of(uint32_t v, int lanes) {
  auto dpp = [](uint32_t x, auto ctrl) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, decltype(ctrl)::value, 0xf, 0xf, true); };
  if (lanes >= 2) v = max(v, dpp(v, std::integral_constant<int, 0xb1>()));     // quad_perm 1 0 3 2
  if (lanes >= 4) v = max(v, dpp(v, std::integral_constant<int, 0x4e>()));     // quad_perm 2 3 0 1
  if (lanes >= 8) v = max(v, dpp(v, std::integral_constant<int, 0x141>()));    // mirror of 8 lanes
  if (lanes >= 16) v = max(v, dpp(v, std::integral_constant<int, 0x128>()));   // rotation of 16 by 8
  if (lanes >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = max((uint32_t)r[0], (uint32_t)r[1]);
  }
  if (lanes >= 64) {
    const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    v = max((uint32_t)r[0], (uint32_t)r[1]);
  }
  return v;
}
template <int LANES> __device__ __forceinline__ uint32_t lanes_most(uint32_t v) { return lanes_most_of(v, LANES); }
__device__ __forceinline__ uint32_t most_of(const float (&v)[8], uint32_t m) {
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
  return m;
}
#endif

}  // namespace ppll
