// Device helpers shared by the kernels of attention over the 8-bit paged cache.
//
// Codes are whole numbers below 2^7, which f16 holds exactly, so the products run on the f16 matrix
// instruction and the blocks' scales are applied to scores and weights.  Queries enter scaled by
// a power of two that puts their row's largest element into [2^14, 2^15): bf16 ones as one f16
// plane (11 bits against their 8), float32 ones as two (22 bits: an element is off by at most
// 2^-23 of itself, less than a sum of 64 products in float32 loses).  Weights, scaled likewise, are
// one plane for bf16 rows (2^-11, an eighth of the output's own rounding) and two for float32.
// Below 2^-29 of a row's largest, where f16's exponents end, they are off by 2^-40 of it.
#pragma once

#include "device.h"
#include "kernels.h"

#include <cfloat>
#include <cmath>

namespace ssd {

typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));

constexpr float LOG2E = 1.4426950408889634f;
constexpr float W_TOP = 32768.f;  // weights' scale

template <typename T> struct Planes { static constexpr int N = sizeof(T) == 4 ? 2 : 1; };

__device__ __forceinline__ uint32_t pack_f16x2(float a, float b) {
  const f16x2_t v = {(_Float16)a, (_Float16)b};
  return __builtin_bit_cast(uint32_t, v);
}

__device__ __forceinline__ f16x8_t f16_frag(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __builtin_bit_cast(f16x8_t, make_uint4(a, b, c, d));
}

// Codes of dword w as f16: 0x64XX is 1024 + XX, from which 1152 leaves XX - 128, XX the code's
// byte with its top bit flipped.
__device__ __forceinline__ uint32_t code_pair(uint32_t w_flipped, uint32_t sel) {
  const f16x2_t off = {(_Float16)-1152.f, (_Float16)-1152.f};
  return __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2_t, __builtin_amdgcn_perm(0x64646464u, w_flipped, sel)) + off);
}

// Eight consecutive codes of a row.
__device__ __forceinline__ f16x8_t codes8(uint32_t a, uint32_t b) {
  a ^= 0x80808080u;
  b ^= 0x80808080u;
  return f16_frag(code_pair(a, 0x04010400), code_pair(a, 0x04030402), code_pair(b, 0x04010400), code_pair(b, 0x04030402));
}

// Eight rows' dwords, four dimensions each: operand d is dimension d of the eight keys.
__device__ __forceinline__ void columns4(const uint32_t (&w)[8], f16x8_t (&out)[4]) {
  uint32_t p[4][4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const uint32_t a = w[2 * k] ^ 0x80808080u, b = w[2 * k + 1] ^ 0x80808080u;
    const uint32_t x = __builtin_amdgcn_perm(b, a, 0x05010400), y = __builtin_amdgcn_perm(b, a, 0x07030602);
    p[0][k] = code_pair(x, 0x04010400);
    p[1][k] = code_pair(x, 0x04030402);
    p[2][k] = code_pair(y, 0x04010400);
    p[3][k] = code_pair(y, 0x04030402);
  }
#pragma unroll
  for (int d = 0; d < 4; ++d) out[d] = f16_frag(p[d][0], p[d][1], p[d][2], p[d][3]);
}

// Eight floats as N f16 planes, each the rounding of what the one before leaves.
template <int N>
__device__ __forceinline__ void f16_planes(const float (&f)[8], f16x8_t (&out)[N]) {
  uint32_t h[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = pack_f16x2(f[2 * i], f[2 * i + 1]);
  out[0] = f16_frag(h[0], h[1], h[2], h[3]);
  if constexpr (N == 2) {
    uint32_t l[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f16x2_t v = __builtin_bit_cast(f16x2_t, h[i]);
      l[i] = pack_f16x2(f[2 * i] - (float)v[0], f[2 * i + 1] - (float)v[1]);
    }
    out[1] = f16_frag(l[0], l[1], l[2], l[3]);
  }
}

// The maximum over the four lanes l % 16 + 16 g of a column.
__device__ __forceinline__ float col_max(float v) {
  v = fmaxf(v, __shfl_xor(v, 16, SSD_WAVE));
  return fmaxf(v, __shfl_xor(v, 32, SSD_WAVE));
}
__device__ __forceinline__ float col_sum(float v) {
  v += __shfl_xor(v, 16, SSD_WAVE);
  return v + __shfl_xor(v, 32, SSD_WAVE);
}

// The matrix operand of a query row: lane (row l % 16, g = l / 16) takes elements g DH / 4 + 8 t + i
// of step t.  Returns what turns a product with it into a score over `scale`: 2^(e - 14), or NaN
// where an element is not finite.
template <typename T, int DH>
__device__ __forceinline__ float load_query(const T* row, int g, f16x8_t (&q)[DH / 32][Planes<T>::N]) {
  float f[DH / 32][8], top = 0.f;
  bool bad = false;
#pragma unroll
  for (int t = 0; t < DH / 32; ++t)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float v = load_elem(row + g * (DH / 4) + 8 * t + i);
      f[t][i] = v;
      top = fmaxf(top, fabsf(v));
      bad |= !(fabsf(v) <= FLT_MAX);
    }
  top = col_max(bad ? INFINITY : top);
  const int e = ilogbf(top);  // (INT_MAX or so where top is 0 or infinite: no use is made of it)
  const bool fine = top <= FLT_MAX, some = top > 0.f && fine;
#pragma unroll
  for (int t = 0; t < DH / 32; ++t) {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[t][i] = some ? ldexpf(f[t][i], 14 - e) : 0.f;
    f16_planes<Planes<T>::N>(f[t], q[t]);
  }
  return fine ? (some ? ldexpf(1.f, e - 14) : 0.f) : NAN;
}

// The rows of sequence b: first row and count, kept inside the buffers whatever row_start holds.
__device__ __forceinline__ void seq_rows(const CacheAttnArgs& a, int b, int& r0, int& n) {
  if (!a.row_start) {
    r0 = b * a.max_rows;
    n = min(a.max_rows, a.rows - r0);
    return;
  }
  r0 = a.row_start[b];
  const int r1 = min(a.row_start[b + 1], a.rows);
  if (r0 < 0 || r0 > r1) { r0 = 0; n = 0; return; }
  n = r1 - r0;
  if (n > a.max_rows) {
    n = a.max_rows;
    atomicOr(a.status, SSD_DEV_CAPACITY);
  }
}

// N consecutive outputs of a row.
template <typename T, int N>
__device__ __forceinline__ void store_out(T* o, const float* f, bool vec) {
  if (!vec) {
#pragma unroll
    for (int i = 0; i < N; ++i) store_elem(o + i, f[i]);
  } else if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < N; i += 4) *reinterpret_cast<float4*>(o + i) = make_float4(f[i], f[i + 1], f[i + 2], f[i + 3]);
  } else {
#pragma unroll
    for (int i = 0; i < N; i += 4)
      *reinterpret_cast<uint2*>(o + i) = make_uint2(pack_bf16x2(f[i], f[i + 1]), pack_bf16x2(f[i + 2], f[i + 3]));
  }
}

// No row: what a key outside the sequence or on a page outside the pools has for its row of codes.
// (Row (page n_heads + head) page_size + offset of the pools; there are fewer than 2^32 of them.)
constexpr uint32_t NO_ROW = 0xffffffffu;

// i / page_size for i < 2^24, page_size <= 256, with inv = ceil(2^32 / page_size) (page_size 1: the
// quotient is i)
__device__ __forceinline__ int page_of(int i, int page_size, uint32_t inv) {
  return page_size == 1 ? i : (int)__umulhi((uint32_t)i, inv);
}

}  // namespace ssd
