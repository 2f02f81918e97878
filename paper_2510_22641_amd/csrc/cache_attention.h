// Device helpers shared by the kernels of attention over the 8-bit paged cache.
//
// Codes are whole numbers below 2^7 and scales powers of two: a code, or a code times a ratio of scales
// down to 2^-24, is exact in f16, so the products run on the f16 matrix instruction.  Queries enter scaled by a power of two that puts
// their row's largest element into [2^14, 2^15): bf16 ones as one f16 plane (11 bits against
// their 8), float32 ones as two (22 bits: an element is off by at most 2^-23 of itself, less than a
// sum of 64 products in float32 loses), either to 2^-39 of the row's largest.
//
// Weights enter the second product times their key's value scale, under a power of two of the
// row's own that follows the largest such product (struct Reference): a key counts there by what it
// adds to the output, so a block of large values with no weight, or one that the row may not attend,
// takes no bits from the others.  They are one plane for bf16 rows (2^-11, an eighth of the
// output's own rounding) and two for float32, up to 2^(W_EXP + REF_STEP) and for the largest seen
// at least 2^(W_EXP - NEAR - 1); those under f16's normal numbers are off by 2^-25.
#pragma once

#include "device.h"
#include "kernels.h"

#include <cfloat>
#include <cmath>

namespace ssd {

typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));

constexpr float LOG2E = 1.4426950408889634f;
constexpr int W_EXP = 7;         // exponent of the weights' scale
constexpr float REF_STEP = 8.f;  // in powers of two
constexpr int NO_EXP = -10000;   // exponent of a scale of 0, whose block has not been written

template <typename T> struct Planes { static constexpr int N = sizeof(T) == 4 ? 2 : 1; };

__device__ __forceinline__ uint32_t pack_f16x2(float a, float b) {
  const f16x2_t v = {(_Float16)a, (_Float16)b};
  return __builtin_bit_cast(uint32_t, v);
}

__device__ __forceinline__ f16x8_t f16_frag(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __builtin_bit_cast(f16x8_t, make_uint4(a, b, c, d));
}

// A pair of keys' scales over the largest, and what takes the codes' offset off again.
struct Ratio {
  f16x2_t r, off;
};
__device__ __forceinline__ Ratio ratio_of(float a, float b) {
  Ratio t;
  t.r = f16x2_t{(_Float16)a, (_Float16)b};
  t.off = t.r * f16x2_t{(_Float16)-1152.f, (_Float16)-1152.f};
  return t;
}

// Two bytes of dword w as f16 times their ratios: 0x64XX is 1024 + XX, so 1152 less leaves XX - 128,
// XX the code's byte with its top bit flipped.
__device__ __forceinline__ uint32_t code_pair(uint32_t w_flipped, uint32_t sel, const Ratio& t) {
  const f16x2_t v = __builtin_bit_cast(f16x2_t, __builtin_amdgcn_perm(0x64646464u, w_flipped, sel));
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(v, t.r, t.off));
}

// The codes themselves.
__device__ __forceinline__ uint32_t code_pair(uint32_t w_flipped, uint32_t sel) {
  const f16x2_t v = __builtin_bit_cast(f16x2_t, __builtin_amdgcn_perm(0x64646464u, w_flipped, sel));
  return __builtin_bit_cast(uint32_t, v - f16x2_t{(_Float16)1152.f, (_Float16)1152.f});
}

// Eight consecutive codes of a key's row, by code_pair's last argument.
template <typename... R>
__device__ __forceinline__ f16x8_t codes8(uint32_t a, uint32_t b, const R&... t) {
  a ^= 0x80808080u;
  b ^= 0x80808080u;
  return f16_frag(code_pair(a, 0x04010400, t...), code_pair(a, 0x04030402, t...), code_pair(b, 0x04010400, t...),
                  code_pair(b, 0x04030402, t...));
}

// Eight keys' dwords, four dimensions each: operand d is dimension d of the eight keys, by code_pair's
// last arguments t[k] of keys 2 k and 2 k + 1.
template <typename... R>
__device__ __forceinline__ void columns4(const uint32_t (&w)[8], f16x8_t (&out)[4], const R (&... t)[4]) {
  uint32_t p[4][4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const uint32_t a = w[2 * k] ^ 0x80808080u, b = w[2 * k + 1] ^ 0x80808080u;
    const uint32_t x = __builtin_amdgcn_perm(b, a, 0x05010400), y = __builtin_amdgcn_perm(b, a, 0x07030602);
    p[0][k] = code_pair(x, 0x04010400, t[k]...);
    p[1][k] = code_pair(x, 0x04030402, t[k]...);
    p[2][k] = code_pair(y, 0x04010400, t[k]...);
    p[3][k] = code_pair(y, 0x04030402, t[k]...);
  }
#pragma unroll
  for (int d = 0; d < 4; ++d) out[d] = f16_frag(p[d][0], p[d][1], p[d][2], p[d][3]);
}

// A scale's exponent.
__device__ __forceinline__ int exp_of(float s) {
  const int e = (int)(__float_as_uint(s) >> 23 & 0xff);
  return e ? e - 127 : NO_EXP;
}

// Two exponents in one word.
__device__ __forceinline__ int pair_of(int k, int v) { return v << 16 | (k & 0xffff); }
__device__ __forceinline__ int first_of(int p) { return (int16_t)p; }
__device__ __forceinline__ int second_of(int p) { return p >> 16; }

// What turns a product of a row of exponent qe and keys of scale 2^ke into a score, positive: |scale|,
// `unit` times, its mantissa and exponent apart, so that no part alone has to be in range.  (Products
// stay under 2^30: a score whose factor is no normal number is nothing.)
struct Factor {
  float m;
  int e;
  __device__ __forceinline__ Factor(float scale, float unit) {
    m = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(frexpf(fabsf(scale), &e) * unit)));
    e = __builtin_amdgcn_readfirstlane(e);
  }
  __device__ __forceinline__ float of(int qe, int ke) const { return fmaxf(ldexpf(m, e + qe + ke), FLT_MIN); }
};

// A product that is rounded whatever becomes of it.
__device__ __forceinline__ float rounded(float a, float b) {
#pragma clang fp contract(off)
  return a * b;
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

// The largest of three, or NaN (one instruction: the other maximum would first bring each to
// canonical form).
__device__ __forceinline__ float max3(float a, float b, float c) {
  return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c);
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

// The matrix operand of a query row: lane (row l % 16, g = l / 16) takes elements 64 (t / 2) + 16 g +
// 8 (t % 2) + i at step t, with the sign of `scale`, times 2^-(the exponent returned); NaN throughout
// where an element or `scale` is not finite.
template <typename T, int DH>
__device__ __forceinline__ int load_query(const T* row, int g, float scale, f16x8_t (&q)[DH / 32][Planes<T>::N]) {
  float f[DH / 32][8], top = 0.f;
  bool bad = false;
#pragma unroll
  for (int t = 0; t < DH / 32; ++t)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float v = load_elem(row + 64 * (t / 2) + 16 * g + 8 * (t % 2) + i);
      f[t][i] = v;
      top = fmaxf(top, fabsf(v));
      bad |= !(fabsf(v) <= FLT_MAX);
    }
  top = col_max(bad ? INFINITY : top);
  const bool fine = top <= FLT_MAX && fabsf(scale) <= FLT_MAX, some = top > 0.f && fine && scale != 0.f;
  const int e = some ? ilogbf(top) : 0;
#pragma unroll
  for (int t = 0; t < DH / 32; ++t) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      f[t][i] = some ? ldexpf(scale < 0.f ? -f[t][i] : f[t][i], 14 - e) : fine ? 0.f : NAN;
    f16_planes<Planes<T>::N>(f[t], q[t]);
  }
  return some ? e - 14 : 0;
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

// N (a multiple of 4) consecutive outputs of row `row` from dimension d of head `head` on.
template <typename T, int DH, int N>
__device__ __forceinline__ void store_result(const CacheAttnArgs& a, size_t row, size_t head, int d, const float* f) {
  if constexpr (sizeof(T) == 4) {
    if (a.out_planes) {
#pragma unroll
      for (int i = 0; i < N; i += 4)
        store_planes4(a.out_planes + plane_at((int)row, (int)head * DH + d + i, (a.rows + 15) >> 4), f[i], f[i + 1],
                      f[i + 2], f[i + 3]);
      return;
    }
  }
  store_out<T, N>(reinterpret_cast<T*>(a.out) + row * a.ldo + head * DH + d, f, a.out_vec);
}

// No row: what a key outside the sequence or on a page outside the pools has for its row of codes.
// (Row (page n_heads + head) page_size + offset of the pools; there are fewer than 2^32 of them.)
constexpr uint32_t NO_ROW = 0xffffffffu;

// Value (key) scales of keys that one exponent serves differ by at most this many powers of two.
constexpr int NEAR = 4, K_NEAR = 16;

// The running references of a row's softmax.  Scores are t = s * f (+ bias); without a bias f carries
// log2 e and t is in powers of two, with one t stays in natural units, where the type's lowest value
// is a finite number (times log2 e it would not be).  The weights e^(t - ref) sum up to the
// denominator; the second product takes them times 2^(value exponent + W_EXP - num).  Both begin
// below what any key has: the lowest value is its own reference, and -inf stays under it.
template <bool BIAS>
struct Reference {
  static constexpr float UNIT = BIAS ? LOG2E : 1.f;  // of t, in powers of two
  float ref = -FLT_MAX;      // subtracted from the scores
  float num = 2.f * NO_EXP;  // a whole number of powers of two beside it, the numerator's

  // Takes in new keys: `top`, their largest score, and `e`, the largest of their scores less top plus
  // the value exponents, in powers of two, or up to NEAR more (both the same in the row's four
  // lanes).  Whether any row of the wave moves, and then by what its sums shrink.
  __device__ __forceinline__ bool move(float top, float e, float& drop, float& num_drop) {
    drop = num_drop = 1.f;
    if (!__any(top - ref > fminf(REF_STEP / UNIT, (num + REF_STEP - e) * (1.f / UNIT)))) return false;
    const float next = fmaxf(ref, top), shift = (ref - next) * UNIT;
    const float n = ceilf(fmaxf(num + shift, fmaf(top - next, UNIT, e)));
    drop = __builtin_amdgcn_exp2f(shift);
    num_drop = __builtin_amdgcn_exp2f(num - n + shift);
    ref = next;
    num = n;
    return true;
  }
};

}  // namespace ssd
