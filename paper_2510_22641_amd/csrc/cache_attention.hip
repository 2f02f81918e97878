// Softmax attention over the 8-bit paged cache.
//
// Query row j of sequence b sits at position p = seq_len[b] + pos_off + j and attends positions
// 0 .. p of its pages; the scores are q . c s_k scale + bias[h][p - i] with c the key's codes and s_k
// its block's scale, the output sum_i w_i s_v c_i over the softmax weights w.  Codes are whole numbers
// below 2^7, which bf16 holds exactly, so the products run on the bf16 matrix instruction with the
// scales applied to scores and weights: float32 queries and weights enter as three bf16 planes
// (24 bits, as float32 itself), bf16 queries as they are and their weights as two planes.
#include "device.h"
#include "kernels.h"

#include <cmath>

namespace ssd {

namespace {

constexpr float LOG2E = 1.4426950408889634f;

// bf16 pairs of two codes' bytes.
__device__ __forceinline__ float code_f(uint32_t w, int i) { return (float)(int8_t)(w >> (8 * i)); }

__device__ __forceinline__ bf16x8_t as_frag(const uint32_t (&w)[4]) {
  return __builtin_bit_cast(bf16x8_t, make_uint4(w[0], w[1], w[2], w[3]));
}

// Eight consecutive codes as a matrix operand.
__device__ __forceinline__ bf16x8_t frag_of(uint32_t a, uint32_t b) {
  const uint32_t w[4] = {pack_bf16x2(code_f(a, 0), code_f(a, 1)), pack_bf16x2(code_f(a, 2), code_f(a, 3)),
                         pack_bf16x2(code_f(b, 0), code_f(b, 1)), pack_bf16x2(code_f(b, 2), code_f(b, 3))};
  return as_frag(w);
}

// Eight floats as NP bf16 planes: each the rounding of what the planes before it leave.
template <int NP>
__device__ __forceinline__ void planes_of(const float* f, bf16x8_t (&out)[NP]) {
  float r[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = f[i];
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w[i] = pack_bf16x2(r[2 * i], r[2 * i + 1]);
      r[2 * i] -= __uint_as_float(w[i] << 16);
      r[2 * i + 1] -= __uint_as_float(w[i] & 0xffff0000u);
    }
    out[p] = as_frag(w);
  }
}

template <typename T> struct Planes;                       // planes of queries, of weights
template <> struct Planes<float> { static constexpr int Q = 3, P = 3; };
template <> struct Planes<bf16_t> { static constexpr int Q = 1, P = 2; };

constexpr int AW = 4;   // waves a block
constexpr int UNIT = 32;  // keys a wave takes at once

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

// DT consecutive outputs of a row.
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

// 16 (row, head) pairs of one sequence and cache head a block, one of `splits` ranges of their keys.
// Pair u of the sequence is row u / G, head hk G + u % G.  A wave takes units of 32 keys straight
// from memory to matrix operands: lane (r = l % 16, g = l / 16) loads d_head / 4 codes of keys r and
// 16 + r, which are its rows of S^T = K Q^T (key order and the order of d are free as long as both
// operands agree); the scores land with lane (pair l % 16, keys 4 g + e of either half), which is
// again the operand layout of the weights in O^T = V^T P^T when its K index 8 g + i names key
// 4 g + i % 4 of half i / 4, so neither scores nor weights cross lanes but for the maximum.  V is
// read row by row, d_head / 16 codes a lane, and its bytes picked per output dimension while they
// are converted.  Each wave keeps its own maximum and sum; they meet in LDS once.
template <typename T, int DH, bool BIAS>
__global__ __launch_bounds__(64 * AW) void cache_attn_kernel(const CacheAttnArgs a, const int tiles, const int splits) {
  constexpr int KS = DH / 32;   // steps of 32 over d_head
  constexpr int NB = DH / 16;   // output blocks of 16 dimensions
  constexpr int KW = DH / 16;   // dwords of K a lane and key half
  constexpr int VW = DH / 64;   // dwords of V a lane and key
  constexpr int NQ = Planes<T>::Q, NP = Planes<T>::P;
  __shared__ float xo[AW][16][DH + 4];
  __shared__ float xm[AW][16], xl[AW][16];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, g = lane >> 4;
  const int hk = blockIdx.x % a.n_heads, bt = blockIdx.x / a.n_heads;
  const int b = bt / tiles, tile = bt - b * tiles, split = blockIdx.y;
  const int G = a.n_q_heads / a.n_heads;
  int r0, nr;
  seq_rows(a, b, r0, nr);
  const int u0 = tile * 16;
  if (u0 >= nr * G) return;  // whole blocks
  const int u = min(u0 + n, nr * G - 1), j = u / G, hq = hk * G + (u - j * G);
  const int base = a.seq_len[b] + a.pos_off;
  const long long cap = (long long)a.max_pages * a.page_size;
  const int pos = base + j;                                    // this lane's row
  const int last = base + (min(u0 + 15, nr * G - 1)) / G;      // the tile's last row
  const int kend = (int)min((long long)last + 1, cap);
  if (last >= cap && tid == 0 && split == 0) atomicOr(a.status, SSD_DEV_CAPACITY);
  const int units = kend > 0 ? (kend + UNIT - 1) / UNIT : 0;
  const int per = (units + splits - 1) / splits;
  const int x0 = split * per, x1 = min(x0 + per, units);

  bf16x8_t q[KS][NQ];
  {
    const T* qp = reinterpret_cast<const T*>(a.q) + (size_t)(r0 + j) * a.ldq + (size_t)hq * DH + g * (DH / 4);
#pragma unroll
    for (int t = 0; t < KS; ++t) {
      float f[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = load_elem(qp + 8 * t + i);
      planes_of<NQ>(f, q[t]);
    }
  }
  f32x4_t o[NB];
#pragma unroll
  for (int i = 0; i < NB; ++i) o[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;
  const int32_t* table = a.page_table + (size_t)b * a.max_pages;
  const size_t head_bytes = (size_t)a.page_size * DH;

  for (int x = x0 + wave; x < x1; x += AW) {
    // page, offset and scales of key x 32 + lane % 32
    const int key = x * UNIT + (lane & 31);
    int page = -1, off = 0;
    float ks = 0.f, vs = 0.f;
    if (key < kend) {
      const int pi = key / a.page_size;
      off = key - pi * a.page_size;
      page = table[pi];
      if (page < 0 || page >= a.n_pages) {
        atomicOr(a.status, SSD_DEV_BAD_PAGE);
        page = -1;
      } else {
        const size_t sc = (size_t)page * a.n_heads + hk;
        ks = a.k_scale[sc];
        vs = a.v_scale[sc];
      }
    }
    uint4 kr[2][KW / 4];
    uint32_t vr[8][VW];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int kp = __shfl(page, 16 * h + n, SSD_WAVE), ko = __shfl(off, 16 * h + n, SSD_WAVE);
#pragma unroll
      for (int i = 0; i < KW / 4; ++i) kr[h][i] = make_uint4(0, 0, 0, 0);
      if (kp >= 0) {
        const int8_t* p = a.k_codes + ((size_t)kp * a.n_heads + hk) * head_bytes + (size_t)ko * DH + g * (DH / 4);
#pragma unroll
        for (int i = 0; i < KW / 4; ++i) kr[h][i] = reinterpret_cast<const uint4*>(p)[i];
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int vp = __shfl(page, 16 * h + 4 * g + e, SSD_WAVE), vo = __shfl(off, 16 * h + 4 * g + e, SSD_WAVE);
#pragma unroll
        for (int i = 0; i < VW; ++i) vr[4 * h + e][i] = 0;
        if (vp >= 0) {
          const int8_t* p = a.v_codes + ((size_t)vp * a.n_heads + hk) * head_bytes + (size_t)vo * DH + n * (DH / 16);
#pragma unroll
          for (int i = 0; i < VW; ++i) vr[4 * h + e][i] = reinterpret_cast<const uint32_t*>(p)[i];
        }
      }
    }
    float s[8], vsc[8];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int t = 0; t < KS; ++t) {
        const uint32_t* kw = reinterpret_cast<const uint32_t*>(&kr[h][0]);
        const bf16x8_t kf = frag_of(kw[2 * t], kw[2 * t + 1]);
#pragma unroll
        for (int p = 0; p < NQ; ++p) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, q[t][NQ - 1 - p], acc, 0, 0, 0);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int src = 16 * h + 4 * g + e, i = x * UNIT + src;
        const int kp = __shfl(page, src, SSD_WAVE);
        float v = acc[e] * __shfl(ks, src, SSD_WAVE) * a.scale;
        vsc[4 * h + e] = __shfl(vs, src, SSD_WAVE);
        const bool in = i <= pos && kp >= 0;
        if (BIAS && in) v += a.bias[(size_t)hq * a.n_bias + min(pos - i, a.n_bias - 1)];
        s[4 * h + e] = in ? v : -INFINITY;
      }
    }
    float mx = s[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) mx = fmaxf(mx, s[i]);
    mx = fmaxf(mx, __shfl_xor(mx, 16, SSD_WAVE));
    mx = fmaxf(mx, __shfl_xor(mx, 32, SSD_WAVE));
    const float mn = fmaxf(m, mx), mu = mn == -INFINITY ? 0.f : mn;  // rows without a key yet: weights of zero
    const float al = __builtin_amdgcn_exp2f((m - mu) * LOG2E);
    m = mn;
    float w[8], sum = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      w[i] = __builtin_amdgcn_exp2f((s[i] - mu) * LOG2E);
      sum += w[i];
      w[i] = s[i] == -INFINITY ? 0.f : w[i] * vsc[i];
    }
    l = l * al + sum;
    bf16x8_t pf[NP];
    planes_of<NP>(w, pf);
#pragma unroll
    for (int d = 0; d < NB; ++d) {
      uint32_t f[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        f[i] = pack_bf16x2(code_f(vr[2 * i][d / 4], d % 4), code_f(vr[2 * i + 1][d / 4], d % 4));
      const bf16x8_t vf = as_frag(f);
      f32x4_t acc = {o[d][0] * al, o[d][1] * al, o[d][2] * al, o[d][3] * al};
#pragma unroll
      for (int p = 0; p < NP; ++p) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[NP - 1 - p], acc, 0, 0, 0);
      o[d] = acc;
    }
  }
  l += __shfl_xor(l, 16, SSD_WAVE);
  l += __shfl_xor(l, 32, SSD_WAVE);
  // O^T block d, row 4 g + e: dimension NB (4 g + e) + d, so a lane holds d_head / 4 consecutive ones
#pragma unroll
  for (int e = 0; e < 4; ++e)
#pragma unroll
    for (int d = 0; d < NB; ++d) xo[wave][n][NB * (4 * g + e) + d] = o[d][e];
  if (g == 0) { xm[wave][n] = m; xl[wave][n] = l; }
  __syncthreads();
  // thread (pair, part): the waves' results
  constexpr int PART = DH / 16;
  const int pn = tid >> 4, d0 = (tid & 15) * PART;
  const int pu = u0 + pn;
  if (pu >= nr * G) return;
  float M = xm[0][pn];
#pragma unroll
  for (int w = 1; w < AW; ++w) M = fmaxf(M, xm[w][pn]);
  const float Mu = M == -INFINITY ? 0.f : M;
  float L = 0.f, f[PART];
#pragma unroll
  for (int i = 0; i < PART; ++i) f[i] = 0.f;
#pragma unroll
  for (int w = 0; w < AW; ++w) {
    const float c = __builtin_amdgcn_exp2f((xm[w][pn] - Mu) * LOG2E);
    L += c * xl[w][pn];
#pragma unroll
    for (int i = 0; i < PART; ++i) f[i] += c * xo[w][pn][d0 + i];
  }
  const int pj = pu / G, ph = hk * G + (pu - pj * G);
  const size_t row = (size_t)(r0 + pj);
  if (splits > 1) {
    float* p = a.part + ((row * a.n_q_heads + ph) * splits + split) * (DH + 2);
#pragma unroll
    for (int i = 0; i < PART; ++i) p[d0 + i] = f[i];
    if (d0 == 0) { p[DH] = M; p[DH + 1] = L; }
    return;
  }
  const float inv = L == 0.f ? 0.f : 1.f / L;  // (NaN stays)
#pragma unroll
  for (int i = 0; i < PART; ++i) f[i] *= inv;
  store_out<T, PART>(reinterpret_cast<T*>(a.out) + row * a.ldo + (size_t)ph * DH + d0, f, a.out_vec);
}

// The splits' results of row blockIdx.y of sequence blockIdx.z and one head, in split order.
template <typename T, int DH>
__global__ __launch_bounds__(DH) void cache_attn_merge_kernel(const CacheAttnArgs a, const int splits) {
  const int h = blockIdx.x;
  int r0, nr;
  seq_rows(a, blockIdx.z, r0, nr);
  if ((int)blockIdx.y >= nr) return;
  const int r = r0 + blockIdx.y;
  const float* p = a.part + ((size_t)r * a.n_q_heads + h) * splits * (DH + 2);
  float M = -INFINITY;
  for (int s = 0; s < splits; ++s) M = fmaxf(M, p[(size_t)s * (DH + 2) + DH]);
  const float Mu = M == -INFINITY ? 0.f : M;
  float L = 0.f, f = 0.f;
  for (int s = 0; s < splits; ++s) {
    const float* ps = p + (size_t)s * (DH + 2);
    const float c = __builtin_amdgcn_exp2f((ps[DH] - Mu) * LOG2E);
    L += c * ps[DH + 1];
    f += c * ps[threadIdx.x];
  }
  const float inv = L == 0.f ? 0.f : 1.f / L;
  store_elem(reinterpret_cast<T*>(a.out) + (size_t)r * a.ldo + (size_t)h * DH + threadIdx.x, f * inv);
}

template <typename T, int DH>
hipError_t launch_t(const CacheAttnArgs& a, hipStream_t s) {
  const int G = a.n_q_heads / a.n_heads, tiles = (a.max_rows * G + 15) / 16;
  const int splits = cache_attn_splits(a);
  const dim3 grid((unsigned)((size_t)a.B * tiles * a.n_heads), splits);
  if (a.bias) hipLaunchKernelGGL((cache_attn_kernel<T, DH, true>), grid, dim3(64 * AW), 0, s, a, tiles, splits);
  else hipLaunchKernelGGL((cache_attn_kernel<T, DH, false>), grid, dim3(64 * AW), 0, s, a, tiles, splits);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || splits == 1) return e;
  hipLaunchKernelGGL((cache_attn_merge_kernel<T, DH>), dim3(a.n_q_heads, a.max_rows, a.B), dim3(DH), 0, s, a, splits);
  return hipGetLastError();
}

}  // namespace

// Key ranges a (row, head) pair's keys are split into: enough blocks to give each compute unit four,
// while a range keeps 128 keys (one unit a wave).
int cache_attn_splits(const CacheAttnArgs& a) {
  const int G = a.n_q_heads / a.n_heads;
  const long long blocks = (long long)a.B * ((a.max_rows * (long long)G + 15) / 16) * a.n_heads;
  long long want = (4LL * 256 + blocks - 1) / blocks;
  const long long most = (a.max_len + AW * UNIT - 1) / (AW * UNIT);
  if (want > most) want = most;
  if (want > CACHE_SPLITS_MAX) want = CACHE_SPLITS_MAX;
  return want < 1 ? 1 : (int)want;
}

size_t cache_attn_part_floats(const CacheAttnArgs& a) {
  const int splits = cache_attn_splits(a);
  return splits > 1 ? (size_t)a.rows * a.n_q_heads * splits * (a.d_head + 2) : 0;
}

hipError_t launch_cache_attention(const CacheAttnArgs& a, hipStream_t s) {
  if (a.rows < 1) return hipSuccess;
  if (a.dtype == 1) return a.d_head == 64 ? launch_t<bf16_t, 64>(a, s) : launch_t<bf16_t, 128>(a, s);
  return a.d_head == 64 ? launch_t<float, 64>(a, s) : launch_t<float, 128>(a, s);
}

}  // namespace ssd
