// Softmax attention over the 8-bit paged cache: many rows a sequence (prompts, long verify chunks).
// Formulas as in cache_attention.hip.
#include "cache_attention.h"

namespace ssd {

namespace {

constexpr int TKEYS = 64;  // keys a block takes at once

// The largest of either half over the wave's lanes.
typedef short s16x2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ s16x2_t wave_max2(s16x2_t v) {
#pragma unroll
  for (int i = 1; i < 64; i <<= 1)
    v = __builtin_elementwise_max(v, __builtin_bit_cast(s16x2_t, __shfl_xor(__builtin_bit_cast(int, v), i, SSD_WAVE)));
  return v;
}

// A value that is the same in every lane, known to be.
__device__ __forceinline__ uint64_t uniform(uint64_t v) {
  return (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32 |
         (uint32_t)__builtin_amdgcn_readfirstlane((int)v);
}
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// TW * NT * 16 (row, head) pairs of one sequence and cache head a block, NT tiles of 16 a wave.  The
// block turns 64 keys at a time into f16 operands in LDS, in the order in which the matrix
// instruction's lanes take them (each a contiguous kilobyte), so a code is converted once for all
// pairs; a wave's scores stay in its registers and are the operand of the second product, as in
// the kernel of few rows.  While a unit is worked on, the next one's codes are on their way to
// registers and the page entries of the one after it to LDS; two buffers, one barrier a unit.
// Scales enter the operands as their ratios to the largest of the unit, which then serves all its
// scores or weights.  That takes bits only where scales lie far apart: such a unit, rare in a
// sequence's own cache, is gone through once for each group of keys whose scales are near each
// other, the others masked (scales in registers beside the scores would spill).
// Bound: vector instructions of the softmax (about nine slots a score, four of them the
// exponential) beside the matrix instructions (two a 16 x 16 x 32 piece for bf16 rows, four for
// float32).  4096 bf16 rows of 32 heads of 128 behind 4096 positions: 412 GFLOP in 484 us, 0.85
// PFLOP/s, the vector instructions busy for half of the time and the matrix instructions for a
// third.  Few units a block are round trips: three times 608 float32 rows 39 us, ragged chunks of 17
// rows over up to 2777 positions 18 us.
template <typename T, int DH, bool BIAS, int NT, int TW>
__global__ __launch_bounds__(64 * TW, 2) void cache_attn_tile_kernel(const CacheAttnArgs a, const int tiles,
                                                                     const int splits, const uint32_t ps_inv) {
  constexpr int KS = DH / 32;   // steps of 32 over d_head
  constexpr int NB = DH / 16;   // output blocks of 16 dimensions
  constexpr int NP = Planes<T>::N;
  constexpr bool EXACT = BIAS || sizeof(T) == 4;  // weights from the scores' differences alone
  __shared__ uint4 kf[2][TKEYS / 16][KS][64], vf[2][TKEYS / 32][NB][64];
  // by unit modulo 3 (one in work, one to convert, one being written): scales over its largest
  __shared__ __attribute__((aligned(16))) float ksc[3][TKEYS], vsc[3][TKEYS];
  __shared__ __attribute__((aligned(16))) uint64_t rows[2][TKEYS];  // bytes from the pools' begin on, of the unit to load next
  struct Unit {
    uint64_t live;  // keys that have a row
    int top;        // exponents of the largest key and value scale
    int apart;      // whether there are several groups
  };
  __shared__ __attribute__((aligned(16))) Unit facts[3];
  __shared__ int group[3][TKEYS];  // exponents of each key's group
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, g = lane >> 4;
  const int hk = blockIdx.x % a.n_heads, bt = blockIdx.x / a.n_heads;
  const int b = bt / tiles, tile = tiles - 1 - (bt - b * tiles), split = blockIdx.y;  // the longest rows first
  const int G = a.n_q_heads / a.n_heads;
  int r0, nr;
  seq_rows(a, b, r0, nr);
  const int pairs = nr * G, u0 = tile * 16 * NT * TW;
  if (u0 >= pairs) return;  // whole blocks
  const int base = a.seq_len[b] + a.pos_off;
  const int cap = a.max_pages * a.page_size;
  const int last = base + min(u0 + 16 * NT * TW - 1, pairs - 1) / G;  // the block's last row
  if (last >= cap && tid == 0 && split == 0) atomicOr(a.status, SSD_DEV_CAPACITY);
  const int kend = min(last, cap - 1) + 1;
  const int units = kend > 0 ? (kend + TKEYS - 1) / TKEYS : 0;
  const int per = (units + splits - 1) / splits;
  const int x0 = split * per, x1 = min(x0 + per, units);
  const int32_t* table = a.page_table + (size_t)b * a.max_pages;
  bool bad_page = false;

  // this wave's pairs
  const int uw = u0 + 16 * NT * wave;
  const bool idle = uw >= pairs;
  const int first = base + min(uw, pairs - 1) / G, wlast = base + min(uw + 16 * NT - 1, pairs - 1) / G;
  const Factor factor(a.scale, BIAS ? 1.f : LOG2E);
  int pos[NT], hq[NT], qe[NT];
  f16x8_t q[NT][KS][NP];
  float l[NT];
  Reference<BIAS> ref[NT];
  f32x4_t o[NT][NB];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int u = min(uw + 16 * t + n, pairs - 1), j = u / G;
    hq[t] = hk * G + (u - j * G);
    pos[t] = base + j;
    const T* qp = reinterpret_cast<const T*>(a.q) + (size_t)(r0 + j) * a.ldq + (size_t)hq[t] * DH;
    qe[t] = load_query<T, DH>(qp, g, a.scale, q[t]);
    l[t] = 0.f;
#pragma unroll
    for (int d = 0; d < NB; ++d) o[t][d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }

  // wave 0, lane = key of a unit
  auto entry = [&](int x) -> int {
    const int key = x * TKEYS + lane;
    return x < x1 && key < kend ? table[page_of(key, a.page_size, ps_inv)] : -1;
  };
  auto row_of = [&](int x, int page) -> uint32_t {
    const int key = x * TKEYS + lane;
    if (x >= x1 || key >= kend) return NO_ROW;
    if (page < 0 || page >= a.n_pages) {
      bad_page = true;
      return NO_ROW;
    }
    return ((uint32_t)page * a.n_heads + hk) * a.page_size + (key - page_of(key, a.page_size, ps_inv) * a.page_size);
  };
  // Shares of a unit: four waves take a quarter of the keys' K codes each, four (the same where the
  // block has no more) a half of the keys and, for DH 128, of the dimensions of V; DH 64: two.
  constexpr int VFIRST = TW == 8 ? 4 : 0;
  const bool k_mine = wave < 4, v_mine = wave >= VFIRST && (DH == 128 || wave < VFIRST + 2);
  const int vhalf = wave & 1, vpart = wave >> 1 & (DH / 64 - 1);
  uint4 kc[DH / 64];
  uint32_t vc[8];
  auto request = [&](int buf) {
    if (k_mine) {
      const int8_t* kp = a.k_codes + rows[buf][16 * (wave & 3) + n] + 16 * g;
#pragma unroll
      for (int i = 0; i < DH / 64; ++i) kc[i] = *reinterpret_cast<const uint4*>(kp + 64 * i);
    }
    if (v_mine) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          vc[4 * h + e] = *reinterpret_cast<const uint32_t*>(a.v_codes + rows[buf][32 * vhalf + 16 * h + 4 * g + e] +
                                                             n * (DH / 16) + 4 * vpart);
    }
  };
  auto convert = [&](int buf, int sc) {
    if (k_mine) {
      const float k = ksc[sc][16 * (wave & 3) + n];
      const Ratio t = ratio_of(k, k);
      const uint32_t* kw = reinterpret_cast<const uint32_t*>(&kc[0]);
#pragma unroll
      for (int st = 0; st < KS; ++st)
        kf[buf][wave & 3][st][lane] = __builtin_bit_cast(uint4, codes8(kw[2 * st], kw[2 * st + 1], t));
    }
    if (v_mine) {
      Ratio t[4];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float4 c = *reinterpret_cast<const float4*>(&vsc[sc][32 * vhalf + 16 * h + 4 * g]);
        t[2 * h] = ratio_of(c.x, c.y);
        t[2 * h + 1] = ratio_of(c.z, c.w);
      }
      f16x8_t f[4];
      columns4(vc, f, t);
#pragma unroll
      for (int d = 0; d < 4; ++d) vf[buf][vhalf][4 * vpart + d][lane] = __builtin_bit_cast(uint4, f[d]);
    }
  };
  // Wave 0: scales, live keys and rows of the units to come.
  float ks1 = 0.f, vs1 = 0.f;
  auto request_scales = [&](uint32_t row, int page) {
    ks1 = vs1 = 0.f;
    if (row != NO_ROW) {
      const size_t sc = (size_t)page * a.n_heads + hk;
      ks1 = a.k_scale[sc];
      vs1 = a.v_scale[sc];
    }
  };
  auto store_scales = [&](int sc, uint32_t row) {
    // the largest exponents of the unit's keys, and the smallest ones' negatives
    const int ke = exp_of(ks1), ve = exp_of(vs1);
    const s16x2_t k = wave_max2(s16x2_t{(short)ke, (short)(row == NO_ROW ? NO_EXP : -ke)}),
                  v = wave_max2(s16x2_t{(short)ve, (short)(row == NO_ROW ? NO_EXP : -ve)});
    const bool far = k[0] + k[1] > K_NEAR || v[0] + v[1] > NEAR;
    const int kt = far ? (ke + K_NEAR - 1) & -K_NEAR : k[0], vt = far ? (ve + NEAR - 1) & -NEAR : v[0];
    ksc[sc][lane] = ldexpf(1.f, ke - kt);
    vsc[sc][lane] = ldexpf(1.f, ve - vt);
    group[sc][lane] = pair_of(kt, vt);
    const uint64_t in = __ballot(row != NO_ROW);
    if (lane == 0) facts[sc] = Unit{in, pair_of(kt, vt), far};
  };
  auto store_row = [&](int buf, uint32_t row) {  // keys without a row read the pools' first: they are masked
    rows[buf][lane] = row == NO_ROW ? 0 : (uint64_t)row * DH;
  };

  // Before unit x is worked on: its operands; scales and live keys of x and x + 1; the rows of x + 1;
  // in wave 0's registers, page and row of x + 2.  What an iteration writes nobody reads before its
  // barrier.
  int page2 = -1;
  uint32_t row2 = NO_ROW;
  if (x0 < x1) {
    if (wave == 0) {
      const int p0 = entry(x0), p1 = entry(x0 + 1);
      page2 = entry(x0 + 2);
      const uint32_t r0 = row_of(x0, p0), r1 = row_of(x0 + 1, p1);
      row2 = row_of(x0 + 2, page2);
      store_row(0, r0);
      store_row(1, r1);
      request_scales(r0, p0);
      store_scales(0, r0);
      request_scales(r1, p1);
      store_scales(1, r1);
    }
    __syncthreads();
    request(0);
    convert(0, 0);
    __syncthreads();
  }

  // (a unit's own is read before the barrier in front of it, and known to be the same in every lane)
  auto unit_at = [&](int sc) {
    const Unit u = facts[sc];
    return Unit{uniform(u.live), uniform(u.top), uniform(u.apart)};
  };
  Unit unit = {};
  if (x0 < x1) unit = unit_at(0);
  for (int x = x0, i0 = 0, i1 = 1, i2 = 2; x < x1; ++x) {
    const int buf = (x - x0) & 1;
    int page3 = -1;
    if (x + 1 < x1) {
      request(buf ^ 1);
      if (wave == 0) {
        request_scales(row2, page2);
        page3 = entry(x + 3);
      }
    }
    uint64_t rest = !idle && x * TKEYS <= wlast ? unit.live : 0;
    while (rest) {
      // (one turn, but for rare units: what each turn loads and computes stays in it)
      int key0 = x * TKEYS;
      asm volatile("" : "+s"(key0) : : "memory");
      uint64_t in = rest;  // the keys of this turn
      int top = unit.top;
      if (unit.apart) {
        const int own = group[i0][lane];
        top = __builtin_amdgcn_readlane(own, __builtin_ctzll(rest));
        in &= __ballot(own == top);
      }
      const int ktop = first_of(top), vtop = second_of(top);
      rest &= ~in;
      // (operands are read from LDS a group ahead of their products; the scheduler would read each
      // where it is used and wait)
      f32x4_t s[NT][TKEYS / 16];
      f16x8_t fr[2][4];
#pragma unroll
      for (int st = 0; st < KS; ++st) fr[0][st] = __builtin_bit_cast(f16x8_t, kf[buf][0][st][lane]);
#pragma unroll
      for (int k = 0; k < TKEYS / 16; ++k) {
        if (k + 1 < TKEYS / 16) {
#pragma unroll
          for (int st = 0; st < KS; ++st) fr[(k + 1) & 1][st] = __builtin_bit_cast(f16x8_t, kf[buf][k + 1][st][lane]);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int t = 0; t < NT; ++t) s[t][k] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int st = 0; st < KS; ++st)
#pragma unroll
          for (int p = NP - 1; p >= 0; --p)
#pragma unroll
            for (int t = 0; t < NT; ++t)
              s[t][k] = __builtin_amdgcn_mfma_f32_16x16x32_f16(fr[k & 1][st], q[t][st][p], s[t][k], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
      const bool full = in == ~0ull && key0 + TKEYS - 1 <= first;  // no key of the unit is masked
      f16x8_t pf[NT][TKEYS / 32][NP];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        float f = factor.of(qe[t], ktop);
        if constexpr (BIAS) {
          const float* bp = a.bias + (size_t)hq[t] * a.n_bias;
#pragma unroll
          for (int i = 0; i < TKEYS / 4; ++i)
            s[t][i / 4][i % 4] = fmaf(s[t][i / 4][i % 4], f,
                                      bp[max(0, min(pos[t] - (key0 + 16 * (i / 4) + 4 * g + i % 4), a.n_bias - 1))]);
        }
        if (!full) {  // (uniform)
          const int after = pos[t] - key0 - 4 * g;  // last of the lane's keys, counted from its first
#pragma unroll
          for (int i = 0; i < TKEYS / 4; ++i) {
            const int key = 16 * (i / 4) + i % 4;
            if (!(in >> (key + 4 * g) & 1) || key > after) s[t][i / 4][i % 4] = -INFINITY;
          }
        }
        float mx = s[t][0][0];
#pragma unroll
        for (int i = 1; i < TKEYS / 4; i += 2)  // (the last one twice)
          mx = max3(mx, s[t][i / 4][i % 4], s[t][(i + 1 < TKEYS / 4 ? i + 1 : i) / 4][(i + 1 < TKEYS / 4 ? i + 1 : i) % 4]);
        mx = BIAS ? col_max(mx) : rounded(col_max(mx), f);
        float drop, num_drop;
        if (ref[t].move(mx, (float)vtop, drop, num_drop)) {  // rare once a few units are seen
          l[t] *= drop;
#pragma unroll
          for (int d = 0; d < NB; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[t][d][e] *= num_drop;
        }
        if (t == NT - 1) {  // the second product's first operands
#pragma unroll
          for (int d = 0; d < 4; ++d) fr[0][d] = __builtin_bit_cast(f16x8_t, (&vf[buf][0][0][0])[d * 64 + lane]);
        }
        // (under 2^-60 the keys add nothing in f16; the bound keeps the sum's own scale finite)
        const float we = (float)(vtop + W_EXP) - ref[t].num, se = fmaxf(we, -60.f);
        float from = (EXACT ? 0.f : se) - ref[t].ref;
        // A fused product less the reference, which is a rounded one: large scores are rounded first (one
        // step of 2^16 is 2^-7).
        const bool large = !BIAS && fabsf(ref[t].ref) > 65536.f;
        if (__any(large)) {  // (such rows alone)
#pragma unroll
          for (int i = 0; i < TKEYS / 4; ++i) {
            const float v = s[t][i / 4][i % 4];
            s[t][i / 4][i % 4] = large ? rounded(v, f) - ref[t].ref : v;
          }
          f = large ? 1.f : f;
          from = large ? EXACT ? 0.f : se : from;
        }
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < TKEYS / 32; ++k) {
          float w[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float v = s[t][2 * k + i / 4][i % 4];
            if constexpr (BIAS) w[i] = __builtin_amdgcn_exp2f((v - ref[t].ref) * LOG2E);
            else w[i] = __builtin_amdgcn_exp2f(fmaf(v, f, from));
            sum += w[i];
            if constexpr (EXACT) w[i] = ldexpf(w[i], (int)we);
          }
          f16_planes<NP>(w, pf[t][k]);
        }
        l[t] += EXACT ? sum : ldexpf(sum, -(int)se);
      }
      constexpr int GROUPS = TKEYS / 32 * NB / 4;  // of four operands
#pragma unroll
      for (int i = 0; i < GROUPS; ++i) {
        if (i + 1 < GROUPS) {
#pragma unroll
          for (int d = 0; d < 4; ++d)
            fr[(i + 1) & 1][d] = __builtin_bit_cast(f16x8_t, (&vf[buf][0][0][0])[(4 * (i + 1) + d) * 64 + lane]);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int p = NP - 1; p >= 0; --p)
#pragma unroll
          for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int t = 0; t < NT; ++t) {
              const int k = 4 * i / NB, od = 4 * i % NB + d;
              o[t][od] = __builtin_amdgcn_mfma_f32_16x16x32_f16(fr[i & 1][d], pf[t][k][p], o[t][od], 0, 0, 0);
            }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    if (x + 1 < x1) {
      unit = unit_at(i1);
      convert(buf ^ 1, i1);
      if (wave == 0) {
        store_scales(i2, row2);
        store_row(buf, row2);
        page2 = page3;
        row2 = row_of(x + 3, page2);
      }
    }
    __syncthreads();
    const int i = i0;
    i0 = i1;
    i1 = i2;
    i2 = i;
  }
  if (bad_page) atomicOr(a.status, SSD_DEV_BAD_PAGE);
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int u = uw + 16 * t + n;
    const float L = col_sum(l[t]), back = ldexpf(1.f, (int)ref[t].num - W_EXP);
    if (u >= pairs) continue;
    // O^T block d, row 4 g + e: dimension NB (4 g + e) + d, so a lane holds DH / 4 consecutive ones
    const int j = u / G;
    const size_t row = (size_t)(r0 + j), head = (size_t)(hk * G + (u - j * G));
    const float inv = L == 0.f ? 0.f : 1.f / L;  // (NaN stays; before `back`: the mean may be a number where the sum is none)
    float f[DH / 4];
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int d = 0; d < NB; ++d) f[NB * e + d] = o[t][d][e] * inv * back;
    if (splits > 1) {
      float* p = a.part + (row * a.n_q_heads + head) * splits * (DH + 2);
      store_out<float, DH / 4>(p + (size_t)split * DH + g * (DH / 4), f, false);
      if (g == 0) {
        p[(size_t)splits * DH + 2 * split] = ref[t].ref;
        p[(size_t)splits * DH + 2 * split + 1] = L;
      }
    } else {
      store_result<T, DH, DH / 4>(a, row, head, g * (DH / 4), f);
    }
  }
}

template <typename T, int DH, int NT, int TW>
void launch_tw(const CacheAttnArgs& a, int splits, hipStream_t s) {
  const int pairs = a.max_rows * (a.n_q_heads / a.n_heads), tiles = (pairs + 16 * NT * TW - 1) / (16 * NT * TW);
  const dim3 grid((unsigned)((size_t)a.B * tiles * a.n_heads), splits), block(64 * TW);
  const uint32_t inv = page_inv(a.page_size);
  if (a.bias) hipLaunchKernelGGL((cache_attn_tile_kernel<T, DH, true, NT, TW>), grid, block, 0, s, a, tiles, splits, inv);
  else hipLaunchKernelGGL((cache_attn_tile_kernel<T, DH, false, NT, TW>), grid, block, 0, s, a, tiles, splits, inv);
}

template <typename T, int DH>
void launch_t(const CacheAttnArgs& a, int n, int splits, hipStream_t s) {
  if (n == 64) launch_tw<T, DH, 1, 4>(a, splits, s);
  else if (n == 128) launch_tw<T, DH, 1, 8>(a, splits, s);
  else if constexpr (!(DH == 128 && sizeof(T) == 4)) launch_tw<T, DH, 2, 8>(a, splits, s);
}

}  // namespace

hipError_t launch_cache_attn_tile(const CacheAttnArgs& a, int n, int splits, hipStream_t s) {
  if (a.dtype == 1) a.d_head == 64 ? launch_t<bf16_t, 64>(a, n, splits, s) : launch_t<bf16_t, 128>(a, n, splits, s);
  else a.d_head == 64 ? launch_t<float, 64>(a, n, splits, s) : launch_t<float, 128>(a, n, splits, s);
  return hipGetLastError();
}

}  // namespace ssd
