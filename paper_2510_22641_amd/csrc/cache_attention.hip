// Softmax attention over the 8-bit paged cache: few rows a sequence (decode steps, verify chunks).
//
// Query row j of sequence b sits at position p = seq_len[b] + pos_off + j and attends positions
// 0 .. p of its pages; the scores are q . c s_k scale + bias[h][p - i] with c the key's codes and s_k
// its block's scale, the output sum_i w_i s_v c_i over the softmax weights w.
#include "cache_attention.h"

namespace ssd {

namespace {

constexpr int UNIT = 32;  // keys a wave takes at once

// Where a unit's keys are, and their scales.  EVEN: of its two halves, the same in every lane; else
// [0] of key lane % 32.
template <bool EVEN>
struct Keys {
  float ks[EVEN ? 2 : 1], vs[EVEN ? 2 : 1];
  uint32_t row[EVEN ? 2 : 1];
};

// Reads through the scalar unit, for addresses that are the same in every lane.
template <typename V>
__device__ __forceinline__ V scalar_load(const V* p) {
  return *(const __attribute__((address_space(4))) V*)(uintptr_t)p;
}

// 16 (row, head) pairs of one sequence and cache head a block, one of `splits` ranges of their keys.
// Pair u of the sequence is row u / G, head hk G + u % G.  A wave takes units of 32 keys straight from
// memory to matrix operands: lane (r = l % 16, g = l / 16) loads 16 codes of each 64 of keys r and
// 16 + r, which are its rows of S^T = K Q^T (key order and the order of d are free as long as both
// operands agree); the scores land with lane (pair l % 16, keys 4 g + e of either half), which is
// again the operand layout of the weights in O^T = V^T P^T when its K index 8 g + i names key
// 4 g + i % 4 of half i / 4, so neither scores nor weights cross lanes but for the maximum.  V is
// read row by row, DH / 16 codes a lane, and its bytes turned to columns in registers.  The next
// unit's codes are requested into the registers that this one's have just left, a whole unit before
// their use; its scales one unit ahead and its page-table entries two (codes of a second or third
// unit on their way in registers of their own measured 2 and 3% slower).  EVEN:
// pages hold a multiple of 16 positions, so a half lies in one page and its entry and scales are
// scalars; else every key has its own, which cross lanes.  The codes are operands as they are; their
// scales multiply the scores and the weights.  Each wave keeps its own references and sums; they
// meet in LDS once.
// Bound: for long contexts the bytes of the codes, which lie scattered in pieces of a page and head
// (one token, 32 heads of 128 over 32768 positions: 269 MB in 50 us and 5 for the merge; 32 tokens of
// 2048 positions, 8 cache heads: 134 MB in 31 us; of 1 to 4096: 130 MB in 41); for short ones the
// chain lengths -> table -> codes (70 positions: 5.5 us, of which an empty kernel takes 3.9).
template <typename T, int DH, bool BIAS, bool EVEN, int AW>
__global__ __launch_bounds__(64 * AW, DH == 64 && AW == 4 ? 3 : 2) void cache_attn_kernel(const CacheAttnArgs a, const int tiles,
                                                                               const int splits, const uint32_t ps_inv) {
  constexpr int KS = DH / 32;  // steps of 32 over d_head
  constexpr int NB = DH / 16;  // output blocks of 16 dimensions
  constexpr int VW = DH / 64;  // dwords of V a lane and key
  constexpr int NP = Planes<T>::N;
  __shared__ float xo[AW][16][DH + 4];
  __shared__ float xm[AW][16], xl[AW][16];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, g = lane >> 4;
  const int hk = blockIdx.x % a.n_heads, bt = blockIdx.x / a.n_heads;
  const int b = bt / tiles, tile = bt - b * tiles, split = blockIdx.y;
  const int G = a.n_q_heads / a.n_heads;
  int r0, nr;
  seq_rows(a, b, r0, nr);
  const int pairs = nr * G, u0 = tile * 16;
  if (u0 >= pairs) return;  // whole blocks
  const int base = a.seq_len[b] + a.pos_off;
  const int cap = a.max_pages * a.page_size;
  const int first = base + u0 / G, last = base + min(u0 + 15, pairs - 1) / G;  // rows of the block
  if (last >= cap && tid == 0 && split == 0) atomicOr(a.status, SSD_DEV_CAPACITY);
  const int kend = min(last, cap - 1) + 1;
  const int units = kend > 0 ? (kend + UNIT - 1) / UNIT : 0;
  // ranges of one length for all sequences, so that no block has more to do than another
  int most = 0;
  if (splits > 1) {
    for (int i = lane; i < a.B; i += 64) most = max(most, a.seq_len[i]);
#pragma unroll
    for (int i = 1; i < 64; i <<= 1) most = max(most, __shfl_xor(most, i, SSD_WAVE));
    // (one value in all lanes; known to be, so that what follows from it stays scalar)
    most = __builtin_amdgcn_readfirstlane(min(max(most + a.pos_off + a.max_rows, kend), cap));
  }
  const int per = splits > 1 ? ((most + UNIT - 1) / UNIT + splits - 1) / splits : units;
  const int x0 = split * per, x1 = min(x0 + per, units);
  const int32_t* table = a.page_table + (size_t)b * a.max_pages;
  bool bad_page = false;

  const uint32_t k_off = n * DH + 16 * g, v_off = 4 * g * DH + n * (DH / 16);  // in a half of one page
  constexpr int NE = EVEN ? 2 : 1;  // entries of a unit a lane holds
  struct Entries { int page[NE]; };
  // (pages of one position are never EVEN)
  auto page_index = [&](int key) { return EVEN ? (int)__umulhi((uint32_t)key, ps_inv) : page_of(key, a.page_size, ps_inv); };
  // (No load depends on a branch, here and in `request`: the counts by which a wave waits for its
  // loads stay known, and it waits for no later one.)
  auto entries = [&](int x) {
    Entries t;
#pragma unroll
    for (int h = 0; h < NE; ++h) {
      const int key = min(x * UNIT + (EVEN ? 16 * h : lane & 31), kend - 1);
      const int32_t* p = table + page_index(key);
      t.page[h] = EVEN ? scalar_load(p) : *p;
    }
    return t;
  };
  auto locate = [&](Keys<EVEN>& u, int x, const Entries& t) {
#pragma unroll
    for (int h = 0; h < NE; ++h) {
      const int key = x * UNIT + (EVEN ? 16 * h : lane & 31), page = t.page[h];
      const bool in = x < x1 && key < kend, ok = in && page >= 0 && page < a.n_pages;
      bad_page |= in && !ok;
      const uint32_t sc = (uint32_t)(ok ? page : 0) * a.n_heads + hk;  // (below 2^32, as the rows)
      u.ks[h] = EVEN ? scalar_load(a.k_scale + sc) : a.k_scale[sc];
      u.vs[h] = EVEN ? scalar_load(a.v_scale + sc) : a.v_scale[sc];
      u.row[h] = ok ? sc * a.page_size + (key - page_index(key) * a.page_size) : NO_ROW;
    }
  };
  // Codes as loaded: of keys 16 h + lane % 16, 16 from 64 i + 16 g on; and of keys 16 h + 4 g + e
  // (8 = 4 h + e), DH / 16 from lane % 16 on.  Keys without a row read the pools' first rows: their
  // scores are masked.
  uint4 kc[2][DH / 64];
  uint32_t vc[VW][8];
  auto first_byte = [&](const Keys<EVEN>& u, int h, int key) -> size_t {  // of a key of half h
    const uint32_t r = EVEN ? u.row[h % NE] : (uint32_t)__shfl(u.row[0], 16 * h + key, SSD_WAVE);
    return (size_t)(r == NO_ROW ? 0 : r) * DH;
  };
  auto request_k = [&](const Keys<EVEN>& u) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int8_t* p = a.k_codes + first_byte(u, h, n) + (EVEN ? k_off : 16 * g);
#pragma unroll
      for (int i = 0; i < DH / 64; ++i) kc[h][i] = *reinterpret_cast<const uint4*>(p + 64 * i);
    }
  };
  auto request_v = [&](const Keys<EVEN>& u) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int8_t* p = a.v_codes + first_byte(u, h, 4 * g + e) + (EVEN ? v_off + e * DH : n * (DH / 16));
#pragma unroll
        for (int i = 0; i < VW; ++i) vc[i][4 * h + e] = *reinterpret_cast<const uint32_t*>(p + 4 * i);
      }
  };

  // (the first unit's entries before the queries: neither waits for the other)
  Entries ahead = {};
  if (x0 + wave < x1) ahead = entries(x0 + wave);
  const int ul = min(u0 + n, pairs - 1), jl = ul / G, hq = hk * G + (ul - jl * G), pos = base + jl;  // this lane's pair
  f16x8_t q[KS][NP];
  const Factor factor(a.scale, BIAS ? 1.f : LOG2E);
  const int qe = load_query<T, DH>(reinterpret_cast<const T*>(a.q) + (size_t)(r0 + jl) * a.ldq + (size_t)hq * DH, g,
                                   a.scale, q);
  const float* bias_row = BIAS ? a.bias + (size_t)hq * a.n_bias : nullptr;
  Reference<BIAS> ref;
  float l = 0.f;  // sum of the weights
  f32x4_t o[NB];
#pragma unroll
  for (int d = 0; d < NB; ++d) o[d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  Keys<EVEN> cur = {}, next;
  float bias[8];
  auto request_bias = [&](int x) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      bias[i] = bias_row[max(0, min(pos - (x * UNIT + 16 * (i / 4) + 4 * g + i % 4), a.n_bias - 1))];
  };

  if (x0 + wave < x1) {
    const Entries then = entries(x0 + wave + AW);
    locate(cur, x0 + wave, ahead);
    if constexpr (BIAS) request_bias(x0 + wave);
    request_k(cur);
    request_v(cur);
    ahead = then;
  }
  // The next unit's codes are requested as soon as this one's have left their registers.
  for (int x = x0 + wave; x < x1; x += AW, cur = next) {
    const Entries then = entries(x + 2 * AW);  // before the codes, for which it must not wait
    locate(next, x + AW, ahead);
    ahead = then;
    const bool rows = EVEN ? cur.row[0] != NO_ROW && cur.row[NE - 1] != NO_ROW : __all(cur.row[0] != NO_ROW);
    const bool full = rows && x * UNIT + UNIT - 1 <= first;  // no key of it is masked
    // exponents of the scales: of the halves, or the lane's keys
    int ke[EVEN ? 2 : 8], ve[EVEN ? 2 : 8];
#pragma unroll
    for (int h = 0; h < NE; ++h) {
      ke[h] = cur.row[h] != NO_ROW ? exp_of(cur.ks[h]) : NO_EXP;
      ve[h] = cur.row[h] != NO_ROW ? exp_of(cur.vs[h]) : NO_EXP;
    }
    if constexpr (!EVEN) {
      const int own = pair_of(ke[0], ve[0]);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int p = __shfl(own, 16 * (i / 4) + 4 * g + i % 4, SSD_WAVE);
        ke[i] = first_of(p);
        ve[i] = second_of(p);
      }
    }
    f32x4_t s[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      s[h] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      const uint32_t* kw = reinterpret_cast<const uint32_t*>(&kc[h][0]);
#pragma unroll
      for (int st = 0; st < KS; ++st) {
        const f16x8_t kf = codes8(kw[2 * st], kw[2 * st + 1]);
#pragma unroll
        for (int p = NP - 1; p >= 0; --p) s[h] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf, q[st][p], s[h], 0, 0, 0);
      }
    }
    // (scores are rounded before anything is subtracted: a product and its reference that went through
    // other roundings would differ by far more than REF_STEP where scores are large)
    float f[EVEN ? 2 : 8];
#pragma unroll
    for (int i = 0; i < (EVEN ? 2 : 8); ++i) f[i] = factor.of(qe, ke[i]);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float v = s[i / 4][i % 4], c = f[EVEN ? i / 4 : i];
      s[i / 4][i % 4] = BIAS ? fmaf(v, c, bias[i]) : rounded(v, c);
    }
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (BIAS) request_bias(x + AW);
    request_k(next);
    __builtin_amdgcn_sched_barrier(0);
    if (!full) {  // (uniform)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int src = 16 * (i / 4) + 4 * g + i % 4;
        const uint32_t row = EVEN ? cur.row[i / 4 % NE] : (uint32_t)__shfl(cur.row[0], src, SSD_WAVE);
        if (row == NO_ROW || x * UNIT + src > pos) s[i / 4][i % 4] = -INFINITY;
      }
    }
    auto half_max = [&](int h) { return max3(max3(s[h][0], s[h][1], s[h][2]), s[h][3], s[h][3]); };
    const float mx = col_max(max3(half_max(0), half_max(1), half_max(1)));
    float ex;
    if constexpr (EVEN) {
      ex = (float)max(ve[0], ve[1]);
      if (abs(ve[0] - ve[1]) > NEAR)  // (uniform)
        ex = fmaxf(fmaf(col_max(half_max(0)) - mx, ref.UNIT, (float)ve[0]),
                   fmaf(col_max(half_max(1)) - mx, ref.UNIT, (float)ve[1]));
    } else {
      ex = -INFINITY;
#pragma unroll
      for (int i = 0; i < 8; ++i) ex = fmaxf(ex, fmaf(s[i / 4][i % 4] - mx, ref.UNIT, (float)ve[i]));
      ex = col_max(ex);
    }
    float drop, num_drop;
    if (ref.move(mx, ex, drop, num_drop)) {  // rare once a few units are seen
      l *= drop;
#pragma unroll
      for (int d = 0; d < NB; ++d)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[d][e] *= num_drop;
    }
    const int to = W_EXP - (int)ref.num;
    float w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      w[i] = __builtin_amdgcn_exp2f((s[i / 4][i % 4] - ref.ref) * ref.UNIT);
      l += w[i];
      w[i] = ldexpf(w[i], ve[EVEN ? i / 4 : i] + to);
    }
    f16x8_t pf[NP];
    f16_planes<NP>(w, pf);
#pragma unroll
    for (int i = 0; i < VW; ++i) {
      f16x8_t vf[4];
      columns4(vc[i], vf);
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int p = NP - 1; p >= 0; --p)
          o[4 * i + d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf[d], pf[p], o[4 * i + d], 0, 0, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
    request_v(next);
    __builtin_amdgcn_sched_barrier(0);
  }
  if (bad_page) atomicOr(a.status, SSD_DEV_BAD_PAGE);
  // (divided first: a sum of values may be past the largest number where their mean is not)
  l = col_sum(l);
  const float inv_l = l == 0.f ? 0.f : 1.f / l, back = ldexpf(1.f, (int)ref.num - W_EXP);  // (NaN stays)
  // O^T block d, row 4 g + e: dimension NB (4 g + e) + d, so a lane holds DH / 4 consecutive ones
#pragma unroll
  for (int e = 0; e < 4; ++e)
#pragma unroll
    for (int d = 0; d < NB; d += 4)
      *reinterpret_cast<float4*>(&xo[wave][n][NB * (4 * g + e) + d]) =
          make_float4(o[d][e] * inv_l * back, o[d + 1][e] * inv_l * back, o[d + 2][e] * inv_l * back,
                      o[d + 3][e] * inv_l * back);
  if (g == 0) { xm[wave][n] = ref.ref; xl[wave][n] = l; }
  __syncthreads();
  // thread (pair, part): the waves' results
  constexpr int PART = DH / 16;
  const int pn = tid >> 4, d0 = (tid & 15) * PART;
  const int pu = u0 + pn;
  if (pn >= 16 || pu >= pairs) return;
  float M = xm[0][pn];
#pragma unroll
  for (int w = 1; w < AW; ++w) M = fmaxf(M, xm[w][pn]);
  float L = 0.f, c[AW], f[PART];
#pragma unroll
  for (int w = 0; w < AW; ++w) {
    c[w] = __builtin_amdgcn_exp2f((xm[w][pn] - M) * (BIAS ? LOG2E : 1.f)) * xl[w][pn];
    L += c[w];
  }
  const float inv = L == 0.f ? 0.f : 1.f / L;
#pragma unroll
  for (int i = 0; i < PART; ++i) f[i] = 0.f;
#pragma unroll
  for (int w = 0; w < AW; ++w) {
#pragma unroll
    for (int i = 0; i < PART; ++i) f[i] += c[w] * inv * xo[w][pn][d0 + i];
  }
  const int pj = pu / G, ph = hk * G + (pu - pj * G);
  const size_t row = (size_t)(r0 + pj);
  if (splits > 1) {
    float* p = a.part + (row * a.n_q_heads + ph) * splits * (DH + 2);
    store_out<float, PART>(p + (size_t)split * DH + d0, f, false);
    if (d0 == 0) {
      p[(size_t)splits * DH + 2 * split] = M;
      p[(size_t)splits * DH + 2 * split + 1] = L;
    }
    return;
  }
  store_result<T, DH, PART>(a, row, ph, d0, f);
}

// The splits' results of row blockIdx.y of sequence blockIdx.z and one head: per pair `splits` rows
// of DH means, then their (reference, sum of weights) pairs.  Thread groups of DH / 4 lanes take every eighth (or
// sixteenth) split, four dimensions a lane, and meet in LDS: the order of the sums is fixed.
constexpr int MERGE = 256;
template <typename T, int DH>
__global__ __launch_bounds__(MERGE) void cache_attn_merge_kernel(const CacheAttnArgs a, const int splits) {
  constexpr int LANES = DH / 4, GROUPS = MERGE / LANES;
  __shared__ float xo[GROUPS][DH];
  __shared__ float c[CACHE_SPLITS_MAX];  // shares of the splits
  const int h = blockIdx.x, tid = threadIdx.x;
  int r0, nr;
  seq_rows(a, blockIdx.z, r0, nr);
  if ((int)blockIdx.y >= nr) return;
  const int r = r0 + blockIdx.y;
  const float* p = a.part + ((size_t)r * a.n_q_heads + h) * splits * (DH + 2);
  if (tid < 64) {  // CACHE_SPLITS_MAX is a wave's lanes
    const float* ml = p + (size_t)splits * DH + 2 * tid;
    const float mv = tid < splits ? ml[0] : -FLT_MAX, lv = tid < splits ? ml[1] : 0.f;
    const float M = wave_max(mv);
    const float w = __builtin_amdgcn_exp2f((mv - M) * (a.bias ? LOG2E : 1.f)) * lv, L = wave_sum(w);
    c[tid] = L == 0.f ? 0.f : w / L;
  }
  __syncthreads();
  const int grp = tid / LANES, d = (tid % LANES) * 4;
  float4 f = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int s = grp; s < splits; s += GROUPS) {
    const float* v = p + (size_t)s * DH + d;
    const float w = c[s];
    f.x += w * v[0]; f.y += w * v[1]; f.z += w * v[2]; f.w += w * v[3];
  }
  *reinterpret_cast<float4*>(&xo[grp][d]) = f;
  __syncthreads();
  if (tid < DH) {
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < GROUPS; ++k) v += xo[k][tid];
    if (sizeof(T) == 4 && a.out_planes)
      store_planes1(a.out_planes + plane_at(r, h * DH + tid, (a.rows + 15) >> 4), v);
    else
      store_elem(reinterpret_cast<T*>(a.out) + (size_t)r * a.ldo + (size_t)h * DH + tid, v);
  }
}

// (row, head) pairs of the longest sequence and cache head.
long long pairs_of(const CacheAttnArgs& a) { return a.max_rows * (long long)(a.n_q_heads / a.n_heads); }

// Pairs a block takes.  16 in the kernel above.  Beyond, the kernel for many rows:
// * 64 in four waves of one tile each.  (Tiles of 16 of the kernel above measured between half and 1.1
//   of its time.  Eight requests over 1000 positions, 17 to 64 float32 rows of 64 elements and a bias:
//   17 to 22 us against 34 to 42; chunks of 6 to 21 bf16 rows of three heads over pages of seven: 17 to
//   26 against 20 to 24.)
// * 128 in eight waves of one tile (80 and 128 of the former rows: 56 and 59 us, in blocks of 64 49 and 51).
// * 256 in eight waves of two tiles, which share what is read from LDS, where that leaves a block for every
//   compute unit (4096 bf16 rows of 32 heads of 128 over 8192 positions: 484 us against 721 in blocks of
//   128; 1000 of 64 over 3000: 97 either way; 300 float32 rows of 64 with a bias: 98 against 69); not
//   for float32 rows of 128, whose two tiles' operands do not fit the registers.
int block_pairs(const CacheAttnArgs& a) {
  const long long p = pairs_of(a);
  if (p <= 64) return p <= 16 ? 16 : 64;
  const bool two = !(a.dtype == SSD_F32 && a.d_head == 128) && a.B * ((p + 255) / 256) * a.n_heads >= 256;
  return two ? 256 : 128;
}

long long blocks_of(const CacheAttnArgs& a) {
  const int n = block_pairs(a);
  return a.B * ((pairs_of(a) + n - 1) / n) * a.n_heads;
}

template <typename T, int DH>
hipError_t launch_t(const CacheAttnArgs& a, hipStream_t s) {
  const int splits = cache_attn_splits(a), n = block_pairs(a);
  hipError_t e;
  if (n >= 64) {
    e = launch_cache_attn_tile(a, n, splits, s);
  } else {
    const dim3 grid((unsigned)blocks_of(a), splits);
    const int tiles = (int)((pairs_of(a) + 15) / 16);
    const uint32_t inv = page_inv(a.page_size);
    // eight waves where that leaves each two units of the longest range (eight requests of up to 1000
    // positions and nine rows each: 12.7 us against 15.3), four for shorter ones (70 positions: 5.5
    // against 5.6; eight requests of 300, one row each: 7.6 against 7.0)
    const int waves = a.max_len / splits >= 16 * UNIT ? 8 : 4;
    const dim3 block(64 * waves);
#define LAUNCH(BIAS, EVEN)                                                                                          \
  do {                                                                                                              \
    if (waves == 8) hipLaunchKernelGGL((cache_attn_kernel<T, DH, BIAS, EVEN, 8>), grid, block, 0, s, a, tiles, splits, inv); \
    else hipLaunchKernelGGL((cache_attn_kernel<T, DH, BIAS, EVEN, 4>), grid, block, 0, s, a, tiles, splits, inv);            \
  } while (0)
    const bool even = a.page_size % 16 == 0;
    if (a.bias) { if (even) LAUNCH(true, true); else LAUNCH(true, false); }
    else { if (even) LAUNCH(false, true); else LAUNCH(false, false); }
#undef LAUNCH
    e = hipGetLastError();
  }
  if (e != hipSuccess || splits == 1) return e;
  hipLaunchKernelGGL((cache_attn_merge_kernel<T, DH>), dim3(a.n_q_heads, a.max_rows, a.B), dim3(MERGE), 0, s, a, splits);
  return hipGetLastError();
}

}  // namespace

// Key ranges a (row, head) pair's keys are split into: a block for each of the 256 compute units (two
// of the 64-pair kernel's four waves), while a range keeps 128 keys.  More of them measured no
// faster (one token of 32 heads over 32768 positions: 58 us with 256 blocks of eight waves, 61 with
// 512; 32 tokens of 8 cache heads: 40 against 45).  The few-row kernel keeps short ranges whole, where
// the merge would cost more than the waves save (one token of 32 heads of 128: 300 positions 8.0 us
// whole, 9.3 in three ranges; 600: 8.7 and 9.2 in five; 1000: 11.3 and 9.1 in eight; two tokens, 1000:
// 12.7 and 11.9 in four; four, 1000 and 1900: 13.3 and 18.3, 15.0 and 19.3 in two).  The rule counts
// blocks alone: where there are enough of them, one long sequence among short ones is not split (one of
// 32768 positions 58 us, seven of 100 beside it 212).
int cache_attn_splits(const CacheAttnArgs& a) {
  const long long blocks = blocks_of(a);
  long long want = (256LL * (block_pairs(a) == 64 ? 2 : 1) + blocks - 1) / blocks;
  const long long most = (a.max_len + 127) / 128;
  if (want > most) want = most;
  if (want > CACHE_SPLITS_MAX) want = CACHE_SPLITS_MAX;
  if (block_pairs(a) == 16 && (a.max_len <= 512 || (want < 4 && a.max_len < 2048))) want = 1;
  // Blocks of n pairs hold rows * n_q_heads <= blocks n pairs, and a split call has blocks * splits <
  // 256 + blocks <= 512 of them (n <= 128), or with n = 64 < 512 + blocks <= 1024: CACHE_PARTS_MAX
  // splits of a pair, but for rows that belong to no sequence.
  const long long room = CACHE_PARTS_MAX / ((long long)a.rows * a.n_q_heads);
  if (want > room) want = room;
  return want < 1 ? 1 : (int)want;
}

bool cache_attn_fits(const CacheAttnArgs& a) {  // (blocks of up to eight waves)
  return (uint64_t)blocks_of(a) * 512 <= MAX_GRID_THREADS;
}

size_t cache_attn_part_floats(size_t rows, int n_q_heads, int d_head, int max_len) {
  size_t splits = ((size_t)max_len + 127) / 128;
  if (splits > CACHE_SPLITS_MAX) splits = CACHE_SPLITS_MAX;
  if (splits < 2) return 0;
  const size_t n = rows * n_q_heads * splits;
  return (n < CACHE_PARTS_MAX ? n : CACHE_PARTS_MAX) * (d_head + 2);
}

hipError_t launch_cache_attention(const CacheAttnArgs& a, hipStream_t s) {
  if (a.rows < 1) return hipSuccess;
  if (a.dtype == 1) return a.d_head == 64 ? launch_t<bf16_t, 64>(a, s) : launch_t<bf16_t, 128>(a, s);
  return a.d_head == 64 ? launch_t<float, 64>(a, s) : launch_t<float, 128>(a, s);
}

}  // namespace ssd
