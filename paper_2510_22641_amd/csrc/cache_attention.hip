// Softmax attention over the 8-bit paged cache: few rows a sequence (decode steps, verify chunks).
//
// Query row j of sequence b sits at position p = seq_len[b] + pos_off + j and attends positions
// 0 .. p of its pages; the scores are q . c s_k scale + bias[h][p - i] with c the key's codes and s_k
// its block's scale, the output sum_i w_i s_v c_i over the softmax weights w.
#include "cache_attention.h"

namespace ssd {

namespace {

constexpr int AW = 4;     // waves a block
constexpr int UNIT = 32;  // keys a wave takes at once

// What a wave needs of a unit before its products: codes as loaded, and scales.
template <int DH>
struct Unit {
  uint4 k[2][DH / 64];        // keys 16 h + lane % 16: DH / 4 codes from g DH / 4 on
  uint32_t v[DH / 64][8];     // keys 16 h + 4 g + e (8 = 4 h + e): DH / 16 codes from lane % 16 on
  float ks, vs;               // of key lane % 32
  uint32_t row;               // of key lane % 32
};

// NT times 16 (row, head) pairs of one sequence and cache head a block, one of `splits` ranges of
// their keys.  Pair u of the sequence is row u / G, head hk G + u % G.  A wave takes units of 32 keys
// straight from memory to matrix operands: lane (r = l % 16, g = l / 16) loads DH / 4 codes of keys
// r and 16 + r, which are its rows of S^T = K Q^T (key order and the order of d are free as long as
// both operands agree); the scores land with lane (pair l % 16, keys 4 g + e of either half), which
// is again the operand layout of the weights in O^T = V^T P^T when its K index 8 g + i names key
// 4 g + i % 4 of half i / 4, so neither scores nor weights cross lanes but for the maximum.  V is
// read row by row, DH / 16 codes a lane, and its bytes turned to columns in registers.  A unit's
// codes and scales are requested one unit ahead of their use and its page-table entries two.  Each
// wave keeps its own maximum, sum and reference scale; they meet in LDS once.
// With a bias the scores stay in natural units, where the type's lowest value is a finite one (times
// log2 e it would not be); without one they carry the log2 e of exp2.
// Bound: bytes of codes for long contexts, the chain lengths -> table -> codes for short ones.
template <typename T, int DH, bool BIAS, int NT>
__global__ __launch_bounds__(64 * AW, NT == 1 ? 3 : 2) void cache_attn_kernel(const CacheAttnArgs a, const int tiles,
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
  const int pairs = nr * G, u0 = tile * 16 * NT;
  if (u0 >= pairs) return;  // whole blocks
  const int base = a.seq_len[b] + a.pos_off;
  const int cap = a.max_pages * a.page_size;
  const int first = base + u0 / G, last = base + min(u0 + 16 * NT - 1, pairs - 1) / G;  // rows of the block
  if (last >= cap && tid == 0 && split == 0) atomicOr(a.status, SSD_DEV_CAPACITY);
  const int kend = min(last, cap - 1) + 1;
  const int units = kend > 0 ? (kend + UNIT - 1) / UNIT : 0;
  const int per = (units + splits - 1) / splits;
  const int x0 = split * per, x1 = min(x0 + per, units);
  const int32_t* table = a.page_table + (size_t)b * a.max_pages;
  bool bad_page = false;

  // row of codes of key x 32 + lane % 32
  auto entry = [&](int x) -> int {
    const int key = x * UNIT + (lane & 31);
    return x < x1 && key < kend ? table[page_of(key, a.page_size, ps_inv)] : -1;
  };
  auto row_of = [&](int x, int page) -> uint32_t {
    const int key = x * UNIT + (lane & 31);
    if (x >= x1 || key >= kend) return NO_ROW;
    if (page < 0 || page >= a.n_pages) {
      bad_page = true;
      return NO_ROW;
    }
    return ((uint32_t)page * a.n_heads + hk) * a.page_size + (key - page_of(key, a.page_size, ps_inv) * a.page_size);
  };
  auto request = [&](Unit<DH>& u, uint32_t row, int page) {
    u.row = row;
    u.ks = u.vs = 0.f;
    if (row != NO_ROW) {
      const size_t sc = (size_t)page * a.n_heads + hk;
      u.ks = a.k_scale[sc];
      u.vs = a.v_scale[sc];
    }
    // keys without a row read the pools' first bytes: their scores are masked
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t kr = __shfl(row, 16 * h + n, SSD_WAVE);
      const uint4* p = reinterpret_cast<const uint4*>(a.k_codes + (size_t)(kr == NO_ROW ? 0 : kr) * DH + g * (DH / 4));
#pragma unroll
      for (int i = 0; i < DH / 64; ++i) u.k[h][i] = p[i];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t vr = __shfl(row, 16 * h + 4 * g + e, SSD_WAVE);
        const uint32_t* pv = reinterpret_cast<const uint32_t*>(a.v_codes + (size_t)(vr == NO_ROW ? 0 : vr) * DH + n * (DH / 16));
#pragma unroll
        for (int i = 0; i < VW; ++i) u.v[i][4 * h + e] = pv[i];
      }
    }
  };

  int pos[NT], hq[NT];
  f16x8_t q[NT][KS][NP];
  float qf[NT];
  f32x4_t o[NT][NB];
  float m[NT], l[NT];
  // (the first unit's entries before the queries: neither waits for the other)
  int page1 = entry(x0 + wave);
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int u = min(u0 + 16 * t + n, pairs - 1), j = u / G;
    hq[t] = hk * G + (u - j * G);
    pos[t] = base + j;
    const T* qp = reinterpret_cast<const T*>(a.q) + (size_t)(r0 + j) * a.ldq + (size_t)hq[t] * DH;
    qf[t] = load_query<T, DH>(qp, g, q[t]) * a.scale * (BIAS ? 1.f : LOG2E);
    m[t] = -INFINITY;
    l[t] = 0.f;
#pragma unroll
    for (int d = 0; d < NB; ++d) o[t][d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  float vref = 0.f;  // weights are held over the largest value scale so far
  Unit<DH> next;
  request(next, row_of(x0 + wave, page1), page1);
  page1 = entry(x0 + wave + AW);

  for (int x = x0 + wave; x < x1; x += AW) {
    const Unit<DH> cur = next;
    if (x + AW < x1) {
      request(next, row_of(x + AW, page1), page1);
      page1 = entry(x + 2 * AW);
    }
    float bias[NT][8];
    if (BIAS) {
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const float* bp = a.bias + (size_t)hq[t] * a.n_bias;
#pragma unroll
        for (int i = 0; i < 8; ++i)
          bias[t][i] = bp[max(0, min(pos[t] - (x * UNIT + 16 * (i / 4) + 4 * g + i % 4), a.n_bias - 1))];
      }
    }
    // weights are multiplied by vs W_TOP / vref
    float vm = cur.vs;
#pragma unroll
    for (int s = 1; s < 32; s <<= 1) vm = fmaxf(vm, __shfl_xor(vm, s, SSD_WAVE));
    const float vnew = fmaxf(vref, vm), vdrop = vnew > 0.f ? vref / vnew : 1.f;
    const float vmul = vnew > 0.f ? cur.vs * (W_TOP / vnew) : cur.vs;
    vref = vnew;
    float ks[8], vs[8];
    bool in[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int src = 16 * (i / 4) + 4 * g + i % 4;
      ks[i] = __shfl(cur.ks, src, SSD_WAVE);
      vs[i] = __shfl(vmul, src, SSD_WAVE);
      in[i] = __shfl(cur.row, src, SSD_WAVE) != NO_ROW;
    }
    const bool all = __all(cur.row != NO_ROW) && x * UNIT + UNIT - 1 <= first;  // nothing to mask
    f32x4_t s[NT][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int t = 0; t < NT; ++t) s[t][h] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      const uint32_t* kw = reinterpret_cast<const uint32_t*>(&cur.k[h][0]);
#pragma unroll
      for (int st = 0; st < KS; ++st) {
        const f16x8_t kf = codes8(kw[2 * st], kw[2 * st + 1]);
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int p = NP - 1; p >= 0; --p) s[t][h] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf, q[t][st][p], s[t][h], 0, 0, 0);
      }
    }
    f16x8_t pf[NT][NP];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      float w[8], mx = -INFINITY, sum = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        w[i] = s[t][i / 4][i % 4] * (ks[i] * qf[t]);
        if (BIAS) w[i] += bias[t][i];
        if (!all) w[i] = in[i] && x * UNIT + 16 * (i / 4) + 4 * g + i % 4 <= pos[t] ? w[i] : -INFINITY;
        mx = fmaxf(mx, w[i]);
      }
      mx = fmaxf(m[t], col_max(mx));
      const float mu = mx == -INFINITY ? 0.f : mx;  // rows without a key yet: weights of zero
      const float al = __builtin_amdgcn_exp2f((m[t] - mu) * (BIAS ? LOG2E : 1.f));
      m[t] = mx;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const bool none = w[i] == -INFINITY;
        w[i] = __builtin_amdgcn_exp2f((w[i] - mu) * (BIAS ? LOG2E : 1.f));
        sum += w[i];
        w[i] *= vs[i];
        if ((BIAS || !all) && none) w[i] = 0.f;
      }
      l[t] = l[t] * al + sum;
      f16_planes<NP>(w, pf[t]);
      const float drop = al * vdrop;
      if (__any(drop != 1.f)) {
#pragma unroll
        for (int d = 0; d < NB; ++d)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[t][d][e] *= drop;
      }
    }
#pragma unroll
    for (int i = 0; i < VW; ++i) {
      f16x8_t vf[4];
      columns4(cur.v[i], vf);
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int p = NP - 1; p >= 0; --p)
            o[t][4 * i + d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf[d], pf[t][p], o[t][4 * i + d], 0, 0, 0);
    }
  }
  if (bad_page) atomicOr(a.status, SSD_DEV_BAD_PAGE);
  const float back = vref * (1.f / W_TOP);
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    if (u0 + 16 * t >= pairs) break;  // whole blocks
    if (t) __syncthreads();  // the previous tile's results are out
    const float lt = col_sum(l[t]);
    // O^T block d, row 4 g + e: dimension NB (4 g + e) + d, so a lane holds DH / 4 consecutive ones
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int d = 0; d < NB; d += 4)
        *reinterpret_cast<float4*>(&xo[wave][n][NB * (4 * g + e) + d]) =
            make_float4(o[t][d][e] * back, o[t][d + 1][e] * back, o[t][d + 2][e] * back, o[t][d + 3][e] * back);
    if (g == 0) { xm[wave][n] = m[t]; xl[wave][n] = lt; }
    __syncthreads();
    // thread (pair, part): the waves' results
    constexpr int PART = DH / 16;
    const int pn = tid >> 4, d0 = (tid & 15) * PART;
    const int pu = u0 + 16 * t + pn;
    if (pu < pairs) {
      float M = xm[0][pn];
#pragma unroll
      for (int w = 1; w < AW; ++w) M = fmaxf(M, xm[w][pn]);
      const float Mu = M == -INFINITY ? 0.f : M;
      float L = 0.f, f[PART];
#pragma unroll
      for (int i = 0; i < PART; ++i) f[i] = 0.f;
#pragma unroll
      for (int w = 0; w < AW; ++w) {
        const float c = __builtin_amdgcn_exp2f((xm[w][pn] - Mu) * (BIAS ? LOG2E : 1.f));
        L += c * xl[w][pn];
#pragma unroll
        for (int i = 0; i < PART; ++i) f[i] += c * xo[w][pn][d0 + i];
      }
      const int pj = pu / G, ph = hk * G + (pu - pj * G);
      const size_t row = (size_t)(r0 + pj);
      if (splits > 1) {
        float* p = a.part + (row * a.n_q_heads + ph) * splits * (DH + 2) + (size_t)split * DH + d0;
        store_out<float, PART>(p, f, false);
        float* ml = a.part + (row * a.n_q_heads + ph) * splits * (DH + 2) + (size_t)splits * DH + 2 * split;
        if (d0 == 0) { ml[0] = M; ml[1] = L; }
      } else {
        const float inv = L == 0.f ? 0.f : 1.f / L;  // (NaN stays)
#pragma unroll
        for (int i = 0; i < PART; ++i) f[i] *= inv;
        store_out<T, PART>(reinterpret_cast<T*>(a.out) + row * a.ldo + (size_t)ph * DH + d0, f, a.out_vec);
      }
    }
  }
}

// The splits' results of row blockIdx.y of sequence blockIdx.z and one head: per pair `splits` rows
// of DH sums, then their (maximum, sum) pairs.  Thread groups of DH / 4 lanes take every eighth (or
// sixteenth) split, four dimensions a lane, and meet in LDS: the order of the sums is fixed.
constexpr int MERGE = 256;
template <typename T, int DH>
__global__ __launch_bounds__(MERGE) void cache_attn_merge_kernel(const CacheAttnArgs a, const int splits) {
  constexpr int LANES = DH / 4, GROUPS = MERGE / LANES;
  __shared__ float xo[GROUPS][DH];
  __shared__ float c[CACHE_SPLITS_MAX], xl[CACHE_SPLITS_MAX];
  const int h = blockIdx.x, tid = threadIdx.x;
  int r0, nr;
  seq_rows(a, blockIdx.z, r0, nr);
  if ((int)blockIdx.y >= nr) return;
  const int r = r0 + blockIdx.y;
  const float* p = a.part + ((size_t)r * a.n_q_heads + h) * splits * (DH + 2);
  if (tid < 64) {  // CACHE_SPLITS_MAX is a wave's lanes
    const float* ml = p + (size_t)splits * DH + 2 * tid;
    const float mv = tid < splits ? ml[0] : -INFINITY, lv = tid < splits ? ml[1] : 0.f;
    const float M = wave_max(mv);
    const float w = __builtin_amdgcn_exp2f((mv - (M == -INFINITY ? 0.f : M)) * (a.bias ? LOG2E : 1.f));
    c[tid] = w;
    xl[tid] = w * lv;
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
    float L = 0.f, v = 0.f;
    for (int s = 0; s < splits; ++s) L += xl[s];
#pragma unroll
    for (int k = 0; k < GROUPS; ++k) v += xo[k][tid];
    const float inv = L == 0.f ? 0.f : 1.f / L;
    store_elem(reinterpret_cast<T*>(a.out) + (size_t)r * a.ldo + (size_t)h * DH + tid, v * inv);
  }
}

// Tiles of 16 (row, head) pairs a block takes: two where a sequence has more than one, which halves
// the reads and conversions of its keys.
int tiles_of(const CacheAttnArgs& a) { return a.max_rows * (a.n_q_heads / a.n_heads) > 16 ? 2 : 1; }

long long blocks_of(const CacheAttnArgs& a, int nt) {
  const long long pairs = a.max_rows * (long long)(a.n_q_heads / a.n_heads);
  return a.B * ((pairs + 16 * nt - 1) / (16 * nt)) * a.n_heads;
}

template <typename T, int DH, int NT>
void launch_nt(const CacheAttnArgs& a, int splits, hipStream_t s) {
  const int pairs = a.max_rows * (a.n_q_heads / a.n_heads), tiles = (pairs + 16 * NT - 1) / (16 * NT);
  const dim3 grid((unsigned)blocks_of(a, NT), splits), block(64 * AW);
  const uint32_t inv = (uint32_t)(((1ull << 32) + a.page_size - 1) / a.page_size);
  if (a.bias) hipLaunchKernelGGL((cache_attn_kernel<T, DH, true, NT>), grid, block, 0, s, a, tiles, splits, inv);
  else hipLaunchKernelGGL((cache_attn_kernel<T, DH, false, NT>), grid, block, 0, s, a, tiles, splits, inv);
}

template <typename T, int DH>
hipError_t launch_t(const CacheAttnArgs& a, hipStream_t s) {
  const int splits = cache_attn_splits(a);
  if (tiles_of(a) == 2) launch_nt<T, DH, 2>(a, splits, s);
  else launch_nt<T, DH, 1>(a, splits, s);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || splits == 1) return e;
  hipLaunchKernelGGL((cache_attn_merge_kernel<T, DH>), dim3(a.n_q_heads, a.max_rows, a.B), dim3(MERGE), 0, s, a, splits);
  return hipGetLastError();
}

}  // namespace

// Key ranges a (row, head) pair's keys are split into: enough blocks to give each compute unit
// three, while a range keeps 128 keys (one unit a wave).
int cache_attn_splits(const CacheAttnArgs& a) {
  const long long blocks = blocks_of(a, tiles_of(a));
  long long want = (3LL * 256 + blocks - 1) / blocks;
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
