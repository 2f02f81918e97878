// The 8-bit paged cache: slot maps from request lengths, storing rows as codes, reading them back.
//
// A block is one page of one head: page_size rows of d_head int8 codes c with one scale s, a power
// of two; the row's values are c s.  With the largest magnitude a of the block's rows, s is the
// smallest 2^e (e >= -100) with a <= 127 2^e: dividing by it is exact, so a store rounds a value once, by
// at most half a code, s / 2 <= a / 127.  A later store on its block that raises the scale rounds it
// again, by half a code of the new scale: over all of them less than one code of the largest scale
// that the block has had since the row came, rows given up again among its causes.  A scale that
// falls rounds nothing, and brings nothing back.
#include "device.h"
#include "kernels.h"

#include <cfloat>

namespace ssd {

namespace {

constexpr int MAP_THREADS = 256;

// Exclusive prefix sums over the block's threads of one value each; *total receives the sum.
__device__ __forceinline__ long long block_scan(long long v, long long* waves, long long* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  long long x = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const long long y = __shfl_up(x, o, SSD_WAVE);
    if (lane >= o) x += y;
  }
  __syncthreads();  // the previous use of waves[]
  if (lane == 63) waves[wave] = x;
  __syncthreads();
  long long before = 0, sum = 0;
#pragma unroll
  for (int w = 0; w < MAP_THREADS / 64; ++w) {
    if (w < wave) before += waves[w];
    sum += waves[w];
  }
  *total = sum;
  return before + x - v;
}

// Largest b in [0, B) with start[b] <= r (start[0] = 0, non-decreasing).
__device__ __forceinline__ int find_seq(const int* start, int B, int r) {
  int lo = 0, hi = B;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (start[mid] <= r) lo = mid; else hi = mid;
  }
  return lo;
}

// Slot map and page table of B <= PAGE_MAP_MAX_BATCH sequences.  Every block repeats the two prefix
// sums over the sequences (a few loads a thread), so that one launch does it all: no block waits for
// another, and a new page's id comes from the free list by its rank instead of from the table that
// other blocks are writing.  Then a block writes its share of the new table entries and the slots
// of its 256 rows, each finding its sequence by bisection in LDS.  Bound: launch latency and
// one dependent chain (lengths, sums, table entry), not bytes (8 sequences 3.6 us, an empty kernel's;
// 1024 with 83 thousand rows 8.2).
__global__ __launch_bounds__(MAP_THREADS) void page_map_kernel(const PageMapArgs a, const uint32_t ps_inv) {
  extern __shared__ int map_lds[];
  int* row0 = map_lds;               // [B + 1] first row of each sequence
  int* page0 = map_lds + a.B + 1;    // [B + 1] rank in the free list of its first new page
  int* len0 = page0 + a.B + 1;       // [B] positions it holds
  __shared__ long long waves[MAP_THREADS / 64];
  const int tid = threadIdx.x;
  const int cap = a.cap;
  int fault = 0;
  auto pages_of = [&](int positions) { return page_of(positions + a.page_size - 1, a.page_size, ps_inv); };  // <= cap
  // pages of a sequence with `len` positions held and n new rows: the first and how many
  auto need = [&](int len, int n, int& first) {
    first = 0;
    if (!a.free_pages || len < 0 || len > cap || n <= 0) return 0;
    first = pages_of(len);
    return pages_of(n < cap - len ? len + n : cap) - first;
  };
  // counts and lengths first, where the sums will be
  for (int b = tid; b < a.B; b += MAP_THREADS) {
    const int len = a.seq_len[b] + a.pos_off, n = a.new_rows ? a.new_rows[b] : a.new_const;
    if (n < 0 || (n > 0 && (len < 0 || (long long)len + n > cap))) fault = 1;
    row0[b] = max(n, 0);
    len0[b] = len;
  }
  __syncthreads();
  // a thread takes `per` sequences one after the other
  const int per = (a.B + MAP_THREADS - 1) / MAP_THREADS, b0 = min(tid * per, a.B), b1 = min(b0 + per, a.B);
  long long rows, pages, sum = 0;
  for (int b = b0; b < b1; ++b) sum += row0[b];
  long long r = block_scan(sum, waves, &rows);
  sum = 0;
  for (int b = b0; b < b1; ++b) {
    // rows past max_rows are cut: they get no slot and no page
    const int lo = (int)(r < a.max_rows ? r : a.max_rows);
    r += row0[b];
    int first;
    sum += need(len0[b], (int)(r < a.max_rows ? r : a.max_rows) - lo, first);
    row0[b] = lo;
  }
  if (tid == 0) row0[a.B] = (int)(rows < a.max_rows ? rows : a.max_rows);
  long long p = block_scan(sum, waves, &pages);  // (and its barriers: every row0 is in place)
  for (int b = b0; b < b1; ++b) {
    int first;
    const int n = need(len0[b], row0[b + 1] - row0[b], first);
    page0[b] = (int)(p < a.n_free ? p : a.n_free);
    p += n;
  }
  if (rows > a.max_rows || pages > a.n_free) fault = 1;
  const int n_rows = (int)(rows < a.max_rows ? rows : a.max_rows);
  const int n_pages = (int)(pages < a.n_free ? pages : a.n_free);
  if (tid == 0) page0[a.B] = n_pages;
  __syncthreads();
  if (blockIdx.x == 0) {
    if (fault) atomicOr(a.status, SSD_DEV_CAPACITY);  // (each thread knows of its own)
    if (a.row_start)
      for (int b = tid; b <= a.B; b += MAP_THREADS) a.row_start[b] = row0[b];
    if (tid == 0 && a.taken) *a.taken = n_pages;
  }
  // new table entries: rank t of the free list belongs to the sequence with page0[b] <= t
  for (int t = blockIdx.x * MAP_THREADS + tid; t < n_pages; t += gridDim.x * MAP_THREADS) {
    const int b = find_seq(page0, a.B, t);
    int first;
    need(len0[b], row0[b + 1] - row0[b], first);
    a.page_table[(size_t)b * a.max_pages + first + t - page0[b]] = a.free_pages[t];
  }
  // entries that the free list could not fill: the last sequences' (none unless `fault`)
  if (a.free_pages && pages > a.n_free && blockIdx.x == 0) {
    for (int b = tid; b < a.B; b += MAP_THREADS) {
      int first;
      const int n = need(len0[b], row0[b + 1] - row0[b], first);
      for (int i = page0[b + 1] - page0[b]; i < n; ++i) a.page_table[(size_t)b * a.max_pages + first + i] = -1;
    }
  }
  if (!a.slot) return;
  {
    const int r = blockIdx.x * MAP_THREADS + tid;
    if (r >= a.max_rows) return;
    int64_t s = -1;
    if (r < n_rows) {
      const int b = find_seq(row0, a.B, r);
      const int len = len0[b];
      const long long p = (long long)len + r - row0[b];
      if (len >= 0 && p < cap) {
        const int i = page_of((int)p, a.page_size, ps_inv);
        int first;
        const int n = need(len, row0[b + 1] - row0[b], first);
        const bool is_new = a.free_pages && i >= first && n > 0;
        const int t = page0[b] + i - first;
        if (!is_new || t < page0[b + 1]) {  // else the free list has ended
          const int page = is_new ? a.free_pages[t] : a.page_table[(size_t)b * a.max_pages + i];
          if (page < 0 || page >= a.n_pages) atomicOr(a.status, SSD_DEV_BAD_PAGE);
          else s = (int64_t)page * a.page_size + ((int)p - i * a.page_size);
        }
      }
    }
    a.slot[r] = s;
  }
}

// Four consecutive elements of a row as they are stored; VEC: the row is aligned for one load.
template <typename T> struct Raw4;
template <> struct Raw4<float> {
  float4 v;
  __device__ __forceinline__ float4 values() const { return v; }
};
template <> struct Raw4<bf16_t> {
  uint2 v;
  __device__ __forceinline__ float4 values() const {
    return make_float4(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u),
                       __uint_as_float(v.y << 16), __uint_as_float(v.y & 0xffff0000u));
  }
};
template <typename T, bool VEC>
__device__ __forceinline__ Raw4<T> load4(const T* p) {
  Raw4<T> r;
  if constexpr (VEC) r.v = *reinterpret_cast<const decltype(r.v)*>(p);
  else if constexpr (sizeof(T) == 4) r.v = make_float4(p[0], p[1], p[2], p[3]);
  else r.v = make_uint2(p[0] | (uint32_t)p[1] << 16, p[2] | (uint32_t)p[3] << 16);
  return r;
}

// Exponent e >= -100 of the smallest scale 2^e with top <= 127 2^e (top >= 0, finite).
__device__ __forceinline__ int scale_exp(float top) {
  const uint32_t u = __float_as_uint(top);
  const int e = (int)(u >> 23) - 133 + ((u & 0x7fffffu) > 0x7e0000u ? 1 : 0);  // 127 = 1.984375 2^6
  return e < -100 ? -100 : e;
}

// Codes of v / s, with inv = 1 / s: nearest (even).  For finite v, whose quotients are at most 127, the
// sum with 1.5 2^23 rounds to a whole number and has it in its low bits.  ANY: an infinity gets the
// largest code, a NaN zero.
template <bool ANY>
__device__ __forceinline__ uint32_t codes_of(const float4& v, float inv) {
  auto code = [&](float x) -> uint32_t {
    if (ANY) {
      const float r = fminf(fmaxf(rintf(x * inv), -127.f), 127.f);
      return (uint32_t)(int)(x == x ? r : 0.f);
    }
    return __float_as_uint(fmaf(x, inv, 12582912.f));
  };
  const uint32_t lo = __builtin_amdgcn_perm(code(v.y), code(v.x), 0x0c0c0400),
                 hi = __builtin_amdgcn_perm(code(v.w), code(v.z), 0x04000c0c);
  return lo | hi;
}

__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }
__device__ __forceinline__ uint32_t abs_bits(const float4& v, uint32_t top) {
  return max(max(max(top, abs_bits(v.x)), max(abs_bits(v.y), abs_bits(v.z))), abs_bits(v.w));
}
__device__ __forceinline__ float finite_abs(const float4& v, float top) {
  const float f[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (fabsf(f[i]) <= FLT_MAX) top = fmaxf(top, fabsf(f[i]));
  return top;
}

__device__ __forceinline__ float code_at(uint32_t w, int i) { return (float)(int8_t)(w >> (8 * i)); }

// slot / page_size for slots below 2^40, ps_inv = 1 / page_size: the rounded product is within one
// of the quotient.
__device__ __forceinline__ int slot_page(int64_t s, int ps, double ps_inv) {
  int q = (int)((double)s * ps_inv);
  const int64_t r = s - (int64_t)q * ps;
  q -= r < 0;
  return q + (r >= ps);
}

constexpr int STORE_WAVES = 4;
constexpr int STORE_HELD = 8;  // passes of rows kept in registers between the maximum and the codes

// Rows into their blocks.  A run is the rows on consecutive slots of one page; a wave owns, for one
// head of K or V, the stretches of rows on one page (rows without a slot do not interrupt them) that
// begin in `window` consecutive rows, and stores a stretch's runs one after the other.  For a run it
// takes the largest magnitude over the run and over the rows the block already holds in front of it
// (their codes times the old scale), rescales those where the block's scale changes, and writes the
// run's codes; 32 (or 16) lanes take four elements each of a row.  Every block belongs to one wave,
// so nothing is atomic.  Bound: bytes for long prompts (8192 bf16 rows of 32 heads of 128, K and V:
// 201 MB in 50 us, 4.1 TB/s, where a large copy reaches 4.9; float32: 336 MB in 78, 4.3); the chain slot -> rows, codes and
// scale -> reduction -> store for single tokens (29 float32 rows of 32 heads of 64: 5.0 us).
template <typename T, int DH, bool VEC>
__global__ __launch_bounds__(64 * STORE_WAVES) void cache_store_kernel(const CacheRowsArgs a, const int window,
                                                                       const int groups, const double ps_inv) {
  constexpr int LPR = DH / 4, RPP = 64 / LPR;  // lanes a row, rows a pass
  const int lane = threadIdx.x & 63;
  // (neighbouring blocks on neighbouring heads: together they read whole rows)
  const int w = blockIdx.x / groups;
  const int task = __builtin_amdgcn_readfirstlane((blockIdx.x - w * groups) * STORE_WAVES + (threadIdx.x >> 6));
  if (task >= 2 * a.n_heads) return;  // whole waves
  const bool is_v = task >= a.n_heads;
  const int h = is_v ? task - a.n_heads : task;
  const int ps = a.page_size;
  const int64_t n_slots = (int64_t)a.n_pages * ps;
  const T* src = reinterpret_cast<const T*>(is_v ? a.v : a.k) + (size_t)h * DH + (lane % LPR) * 4;
  int8_t* codes = is_v ? a.v_codes : a.k_codes;
  float* scales = is_v ? a.v_scale : a.k_scale;
  const int lr = lane / LPR, lc = (lane % LPR) * 4;
  // the stretches that begin in this window
  const int w0 = w * window, w1 = min(w0 + window, a.rows);
  auto fits = [&](int64_t v) { return v >= 0 && v < n_slots; };
  const int64_t mine = w0 + lane < a.rows ? a.slot[w0 + lane] : -1;
  const int64_t before = w0 > 0 ? a.slot[w0 - 1] : -1;
  bool first = false, back = false;
  {
    const int r = w0 + lane;
    int64_t prev = __shfl_up(mine, 1, SSD_WAVE);
    if (lane == 0) prev = before;
    if (r < w1) {
      if (fits(mine)) {
        first = r == 0 || (fits(prev) && slot_page(prev, ps, ps_inv) != slot_page(mine, ps, ps_inv));
        back = r > 0 && !fits(prev);
      } else if (mine != -1 && task == 0) {
        atomicOr(a.status, SSD_DEV_BAD_PAGE);
      }
    }
  }
  uint64_t starts = __ballot(first), backs = __ballot(back);
  while (backs) {  // behind a row without a slot: the nearest row that has one decides
    const int at = __builtin_ctzll(backs);
    backs &= backs - 1;
    const int page = slot_page(__shfl(mine, at, SSD_WAVE), ps, ps_inv);
    bool own = true;
    for (int e = w0 + at - 2; e >= 0; e -= 64) {
      const int64_t v = e - lane >= 0 ? a.slot[e - lane] : -1;
      const uint64_t m = __ballot(fits(v));
      if (m) {
        own = slot_page(__shfl(v, __builtin_ctzll(m), SSD_WAVE), ps, ps_inv) != page;
        break;
      }
    }
    if (own) starts |= 1ull << at;
  }
  bool bad = false;
  int r0 = -1, page = -1;  // the next run, of the current stretch where r0 >= 0
  int64_t s0 = 0;
  while (r0 >= 0 || starts) {
    if (r0 < 0) {
      const int at = __builtin_ctzll(starts);
      starts &= starts - 1;
      r0 = w0 + at;
      s0 = __shfl(mine, at, SSD_WAVE);
      page = slot_page(s0, ps, ps_inv);
    }
    const int off = (int)(s0 - (int64_t)page * ps), run = r0;
    // rows of the run, up to the page's end, and the row with a slot that follows it
    int n = 0;
    int64_t next = -1;
    r0 = -1;
    for (int e = run; e < a.rows; e += 64) {
      int64_t v = mine;  // (the window's first run is looked at already)
      if (e != w0) v = e + lane < a.rows ? a.slot[e + lane] : -1;
      const int i = e + lane - run;
      const uint64_t in = __ballot(i == n + lane && off + i < ps && v == s0 + i);
      const int k = ~in ? __builtin_ctzll(~in) : 64;
      n += k;
      const uint64_t more = __ballot(lane >= k && fits(v));
      if (more) {
        const int at = __builtin_ctzll(more);
        next = __shfl(v, at, SSD_WAVE);
        if (slot_page(next, ps, ps_inv) == page) r0 = e + at;
        break;
      }
    }
    int8_t* block = codes + ((size_t)page * a.n_heads + h) * ps * DH;
    float* sp = scales + (size_t)page * a.n_heads + h;
    const float s_old = off ? *sp : 0.f;
    // elements of the run's rows, counted from its first (VEC: ld < 2^20, so a byte count fits 32 bits)
    const T* rows = src + (size_t)run * a.ld;
    auto at = [&](int r) -> Raw4<T> {
      if constexpr (VEC) return load4<T, VEC>(rows + (uint32_t)r * (uint32_t)a.ld);
      else return load4<T, VEC>(rows + (size_t)r * a.ld);
    };
    Raw4<T> kept[STORE_HELD];
#pragma unroll
    for (int p = 0; p < STORE_HELD; ++p) {
      if (p * RPP < n) {  // uniform; a row past the run repeats its last: no other maximum
        const int r = p * RPP + lr;
        kept[p] = at(min(r, n - 1));
      }
    }
    float held = 0.f;
    for (int r = lr; r < off; r += RPP) {
      const uint32_t w = *reinterpret_cast<const uint32_t*>(block + (size_t)r * DH + lc);
#pragma unroll
      for (int i = 0; i < 4; ++i) held = fmaxf(held, fabsf(code_at(w, i)));
    }
    held *= s_old;
    // codes over 63 of scale 2^122 are past the largest number (a stored scale that is none counts as zero)
    if (!(held <= FLT_MAX)) held = s_old <= FLT_MAX ? FLT_MAX : 0.f;
    // largest magnitude as bits, which order as the numbers do
    uint32_t top = __float_as_uint(held);
#pragma unroll
    for (int p = 0; p < STORE_HELD; ++p)
      if (p * RPP < n) top = abs_bits(kept[p].values(), top);
    for (int r = STORE_HELD * RPP + lr; r < n; r += RPP) top = abs_bits(at(r).values(), top);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o, SSD_WAVE));
    const bool any = top >= 0x7f800000u;  // uniform: something is not finite, and the finite ones count
    if (any) {
      bad = true;
      float f = held;
      for (int r = lr; r < n; r += RPP) f = finite_abs(at(r).values(), f);
      top = __float_as_uint(wave_max(f));
    }
    const int e = scale_exp(__uint_as_float(top));
    const float s_new = __uint_as_float((uint32_t)(e + 127) << 23);
    const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
    if (off && s_new != s_old) {
      for (int r = lr; r < off; r += RPP) {
        uint32_t* p = reinterpret_cast<uint32_t*>(block + (size_t)r * DH + lc);
        const uint32_t w = *p;
        *p = codes_of<true>(make_float4(code_at(w, 0) * s_old, code_at(w, 1) * s_old, code_at(w, 2) * s_old,
                                        code_at(w, 3) * s_old), inv);
      }
    }
    uint32_t* dst = reinterpret_cast<uint32_t*>(block + (size_t)off * DH + lc);
    if (any) {
      for (int r = lr; r < n; r += RPP)
        dst[r * LPR] = codes_of<true>(at(r).values(), inv);
    } else {
#pragma unroll
      for (int p = 0; p < STORE_HELD; ++p) {
        const int r = p * RPP + lr;
        if (r < n) dst[r * LPR] = codes_of<false>(kept[p].values(), inv);
      }
      for (int r = STORE_HELD * RPP + lr; r < n; r += RPP)
        dst[r * LPR] = codes_of<false>(at(r).values(), inv);
    }
    if (lane == 0) *sp = s_new;
    if (r0 >= 0) {  // another run on this page, which reads what was just written
      s0 = next;
      __threadfence_block();
    }
  }
  if (__any(bad) && lane == 0) atomicOr(a.status, SSD_DEV_NOT_FINITE);
}

// Rows back from their blocks: eight codes a lane, consecutive lanes on consecutive elements of a
// row, K (blockIdx.y 0) or V.  Bound: bytes (the same rows: 201 MB in 44 us, 4.5 TB/s; 336 in 69, 4.9).
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void cache_load_kernel(const CacheRowsArgs a) {
  const int per = a.n_heads * a.d_head / 8;  // lanes a row
  const size_t t = (size_t)blockIdx.x * 256 + threadIdx.x;
  const size_t r = t / per;
  if (r >= (size_t)a.rows) return;
  const int c = (int)(t - r * per) * 8, h = c / a.d_head;
  const bool is_v = blockIdx.y;
  const int64_t s = a.slot[r];
  if (s < 0 || s >= (int64_t)a.n_pages * a.page_size) {
    if (s != -1) atomicOr(a.status, SSD_DEV_BAD_PAGE);
    return;
  }
  const int64_t page = s / a.page_size, off = s - page * a.page_size;
  const size_t block = (size_t)page * a.n_heads + h;
  const int8_t* p = (is_v ? a.v_codes : a.k_codes) + (block * a.page_size + off) * a.d_head + (c - h * a.d_head);
  const uint2 w = *reinterpret_cast<const uint2*>(p);
  const float sc = (is_v ? a.v_scale : a.k_scale)[block];
  float f[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[i] = code_at(w.x, i) * sc;
    f[4 + i] = code_at(w.y, i) * sc;
  }
  if (sc >= 0x1p122f) {  // code 64 stands for the largest numbers, which rounded up to it
    const float most = sizeof(T) == 4 ? FLT_MAX : 0x1.fep127f;
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = fminf(fmaxf(f[i], -most), most);
  }
  T* o = reinterpret_cast<T*>(is_v ? a.v_out : a.k_out) + r * a.ld + c;
  if constexpr (!VEC) {
#pragma unroll
    for (int i = 0; i < 8; ++i) store_elem(o + i, f[i]);
  } else if constexpr (sizeof(T) == 4) {
    reinterpret_cast<float4*>(o)[0] = make_float4(f[0], f[1], f[2], f[3]);
    reinterpret_cast<float4*>(o)[1] = make_float4(f[4], f[5], f[6], f[7]);
  } else {
    *reinterpret_cast<uint4*>(o) = make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]),
                                              pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
  }
}

bool aligned(const void* p, int64_t ld, size_t elem, size_t bytes) {
  return reinterpret_cast<uintptr_t>(p) % bytes == 0 && ((size_t)ld * elem) % bytes == 0;
}

template <typename T>
hipError_t store_t(const CacheRowsArgs& a, int window, int groups, dim3 grid, hipStream_t s) {
  const double ps_inv = 1.0 / a.page_size;
  const bool vec = aligned(a.k, a.ld, sizeof(T), 4 * sizeof(T)) && aligned(a.v, a.ld, sizeof(T), 4 * sizeof(T)) &&
                   a.ld < 1 << 20;
  const dim3 block(64 * STORE_WAVES);
  if (a.d_head == 64) {
    if (vec) hipLaunchKernelGGL((cache_store_kernel<T, 64, true>), grid, block, 0, s, a, window, groups, ps_inv);
    else hipLaunchKernelGGL((cache_store_kernel<T, 64, false>), grid, block, 0, s, a, window, groups, ps_inv);
  } else {
    if (vec) hipLaunchKernelGGL((cache_store_kernel<T, 128, true>), grid, block, 0, s, a, window, groups, ps_inv);
    else hipLaunchKernelGGL((cache_store_kernel<T, 128, false>), grid, block, 0, s, a, window, groups, ps_inv);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_page_map(const PageMapArgs& a, hipStream_t s) {
  if (a.B < 1 || a.B > PAGE_MAP_MAX_BATCH) return hipErrorInvalidValue;
  const int blocks = a.max_rows > MAP_THREADS ? (a.max_rows + MAP_THREADS - 1) / MAP_THREADS : 1;
  hipLaunchKernelGGL(page_map_kernel, dim3(blocks), dim3(MAP_THREADS), (3 * a.B + 2) * sizeof(int), s, a,
                     page_inv(a.page_size));
  return hipGetLastError();
}

// Rows a wave: one while that leaves the device room; of long prompts 16, a usual page's worth, since
// most waves of one row would find that their row begins no run.
static int store_window(const CacheRowsArgs& a) { return a.rows > 256 ? 16 : 1; }
static int store_groups(const CacheRowsArgs& a) { return (2 * a.n_heads + STORE_WAVES - 1) / STORE_WAVES; }
static uint64_t store_blocks(const CacheRowsArgs& a) {
  const int w = store_window(a);
  return (uint64_t)((a.rows + w - 1) / w) * store_groups(a);
}
static uint64_t load_blocks(const CacheRowsArgs& a) {
  return ((uint64_t)a.rows * (a.n_heads * a.d_head / 8) + 255) / 256;
}

bool cache_rows_fit(const CacheRowsArgs& a) {
  return store_blocks(a) * (64 * STORE_WAVES) <= MAX_GRID_THREADS && load_blocks(a) * 256 <= MAX_GRID_THREADS;
}

hipError_t launch_cache_store(const CacheRowsArgs& a, hipStream_t s) {
  if (a.rows < 1) return hipSuccess;
  const int window = store_window(a), groups = store_groups(a);
  const dim3 grid((unsigned)store_blocks(a));
  return a.dtype == 1 ? store_t<bf16_t>(a, window, groups, grid, s) : store_t<float>(a, window, groups, grid, s);
}

hipError_t launch_cache_load(const CacheRowsArgs& a, hipStream_t s) {
  if (a.rows < 1) return hipSuccess;
  const dim3 grid((unsigned)load_blocks(a), 2), block(256);
  const size_t elem = a.dtype == 1 ? 2 : 4;
  const bool vec = aligned(a.k_out, a.ld, elem, 16) && aligned(a.v_out, a.ld, elem, 16);
  if (a.dtype == 1) {
    if (vec) hipLaunchKernelGGL((cache_load_kernel<bf16_t, true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((cache_load_kernel<bf16_t, false>), grid, block, 0, s, a);
  } else {
    if (vec) hipLaunchKernelGGL((cache_load_kernel<float, true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((cache_load_kernel<float, false>), grid, block, 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace ssd
