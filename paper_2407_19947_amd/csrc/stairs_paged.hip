// Operators over paged key/value caches: pages and slots for the requests of a step, storing the new rows and reading rows back,
// attention of the new rows over the pages.  The page layout is the tiled layout of the framework's own half caches (k_cache_off, v_cache_off),
// page by page.
#include "stairs_paged.h"

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <type_traits>

namespace stairs {
namespace {
// ---------------------------------------------------------------------------------------
// pages and slots
// ---------------------------------------------------------------------------------------
constexpr int kPlanThreads = 1024;
static_assert(kPlanThreads >= STAIRS_PAGED_MAX_SEQS, "a thread per sequence");

// Sums that stop at 2^31 - 1: counts that make no sense stay counts, ascending, and whatever is compared with fewer pages than that
// compares as it would in the integers.
struct Counts { unsigned rows, ask, drop; };
__device__ __forceinline__ unsigned capped(unsigned a, unsigned b) { return min(a + b, (unsigned)INT32_MAX); }
__device__ __forceinline__ Counts plus(const Counts& a, const Counts& b) { return {capped(a.rows, b.rows), capped(a.ask, b.ask), capped(a.drop, b.drop)}; }

// the last index b < n with first[b] <= i, first ascending, first[0] <= i; ten steps for any n up to 1024, so that several searches
// run side by side
__device__ __forceinline__ int find_seq(const int* first, int n, int i) {
  int b = 0;
#pragma unroll
  for (int step = STAIRS_PAGED_MAX_SEQS / 2; step >= 1; step >>= 1) {
    const int next = b + step;
    if (first[min(next, n - 1)] <= i && next < n) b = next;
  }
  return b;
}
// f(i, sequence of i) for the thread's share of 0 .. n - 1, U searches at a time
template <int U, typename F>
__device__ __forceinline__ void each_of(int n, const int* first, int n_seqs, int begin, int step, F f) {
  for (int i0 = begin; i0 < n; i0 += U * step) {
    int b[U];
#pragma unroll
    for (int k = 0; k < U; ++k) b[k] = find_seq(first, n_seqs, i0 + k * step);
#pragma unroll
    for (int k = 0; k < U; ++k)
      if (i0 + k * step < n) f(i0 + k * step, b[k]);
    if (n - i0 <= U * step) break;                  // (i0 stays an int)
  }
}

// positions and slots of the thread's rows, by the sequences' first rows and lengths
template <int U>
__device__ __forceinline__ void row_slots(const stairs_page_plan& p, const int* first, const int* lens, int rows, int begin, int step) {
  const int total = first[p.n_seqs], shift = __builtin_ctz(p.page_size);
  each_of<U>(min(total, rows), first, p.n_seqs, begin, step, [&](int t, int b) {
    const int len = lens[b];
    int pos = len > 0 ? len - (first[b + 1] - t) : -1, slot = -1;
    if (pos < 0 || pos >= len) pos = -1;            // (counts whose sum is no int)
    const int page = pos < 0 ? -1 : p.block_table[(size_t)b * p.max_blocks + (pos >> shift)];
    if ((unsigned)page < (unsigned)p.n_pages) slot = (page << shift) + (pos & (p.page_size - 1));
    p.position[t] = pos;
    p.slot[t] = slot;
  });
  for (long long t = begin; t < rows; t += step)
    if (t >= total) p.position[t] = p.slot[t] = -1;
}

// One block, bound by the latency of its steps: a thread per sequence counts, sums over the sequences say where everything goes, then the
// pages that change hands and the rows are spread over all threads (a sequence that ends with a thousand pages is not one
// thread's work).  Requests are served in order without overtaking, so whoever gets pages stands behind nobody who asked and got
// none: its pages begin where its share of the asks does.  (16 requests 5.0 us; 1000
// requests, a quarter of them chunks of up to 600 rows, 14.9 and k_paged_slots 4.8; a sum and a search at a time 20 and 5.6.)
__global__ __launch_bounds__(kPlanThreads) void k_paged_plan(stairs_page_plan p, int rows_here) {
  constexpr int kWaves = kPlanThreads / 64;
  __shared__ Counts s_wave[kWaves];
  __shared__ int s_rows[STAIRS_PAGED_MAX_SEQS + 1], s_drop[STAIRS_PAGED_MAX_SEQS], s_ask[STAIRS_PAGED_MAX_SEQS];
  __shared__ int s_need[STAIRS_PAGED_MAX_SEQS], s_held[STAIRS_PAGED_MAX_SEQS], s_granted;
  const int b = threadIdx.x, lane = b & 63, wave = b >> 6;
  const bool here = b < p.n_seqs;
  const int cached = here ? max(p.cached[b], 0) : 0, fresh = here ? max(p.fresh[b], 0) : 0;
  const int held = here ? min(max(p.held[b], 0), p.max_blocks) : 0;
  const int n_free = min(max(p.n_free[0], 0), p.n_pages);
  const unsigned len = (unsigned)cached + (unsigned)fresh;
  const bool fits = len <= (unsigned)p.max_blocks * (unsigned)p.page_size;
  const int need = fits ? (int)((len + p.page_size - 1) >> __builtin_ctz(p.page_size)) : held;
  const int ask = max(need - held, 0), drop = held - min(need, held);
  const Counts mine{(unsigned)fresh, (unsigned)ask, (unsigned)drop};
  Counts to = mine;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const Counts o{__shfl_up(to.rows, off), __shfl_up(to.ask, off), __shfl_up(to.drop, off)};
    if (lane >= off) to = plus(to, o);
  }
  if (lane == 63) s_wave[wave] = to;
  if (b == 0) s_granted = 0;
  __syncthreads();
  Counts front{0, 0, 0}, all{0, 0, 0};
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const Counts o = s_wave[w];
    all = plus(all, o);
    if (w < wave) front = plus(front, o);
  }
  const Counts before = plus(front, {(unsigned)__shfl_up(to.rows, 1), (unsigned)__shfl_up(to.ask, 1), (unsigned)__shfl_up(to.drop, 1)});
  const Counts at = lane == 0 ? front : before;
  const int rows = (int)all.rows, dropped = min((int)all.drop, p.n_pages - n_free), avail = n_free + dropped;
  const bool ok = fits && (ask == 0 || (long long)at.ask + ask <= avail);
  const unsigned long long takers = __ballot(ok && ask > 0);
  if (takers && lane == 63 - __builtin_clzll(takers)) atomicMax(&s_granted, (int)at.ask + ask);   // (the wave's last)
  if (here) {
    s_rows[b] = (int)at.rows;
    s_drop[b] = (int)at.drop;
    s_ask[b] = (int)at.ask;
    s_need[b] = need;
    s_held[b] = held;
  }
  if (b == 0) s_rows[p.n_seqs] = rows;
  __syncthreads();
  const int granted = s_granted;
  // pages given back, behind the free ones
  each_of<4>(dropped, s_drop, p.n_seqs, b, kPlanThreads, [&](int i, int q) {
    p.free_pages[n_free + i] = p.block_table[(size_t)q * p.max_blocks + s_need[q] + (i - s_drop[q])];
  });
  __syncthreads();
  // pages taken, from the end of the stack
  each_of<4>(granted, s_ask, p.n_seqs, b, kPlanThreads, [&](int i, int q) {
    p.block_table[(size_t)q * p.max_blocks + s_held[q] + (i - s_ask[q])] = p.free_pages[avail - 1 - i];
  });
  if (here) {
    p.held_out[b] = ok ? need : held;
    p.row_start[b] = s_rows[b];
    p.seq_len[b] = s_need[b] = ok ? (int)len : 0;    // (s_need: of no more use)
  }
  if (b == 0) {
    p.n_free_out[0] = avail - granted;
    p.row_start[p.n_seqs] = rows;
  }
  __syncthreads();
  row_slots<4>(p, s_rows, s_need, rows_here, b, kPlanThreads);
}

__global__ __launch_bounds__(256) void k_paged_slots(stairs_page_plan p) {
  __shared__ int s_rows[STAIRS_PAGED_MAX_SEQS + 1], s_len[STAIRS_PAGED_MAX_SEQS];
  for (int b = threadIdx.x; b <= p.n_seqs; b += 256) {
    s_rows[b] = p.row_start[b];
    if (b < p.n_seqs) s_len[b] = p.seq_len[b];
  }
  __syncthreads();
  row_slots<1>(p, s_rows, s_len, p.max_rows, blockIdx.x * 256 + threadIdx.x, gridDim.x * 256);
}

// ---------------------------------------------------------------------------------------
// storing rows
// ---------------------------------------------------------------------------------------
template <typename T> struct Elem;
template <> struct Elem<__bf16> {
  typedef bf16x8 x8;
  static __device__ __forceinline__ float up(__bf16 v) { return (float)v; }
  static __device__ __forceinline__ __bf16 down(float v) { return (__bf16)v; }
};
template <> struct Elem<_Float16> {
  typedef f16x8 x8;
  static __device__ __forceinline__ float up(_Float16 v) { return (float)v; }
  static __device__ __forceinline__ _Float16 down(float v) { return (_Float16)v; }
};

// ---- rows in 8 bits -------------------------------------------------------------------------------------------------
// A row of a head is codes times 2^(b - 127): b the smallest byte from 1 on with amax <= 448 * 2^(b - 127) = 1.75 * 2^(b - 119).  A float
// amax = 1.f * 2^(E - 127) asks for b = E - 8, one more where its mantissa is past 1.75.  (A power of two loses nothing against a finer scale: codes are
// floats themselves, with 4 bits down to 2^-14 of the largest, and products with it are exact.)
__device__ __forceinline__ uint32_t finite_bits(float x) {       // of |x|; 0 for infinities and NaN
  const uint32_t u = __float_as_uint(x) & 0x7FFFFFFFu;
  return u < 0x7F800000u ? u : 0u;
}
// Rows of halves: magnitudes past 61440 are held as 61440 (within a half step, 2^-4; the next number is past the largest half).  -> what is then the
// largest finite one
constexpr uint32_t kHalfTop = 0x47700000u;
__device__ __forceinline__ uint32_t cut(float* x, int n) {
#pragma unroll
  for (int i = 0; i < n; ++i)
    if (finite_bits(x[i]) > kHalfTop) x[i] = copysignf(61440.f, x[i]);
  return kHalfTop;
}
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax_bits) {
  const int b = (int)(amax_bits >> 23) - 8 + ((amax_bits & 0x7FFFFFu) > 0x600000u);
  return (uint32_t)max(b, 1);
}
__device__ __forceinline__ float scale_inverse(uint32_t b) { return __uint_as_float((254u - b) << 23); }     // 2^(127 - b), b at most 247
__device__ __forceinline__ float scale_of(uint32_t bytes, int i) {                                           // byte i of four
  return __uint_as_float((i < 3 ? bytes << (23 - 8 * i) : bytes >> 1) & 0x7F800000u);
}
// the largest byte with which all codes are numbers of the type: 448 * 2^(b - 127) is; of four bytes those past it, as their top bits
template <typename T> constexpr uint32_t kMostByte = __is_same(T, __bf16) ? 246 : 134;
template <typename T>
__device__ __forceinline__ uint32_t bytes_past(uint32_t u) { return ((u & 0x7F7F7F7Fu) + (255 - kMostByte<T>) * 0x01010101u) & u & 0x80808080u; }
__device__ __forceinline__ uint32_t codes_of(float a, float b, float c, float d) {
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
}
template <typename T> struct Wide;
template <> struct Wide<__bf16> {
  template <bool HI> static __device__ __forceinline__ uint32_t pair(uint32_t codes, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, HI));
  }
};
template <> struct Wide<_Float16> {
  template <bool HI> static __device__ __forceinline__ uint32_t pair(uint32_t codes, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes, scale, HI));
  }
};
// eight codes as numbers of the type, times a power of two
template <typename T>
__device__ __forceinline__ uint4 widen(uint32_t lo, uint32_t hi, float scale) {
  return make_uint4(Wide<T>::template pair<false>(lo, scale), Wide<T>::template pair<true>(lo, scale), Wide<T>::template pair<false>(hi, scale),
                    Wide<T>::template pair<true>(hi, scale));
}
// the same, a power of two for each: a pair converted with either's
__device__ __forceinline__ uint32_t low_high(uint32_t a, uint32_t b) { return (a & 0xFFFFu) | (b & 0xFFFF0000u); }
template <typename T>
__device__ __forceinline__ uint4 widen(uint32_t lo, uint32_t hi, const float (&f)[8]) {
  typedef Wide<T> W;
  return make_uint4(low_high(W::template pair<false>(lo, f[0]), W::template pair<false>(lo, f[1])), low_high(W::template pair<true>(lo, f[2]), W::template pair<true>(lo, f[3])),
                    low_high(W::template pair<false>(hi, f[4]), W::template pair<false>(hi, f[5])), low_high(W::template pair<true>(hi, f[6]), W::template pair<true>(hi, f[7])));
}
__device__ __forceinline__ uint32_t group_max(uint32_t v, int lanes) {                                       // of 4, 8 or 16 adjacent lanes
  auto step = [&](auto ctrl) { v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, decltype(ctrl)::value, 0xF, 0xF, true)); };
  step(std::integral_constant<int, kDppXor1>{});
  step(std::integral_constant<int, kDppXor2>{});
  if (lanes > 4) step(std::integral_constant<int, kDppHalfMirror>{});
  if (lanes > 8) step(std::integral_constant<int, kDppRor8>{});
  return v;
}

// sine and cosine of `turns` whole turns: the nearest quarter turn, and the series for what is left, |x| <= pi / 4 (the next terms are
// below 2^-28)
__device__ __forceinline__ float2 cos_sin(double turns) {
  const double t = 4.0 * (turns - rint(turns)), quarter = rint(t), x = (t - quarter) * 1.57079632679489661923, y = x * x;
  double s = 1.0 / 362880;
  s = fma(s, y, -1.0 / 5040);
  s = fma(s, y, 1.0 / 120);
  s = fma(s, y, -1.0 / 6);
  s = fma(s * y, x, x);
  double c = -1.0 / 3628800;
  c = fma(c, y, 1.0 / 40320);
  c = fma(c, y, -1.0 / 720);
  c = fma(c, y, 1.0 / 24);
  c = fma(c, y, -0.5);
  c = fma(c, y, 1.0);
  const int q = (int)quarter;
  const float fc = (float)c, fs = (float)s;
  const float2 r = q & 1 ? make_float2(-fs, fc) : make_float2(fc, fs);      // (a quarter turn on: (cos, sin) -> (-sin, cos))
  return q & 2 ? make_float2(-r.x, -r.y) : r;
}

// (streaming hint, for what is read once: 8190 rows of 16 + 16 heads of q and k 36.7 -> 30.5 us; on the stores it costs 9)
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
template <typename X>
__device__ __forceinline__ X ld_once_as(const void* p) {
  return __builtin_bit_cast(X, __builtin_nontemporal_load(static_cast<const u32x4*>(p)));
}

__device__ __forceinline__ void st_once(void* p, uint4 v) { __builtin_nontemporal_store(__builtin_bit_cast(u32x4, v), static_cast<u32x4*>(p)); }

// Bound by memory, with few rows by latency.  Into 8-bit pages a row's largest magnitude is found by the lanes that share it; values become codes on
// their way to LDS, four heads at a time (8190 rows of 48 heads 46 us = 3.7 TB/s, a head at a time 49).  A work-group has 32 rows and some of the n_heads + 2 n_kv_heads heads (so many
// groups of them that there are work for all CUs); the rows' rotations are formed once for all its heads.  q and k: a thread takes 8
// pairs of a row, 16 bytes of either half; in a key tile the same 8 dims of 8 rows are one line.  v: a head's rows go through LDS;
// the eight positions of a value tile that are 16 adjacent bytes a dim (two quads, 16 apart) are stored together where they are rows
// of this call, so that a wave's store is a whole tile row; rows that have not all of them as quads of 8 bytes or single
// values.  (Quads transposed in registers, 8 bytes here and there: 8190 rows of 48 heads 75 us, 40 of them for the
// values; as it is 57.5 = 3.5 TB/s, reading 8 % more than the rows have,
// writing no more.)
constexpr int kAppendRows = 32;
template <typename T, int HD, bool H8>
__global__ __launch_bounds__(256) void k_paged_append(stairs_paged_cache c, stairs_paged_rows a, double log2_theta) {
  constexpr int AHEAD = 19, BEHIND = 16;                        // rows around these that decide how theirs are stored
  constexpr int kHeads = 4;
  __shared__ union {
    float2 cs[kAppendRows][HD / 2];
    T v[H8 ? 1 : kAppendRows + AHEAD][HD];
    uint8_t v8[H8 ? kHeads : 1][kAppendRows + AHEAD][HD];
  } lds;
  __shared__ uint8_t s_vb[H8 ? kHeads : 1][kAppendRows + AHEAD];   // the values' powers of two
  __shared__ int s_slots[BEHIND + kAppendRows + AHEAD], s_pos[kAppendRows], s_unit[kAppendRows], s_units, s_end;
  const int* const s_slot = s_slots + BEHIND;
  // (an XCD takes rows that follow each other: lines that two work-groups share meet in one L2; 16000 rows of 48 heads 104 -> 101 us)
  const int xcd = blockIdx.x & 7, share = gridDim.x >> 3, more = gridDim.x & 7;
  const int t0 = (xcd * share + min(xcd, more) + (int)(blockIdx.x >> 3)) * kAppendRows, n = min(kAppendRows, a.rows - t0);
  // its heads: a run of q's, one of k's and v's
  const int nq = a.n_heads, nk = c.n_kv_heads, y = blockIdx.y, groups = gridDim.y;
  const int only = gridDim.z == 1 ? -1 : (int)blockIdx.z;      // (few rows: q, k and v each a work-group of their own)
  const int q0 = nq * y / groups, q1 = only > 0 ? q0 : nq * (y + 1) / groups, k0 = nk * y / groups, k1 = only == 0 ? k0 : nk * (y + 1) / groups;
  const bool rotate = a.rope_theta > 0.f;
  const int tid = threadIdx.x, lane = tid & 63;
  const unsigned slots = (unsigned)c.n_pages * (unsigned)c.page_size;
  if (tid < BEHIND + kAppendRows + AHEAD) {
    const int t = t0 - BEHIND + tid, slot = t >= 0 && t < a.rows ? a.slot[t] : -1;
    s_slots[tid] = (unsigned)slot < slots ? slot : -1;
  }
  if (tid < kAppendRows) s_pos[tid] = tid < n ? (rotate ? a.position[t0 + tid] : 0) : -1;
  __syncthreads();
  if (tid < 64) {
    // whether row r begins four of one quad; whether that and row r + 16 begin the two quads that are stored together
    auto quad = [&](int r) { return s_slot[r] >= 0 && (s_slot[r] & 3) == 0 && s_slot[r + 1] == s_slot[r] + 1 && s_slot[r + 2] == s_slot[r] + 2 && s_slot[r + 3] == s_slot[r] + 3; };
    auto pair = [&](int r) { return quad(r) && (s_slot[r] & 16) == 0 && s_slot[r + 16] == s_slot[r] + 16 && quad(r + 16); };
    int kind = 0;                                               // 3: two quads, 2: one, 1: a single row, 0: stored with another
    if (lane < n && s_slot[lane] >= 0) {
      const int first = lane - (s_slot[lane] & 3);
      if (first < -BEHIND || !quad(first)) kind = 1;
      else if (first == lane) kind = pair(lane) ? 3 : (s_slot[lane] & 16) && lane >= 16 - BEHIND && pair(lane - 16) ? 0 : 2;
    }
    const unsigned long long units = __ballot(kind > 0);
    if (kind > 0) s_unit[__popcll(units & ((1ull << lane) - 1))] = lane << 2 | kind;
    int end = kind == 3 ? lane + 20 : kind == 2 ? lane + 4 : lane + 1;   // rows that the units read
    if (kind == 0) end = 0;
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) end = max(end, __shfl_xor(end, off));
    if (lane == 0) {
      s_units = __popcll(units);
      s_end = end;
    }
  }
  __syncthreads();
  if (rotate && (q1 > q0 || (k1 > k0 && only < 2))) {
    const int i = tid % (HD / 2);
    const double turn = exp2(-(2.0 * i / HD) * log2_theta) * 0.15915494309189533577;   // of a position, in whole turns
    for (int r = tid / (HD / 2); r < n; r += 256 / (HD / 2)) lds.cs[r][i] = cos_sin((double)s_pos[r] * turn);
    __syncthreads();
  }
  const size_t head_elems = (size_t)c.page_size * HD;
  const int ps_shift = __builtin_ctz(c.page_size);
  typedef typename Elem<T>::x8 x8;
  constexpr int PAIRS = HD / 16;                                // units of 8 pairs
  auto turn = [&](x8& lo, x8& hi, int r, int e) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float2 v = rope_rotate(Elem<T>::up(lo[k]), Elem<T>::up(hi[k]), lds.cs[r][e + k]);
      lo[k] = Elem<T>::down(v.x);
      hi[k] = Elem<T>::down(v.y);
    }
  };
  const int nqh = q1 - q0, nkh = only < 2 ? k1 - k0 : 0;
  for (int i = tid; i < nqh * n * PAIRS; i += 256) {            // (a row's heads one behind the other in memory)
    const int e = i % PAIRS * 8, h = q0 + i / PAIRS % nqh, r = i / (PAIRS * nqh);
    if (s_pos[r] < 0) continue;
    const T* src = static_cast<const T*>(a.q) + (size_t)(t0 + r) * a.q_stride + h * HD + e;
    x8 lo = ld_once_as<x8>(src), hi = ld_once_as<x8>(src + HD / 2);
    if (rotate) turn(lo, hi, r, e);
    T* dst = static_cast<T*>(a.q_out) + (size_t)(t0 + r) * a.q_out_stride + h * HD + e;
    if constexpr (H8) {                                         // (beside 8-bit pages the streaming hint saves 2 of 50 us)
      st_once(dst, __builtin_bit_cast(uint4, lo));
      st_once(dst + HD / 2, __builtin_bit_cast(uint4, hi));
    } else {
      *reinterpret_cast<x8*>(dst) = lo;
      *reinterpret_cast<x8*>(dst + HD / 2) = hi;
    }
  }
  const size_t head_scales = (size_t)c.page_size * 2;
  uint8_t* const scales = static_cast<uint8_t*>(c.scale);
  if constexpr (H8) {
    // four lanes have a row: each 8 dims of every 32, so that what it stores are whole places of 16 bytes
    constexpr int NX = HD / 32;
    for (int i = tid; i < nkh * kAppendRows * 4; i += 256) {
      const int g = i & 3, r = i / 4 % kAppendRows, h = k0 + i / (4 * kAppendRows), slot = s_slot[r];
      if (r >= n || slot < 0) continue;
      const T* src = static_cast<const T*>(a.k) + (size_t)(t0 + r) * a.k_stride + h * HD + 8 * g;
      x8 in[NX];
#pragma unroll
      for (int j = 0; j < NX; ++j) in[j] = ld_once_as<x8>(src + 32 * j);
      float x[NX][8];
#pragma unroll
      for (int j = 0; j < NX; ++j)
#pragma unroll
        for (int k = 0; k < 8; ++k) x[j][k] = Elem<T>::up(in[j][k]);
      if (rotate) {
#pragma unroll
        for (int j = 0; j < NX / 2; ++j)
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const float2 v = rope_rotate(x[j][k], x[j + NX / 2][k], lds.cs[r][32 * j + 8 * g + k]);
            x[j][k] = v.x;
            x[j + NX / 2][k] = v.y;
          }
      }
      uint32_t top = 0;
#pragma unroll
      for (int j = 0; j < NX; ++j)
#pragma unroll
        for (int k = 0; k < 8; ++k) top = max(top, finite_bits(x[j][k]));
      if (__is_same(T, _Float16) && top > kHalfTop) top = cut(x[0], NX * 8);
      const uint32_t b = scale_byte(group_max(top, 4));
      const float f = scale_inverse(b);
      uint2 code[NX];
#pragma unroll
      for (int j = 0; j < NX; ++j)
        code[j] = make_uint2(codes_of(x[j][0] * f, x[j][1] * f, x[j][2] * f, x[j][3] * f), codes_of(x[j][4] * f, x[j][5] * f, x[j][6] * f, x[j][7] * f));
      const int p = slot & (c.page_size - 1);
      const size_t head = (size_t)(slot >> ps_shift) * nk + h;
      uint8_t* dst = static_cast<uint8_t*>(c.k) + head * head_elems + k_held_off(p, 8 * g, HD);
#pragma unroll
      for (int t = 0; t < HD / 64; ++t) *reinterpret_cast<uint4*>(dst + t * 1024) = make_uint4(code[2 * t].x, code[2 * t].y, code[2 * t + 1].x, code[2 * t + 1].y);
      if (g == 0) scales[head * head_scales + scale_off(p)] = (uint8_t)b;
    }
  } else
  for (int i = tid; i < nkh * kAppendRows * PAIRS; i += 256) {  // (rows that are neighbours in a tile one behind the other)
    const int e = i % PAIRS * 8, r = i / PAIRS % kAppendRows, h = k0 + i / (PAIRS * kAppendRows), slot = s_slot[r];
    if (r >= n || slot < 0) continue;
    const T* src = static_cast<const T*>(a.k) + (size_t)(t0 + r) * a.k_stride + h * HD + e;
    x8 lo = ld_once_as<x8>(src), hi = ld_once_as<x8>(src + HD / 2);
    if (rotate) turn(lo, hi, r, e);
    T* dst = static_cast<T*>(c.k) + ((size_t)(slot >> ps_shift) * nk + h) * head_elems;
    const int p = slot & (c.page_size - 1);
    *reinterpret_cast<x8*>(dst + k_cache_off(p, e, HD)) = lo;
    *reinterpret_cast<x8*>(dst + k_cache_off(p, e + HD / 2, HD)) = hi;
  }
  const int units = only == 1 ? 0 : s_units, staged = s_end;
  if (units == 0) return;
  if constexpr (H8) {
    // four heads at a time: their rows are all requested before the first is waited for
    for (int h0 = k0; h0 < k1; h0 += kHeads) {
      const int nh = min(kHeads, k1 - h0), per_row = nh * (HD / 8);
      __syncthreads();
      for (int i0 = tid; i0 < staged * per_row; i0 += 256 * 8) {
        x8 in[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int i = min(i0 + j * 256, staged * per_row - HD / 8 + tid % (HD / 8)), r = i / per_row, e = i % per_row * 8;   // (past the last: the last row's again)
          in[j] = ld_once_as<x8>(static_cast<const T*>(a.v) + (size_t)(t0 + r) * a.v_stride + h0 * HD + e);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int i = i0 + j * 256, r = i / per_row, e = i % per_row * 8;
          if (i >= staged * per_row) break;
          float x[8];
          uint32_t top = 0;
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            x[k] = Elem<T>::up(in[j][k]);
            top = max(top, finite_bits(x[k]));
          }
          if (__is_same(T, _Float16) && top > kHalfTop) top = cut(x, 8);
          const uint32_t b = scale_byte(group_max(top, HD / 8));
          const float f = scale_inverse(b);
          *reinterpret_cast<uint2*>(&lds.v8[e / HD][r][e % HD]) = make_uint2(codes_of(x[0] * f, x[1] * f, x[2] * f, x[3] * f), codes_of(x[4] * f, x[5] * f, x[6] * f, x[7] * f));
          if (e % HD == 0) s_vb[e / HD][r] = (uint8_t)b;
        }
      }
      __syncthreads();
      // a place of 16 bytes: dims e and e + 16, eight positions of either
      for (int i = tid; i < nh * units * (HD / 2); i += 256) {
        const int j = i % (HD / 2), e = (j >> 4) * 32 + (j & 15), at = i / (HD / 2), hh = at / units, u = s_unit[at - hh * units], r = u >> 2, kind = u & 3, slot = s_slot[r];
        const int p = slot & (c.page_size - 1);
        const size_t head = (size_t)(slot >> ps_shift) * nk + h0 + hh;
        uint8_t* dst = static_cast<uint8_t*>(c.v) + head * head_elems + v_held_off(p, e, HD);
        uint8_t* sdst = scales + head * head_scales + scale_off(p) + 8;
        const auto& v8 = lds.v8[hh];
        const auto& vb = s_vb[hh];
        auto four = [&](int row, int dim) { return v8[row][dim] | v8[row + 1][dim] << 8 | v8[row + 2][dim] << 16 | (uint32_t)v8[row + 3][dim] << 24; };
        auto bytes = [&](int row) { return vb[row] | vb[row + 1] << 8 | vb[row + 2] << 16 | (uint32_t)vb[row + 3] << 24; };
        if (kind == 1) {
          dst[0] = v8[r][e];
          dst[8] = v8[r][e + 16];
          if (j == 0) *sdst = vb[r];
        } else if (kind == 2) {
          *reinterpret_cast<uint32_t*>(dst) = four(r, e);
          *reinterpret_cast<uint32_t*>(dst + 8) = four(r, e + 16);
          if (j == 0) *reinterpret_cast<uint32_t*>(sdst) = bytes(r);
        } else {
          *reinterpret_cast<uint4*>(dst) = make_uint4(four(r, e), four(r + 16, e), four(r, e + 16), four(r + 16, e + 16));
          if (j == 0) *reinterpret_cast<uint2*>(sdst) = make_uint2(bytes(r), bytes(r + 16));
        }
      }
    }
    return;
  }
  for (int h = k0; h < k1; ++h) {
    __syncthreads();
    for (int i = tid; i < staged * (HD / 8); i += 256) {
      const int r = i / (HD / 8), e = i % (HD / 8) * 8;
      *reinterpret_cast<x8*>(&lds.v[r][e]) = ld_once_as<x8>(static_cast<const T*>(a.v) + (size_t)(t0 + r) * a.v_stride + h * HD + e);
    }
    __syncthreads();
    for (int i = tid; i < units * HD; i += 256) {
      const int e = i % HD, r = s_unit[i / HD] >> 2, kind = s_unit[i / HD] & 3, slot = s_slot[r];
      T* dst = static_cast<T*>(c.v) + ((size_t)(slot >> ps_shift) * nk + h) * head_elems + v_cache_off(slot & (c.page_size - 1), e, HD);
      if (kind == 1) {
        *dst = lds.v[r][e];
      } else {
        T v[8];
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = lds.v[r + k][e];
        if (kind == 2) {
          *reinterpret_cast<uint2*>(dst) = *reinterpret_cast<const uint2*>(v);
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k) v[4 + k] = lds.v[r + 16 + k][e];
          *reinterpret_cast<uint4*>(dst) = *reinterpret_cast<const uint4*>(v);
        }
      }
    }
  }
}

// ---------------------------------------------------------------------------------------
// reading rows back
// ---------------------------------------------------------------------------------------
// As k_paged_append the other way: a work-group has 32 rows and some of the heads; keys go from a tile's places to the rows directly, values through
// LDS, the eight positions of a place at once where they are rows of the work-group in that order, four or one otherwise.  Bound by memory (24000 rows
// of 8 heads of 128 in 8 bits: 29.4 .. 30.2 us = 5.0 .. 5.2 TB/s, what a copy reaches; 40 without the streaming hint on the stores; in 16 bits 49 = 4.1 TB/s; several
// heads at a time, as in k_paged_append, 1 .. 5 us slower).
// What is past the type's largest comes back as that (a bfloat16 from 1.9375 * 2^127 on is stored as 2^128; halves as large are in pages alone that others
// have filled).  Codes have no infinities, so an infinity is such a number, its bits one more than the largest's: one is taken off whatever has all
// exponent bits (of a NaN, too: it stays one).  (24000 rows of bfloat16 30.2 us, without it 29.7; every number compared as a float 32.0.)
template <typename T> __device__ __forceinline__ uint32_t odd_bits(uint32_t u);
template <typename T>
__device__ __forceinline__ uint4 no_infinities(uint4 v) {
  auto less = [](uint32_t u) { return u - (odd_bits<T>(u) >> 15); };
  return make_uint4(less(v.x), less(v.y), less(v.z), less(v.w));
}
template <typename T, int HD, bool H8>
__global__ __launch_bounds__(256) void k_paged_read(stairs_paged_cache c, stairs_paged_out a) {
  constexpr int R = kAppendRows;
  __shared__ uint16_t s_v[R][HD + 8];
  __shared__ int s_slot[R], s_unit[R], s_units;
  const int xcd = blockIdx.x & 7, share = gridDim.x >> 3, more = gridDim.x & 7;
  const int t0 = (xcd * share + min(xcd, more) + (int)(blockIdx.x >> 3)) * R, n = min(R, a.rows - t0);
  const int nk = c.n_kv_heads, h0 = nk * (int)blockIdx.y / (int)gridDim.y, h1 = nk * ((int)blockIdx.y + 1) / (int)gridDim.y;
  const int tid = threadIdx.x, lane = tid & 63, ps_shift = __builtin_ctz(c.page_size);
  const unsigned slots = (unsigned)c.n_pages * (unsigned)c.page_size;
  if (tid < R) {
    const int slot = tid < n ? a.slot[t0 + tid] : -1;
    s_slot[tid] = (unsigned)slot < slots ? slot : -1;
  }
  __syncthreads();
  if (tid < 64) {
    auto quad = [&](int r) { return r + 3 < n && s_slot[r] >= 0 && (s_slot[r] & 3) == 0 && s_slot[r + 1] == s_slot[r] + 1 && s_slot[r + 2] == s_slot[r] + 2 && s_slot[r + 3] == s_slot[r] + 3; };
    auto pair = [&](int r) { return r + 19 < n && quad(r) && (s_slot[r] & 16) == 0 && s_slot[r + 16] == s_slot[r] + 16 && quad(r + 16); };
    int kind = 0;                                               // 3: two quads, 2: one, 1: a single row, 0: read with another
    if (lane < n && s_slot[lane] >= 0) {
      const int first = lane - (s_slot[lane] & 3);
      if (first < 0 || !quad(first)) kind = 1;
      else if (first == lane) kind = pair(lane) ? 3 : (s_slot[lane] & 16) && lane >= 16 && pair(lane - 16) ? 0 : 2;
    }
    const unsigned long long units = __ballot(kind > 0);
    if (kind > 0) s_unit[__popcll(units & ((1ull << lane) - 1))] = lane << 2 | kind;
    if (lane == 0) s_units = __popcll(units);
  }
  const size_t head_bytes = (size_t)c.page_size * HD * (H8 ? 1 : 2), head_scales = (size_t)c.page_size * 2;
  const uint8_t* const scales = static_cast<const uint8_t*>(c.scale);
  if (a.k && blockIdx.z == 0) {
    for (int i = tid; i < (h1 - h0) * R * 4; i += 256) {
      const int g = i & 3, r = i / 4 % R, h = h0 + i / (4 * R), slot = s_slot[r];
      if (r >= n || slot < 0) continue;
      const int p = slot & (c.page_size - 1);
      const size_t head = (size_t)(slot >> ps_shift) * nk + h;
      const uint8_t* src = static_cast<const uint8_t*>(c.k) + head * head_bytes;
      uint16_t* dst = static_cast<uint16_t*>(a.k) + (size_t)(t0 + r) * a.k_stride + h * HD + 8 * g;
      if constexpr (H8) {
        const float f = scale_of(scales[head * head_scales + scale_off(p)], 0);
#pragma unroll
        for (int t = 0; t < HD / 64; ++t) {
          const uint4 v = *reinterpret_cast<const uint4*>(src + k_held_off(p, 8 * g, HD) + t * 1024);
          st_once(dst + 64 * t, no_infinities<T>(widen<T>(v.x, v.y, f)));
          st_once(dst + 64 * t + 32, no_infinities<T>(widen<T>(v.z, v.w, f)));
        }
      } else {
#pragma unroll
        for (int j = 0; j < HD / 32; ++j) st_once(dst + 32 * j, *reinterpret_cast<const uint4*>(src + 2 * k_cache_off(p, 32 * j + 8 * g, HD)));
      }
    }
  }
  if (!a.v || (gridDim.z > 1 && blockIdx.z == 0)) return;
  constexpr int D = H8 ? HD / 2 : HD;                           // places of 16 bytes of a unit
  for (int h = h0; h < h1; ++h) {
    __syncthreads();
    const int units = s_units;
    for (int i = tid; i < units * D; i += 256) {
      const int j = i % D, e = H8 ? (j >> 4) * 32 + (j & 15) : j, r = s_unit[i / D] >> 2, kind = s_unit[i / D] & 3, slot = s_slot[r], p = slot & (c.page_size - 1);
      const size_t head = (size_t)(slot >> ps_shift) * nk + h;
      if constexpr (H8) {
        const uint8_t* src = static_cast<const uint8_t*>(c.v) + head * head_bytes + v_held_off(p, e, HD);
        const uint8_t* sc = scales + head * head_scales + scale_off(p) + 8;
        auto put = [&](int row, uint32_t codes, uint32_t bytes, int dim, int count) {
          const uint32_t v[4] = {Wide<T>::template pair<false>(codes, scale_of(bytes, 0)), Wide<T>::template pair<false>(codes, scale_of(bytes, 1)) >> 16,
                                 Wide<T>::template pair<true>(codes, scale_of(bytes, 2)), Wide<T>::template pair<true>(codes, scale_of(bytes, 3)) >> 16};
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (k < count) s_v[row + k][dim] = (uint16_t)v[k];
        };
        if (kind == 3) {
          const uint4 v = *reinterpret_cast<const uint4*>(src);
          const uint2 b = *reinterpret_cast<const uint2*>(sc);
          put(r, v.x, b.x, e, 4);
          put(r + 16, v.y, b.y, e, 4);
          put(r, v.z, b.x, e + 16, 4);
          put(r + 16, v.w, b.y, e + 16, 4);
        } else if (kind == 2) {
          const uint32_t b = *reinterpret_cast<const uint32_t*>(sc);
          put(r, *reinterpret_cast<const uint32_t*>(src), b, e, 4);
          put(r, *reinterpret_cast<const uint32_t*>(src + 8), b, e + 16, 4);
        } else {
          put(r, src[0], *sc, e, 1);
          put(r, src[8], *sc, e + 16, 1);
        }
      } else {
        const uint16_t* src = static_cast<const uint16_t*>(c.v) + head * (head_bytes / 2) + v_cache_off(p, e, HD);
        if (kind == 1) {
          s_v[r][e] = *src;
        } else {
          uint16_t v[8];
          if (kind == 3) *reinterpret_cast<uint4*>(v) = *reinterpret_cast<const uint4*>(src);
          else *reinterpret_cast<uint2*>(v) = *reinterpret_cast<const uint2*>(src);
#pragma unroll
          for (int k = 0; k < 4; ++k) s_v[r + k][e] = v[k];
          if (kind == 3)
#pragma unroll
            for (int k = 0; k < 4; ++k) s_v[r + 16 + k][e] = v[4 + k];
        }
      }
    }
    __syncthreads();
    for (int i = tid; i < n * (HD / 8); i += 256) {
      const int r = i / (HD / 8), e = i % (HD / 8) * 8;
      if (s_slot[r] < 0) continue;
      const uint4 v = *reinterpret_cast<const uint4*>(&s_v[r][e]);
      st_once(static_cast<uint16_t*>(a.v) + (size_t)(t0 + r) * a.v_stride + h * HD + e, H8 ? no_infinities<T>(v) : v);
    }
  }
}

// ---------------------------------------------------------------------------------------
// attention
// ---------------------------------------------------------------------------------------
// A tile is up to 16 CT columns of one key head of one sequence; a column is (row, query head of the group), so that heads that
// share keys share the loads.  Scores are computed transposed, S^T = K Q^T: a lane then holds the scores of ONE column for 8 of 32
// keys, which are already the operand O^T = V^T P^T wants from it (the value tiles are laid out for that order of keys), so the
// probabilities never leave their registers, and maximum and sum are per lane but for two exchanges between lane groups.
__device__ __forceinline__ f32x4 mma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mma(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
constexpr float kLog2e = 1.44269504088896340736f;
// The running maximum m follows once a score exceeds it by 2^slack; probabilities are exp2(score + lift - m).  A bfloat16 has a float's
// range: rounded, they keep their relative precision wherever they lie.  A half's steps are 2^-24 all the way below 2^-14, so the largest
// are put next to its end (2^15, and room for what rounding adds): full precision down to 2^-27 of the largest, and keys below that are
// off by 2^-38 of it, 60000 of them together by 2^-22.  (Without the lift the others' share beside keys 13 .. 18 nats above them
// was up to 23 times as far off as roundings of half a step explain.)
template <typename T> struct Headroom;
template <> struct Headroom<__bf16> { static constexpr float slack = 8.f, lift = 0.f; };
template <> struct Headroom<_Float16> { static constexpr float slack = 2.f, lift = 13.f; };

// x >= 0 as two numbers of the type, the one below it and what that leaves, for two products with the values: results are then off by
// their own rounding (with probabilities rounded once they were 1.3 to 1.5 times as far off).  Where the first is not 0 neither is the rest (an
// infinite value times 0 would be NaN): in bfloat16 2^-23 of x is added to it, in half it is the smallest step at least.  The matrix units
// wait for memory in attend_rows, the second product costs 0 .. 1.5 % there (32 verifications 66.4 -> 66.6 us, the mixed batch 78.5 -> 79.0);
// in attend_chunk, which they bound, a third (2048 rows over 8200 positions 241 -> 325 us, 256 over 8000 56 -> 70): probabilities stay
// rounded once there, half a step of the type each.
__device__ __forceinline__ void split(const float (&x)[8], bf16x8& first, bf16x8& rest) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t top = __float_as_uint(x[i]) & 0xFFFF0000u;
    first[i] = __builtin_bit_cast(__bf16, (uint16_t)(top >> 16));
    rest[i] = (__bf16)fmaf(x[i], 1.f + 0x1p-23f, -__uint_as_float(top));
  }
}
__device__ __forceinline__ void split(const float (&x)[8], f16x8& first, f16x8& rest) {
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    const auto top = __builtin_amdgcn_cvt_pkrtz(x[i], x[i + 1]);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const float t = (float)top[k];
      first[i + k] = (_Float16)t;
      rest[i + k] = (_Float16)fmaxf(x[i + k] - t, fminf(t, 0x1p-24f));
    }
  }
}

// (a lane's value, those of the lanes 16, 32 and 48 further) -> the largest / the sum, in all four
__device__ __forceinline__ float groups_max(float v) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float groups_sum(float v) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Whether any of the eight halves of v is an infinity or not a number: exponent bits all ones, found by one carry
template <typename T>
__device__ __forceinline__ uint32_t odd_bits(uint32_t u) {
  constexpr uint32_t m = sizeof(T) == 2 && __is_same(T, __bf16) ? 0x7F807F80u : 0x7C007C00u, one = __is_same(T, __bf16) ? 0x00800080u : 0x04000400u;
  return ((u & m) + one) & 0x80008000u;
}

// Keeps of a pair of values what `keep` says but infinities and NaNs; not 0: there was one
template <typename T>
__device__ __forceinline__ uint32_t clear_odd(uint32_t& v, uint32_t keep) {
  v &= keep;
  const uint32_t e = odd_bits<T>(v);
  v &= ~((e >> 15) * 0xFFFFu);
  return e;
}
// What a pair of values is: 1 for +infinity, 64 for -infinity, 4096 for NaN, as numbers of the type.  Summed over the keys that a
// column sees (32 at most, so the three counts stay apart) they say what belongs in its sum.
template <typename T>
__device__ __forceinline__ uint32_t odd_kinds(uint32_t v) {
  constexpr bool b = __is_same(T, __bf16);
  constexpr uint32_t inf = b ? 0x7F80u : 0x7C00u, one = b ? 0x3F80u : 0x3C00u, k64 = b ? 0x4280u : 0x5400u, k4096 = b ? 0x4580u : 0x6C00u;
  uint32_t kinds = 0;
#pragma unroll
  for (int h = 0; h < 32; h += 16) {
    const uint32_t x = (v >> h) & 0xFFFFu, m = x & 0x7FFFu;
    kinds |= (m < inf ? 0u : m > inf ? k4096 : x > m ? k64 : one) << h;
  }
  return kinds;
}
// a pair of bfloat16s, those past the largest number of type T as infinities (a bfloat16 past its own is one; 65536 is the next number of 4 bits behind
// 65504)
template <typename T>
__device__ __forceinline__ uint32_t infinite_past(uint32_t v) {
  if constexpr (__is_same(T, __bf16)) return v;
  uint32_t out = 0;
#pragma unroll
  for (int h = 0; h < 32; h += 16) {
    const uint32_t x = (v >> h) & 0xFFFFu, m = x & 0x7FFFu;
    out |= (m >= 0x4780u && m <= 0x7F80u ? 0x7F80u | (x ^ m) : x) << h;
  }
  return out;
}
__device__ __forceinline__ float odd_value(float n) {
  const int c = (int)n;
  return (c & 63 ? INFINITY : 0.f) + (c & (63 << 6) ? -INFINITY : 0.f) + (c >> 12 ? __uint_as_float(0x7FC00000u) : 0.f);
}

// ---- which piece of the work a work-group takes -------------------------------------------------------------------
// The lengths are on the device, so the split is made there, by every wave for itself (64 sequences at a time, a lane each; no
// memory but the counts): a tile's keys are cut into pieces of `per` units so that all pieces together are about `slots`, the
// work-groups that run at once.  Then one long sequence among short ones is spread over the chip, and a batch that fills it is not
// split at all.  Work-group i takes key head i % n_kv_heads (neighbouring work-groups go to different XCDs: with 8 key heads and
// more a head's work-groups share an L2).
struct Span {
  int min_cols, max_cols;     // sequences with so many columns (rows times heads a key head has)
  int tile_cols, unit;        // columns of a tile, keys of a unit
  int slots;
  int min_units, whole;       // of a piece; tiles that are not cut (find_piece)
  int first_block;            // the launch's work-groups from here on
  int start;                  // units that a piece's start and join are worth (where they are weighed)
  int tickets;                // its first in the workspace
  int64_t partials;           // bytes in front of its partial results there
};
constexpr int kMaxPieces = 32;        // of a tile: whoever joins them reads them all
struct Piece {
  int seq, row0, rows, len;   // rows of the sequence, its length (not cut to the table)
  int group, piece, pieces;   // tile of the sequence, piece of the tile
  int u0, u1;                 // its units
  int first;                  // number of the tile's first piece among the pieces of split tiles
  int kvh;
};
struct SeqWork { int row0, rows, len, groups, units; };
__device__ __forceinline__ SeqWork seq_work(const stairs_paged_cache& c, const stairs_paged_attn& a, const Span& sp, int b) {
  SeqWork w{0, 0, 0, 0, 0};
  if (b < a.n_seqs) {
    w.row0 = a.row_start[b];
    w.rows = a.row_start[b + 1] - w.row0;
    w.len = a.seq_len[b];
    const long long cols = (long long)w.rows * (a.n_heads / c.n_kv_heads);
    if (w.row0 >= 0 && w.rows > 0 && w.rows <= a.rows - w.row0 && cols >= sp.min_cols && cols <= sp.max_cols) {
      w.groups = (int)((cols + sp.tile_cols - 1) / sp.tile_cols);
      w.units = (min(max(w.len, 0), a.max_blocks * c.page_size) + sp.unit - 1) / sp.unit;
    }
  }
  return w;
}
template <typename T>
__device__ __forceinline__ T wave_scan(T v) {                  // inclusive
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const T o = __shfl_up(v, off);
    if (lane >= off) v += o;
  }
  return v;
}
__device__ __forceinline__ int quotient(long long a, int b) {    // a >= 0, b > 0 (a division of 64 bits is over a hundred instructions)
  return (a >> 32) == 0 ? (int)((unsigned)a / (unsigned)b) : (int)min(a / b, (long long)INT32_MAX);
}
template <bool WEIGH>
__device__ __forceinline__ bool find_piece(const stairs_paged_cache& c, const stairs_paged_attn& a, const Span& sp, Piece& out) {
  const int lane = threadIdx.x & 63;
  const int block = blockIdx.x - sp.first_block, kvh = block % c.n_kv_heads, item = block / c.n_kv_heads;
  long long units = 0;
  int tiles = 0, most = 0;
  SeqWork w;
  for (int b0 = 0; b0 < a.n_seqs; b0 += 64) {
    w = seq_work(c, a, sp, b0 + lane);
    units += (long long)w.groups * w.units;
    tiles += w.groups;
    most = max(most, w.units);
  }
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) {
    units += __shfl_xor(units, off);
    tiles += __shfl_xor(tiles, off);
    most = max(most, __shfl_xor(most, off));
  }
  units *= c.n_kv_heads;
  const long long all_tiles = (long long)tiles * c.n_kv_heads;
  int per;
  if (all_tiles >= sp.whole && units * 4 >= all_tiles * most * 3) {
    // Tiles of about one length for nearly every CU stay whole: half as many streams, and nothing to join (32 sequences of 2048
    // keys, 8 heads: 46 us whole, 58 in halves; of 8192 keys 162 and 189).
    per = max(1, most);
  } else {
    // Pieces of one size, for which they all run at once: a second round, however short, costs a whole piece's latencies (32
    // verifications of 200 .. 8000 keys: 79 us with 612 pieces, 66 with 490).  With more tiles than run at once anyway, or more
    // sequences than lanes, the even share.
    per = max(sp.min_units, quotient(units + sp.slots - 1, sp.slots));
    if (a.n_seqs <= 64 && per > sp.min_units && per < most) {
      const float fit = (float)(sp.slots / c.n_kv_heads);
      int lo = per, hi = 4 * per;                               // (up to 4 shares: beyond that one round is no aim any more)
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        const float pieces = fmaxf(1.f, floorf(((float)(w.units + mid) - 0.5f) * __builtin_amdgcn_rcpf((float)mid)));
        if (__builtin_amdgcn_readfirstlane(__float_as_int(wave_sum((float)w.groups * pieces) - fit)) <= 0) hi = mid;
        else lo = mid + 1;
      }
      if constexpr (WEIGH) {
        // ... or more than run at once: what all pieces take, their starts and joins (of so many units each) with them, and half a piece, for
        // which CUs stand half empty at the end.  (Trees of 61 rows of 32 sequences of 500 .. 6000 keys, 32 heads on 8 of 128, 8-bit pages: one round means
        // whole tiles of up to 94 units, 188 us; 153 .. 145 so, for 4 .. 32 units; trees of 25 rows of 16 sequences 70 with 4, 59 with 8 .. 32.)
        auto cost = [&](int n) {
          const float pieces = fmaxf(1.f, floorf(((float)(w.units + n) - 0.5f) * __builtin_amdgcn_rcpf((float)n)));
          return wave_sum((float)w.groups * pieces) * (float)(c.n_kv_heads * sp.start) * __builtin_amdgcn_rcpf((float)sp.slots) + 0.5f * (float)n;
        };
        float least = cost(lo);
        int best = lo;
#pragma unroll 1
        for (int k = 4; k < 12; ++k) {
          const int n = per * k / 4;
          if (n >= lo) break;
          const float x = cost(n);
          if (x < least) {
            least = x;
            best = n;
          }
        }
        per = best;
      } else if (lo < 4 * per) {
        per = lo;
      }
    }
  }
  per = __builtin_amdgcn_readfirstlane(per);
  auto pieces_of = [&](const SeqWork& q) { return min(kMaxPieces, max(1, (int)((unsigned)(q.units + per - 1) / (unsigned)per))); };
  int seq = lane;
  if (WEIGH && a.n_seqs <= 64 && all_tiles * 2 > sp.slots) {
    // Large pieces first (what starts last is short then): the sequences in the order of their pieces' sizes, one behind the other where
    // they are alike (those trees of 61 rows 145 -> 127 us).
    const int size = w.groups > 0 ? (int)((unsigned)w.units / (unsigned)pieces_of(w)) : -1;
    int rank = 0;
    for (int k = 0; k < a.n_seqs; ++k) {
      const int other = __builtin_amdgcn_readlane(size, k);
      rank += other > size || (other == size && k < lane);
    }
    if (lane >= a.n_seqs) rank = lane;
    auto go = [&](int& v) { v = __builtin_amdgcn_ds_permute(rank * 4, v); };
    go(w.row0); go(w.rows); go(w.len); go(w.groups); go(w.units); go(seq);
  }
  int before = 0, split_before = 0;
  for (int b0 = 0; b0 < a.n_seqs; b0 += 64) {
    if (a.n_seqs > 64) w = seq_work(c, a, sp, b0 + lane);
    const int pieces = pieces_of(w);
    const int mine = w.groups * pieces, split = pieces > 1 ? mine : 0;
    const int to = before + wave_scan(mine), split_to = split_before + wave_scan(split);
    const unsigned long long there = __ballot(to > item);
    if (there) {
      const int l = __builtin_ctzll(there);
      const unsigned at = item - (__builtin_amdgcn_readlane(to, l) - __builtin_amdgcn_readlane(mine, l));
      const unsigned n = __builtin_amdgcn_readlane(pieces, l), group = at / n;
      const int u = __builtin_amdgcn_readlane(w.units, l);
      out.seq = b0 + __builtin_amdgcn_readlane(seq, l);
      out.row0 = __builtin_amdgcn_readlane(w.row0, l);
      out.rows = __builtin_amdgcn_readlane(w.rows, l);
      out.len = __builtin_amdgcn_readlane(w.len, l);
      out.pieces = n;
      out.group = __builtin_amdgcn_readlane(w.groups, l) - 1 - __builtin_amdgcn_readfirstlane(group);   // (the last rows see most: first)
      out.piece = __builtin_amdgcn_readfirstlane(at - group * n);
      out.u0 = __builtin_amdgcn_readfirstlane((unsigned)u * out.piece / n);        // (26 bits of units, 5 of pieces)
      out.u1 = __builtin_amdgcn_readfirstlane((unsigned)u * (out.piece + 1) / n);
      out.first = (__builtin_amdgcn_readlane(split_to, l) - __builtin_amdgcn_readlane(split, l) + (int)at - out.piece) * c.n_kv_heads + kvh;
      out.kvh = kvh;
      return true;
    }
    before = __builtin_amdgcn_readlane(to, 63);
    split_before = __builtin_amdgcn_readlane(split_to, 63);
  }
  return false;
}
// a split tile's pieces are numbered first + piece * n_kv_heads; all of them together are at most this many: a split
// sequence has more units than `per`, so fewer than 2 units / per pieces
__host__ __device__ constexpr int most_pieces(int slots) { return 2 * slots; }

// ---- joining ------------------------------------------------------------------------------------------------------------
// Partial results of a piece: [tile_cols][HD] outputs relative to the column's maximum, then [tile_cols] (maximum, sum) pairs.  The
// workspace begins with all tickets, chunks' and rows', whichever of them a call needs: calls of other head sizes, head counts and
// rows may follow in the same workspace, and none finds partial results where its tickets are.
__device__ __forceinline__ int* tickets(const stairs_paged_attn& a, const Span& sp) { return static_cast<int*>(a.workspace) + sp.tickets; }
__device__ __forceinline__ float* partials(const stairs_paged_attn& a, const Span& sp) { return reinterpret_cast<float*>(static_cast<char*>(a.workspace) + sp.partials); }
template <int HD>
__host__ __device__ constexpr size_t piece_floats(int tile_cols) { return (size_t)tile_cols * (HD + 2); }

template <typename T, int HD>
__device__ __forceinline__ void store_out(const stairs_paged_cache& c, const stairs_paged_attn& a, const Piece& w, int col, int e, float4 v, float l) {
  const int G = a.n_heads / c.n_kv_heads, r = col / G;
  const float f = l == 0.f ? 0.f : 1.f / l;                      // (0: the row has seen nothing)
  T out[4] = {Elem<T>::down(v.x * f), Elem<T>::down(v.y * f), Elem<T>::down(v.z * f), Elem<T>::down(v.w * f)};
  *reinterpret_cast<uint2*>(static_cast<T*>(a.out) + (size_t)(w.row0 + r) * a.out_stride + (w.kvh * G + col - r * G) * HD + e) =
      *reinterpret_cast<const uint2*>(out);
}
__device__ __forceinline__ float weight_of(float m, float all) { return m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - all); }

// 16 bytes past the caches that XCDs do not share (what ld_dev and st_dev do for 4 and 8)
__device__ __forceinline__ float4 ld_dev4(const float* base, int offset) {
  const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(base), 0, 0xFFFFFFFFu, 0x00027000);
  return __builtin_bit_cast(float4, __builtin_amdgcn_raw_buffer_load_b128(r, offset * 4, 0, 16));
}
__device__ __forceinline__ void st_dev4(float* base, int offset, float4 v) {
  const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(base, 0, 0xFFFFFFFFu, 0x00027000);
  __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), r, offset * 4, 0, 16);
}
// The last of a split tile's work-groups joins its pieces, in their order whoever it is.  All maxima and sums are requested at once,
// then sixteen outputs a thread (one after the other, each a round trip past the caches, the maxima and sums alone of 32
// pieces were 30 us); the code is kept short, it runs once and comes from memory (unrolled over everything: 5 us more).
template <typename T, int HD, int COLS>
__device__ __forceinline__ void join_pieces(const stairs_paged_cache& c, const stairs_paged_attn& a, const Span& sp, const Piece& w, float2* s_ml, int* s_last) {
  int* counter = tickets(a, sp) + w.first;
  if (!last_arrival(counter, w.pieces, s_last)) return;
  constexpr int NT = 256, TB = COLS <= 32 ? 1 : 4, PB = 16 / TB;
  const size_t step = piece_floats<HD>(COLS) * c.n_kv_heads;
  float* base = partials(a, sp) + (size_t)w.first * piece_floats<HD>(COLS);
  const int G = a.n_heads / c.n_kv_heads, col0 = w.group * COLS, cols = min(COLS, w.rows * G - col0);
  constexpr int MLS = (kMaxPieces * COLS + NT - 1) / NT;
  float2 ml[MLS];
#pragma unroll
  for (int k = 0; k < MLS; ++k) ml[k] = ld_dev2(base + min((int)(threadIdx.x + k * NT) / COLS, w.pieces - 1) * step + COLS * HD + threadIdx.x % COLS * 2);
  float mine = -INFINITY;
#pragma unroll
  for (int k = 0; k < MLS; ++k) mine = fmaxf(mine, ml[k].x);
  float* s_max = reinterpret_cast<float*>(s_ml + kMaxPieces * COLS);
  s_max[threadIdx.x] = mine;
  __syncthreads();
  float all = -INFINITY;
#pragma unroll
  for (int k = 0; k < NT / COLS; ++k) all = fmaxf(all, s_max[threadIdx.x % COLS + k * COLS]);
#pragma unroll
  for (int k = 0; k < MLS; ++k) {
    const float f = (int)(threadIdx.x + k * NT) / COLS < w.pieces ? weight_of(ml[k].x, all) : 0.f;
    s_ml[threadIdx.x + k * NT] = make_float2(f, f * ml[k].y);
  }
  __syncthreads();
#pragma unroll 1
  for (int t0 = 0; t0 * NT < cols * (HD / 4); t0 += TB) {
    float4 v[TB];
    float l[TB];
#pragma unroll
    for (int t = 0; t < TB; ++t) {
      v[t] = make_float4(0.f, 0.f, 0.f, 0.f);
      l[t] = 0.f;
    }
#pragma unroll 1
    for (int p0 = 0; p0 < w.pieces; p0 += PB) {
      float4 x[PB][TB];
#pragma unroll
      for (int k = 0; k < PB; ++k)
#pragma unroll
        for (int t = 0; t < TB; ++t) x[k][t] = ld_dev4(base + min(p0 + k, w.pieces - 1) * step, (threadIdx.x + (t0 + t) * NT) * 4);
      __builtin_amdgcn_sched_barrier(0);                        // (all of them on their way before the first is waited for)
#pragma unroll
      for (int k = 0; k < PB; ++k) {
        const bool there = p0 + k < w.pieces;                   // (behind the last piece: the last one again, for nothing)
#pragma unroll
        for (int t = 0; t < TB; ++t) {
          const float2 f = s_ml[(p0 + k) * COLS + (threadIdx.x + (t0 + t) * NT) / (HD / 4)];
          l[t] += f.y;
          v[t].x += there ? f.x * x[k][t].x : 0.f;
          v[t].y += there ? f.x * x[k][t].y : 0.f;
          v[t].z += there ? f.x * x[k][t].z : 0.f;
          v[t].w += there ? f.x * x[k][t].w : 0.f;
        }
      }
    }
#pragma unroll
    for (int t = 0; t < TB; ++t) {
      const int i = threadIdx.x + (t0 + t) * NT;
      if (i < cols * (HD / 4)) store_out<T, HD>(c, a, w, col0 + i / (HD / 4), i % (HD / 4) * 4, v[t], l[t]);
    }
  }
  if (threadIdx.x == 0) *counter = 0;
}

// the four waves' results of a piece -> the output, or a partial result
template <typename T, int HD, int COLS>
__device__ __forceinline__ void join_waves(const stairs_paged_cache& c, const stairs_paged_attn& a, const Span& sp, const Piece& w,
                                           float (*s_o)[COLS][HD + 4], float (*s_m)[COLS], float (*s_l)[COLS], int* s_last) {
  static_assert(4 * COLS * (HD + 4) >= 2 * kMaxPieces * COLS + 256, "the pieces' maxima and sums fit where the waves' outputs were");
  const int G = a.n_heads / c.n_kv_heads, col0 = w.group * COLS, cols = min(COLS, w.rows * G - col0);
  float* part = partials(a, sp) +
                (size_t)(w.first + w.piece * c.n_kv_heads) * piece_floats<HD>(COLS);
  for (int i = threadIdx.x; i < cols * (HD / 4); i += 256) {
    const int col = i / (HD / 4), e = i % (HD / 4) * 4;
    float m = s_m[0][col];
#pragma unroll
    for (int k = 1; k < 4; ++k) m = fmaxf(m, s_m[k][col]);
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    float l = 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float f = weight_of(s_m[k][col], m);
      const float4 x = *reinterpret_cast<const float4*>(&s_o[k][col][e]);
      l += f * s_l[k][col];
      v.x += f * x.x;
      v.y += f * x.y;
      v.z += f * x.z;
      v.w += f * x.w;
    }
    if (w.pieces == 1) {
      store_out<T, HD>(c, a, w, col0 + col, e, v, l);
    } else {
      st_dev4(part, col * HD + e, v);
      if (e == 0) st_dev2(part + COLS * HD + col * 2, m, l);
    }
  }
  if (w.pieces > 1) join_pieces<T, HD, COLS>(c, a, sp, w, reinterpret_cast<float2*>(s_o), s_last);
}

// ---- what a column sees -------------------------------------------------------------------------------------------
// Kernels come in forms: keys and values of the cache's type and rows that see the positions up to their own (0); with what a column sees as a count
// of keys in front and 64 bits for those behind them (kMasks: trees, and as bits or as a count every other row); over 8-bit pages (kHeld8, masks always:
// they are looked at only in a sequence's last keys).
constexpr int kMasks = 1, kHeld8 = 2;
struct Sees {
  int open;                   // keys in front of this one
  unsigned long long bits;    // and of the 64 from it on
};
__device__ __forceinline__ bool is_tree(const stairs_paged_attn& a, const Piece& w) { return a.sees && w.rows <= STAIRS_TREE_MAX_ROWS; }
__device__ __forceinline__ Sees sees_of(const stairs_paged_attn& a, const Piece& w, int row, int limit) {
  const int pos0 = w.len - w.rows;
  if (!is_tree(a, w)) return {max(min(pos0 + row, limit - 1) + 1, 0), 0};
  unsigned long long bits = a.sees[w.row0 + row] & (~0ull >> (64 - w.rows));
  if (pos0 < 0) bits = pos0 > -64 ? bits >> -pos0 : 0;           // (rows in front of position 0 are nowhere)
  return {max(min(pos0, limit), 0), bits};
}
__device__ __forceinline__ uint32_t block_of(const Sees& s, int key0) {   // the 32 keys from key0 on
  const int d = key0 - s.open;
  if (d <= -32) return ~0u;
  if (d < 0) return (~0u >> (32 + d)) | (uint32_t)(s.bits << -d);
  return d < 64 ? (uint32_t)(s.bits >> d) : 0u;
}

// ---- few columns: a wave per 32 keys ----------------------------------------------------------------------------------
// Bound by the bytes of the cache.  A work-group takes a piece of a tile of 16 CT columns; its four waves take 32-key blocks in
// turn, straight from memory into the matrix operands (a block of a head is 2 x 64 HD contiguous bytes, every load 1 KiB of a
// wave), no LDS, and are joined at the end.  Values are requested before the scores they wait for, the next block's keys as
// soon as this block's are used.  (3 sequences of 9 rows and 23456 .. 59999 positions, 32 heads of 128: 300 us = 6.6 TB/s; 32 of 5 rows and
// 200 .. 8000 positions, 8 key heads: 66.6 us = 4.3 TB/s, the rest goes into starting and joining pieces; 300 positions alone 6.6 us, one sequence of
// 8000 and 8 key heads 13 us with 1 row, 19 with 5.)  Over 8-bit pages the codes become numbers of the matrix unit's type in registers, two an
// instruction: the same 3 sequences 161 us = 6.2 TB/s, 32 single tokens of 200 .. 8000 positions 32, of which 20 for the bytes (pieces by weight as
// in chunks, or three and four waves a SIMD with as many pieces, were slower: 201 us, 166 .. 284).
constexpr int kRowUnit = 32 * 4;
template <int HD, int CT>
struct RowsLds {
  float o[4][16 * CT][HD + 4], m[4][16 * CT], l[4][16 * CT];
  int last;
};
template <typename T, int HD, int CT, int F>
__device__ __forceinline__ void attend_rows(const stairs_paged_cache& c, const stairs_paged_attn& a, const Span& sp, float scale2, RowsLds<HD, CT>& lds) {
  constexpr bool H8 = F & kHeld8, M = F & kMasks;
  typedef typename Elem<T>::x8 x8;
  // Codes are numbers of either type.  A score is multiplied by its key's power of two, a probability by its value's: in bfloat16, so that whatever
  // power of two that is stays in range; two numbers of it are as exact as half's two.  (But for values of less than 2^-112: times their power
  // the probabilities are then below the normal bfloat16s and lose bits, to 0.3 % of the largest at 2^-116.)
  typedef std::conditional_t<H8, __bf16, T> VT;
  typedef typename Elem<VT>::x8 vx8;
  typedef std::conditional_t<H8, uint8_t, T> PT;
  constexpr int KK = HD / 32, ET = HD / 16, NK = H8 ? KK : 2 * KK, NV = H8 ? ET / 2 : ET;
  Piece w;
  if (!find_piece<false>(c, a, sp, w)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), j = lane & 15, g = lane >> 4;
  const int G = a.n_heads / c.n_kv_heads, cols = w.rows * G, col0 = w.group * 16 * CT;
  const int limit = a.max_blocks * c.page_size;
  const int pos0 = w.len - w.rows;                              // position of the sequence's first row
  const bool tree = M && is_tree(a, w);
  // last position that all of the tile's columns see, that any does
  const int first_last = tree ? min(pos0, limit) - 1 : min(pos0 + col0 / G, limit - 1);
  const int last_last = tree ? min(w.len, limit) - 1 : min(pos0 + (min(cols, col0 + 16 * CT) - 1) / G, limit - 1);
  int last[CT];
  Sees sees[CT];
  x8 q[CT][KK];
  bool had_odd = false;                                         // the wave has left infinities or NaNs in its part of lds.o
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    const int col = col0 + ct * 16 + j;
    last[ct] = -1;
    sees[ct] = {0, 0};
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) q[ct][kk] = x8{};
    if (col < cols) {
      const int r = col / G;
      last[ct] = min(pos0 + r, limit - 1);
      if constexpr (M) sees[ct] = sees_of(a, w, r, limit);
      const T* qp = static_cast<const T*>(a.q) + (size_t)(w.row0 + r) * a.q_stride + (w.kvh * G + col - r * G) * HD + g * 8;
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) q[ct][kk] = *reinterpret_cast<const x8*>(qp + kk * 32);
    }
  }
  f32x4 o[CT][ET];
  float m[CT], l[CT];
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    m[ct] = -INFINITY;
    l[ct] = 0.f;
#pragma unroll
    for (int et = 0; et < ET; ++et) o[ct][et] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const size_t head_elems = (size_t)c.page_size * HD, page_elems = head_elems * c.n_kv_heads;
  const PT* K = static_cast<const PT*>(c.k) + w.kvh * head_elems;
  const PT* V = static_cast<const PT*>(c.v) + w.kvh * head_elems;
  constexpr int PER = 16 / sizeof(PT);                          // elements of a load
  const uint8_t* S = H8 ? static_cast<const uint8_t*>(c.scale) + w.kvh * (size_t)c.page_size * 2 : nullptr;
  const int* table = a.block_table + (size_t)w.seq * a.max_blocks;
  const int ps_shift = __builtin_ctz(c.page_size);

  // the wave's blocks: unit u's block is keys 128 u + 32 wave ..; page numbers 64 units at a time, a lane each
  int pages = -1, pages_at = w.u0;
  const int u1 = min(w.u1, last_last < 0 ? 0 : (last_last - 32 * wave) / kRowUnit + (last_last >= 32 * wave));
  auto fetch_pages = [&](int u) {
    pages_at = u;
    const unsigned key = (unsigned)(u + lane) * kRowUnit + wave * 32;
    pages = u + lane < u1 ? table[key >> ps_shift] : -1;
    if ((unsigned)pages >= (unsigned)c.n_pages) pages = -1;
  };
  auto next_block = [&](int u) {                                // the first unit from u on that has a page
    for (;;) {
      if (u >= u1) return u1;
      if (u >= pages_at + 64) fetch_pages(u);
      const unsigned long long there = __ballot(pages >= 0) & (~0ull << (u - pages_at));
      if (there) return pages_at + (int)__builtin_ctzll(there);
      u = pages_at + 64;
    }
  };
  uint4 kf[NK], vf[NV], scales{};                               // (scales: of the lane's eight keys, then of their values)
  auto block_at = [&](int u) -> size_t {                        // elements in front of the block in its pool
    const int key = u * kRowUnit + wave * 32;
    return (size_t)__builtin_amdgcn_readlane(pages, u - pages_at) * page_elems + (size_t)(key & (c.page_size - 1)) * HD;
  };
  auto load_keys = [&](size_t at) {
#pragma unroll
    for (int i = 0; i < NK; ++i) kf[i] = ld_once_as<uint4>(K + at + (i * 64 + lane) * PER);
    if constexpr (H8) scales = *reinterpret_cast<const uint4*>(S + at / (HD / 2) + g * 16);
  };
  if (w.u0 < u1) fetch_pages(w.u0);
  int u = next_block(w.u0);
  size_t at = 0;
  if (u < u1) {
    at = block_at(u);
    load_keys(at);
  }
  while (u < u1) {
#pragma unroll
    for (int i = 0; i < NV; ++i) vf[i] = ld_once_as<uint4>(V + at + (i * 64 + lane) * PER);
    f32x4 s[CT][2];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        s[ct][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
          uint4 k;
          if constexpr (H8) {
            const uint4 codes = kf[t * (KK / 2) + kk / 2];
            k = kk & 1 ? widen<T>(codes.z, codes.w, 1.f) : widen<T>(codes.x, codes.y, 1.f);
          } else {
            k = kf[t * KK + kk];
          }
          s[ct][t] = mma(__builtin_bit_cast(x8, k), q[ct][kk], s[ct][t]);
        }
      }
    const int key0 = u * kRowUnit + wave * 32;
    const int un = next_block(u + 1);
    const size_t at_here = at;
    uint4 powers = scales;
    if (un < u1) {
      at = block_at(un);
      load_keys(at);
    }
    bool past = false;
    if constexpr (H8) {
      // Powers of two with which a code may be past the type's largest number (of rows that others have stored, or of the largest bfloat16s): such
      // numbers are infinite, as they are in attend_chunk, where numbers of the type are what is multiplied: scores by this, values as odd_values.  Looking for
      // them costs 0 .. 1 % (32 verifications of 8 rows 43.4 us, 42.7 without).  Of keys that a column sees:
      const uint32_t far[2] = {bytes_past<T>(powers.x), bytes_past<T>(powers.y)};
      if (__any((far[0] | far[1] | bytes_past<T>(powers.z) | bytes_past<T>(powers.w)) != 0)) {
        auto seen = [&](int i) {
          const int n = last_last - (key0 + i * 16 + g * 4) + 1;
          return n >= 4 ? ~0u : n <= 0 ? 0u : (1u << (8 * n)) - 1;
        };
        past = __any((((far[0] | bytes_past<T>(powers.z)) & seen(0)) | ((far[1] | bytes_past<T>(powers.w)) & seen(1))) != 0);
        if (past) {
          // scores again, such keys as numbers of the type in the product and their scores multiplied by 1
          auto one = [](uint32_t u, uint32_t bits) { return (u & ~((bits >> 7) * 255u)) | (bits >> 7) * 127u; };
          powers.x = one(powers.x, far[0]);
          powers.y = one(powers.y, far[1]);
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            const uint32_t b = S[at_here / (HD / 2) + scale_off(t * 16 + j)];
            const float f = b > kMostByte<T> ? __uint_as_float(b << 23) : 1.f;
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) s[ct][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) {
              const uint2 codes = *reinterpret_cast<const uint2*>(K + at_here + ((t * (KK / 2) + kk / 2) * 64 + lane) * PER + kk % 2 * 8);
              const x8 k = __builtin_bit_cast(x8, widen<T>(codes.x, codes.y, f));
#pragma unroll
              for (int ct = 0; ct < CT; ++ct) s[ct][t] = mma(k, q[ct][kk], s[ct][t]);
              __builtin_amdgcn_sched_barrier(0);
            }
          }
        }
      }
    }
    float ks[8], vs[8];
    if constexpr (H8) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        ks[i] = scale_of(i < 4 ? powers.x : powers.y, i & 3) * scale2;
        vs[i] = scale_of(i < 4 ? powers.z : powers.w, i & 3);
      }
    }
    const bool full = key0 + 31 <= first_last && !past;
    vx8 p[CT], rest[CT];
    uint32_t seen_bits[CT];                                     // of the lane's keys: (i >> 2) * 16 + (i & 3) for the i-th
    if constexpr (M)
      if (!full) {
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) seen_bits[ct] = block_of(sees[ct], key0) >> (g * 4);
      }
    auto sees_key = [&](int ct, int i) {
      if constexpr (M) return (seen_bits[ct] >> ((i >> 2) * 16 + (i & 3)) & 1) != 0;
      else return key0 + (i >> 2) * 16 + g * 4 + (i & 3) <= last[ct];
    };
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = s[ct][i >> 2][i & 3] * (H8 ? ks[i] : scale2);
      if (!full) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = sees_key(ct, i) ? x[i] : -INFINITY;
      }
      float mx = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
      if (__any(mx - m[ct] > (past ? 0.f : Headroom<VT>::slack))) {   // (the difference is exact where the scores are far
                                                                // from 0; past: probabilities times 2^127 are floats)
        const float mn = fmaxf(m[ct], groups_max(mx));
        const float f = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[ct] - mn);
        m[ct] = mn;
        l[ct] *= f;
#pragma unroll
        for (int et = 0; et < ET; ++et) o[ct][et] *= f;
      }
      const float mr = m[ct] == -INFINITY ? 0.f : m[ct];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] = __builtin_amdgcn_exp2f(x[i] - mr + Headroom<VT>::lift);
        l[ct] += x[i];
        if constexpr (H8) x[i] = full || x[i] != 0.f ? x[i] * vs[i] : 0.f;   // (a power of two that nobody stored may be anything)
      }
      split(x, p[ct], rest[ct]);
    }
    auto value = [&](int et) {
      if constexpr (H8) return et & 1 ? widen<VT>(vf[et / 2].z, vf[et / 2].w, 1.f) : widen<VT>(vf[et / 2].x, vf[et / 2].y, 1.f);
      else return vf[et];
    };
    auto add_value = [&](int et, uint4 v) {
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        o[ct][et] = mma(__builtin_bit_cast(vx8, v), rest[ct], o[ct][et]);
        o[ct][et] = mma(__builtin_bit_cast(vx8, v), p[ct], o[ct][et]);
      }
    };
    if (!full) {
      // Some keys of the block are not seen by all columns.  Their probability is 0, and 0 times what is there must be 0: what
      // no column sees is cleared, and so are infinities and NaNs; those that some columns see are looked at again (odd_values).
      uint32_t keep[4], odd = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int key = key0 + (i >> 1) * 16 + g * 4 + (i & 1) * 2;
        keep[i] = (key <= last_last ? 0xFFFFu : 0u) | (key + 1 <= last_last ? 0xFFFF0000u : 0u);
      }
#pragma unroll
      for (int et = 0; et < ET; ++et) {
        uint4 held = value(et);
        uint4& v = H8 ? held : vf[H8 ? 0 : et];
        odd |= clear_odd<VT>(v.x, keep[0]);
        odd |= clear_odd<VT>(v.y, keep[1]);
        odd |= clear_odd<VT>(v.z, keep[2]);
        odd |= clear_odd<VT>(v.w, keep[3]);
        if constexpr (H8) add_value(et, v);
        __builtin_amdgcn_sched_barrier(0);                      // (one tile after the other: their temporaries share registers)
      }
      if (past || __any(odd != 0)) {
        if (!had_odd)
          for (int i = lane; i < 16 * CT * (HD + 4); i += 64) (&lds.o[wave][0][0])[i] = 0.f;
        had_odd = true;
        vx8 seen[CT];
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
          for (int i = 0; i < 8; ++i) seen[ct][i] = sees_key(ct, i) ? (VT)1.f : (VT)0.f;
#pragma unroll 1
        for (int et = 0; et < ET; ++et) {
          uint4 v = *reinterpret_cast<const uint4*>(V + at_here + ((H8 ? et / 2 : et) * 64 + lane) * PER);
          if constexpr (H8) {
            const uint2 b = *reinterpret_cast<const uint2*>(S + at_here / (HD / 2) + g * 16 + 8), codes = et & 1 ? make_uint2(v.z, v.w) : make_uint2(v.x, v.y);
            auto pair = [&](uint32_t lo, uint32_t hi) {
              __builtin_amdgcn_sched_barrier(0);
              return infinite_past<T>(low_high(lo, hi));
            };
            typedef Wide<VT> W;
            v.x = pair(W::template pair<false>(codes.x, scale_of(b.x, 0)), W::template pair<false>(codes.x, scale_of(b.x, 1)));
            v.y = pair(W::template pair<true>(codes.x, scale_of(b.x, 2)), W::template pair<true>(codes.x, scale_of(b.x, 3)));
            v.z = pair(W::template pair<false>(codes.y, scale_of(b.y, 0)), W::template pair<false>(codes.y, scale_of(b.y, 1)));
            v.w = pair(W::template pair<true>(codes.y, scale_of(b.y, 2)), W::template pair<true>(codes.y, scale_of(b.y, 3)));
          }
          v.x &= keep[0]; v.y &= keep[1]; v.z &= keep[2]; v.w &= keep[3];
          const uint4 kinds = make_uint4(odd_kinds<VT>(v.x), odd_kinds<VT>(v.y), odd_kinds<VT>(v.z), odd_kinds<VT>(v.w));
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) {
            const f32x4 count = mma(__builtin_bit_cast(vx8, kinds), seen[ct], f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
            for (int i = 0; i < 4; ++i) lds.o[wave][ct * 16 + j][et * 16 + g * 4 + i] += odd_value(count[i]);
          }
        }
      }
    }
    if (!H8 || full) {
#pragma unroll
      for (int et = 0; et < ET; ++et) add_value(et, value(et));
    }
    u = un;
  }

  // the four waves: maximum, sum and outputs as they are; whoever adds them scales them
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    const float sum = groups_sum(l[ct]);
    if (g == 0) {
      lds.m[wave][ct * 16 + j] = m[ct];
      lds.l[wave][ct * 16 + j] = sum;
    }
#pragma unroll
    for (int et = 0; et < ET; ++et) {
      float4* dst = reinterpret_cast<float4*>(&lds.o[wave][ct * 16 + j][et * 16 + g * 4]);
      float4 v = make_float4(o[ct][et][0], o[ct][et][1], o[ct][et][2], o[ct][et][3]);
      if (had_odd) {
        const float4 x = *dst;
        v = make_float4(v.x + x.x, v.y + x.y, v.z + x.z, v.w + x.w);
      }
      *dst = v;
    }
  }
  __syncthreads();
  join_waves<T, HD, 16 * CT>(c, a, sp, w, lds.o, lds.m, lds.l, &lds.last);
}
template <typename T, int HD, int CT, int F>
__global__ __launch_bounds__(256, 2) void k_paged_rows(stairs_paged_cache c, stairs_paged_attn a, Span sp, float scale2) {
  __shared__ RowsLds<HD, CT> lds;
  attend_rows<T, HD, CT, F>(c, a, sp, scale2, lds);
}

// ---- many columns: tiles of 128 columns, keys and values shared through LDS ------------------------------------------
// Bound by the matrix units and by the exponentials beside them.  A wave has 32 columns, the work-group's four waves read 64
// keys at a time, copied to LDS while the 64 before are used.  On the 32 x 32 instruction the tiled page layout fits as it is: a
// lane's 16 scores of 32 keys are two operands of the value product (keys 4 h + i and 16 + 4 h + i, and 8 further, of lane
// half h), whose other operand is one 16-byte read of a value tile.  (2048 rows that end at 8200, 32 heads of 128 on 8 key heads: 233 ..
// 249 us by card, 970 .. 1030 TFLOP/s, where a bf16 product of 8192^3 reaches 1181; 2048 rows alone 53.8 us = 640, 256 rows that end at 8000 56.8 =
// 580: partial results of pieces and their joins.)  Over 8-bit pages 258 .. 272 us: a work-group turns the codes of the next 64 keys into numbers on
// their way to LDS, 47 us of the vector units' time, most of it for the values, whose powers of two differ from key to key.  (Requested two units ahead
// instead of one, in registers, the outputs no longer fit in them: 627 us.)
typedef float f32x16 __attribute__((ext_vector_type(16)));
__device__ __forceinline__ f32x16 mma(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 mma(f16x8 a, f16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ float halves_max(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float halves_sum(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// lane l: lds[l] = base[offset / 16 + l]
__device__ __forceinline__ void copy_tile(const void* base, uint32_t offset, uint4* lds, uint32_t lane_bytes) {
  const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, 0xFFFFFFFFu, 0x00027000);
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)(static_cast<uint32_t>(reinterpret_cast<uintptr_t>(lds))), 16,
                                           lane_bytes, offset, 0, 0);
}
constexpr int kChunkCols = 128, kChunkUnit = 64;
constexpr float kFarScore = 4096.f;   // in powers of two; below it the reference point's product is off by 2^-13 of one at most
template <int HD>
struct ChunkLds {
  union {
    uint4 tile[2][2][2][4 * HD];   // [buffer][32-key block][keys, values][64 HD bytes]
    float join[2 * kMaxPieces * kChunkCols + 256];
  };
  int last;
};
// Pieces of a tile joined two at a time, as the leaves of a binary tree: who comes first to a pair leaves its results there, who comes second adds them to
// its own, in registers, and goes on; true where that was the last pair.  The last of n pieces reads log2 n others then, not all of them (2 us each for a
// work-group: trees of 25 rows of 16 sequences, 32 heads on 8 of 128, up to 14 pieces: 86 us with one work-group that reads all, 70 so; 59 with the larger
// pieces that find_piece takes).  Either order gives the same bits: the sums below are symmetric.  A pair's ticket is that of its right half's first piece; a
// half that sees the other's ticket taken does not leave its results first.
template <int HD>
__device__ __forceinline__ bool join_two_by_two(const stairs_paged_cache& c, const stairs_paged_attn& a, const Span& sp, const Piece& w, f32x16 (&o)[HD / 32], float& m, float& l,
                                                bool here, int* s_last) {
#pragma clang fp contract(off)
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, at = wave * (HD / 8) * 256 + lane * 4, at_ml = kChunkCols * HD + wave * 64 + (lane & 31) * 2;
#pragma unroll 1
  for (int s = 1; s < w.pieces; s <<= 1) {
    const int left = w.piece & ~(2 * s - 1), right = left + s;
    if (right >= w.pieces) continue;
    const int mine = w.piece & s ? right : left;
    int* counter = tickets(a, sp) + w.first + right * c.n_kv_heads;
    auto slot = [&](int piece) { return partials(a, sp) + (size_t)(w.first + piece * c.n_kv_heads) * piece_floats<HD>(kChunkCols); };
    __syncthreads();
    if (threadIdx.x == 0) *s_last = __hip_atomic_load(counter, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    if (*s_last == 0 && here) {                                 // (the other half may still come first: then this was for nothing)
      float* dst = slot(mine);
#pragma unroll
      for (int d = 0; d < HD / 32; ++d)
#pragma unroll
        for (int b = 0; b < 4; ++b) st_dev4(dst, at + (d * 4 + b) * 256, make_float4(o[d][b * 4], o[d][b * 4 + 1], o[d][b * 4 + 2], o[d][b * 4 + 3]));
      if (lane < 32) st_dev2(dst + at_ml, m, l);
    }
    if (!last_arrival(counter, 2, s_last)) return false;
    if (here) {
      const float* src = slot(left + right - mine);
      const float2 ml = ld_dev2(src + at_ml);
      float4 x[HD / 8];
#pragma unroll
      for (int i = 0; i < HD / 8; ++i) x[i] = ld_dev4(src, at + i * 256);
      __builtin_amdgcn_sched_barrier(0);                        // (all of them on their way before the first is waited for)
      const float all = fmaxf(m, ml.x), f = weight_of(m, all), g = weight_of(ml.x, all);
      m = all;
      l = l * f + ml.y * g;
#pragma unroll
      for (int i = 0; i < HD / 8; ++i) {
        const int d = i >> 2, b = (i & 3) * 4;
        o[d][b] = o[d][b] * f + x[i].x * g;
        o[d][b + 1] = o[d][b + 1] * f + x[i].y * g;
        o[d][b + 2] = o[d][b + 2] * f + x[i].z * g;
        o[d][b + 3] = o[d][b + 3] * f + x[i].w * g;
      }
    }
    if (threadIdx.x == 0) *counter = 0;
  }
  return true;
}

template <typename T, int HD, int F>
__device__ __forceinline__ void attend_chunk(const stairs_paged_cache& c, const stairs_paged_attn& a, const Span& sp, float scale2, ChunkLds<HD>& lds) {
  constexpr bool H8 = F & kHeld8, M = F & kMasks;
  typedef typename Elem<T>::x8 x8;
  // (Over 8-bit pages the codes times their powers of two are what lies in LDS: numbers of T, exact but where a half has no steps any more.)
  constexpr int KS = HD / 16, DT = HD / 32;                     // steps of 16 dims, tiles of 32 dims
  Piece w;
  if (!find_piece<M>(c, a, sp, w)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 31, h = lane >> 5;
  const int G = a.n_heads / c.n_kv_heads, cols = w.rows * G, col0 = w.group * kChunkCols, wcol = col0 + wave * 32;
  const int limit = a.max_blocks * c.page_size, pos0 = w.len - w.rows;
  // last positions that the work-group's, the wave's and the lane's columns see
  const bool tree = M && is_tree(a, w);
  const int last_tree = min(w.len, limit) - 1;
  const int last_group = tree ? last_tree : min(pos0 + (min(cols, col0 + kChunkCols) - 1) / G, limit - 1);
  const int first_wave = wcol >= cols ? -1 : tree ? min(pos0, limit) - 1 : min(pos0 + wcol / G, limit - 1);
  const int last_wave = wcol >= cols ? -1 : tree ? last_tree : min(pos0 + (min(cols, wcol + 32) - 1) / G, limit - 1);
  const int col = wcol + n, row = col < cols ? col / G : 0;
  const int last = col < cols ? min(pos0 + row, limit - 1) : -1;
  Sees sees{0, 0};
  if constexpr (M)
    if (col < cols) sees = sees_of(a, w, row, limit);
  const size_t at_row = (size_t)(w.row0 + row), at_head = (size_t)(w.kvh * G + (col < cols ? col - row * G : 0)) * HD;
  x8 q[KS];
  {
    const T* qp = static_cast<const T*>(a.q) + at_row * a.q_stride + at_head + h * 8;
#pragma unroll
    for (int k = 0; k < KS; ++k) q[k] = *reinterpret_cast<const x8*>(qp + k * 16);
  }
  f32x16 o[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d) o[d] = f32x16{};
  float m = -INFINITY, l = 0.f;

  const size_t head_elems = (size_t)c.page_size * HD, page_elems = head_elems * c.n_kv_heads;
  // the wave copies block wave / 2 of a unit, its keys or its values
  const T* pool = static_cast<const T*>(wave & 1 ? c.v : c.k) + w.kvh * head_elems;
  const int* table = a.block_table + (size_t)w.seq * a.max_blocks;
  const int ps_shift = __builtin_ctz(c.page_size);
  const int u1 = min(w.u1, last_group < 0 ? 0 : last_group / kChunkUnit + 1);
  int pages = -1, pages_at = w.u0;                              // of the blocks 2 pages_at .., a lane each
  auto fetch_pages = [&](int u) {
    pages_at = u;
    const unsigned key = u * kChunkUnit + lane * 32u;           // (lanes behind the last key: past 2^31 perhaps)
    pages = key <= (unsigned)last_group ? table[key >> ps_shift] : -1;
    if ((unsigned)pages >= (unsigned)c.n_pages) pages = -1;
  };
  auto page_of = [&](int u, int block) { return __builtin_amdgcn_readlane(pages, (u - pages_at) * 2 + block); };
  // 8-bit pages: a wave takes 16 keys of a block and half of the dims of its values, through registers
  constexpr int NS = HD / 64;
  uint4 kr[NS], vr[NS];
  uint32_t kb = 0;
  uint2 vb{};
  auto request = [&](int u, int buf) {                          // (a block without a page: another's bytes, masked below)
    const int b = wave >> 1, key = u * kChunkUnit + b * 32;
    const size_t at = (size_t)max(page_of(u, b), 0) * page_elems + (size_t)(key & (c.page_size - 1)) * HD;
    if constexpr (H8) {
      const size_t from = at + w.kvh * head_elems + (wave & 1) * NS * 1024;
      const uint8_t* s = static_cast<const uint8_t*>(c.scale) + (at + w.kvh * head_elems) / (HD / 2);
#pragma unroll
      for (int i = 0; i < NS; ++i) {
        kr[i] = *reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(c.k) + from + i * 1024 + lane * 16);
        vr[i] = *reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(c.v) + from + i * 1024 + lane * 16);
      }
      kb = s[(lane & 15) / 4 * 16 + (wave & 1) * 4 + (lane & 3)];
      vb = *reinterpret_cast<const uint2*>(s + (lane >> 4) * 16 + 8);
    } else {
      const T* src = pool + at;
#pragma unroll
      for (int i = 0; i < HD / 16; ++i) copy_tile(src, i * 1024, &lds.tile[buf][b][wave & 1][i * 64], lane * 16);
    }
  };
  auto stage = [&](int buf) {                                   // what was requested, as it is used, into its buffer
    if constexpr (H8) {
      uint4* kd = &lds.tile[buf][wave >> 1][0][(wave & 1) * (HD / 32) * 64 + lane];
      uint4* vd = &lds.tile[buf][wave >> 1][1][(wave & 1) * (HD / 32) * 64 + lane];
      const float kf = __uint_as_float(kb << 23);
      float vf[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) vf[i] = scale_of(i < 4 ? vb.x : vb.y, i & 3);
#pragma unroll
      for (int i = 0; i < NS; ++i) {
        kd[2 * i * 64] = widen<T>(kr[i].x, kr[i].y, kf);
        kd[(2 * i + 1) * 64] = widen<T>(kr[i].z, kr[i].w, kf);
        vd[2 * i * 64] = widen<T>(vr[i].x, vr[i].y, vf);
        vd[(2 * i + 1) * 64] = widen<T>(vr[i].z, vr[i].w, vf);
      }
    }
  };
  __syncthreads();
  if (w.u0 < u1) {
    fetch_pages(w.u0);
    request(w.u0, w.u0 & 1);
    stage(w.u0 & 1);
  }
  // Two loops of one body: units that all of the wave's columns see, then those with masks (with both in one loop the 64 output
  // registers were copied twice a unit).  A wave goes from one to the other when it has to; barriers are one a unit in both.
  int u = w.u0;
  int page0 = -1, page1 = -1;
  auto next_unit = [&]() {                                      // unit u is in LDS, the next one on its way
    page0 = page_of(u, 0);
    page1 = page_of(u, 1);
    if (u + 1 - pages_at >= 32) fetch_pages(u + 1);
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");   // unit u is there, the other buffer has been read
    if (u + 1 < u1) request(u + 1, (u + 1) & 1);
  };
  auto scores = [&](f32x16 (&s)[2]) {
    s[0] = s[1] = f32x16{};
    const uint4* kt = lds.tile[u & 1][0][0] + (n >> 4) * (HD / 32) * 64 + (n & 15) + 16 * h;
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int b = 0; b < 2; ++b) s[b] = mma(__builtin_bit_cast(x8, kt[b * 8 * HD + (k >> 1) * 64 + 32 * (k & 1)]), q[k], s[b]);
  };
  // (m: the reference point in units of the raw score)
  auto probabilities = [&](f32x16 (&s)[2], x8 (&p)[2][2]) {
    // (the maximum that passes NaN on, one instruction for three values; a NaN makes the column's sum NaN whatever m is)
    float mx = __builtin_elementwise_maximum(s[0][0], s[1][0]);
#pragma unroll
    for (int i = 1; i < 16; ++i) mx = __builtin_elementwise_maximum(mx, __builtin_elementwise_maximum(s[0][i], s[1][i]));
    if (__any((mx - m) * scale2 > Headroom<T>::slack)) {
      const float mn = fmaxf(m, halves_max(mx));
      const float f = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m - mn) * scale2);
      m = mn;
      l *= f;
#pragma unroll
      for (int d = 0; d < DT; ++d) o[d] *= f;
    }
    float mr = m == -INFINITY ? 0.f : Headroom<T>::lift - m * scale2;
    if (__any(fabsf(mr) > kFarScore)) {
      // Far from 0 the reference point's product is rounded by whole powers of two (probabilities past the largest half, in bfloat16 ones
      // that are none of 1): there it is taken off the raw scores.
#pragma unroll
      for (int i = 0; i < 32; ++i) s[i >> 4][i & 15] -= m == -INFINITY ? 0.f : m;
      mr = Headroom<T>::lift;
    }
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      const float x = __builtin_amdgcn_exp2f(fmaf(s[i >> 4][i & 15], scale2, mr));
      sum[i & 3] += x;
      p[i >> 4][i >> 2 & 1][(i & 3) + 4 * (i >> 3 & 1)] = Elem<T>::down(x);
    }
    l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
  };
  for (; u < u1; ++u) {
    const int key0 = u * kChunkUnit;
    if (key0 + kChunkUnit - 1 > first_wave || page_of(u, 0) < 0 || page_of(u, 1) < 0) break;
    next_unit();
    f32x16 s[2];
    x8 p[2][2];
    scores(s);
    probabilities(s, p);
    const uint4* vt = lds.tile[u & 1][0][1] + (n >> 4) * 64 + (n & 15) + 16 * h;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int d = 0; d < DT; ++d) o[d] = mma(__builtin_bit_cast(x8, vt[b * 8 * HD + d * 128 + r * 32]), p[b][r], o[d]);
    if (H8 && u + 1 < u1) stage((u + 1) & 1);
  }
#pragma unroll 1
  for (; u < u1; ++u) {
    const int key0 = u * kChunkUnit;
    next_unit();
    if (H8 && u + 1 < u1) stage((u + 1) & 1);
    if (key0 > last_wave) continue;                             // (nothing for this wave any more)
    f32x16 s[2];
    x8 p[2][2];
    scores(s);
    uint32_t seen_bits[2];                                      // of the lane's keys of a block: (key - 4 h) of the 32
    if constexpr (M) {
      seen_bits[0] = page0 < 0 ? 0 : block_of(sees, key0) >> (4 * h);
      seen_bits[1] = page1 < 0 ? 0 : block_of(sees, key0 + 32) >> (4 * h);
    }
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      const int key = key0 + (i >> 4) * 32 + (i >> 2 & 3) * 8 + h * 4 + (i & 3);
      float& x = reinterpret_cast<float*>(&s[i >> 4])[i & 15];
      if constexpr (M) x = seen_bits[i >> 4] >> ((i >> 2 & 3) * 8 + (i & 3)) & 1 ? x : -INFINITY;
      else x = key <= last && (i < 16 ? page0 : page1) >= 0 ? x : -INFINITY;
    }
    probabilities(s, p);
    // as in attend_rows: what no column of the wave sees is cleared, infinities and NaNs go to the columns that see them
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const int end = (b ? page1 : page0) < 0 ? -1 : last_wave, mine = (b ? page1 : page0) < 0 ? -1 : last;
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const int key = key0 + b * 32 + r * 8 + h * 4;
        uint32_t keep[4], odd = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int k = key + (i >> 1) * 16 + (i & 1) * 2;
          keep[i] = (k <= end ? 0xFFFFu : 0u) | (k + 1 <= end ? 0xFFFF0000u : 0u);
        }
        const uint4* vt = lds.tile[u & 1][b][1] + (n >> 4) * 64 + (n & 15) + 16 * h + r * 32;
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          uint4 v = vt[d * 128];
          odd |= clear_odd<T>(v.x, keep[0]) | clear_odd<T>(v.y, keep[1]) | clear_odd<T>(v.z, keep[2]) | clear_odd<T>(v.w, keep[3]);
          o[d] = mma(__builtin_bit_cast(x8, v), p[b][r], o[d]);
        }
        if (__any(odd != 0)) {
          x8 seen;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const bool sees_key = M ? (seen_bits[b] >> (r * 8 + (i >> 2) * 16 + (i & 3)) & 1) != 0 : key + (i >> 2) * 16 + (i & 3) <= mine;
            seen[i] = sees_key ? (T)1.f : (T)0.f;
          }
#pragma unroll
          for (int d = 0; d < DT; ++d) {
            uint4 v = vt[d * 128];
            v.x &= keep[0]; v.y &= keep[1]; v.z &= keep[2]; v.w &= keep[3];
            const uint4 kinds = make_uint4(odd_kinds<T>(v.x), odd_kinds<T>(v.y), odd_kinds<T>(v.z), odd_kinds<T>(v.w));
            const f32x16 count = mma(__builtin_bit_cast(x8, kinds), seen, f32x16{});
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] += odd_value(count[i]);
          }
        }
      }
    }
  }
  l = halves_sum(l);
  m = m == -INFINITY ? m : m * scale2;                          // (what the join works with)
  if constexpr (M) {
    if (!join_two_by_two<HD>(c, a, sp, w, o, m, l, wcol < cols, &lds.last)) return;
  }
  if (M || w.pieces == 1) {
    if (col < cols) {
      const float f = l == 0.f ? 0.f : 1.f / l;
      T* dst = static_cast<T*>(a.out) + at_row * a.out_stride + at_head + h * 4;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          T v[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] = Elem<T>::down(o[d][b * 4 + i] * f);
          *reinterpret_cast<uint2*>(dst + d * 32 + b * 8) = *reinterpret_cast<const uint2*>(v);
        }
    }
    return;
  }
  if constexpr (M) return;
  float* part = partials(a, sp) + (size_t)(w.first + w.piece * c.n_kv_heads) * piece_floats<HD>(kChunkCols);
  if (col < cols) {
    const int dst = (col - col0) * HD + h * 4;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        st_dev4(part, dst + d * 32 + b * 8, make_float4(o[d][b * 4], o[d][b * 4 + 1], o[d][b * 4 + 2], o[d][b * 4 + 3]));
      }
    if (h == 0) st_dev2(part + kChunkCols * HD + (col - col0) * 2, m, l);
  }
  __syncthreads();                                              // (the tiles have been read: their place serves the join)
  join_pieces<T, HD, kChunkCols>(c, a, sp, w, reinterpret_cast<float2*>(lds.join), &lds.last);
}
template <typename T, int HD, int F>
__global__ __launch_bounds__(256, 2) void k_paged_chunk(stairs_paged_cache c, stairs_paged_attn a, Span sp, float scale2) {
  __shared__ ChunkLds<HD> lds;
  attend_chunk<T, HD, F>(c, a, sp, scale2, lds);
}
// both in one launch: the chunks' work-groups first, the few rows of the others where there is room (2 chunks of 509 rows among 22
// sequences of 3, 90 .. 5000 positions, 16 heads of 128: 79 us = 3.3 TB/s)
template <typename T, int HD, int F>
__global__ __launch_bounds__(256, 2) void k_paged_mixed(stairs_paged_cache c, stairs_paged_attn a, Span chunk, Span rows, float scale2) {
  __shared__ union { ChunkLds<HD> chunk; RowsLds<HD, 2> rows; } lds;
  if ((int)blockIdx.x < rows.first_block) attend_chunk<T, HD, F>(c, a, chunk, scale2, lds.chunk);
  else attend_rows<T, HD, 2, F>(c, a, rows, scale2, lds.rows);
}

}  // namespace

int check_stream(hipStream_t st) {
  int here = -1;
  if (hipGetDevice(&here) != hipSuccess) return STAIRS_EHIP;
  if (!st) return STAIRS_OK;
  hipDevice_t its = -1;
  if (hipStreamGetDevice(st, &its) != hipSuccess) return STAIRS_EHIP;
  return its == here ? STAIRS_OK : STAIRS_EINVAL;
}

}  // namespace stairs

using namespace stairs;

namespace {

constexpr int kCus = 256;
constexpr int64_t kMostGroups = (1ll << 24) - 1;     // work-groups of 256 threads in a launch

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

}  // namespace

bool stairs::paged_cache_ok(const stairs_paged_cache* c) {
  if (!c || (c->dtype != STAIRS_DTYPE_BF16 && c->dtype != STAIRS_DTYPE_FP16)) return false;
  if (c->page_size != 32 && c->page_size != 64 && c->page_size != 128 && c->page_size != 256) return false;
  if (c->head_dim != 64 && c->head_dim != 128) return false;
  if (c->n_kv_heads < 1 || c->n_kv_heads > 4096 || c->n_pages < 1 || (int64_t)c->n_pages * c->page_size > INT32_MAX) return false;
  if (c->held != 0 && (c->held != STAIRS_DTYPE_E4M3 || !c->scale || !aligned16(c->scale))) return false;
  return c->k && c->v && aligned16(c->k) && aligned16(c->v);
}

namespace {

// every stride holds a row and keeps its 16-byte alignment
bool stride_ok(int64_t stride, int heads, int hd) { return stride >= (int64_t)heads * hd && stride % 8 == 0; }

int launched() { return hipGetLastError() == hipSuccess ? STAIRS_OK : STAIRS_EHIP; }

// f(type, head_dim) for the cache's
template <typename F>
void by_type(const stairs_paged_cache* c, F f) {
  const bool b = c->dtype == STAIRS_DTYPE_BF16;
  if (c->head_dim == 64) b ? f(__bf16{}, std::integral_constant<int, 64>{}) : f(_Float16{}, std::integral_constant<int, 64>{});
  else b ? f(__bf16{}, std::integral_constant<int, 128>{}) : f(_Float16{}, std::integral_constant<int, 128>{});
}

// f(type, head_dim, whether pages hold 8 bits)
template <typename F>
void by_pages(const stairs_paged_cache* c, F f) {
  by_type(c, [&](auto type, auto hd) { c->held ? f(type, hd, std::true_type{}) : f(type, hd, std::false_type{}); });
}
// f(type, head_dim, form of the attention kernels)
template <typename F>
void by_form(const stairs_paged_cache* c, const stairs_paged_attn* a, F f) {
  by_type(c, [&](auto type, auto hd) {
    if (c->held) f(type, hd, std::integral_constant<int, kMasks | kHeld8>{});
    else if (a->sees) f(type, hd, std::integral_constant<int, kMasks>{});
    else f(type, hd, std::integral_constant<int, 0>{});
  });
}

bool attn_sizes_ok(const stairs_paged_cache* c, const stairs_paged_attn* a) {
  if (!paged_cache_ok(c) || !a) return false;
  if (a->n_seqs < 0 || a->n_seqs > STAIRS_PAGED_MAX_SEQS || a->max_blocks < 1 || a->rows < 0 || a->max_fresh < 0) return false;
  if ((int64_t)a->max_blocks * c->page_size > INT32_MAX) return false;
  if (a->n_heads < 1 || (int64_t)a->rows * a->n_heads / c->n_kv_heads > 1 << 24) return false;   // (counts of tiles stay ints)
  return a->n_heads >= 1 && a->n_heads <= 4096 && a->n_heads % c->n_kv_heads == 0;
}

}  // namespace

extern "C" int stairs_paged_plan(const stairs_page_plan* p, void* hip_stream) {
  if (!p || p->n_seqs < 0 || p->n_seqs > STAIRS_PAGED_MAX_SEQS || p->max_blocks < 1 || p->max_rows < 0 || p->n_pages < 1) return STAIRS_EINVAL;
  if (p->page_size != 32 && p->page_size != 64 && p->page_size != 128 && p->page_size != 256) return STAIRS_EINVAL;
  if ((int64_t)p->n_pages * p->page_size > INT32_MAX || (int64_t)p->max_blocks * p->page_size > INT32_MAX) return STAIRS_EINVAL;
  if (!p->n_free || !p->n_free_out || !p->free_pages || !p->row_start) return STAIRS_EINVAL;
  if (p->n_seqs > 0 && (!p->cached || !p->fresh || !p->held || !p->held_out || !p->block_table || !p->seq_len)) return STAIRS_EINVAL;
  if (p->max_rows > 0 && (!p->position || !p->slot)) return STAIRS_EINVAL;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (const int rc = check_stream(st)) return rc;
  const bool one = p->max_rows <= 4 * kPlanThreads;
  hipLaunchKernelGGL(k_paged_plan, dim3(1), dim3(kPlanThreads), 0, st, *p, one ? p->max_rows : 0);
  if (!one) hipLaunchKernelGGL(k_paged_slots, dim3(std::min((p->max_rows - 1) / 256 + 1, 8 * kCus)), dim3(256), 0, st, *p);
  return launched();
}

extern "C" int stairs_paged_append(const stairs_paged_cache* c, const stairs_paged_rows* a, void* hip_stream) {
  if (!paged_cache_ok(c) || !a || a->rows < 0 || a->rows > kMostGroups * kAppendRows || a->n_heads < 0 || a->n_heads > 4096) return STAIRS_EINVAL;
  if (!(a->rope_theta >= 0.f) || std::isinf(a->rope_theta)) return STAIRS_EINVAL;
  if (a->rows == 0) return STAIRS_OK;
  if (!a->k || !a->v || !a->slot || (a->rope_theta > 0.f && !a->position)) return STAIRS_EINVAL;
  if (!aligned16(a->k) || !aligned16(a->v) || !stride_ok(a->k_stride, c->n_kv_heads, c->head_dim) || !stride_ok(a->v_stride, c->n_kv_heads, c->head_dim))
    return STAIRS_EINVAL;
  if (a->n_heads > 0 && (!a->q || !a->q_out || !aligned16(a->q) || !aligned16(a->q_out) || !stride_ok(a->q_stride, a->n_heads, c->head_dim) ||
                         !stride_ok(a->q_out_stride, a->n_heads, c->head_dim) || (a->q == a->q_out && a->q_stride != a->q_out_stride)))
    return STAIRS_EINVAL;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (const int rc = check_stream(st)) return rc;
  stairs_paged_rows r = *a;
  if (r.rope_theta == 0.f && r.q == r.q_out) r.n_heads = 0;       // nothing happens to q
  const int heads = std::max(r.n_heads, c->n_kv_heads), tiles = (r.rows - 1) / kAppendRows + 1;
  const int groups = std::max(1, std::min((4 * kCus + tiles - 1) / tiles, heads));
  const double log2_theta = r.rope_theta > 0.f ? std::log2((double)r.rope_theta) : 0.0;
  by_pages(c, [&](auto type, auto hd, auto h8) {
    hipLaunchKernelGGL((k_paged_append<decltype(type), decltype(hd)::value, decltype(h8)::value>), dim3(tiles, groups, tiles * groups < 2 * kCus ? 3 : 1), dim3(256), 0, st, *c, r, log2_theta);
  });
  return launched();
}

extern "C" int stairs_paged_read(const stairs_paged_cache* c, const stairs_paged_out* a, void* hip_stream) {
  if (!paged_cache_ok(c) || !a || a->rows < 0 || a->rows > kMostGroups * kAppendRows) return STAIRS_EINVAL;
  if (a->rows == 0 || (!a->k && !a->v)) return STAIRS_OK;
  if (!a->slot) return STAIRS_EINVAL;
  if (a->k && (!aligned16(a->k) || !stride_ok(a->k_stride, c->n_kv_heads, c->head_dim))) return STAIRS_EINVAL;
  if (a->v && (!aligned16(a->v) || !stride_ok(a->v_stride, c->n_kv_heads, c->head_dim))) return STAIRS_EINVAL;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (const int rc = check_stream(st)) return rc;
  const int tiles = (a->rows - 1) / kAppendRows + 1, groups = std::max(1, std::min((8 * kCus + tiles - 1) / tiles, c->n_kv_heads));
  by_pages(c, [&](auto type, auto hd, auto h8) {
    hipLaunchKernelGGL((k_paged_read<decltype(type), decltype(hd)::value, decltype(h8)::value>), dim3(tiles, groups, a->k && a->v ? 2 : 1), dim3(256), 0, st, *c, *a);
  });
  return launched();
}

namespace {

// ---- how a call is spread: by its sizes on the host, by the lengths on the device (find_piece) ------------------------
// A sequence's columns are its rows times the query heads of a key head.  Up to 32 of them (16 in one tile) go to attend_rows, more to
// attend_chunk; max_fresh says which of the two a call needs, and with one sequence, or none with more, one kernel
// takes whatever it finds.
constexpr int kFewCols = 32;
struct Launch {
  int ct;                      // column tiles of the rows' part, 0: there is none
  bool chunk;
  Span rows, chunks;
  int64_t work_bytes, grid;
};
Launch plan_attention(const stairs_paged_cache* c, const stairs_paged_attn* a) {
  const int G = a->n_heads / c->n_kv_heads;
  const int64_t cols = (int64_t)a->max_fresh * G;
  Launch l{};
  l.chunk = cols > kFewCols;
  l.ct = cols <= 16 ? 1 : !l.chunk || a->n_seqs > 1 ? 2 : 0;
  constexpr int kSlots = 2 * kCus;
  l.work_bytes = 2 * most_pieces(kSlots) * (int64_t)sizeof(int);
  auto add = [&](Span& s) {
    s.first_block = (int)l.grid;
    s.partials = l.work_bytes;
    // at most `slots` pieces and one a tile
    const int64_t tiles = a->n_seqs + (int64_t)a->rows * G / s.tile_cols;
    l.grid += s.slots + tiles * c->n_kv_heads;
    l.work_bytes += most_pieces(s.slots) * (int64_t)(s.tile_cols * (c->head_dim + 2) * sizeof(float));
  };
  if (l.chunk) {
    l.chunks = Span{l.ct ? kFewCols + 1 : 1, INT32_MAX, kChunkCols, kChunkUnit, kSlots, 8, 400, 0, 32, 0, 0};
    add(l.chunks);
  }
  if (l.ct) {
    // pieces of 4 units and more: shorter ones cost more to join than they save (8000 keys of 8 heads alone: 25 us with 2, 19 with 4)
    l.rows = Span{1, l.chunk ? kFewCols : INT32_MAX, 16 * l.ct, kRowUnit, kSlots, 4, 200, 0, 0, most_pieces(kSlots), 0};
    add(l.rows);
  }
  return l;
}

}  // namespace

extern "C" int64_t stairs_paged_attention_workspace(const stairs_paged_cache* c, const stairs_paged_attn* a) {
  if (!attn_sizes_ok(c, a)) return STAIRS_EINVAL;
  const Launch l = plan_attention(c, a);
  return l.grid <= kMostGroups ? l.work_bytes : (int64_t)STAIRS_EINVAL;
}

extern "C" int stairs_paged_attention(const stairs_paged_cache* c, const stairs_paged_attn* a, void* hip_stream) {
  if (!attn_sizes_ok(c, a) || std::isnan(a->scale) || std::isinf(a->scale)) return STAIRS_EINVAL;
  if (a->n_seqs == 0 || a->rows == 0) return STAIRS_OK;
  if (!a->q || !a->out || a->q == a->out || !a->block_table || !a->row_start || !a->seq_len) return STAIRS_EINVAL;
  if (!aligned16(a->q) || !aligned16(a->out) || !stride_ok(a->q_stride, a->n_heads, c->head_dim) || !stride_ok(a->out_stride, a->n_heads, c->head_dim))
    return STAIRS_EINVAL;
  if (!a->workspace || !aligned16(a->workspace) || reinterpret_cast<uintptr_t>(a->sees) % 8 != 0) return STAIRS_EINVAL;
  const Launch l = plan_attention(c, a);
  if (l.grid > kMostGroups) return STAIRS_EINVAL;
  if (a->workspace_bytes < l.work_bytes) return STAIRS_ECAPACITY;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (const int rc = check_stream(st)) return rc;
  const float scale2 = (a->scale > 0.f ? a->scale : 1.0f / sqrtf((float)c->head_dim)) * kLog2e;
  by_form(c, a, [&](auto type, auto hd, auto form) {
    typedef decltype(type) T;
    constexpr int HD = decltype(hd)::value, F = decltype(form)::value;
    const dim3 grid((unsigned)l.grid), block(256);
    if (l.chunk && l.ct) hipLaunchKernelGGL((k_paged_mixed<T, HD, F>), grid, block, 0, st, *c, *a, l.chunks, l.rows, scale2);
    else if (l.chunk) hipLaunchKernelGGL((k_paged_chunk<T, HD, F>), grid, block, 0, st, *c, *a, l.chunks, scale2);
    else if (l.ct == 1) hipLaunchKernelGGL((k_paged_rows<T, HD, 1, F>), grid, block, 0, st, *c, *a, l.rows, scale2);
    else hipLaunchKernelGGL((k_paged_rows<T, HD, 2, F>), grid, block, 0, st, *c, *a, l.rows, scale2);
  });
  return launched();
}
