// Operators over paged key/value caches: pages and slots for the requests of a step, storing the new rows, attention of the
// new rows over the pages.  The page layout is the tiled layout of the framework's own half caches (k_cache_off, v_cache_off),
// page by page.
#include "../../include/stairs.h"
#include "stairs_device.h"

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

// Bound by memory, with few rows by latency.  A work-group has 32 rows and some of the n_heads + 2 n_kv_heads heads (so many
// groups of them that there are work for all CUs); the rows' rotations are formed once for all its heads.  q and k: a thread takes 8
// pairs of a row, 16 bytes of either half; in a key tile the same 8 dims of 8 rows are one line.  v: a head's rows go through LDS;
// the eight positions of a value tile that are 16 adjacent bytes a dim (two quads, 16 apart) are stored together where they are rows
// of this call, so that a wave's store is a whole tile row; rows that have not all of them as quads of 8 bytes or single
// values.  (Quads transposed in registers, 8 bytes here and there: 8190 rows of 48 heads 75 us, 40 of them for the
// values; as it is 57.5 = 3.5 TB/s, reading 8 % more than the rows have,
// writing no more.)
constexpr int kAppendRows = 32;
template <typename T, int HD>
__global__ __launch_bounds__(256) void k_paged_append(stairs_paged_cache c, stairs_paged_rows a, double log2_theta) {
  constexpr int AHEAD = 19, BEHIND = 16;                        // rows around these that decide how theirs are stored
  __shared__ union {
    float2 cs[kAppendRows][HD / 2];
    T v[kAppendRows + AHEAD][HD];
  } lds;
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
    *reinterpret_cast<x8*>(dst) = lo;
    *reinterpret_cast<x8*>(dst + HD / 2) = hi;
  }
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
      if (lo < 4 * per) per = lo;
    }
  }
  per = __builtin_amdgcn_readfirstlane(per);
  int before = 0, split_before = 0;
  for (int b0 = 0; b0 < a.n_seqs; b0 += 64) {
    if (a.n_seqs > 64) w = seq_work(c, a, sp, b0 + lane);
    const int pieces = min(kMaxPieces, max(1, (int)((unsigned)(w.units + per - 1) / (unsigned)per)));
    const int mine = w.groups * pieces, split = pieces > 1 ? mine : 0;
    const int to = before + wave_scan(mine), split_to = split_before + wave_scan(split);
    const unsigned long long there = __ballot(to > item);
    if (there) {
      const int l = __builtin_ctzll(there);
      const unsigned at = item - (__builtin_amdgcn_readlane(to, l) - __builtin_amdgcn_readlane(mine, l));
      const unsigned n = __builtin_amdgcn_readlane(pieces, l), group = at / n;
      const int u = __builtin_amdgcn_readlane(w.units, l);
      out.seq = b0 + l;
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

// ---- few columns: a wave per 32 keys ----------------------------------------------------------------------------------
// Bound by the bytes of the cache.  A work-group takes a piece of a tile of 16 CT columns; its four waves take 32-key blocks in
// turn, straight from memory into the matrix operands (a block of a head is 2 x 64 HD contiguous bytes, every load 1 KiB of a
// wave), no LDS, and are joined at the end.  Values are requested before the scores they wait for, the next block's keys as
// soon as this block's are used.  (3 sequences of 9 rows and 23456 .. 59999 positions, 32 heads of 128: 300 us = 6.6 TB/s; 32 of 5 rows and
// 200 .. 8000 positions, 8 key heads: 66.6 us = 4.3 TB/s, the rest goes into starting and joining pieces; 300 positions alone 6.6 us, one sequence of
// 8000 and 8 key heads 13 us with 1 row, 19 with 5.)
constexpr int kRowUnit = 32 * 4;
template <int HD, int CT>
struct RowsLds {
  float o[4][16 * CT][HD + 4], m[4][16 * CT], l[4][16 * CT];
  int last;
};
template <typename T, int HD, int CT>
__device__ __forceinline__ void attend_rows(const stairs_paged_cache& c, const stairs_paged_attn& a, const Span& sp, float scale2, RowsLds<HD, CT>& lds) {
  typedef typename Elem<T>::x8 x8;
  constexpr int KK = HD / 32, ET = HD / 16;
  Piece w;
  if (!find_piece(c, a, sp, w)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), j = lane & 15, g = lane >> 4;
  const int G = a.n_heads / c.n_kv_heads, cols = w.rows * G, col0 = w.group * 16 * CT;
  const int limit = a.max_blocks * c.page_size;
  const int pos0 = w.len - w.rows;                              // position of the sequence's first row
  const int first_last = min(pos0 + col0 / G, limit - 1);        // last position the tile's first and last column see
  const int last_last = min(pos0 + (min(cols, col0 + 16 * CT) - 1) / G, limit - 1);
  int last[CT];
  x8 q[CT][KK];
  bool had_odd = false;                                         // the wave has left infinities or NaNs in its part of lds.o
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    const int col = col0 + ct * 16 + j;
    last[ct] = -1;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) q[ct][kk] = x8{};
    if (col < cols) {
      const int r = col / G;
      last[ct] = min(pos0 + r, limit - 1);
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
  const T* K = static_cast<const T*>(c.k) + w.kvh * head_elems;
  const T* V = static_cast<const T*>(c.v) + w.kvh * head_elems;
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
  uint4 kf[2 * KK], vf[ET];
  auto block_at = [&](int u) -> size_t {                        // elements in front of the block in its pool
    const int key = u * kRowUnit + wave * 32;
    return (size_t)__builtin_amdgcn_readlane(pages, u - pages_at) * page_elems + (size_t)(key & (c.page_size - 1)) * HD;
  };
  auto load_keys = [&](size_t at) {
#pragma unroll
    for (int i = 0; i < 2 * KK; ++i) kf[i] = ld_once_as<uint4>(K + at + (i * 64 + lane) * 8);
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
    for (int i = 0; i < ET; ++i) vf[i] = ld_once_as<uint4>(V + at + (i * 64 + lane) * 8);
    f32x4 s[CT][2];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        s[ct][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) s[ct][t] = mma(__builtin_bit_cast(x8, kf[t * KK + kk]), q[ct][kk], s[ct][t]);
      }
    const int key0 = u * kRowUnit + wave * 32;
    const int un = next_block(u + 1);
    const size_t at_here = at;
    if (un < u1) {
      at = block_at(un);
      load_keys(at);
    }
    const bool full = key0 + 31 <= first_last;
    x8 p[CT], rest[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = s[ct][i >> 2][i & 3] * scale2;
      if (!full) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = key0 + (i >> 2) * 16 + g * 4 + (i & 3) <= last[ct] ? x[i] : -INFINITY;
      }
      float mx = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
      if (__any(mx - m[ct] > Headroom<T>::slack)) {             // (the difference is exact where the scores are far from 0)
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
        x[i] = __builtin_amdgcn_exp2f(x[i] - mr + Headroom<T>::lift);
        l[ct] += x[i];
      }
      split(x, p[ct], rest[ct]);
    }
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
        odd |= clear_odd<T>(vf[et].x, keep[0]);
        odd |= clear_odd<T>(vf[et].y, keep[1]);
        odd |= clear_odd<T>(vf[et].z, keep[2]);
        odd |= clear_odd<T>(vf[et].w, keep[3]);
        __builtin_amdgcn_sched_barrier(0);                      // (one tile after the other: their temporaries share registers)
      }
      if (__any(odd != 0)) {
        if (!had_odd)
          for (int i = lane; i < 16 * CT * (HD + 4); i += 64) (&lds.o[wave][0][0])[i] = 0.f;
        had_odd = true;
        x8 seen[CT];
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
          for (int i = 0; i < 8; ++i) seen[ct][i] = key0 + (i >> 2) * 16 + g * 4 + (i & 3) <= last[ct] ? (T)1.f : (T)0.f;
#pragma unroll 1
        for (int et = 0; et < ET; ++et) {
          uint4 v = *reinterpret_cast<const uint4*>(V + at_here + (et * 64 + lane) * 8);
          v.x &= keep[0]; v.y &= keep[1]; v.z &= keep[2]; v.w &= keep[3];
          const uint4 kinds = make_uint4(odd_kinds<T>(v.x), odd_kinds<T>(v.y), odd_kinds<T>(v.z), odd_kinds<T>(v.w));
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) {
            const f32x4 count = mma(__builtin_bit_cast(x8, kinds), seen[ct], f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
            for (int i = 0; i < 4; ++i) lds.o[wave][ct * 16 + j][et * 16 + g * 4 + i] += odd_value(count[i]);
          }
        }
      }
    }
#pragma unroll
    for (int et = 0; et < ET; ++et)
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        o[ct][et] = mma(__builtin_bit_cast(x8, vf[et]), rest[ct], o[ct][et]);
        o[ct][et] = mma(__builtin_bit_cast(x8, vf[et]), p[ct], o[ct][et]);
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
template <typename T, int HD, int CT>
__global__ __launch_bounds__(256, 2) void k_paged_rows(stairs_paged_cache c, stairs_paged_attn a, Span sp, float scale2) {
  __shared__ RowsLds<HD, CT> lds;
  attend_rows<T, HD, CT>(c, a, sp, scale2, lds);
}

// ---- many columns: tiles of 128 columns, keys and values shared through LDS ------------------------------------------
// Bound by the matrix units and by the exponentials beside them.  A wave has 32 columns, the work-group's four waves read 64
// keys at a time, copied to LDS while the 64 before are used.  On the 32 x 32 instruction the tiled page layout fits as it is: a
// lane's 16 scores of 32 keys are two operands of the value product (keys 4 h + i and 16 + 4 h + i, and 8 further, of lane
// half h), whose other operand is one 16-byte read of a value tile.  (2048 rows that end at 8200, 32 heads of 128 on 8 key heads: 233 ..
// 249 us by card, 970 .. 1030 TFLOP/s, where a bf16 product of 8192^3 reaches 1181; 2048 rows alone 53.8 us = 640, 256 rows that end at 8000 56.8 =
// 580: partial results of pieces and their joins.)
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
template <typename T, int HD>
__device__ __forceinline__ void attend_chunk(const stairs_paged_cache& c, const stairs_paged_attn& a, const Span& sp, float scale2, ChunkLds<HD>& lds) {
  typedef typename Elem<T>::x8 x8;
  constexpr int KS = HD / 16, DT = HD / 32;                     // steps of 16 dims, tiles of 32 dims
  Piece w;
  if (!find_piece(c, a, sp, w)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 31, h = lane >> 5;
  const int G = a.n_heads / c.n_kv_heads, cols = w.rows * G, col0 = w.group * kChunkCols, wcol = col0 + wave * 32;
  const int limit = a.max_blocks * c.page_size, pos0 = w.len - w.rows;
  // last positions that the work-group's, the wave's and the lane's columns see
  const int last_group = min(pos0 + (min(cols, col0 + kChunkCols) - 1) / G, limit - 1);
  const int first_wave = wcol < cols ? min(pos0 + wcol / G, limit - 1) : -1;
  const int last_wave = wcol < cols ? min(pos0 + (min(cols, wcol + 32) - 1) / G, limit - 1) : -1;
  const int col = wcol + n, row = col < cols ? col / G : 0;
  const int last = col < cols ? min(pos0 + row, limit - 1) : -1;
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
  auto request = [&](int u, int buf) {                          // (a block without a page: another's bytes, masked below)
    const int b = wave >> 1, key = u * kChunkUnit + b * 32;
    const T* src = pool + (size_t)max(page_of(u, b), 0) * page_elems + (size_t)(key & (c.page_size - 1)) * HD;
#pragma unroll
    for (int i = 0; i < HD / 16; ++i) copy_tile(src, i * 1024, &lds.tile[buf][b][wave & 1][i * 64], lane * 16);
  };
  __syncthreads();
  if (w.u0 < u1) {
    fetch_pages(w.u0);
    request(w.u0, w.u0 & 1);
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
  }
#pragma unroll 1
  for (; u < u1; ++u) {
    const int key0 = u * kChunkUnit;
    next_unit();
    if (key0 > last_wave) continue;                             // (nothing for this wave any more)
    f32x16 s[2];
    x8 p[2][2];
    scores(s);
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      const int key = key0 + (i >> 4) * 32 + (i >> 2 & 3) * 8 + h * 4 + (i & 3);
      float& x = reinterpret_cast<float*>(&s[i >> 4])[i & 15];
      x = key <= last && (i < 16 ? page0 : page1) >= 0 ? x : -INFINITY;
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
          for (int i = 0; i < 8; ++i) seen[i] = key + (i >> 2) * 16 + (i & 3) <= mine ? (T)1.f : (T)0.f;
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
  if (w.pieces == 1) {
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
template <typename T, int HD>
__global__ __launch_bounds__(256, 2) void k_paged_chunk(stairs_paged_cache c, stairs_paged_attn a, Span sp, float scale2) {
  __shared__ ChunkLds<HD> lds;
  attend_chunk<T, HD>(c, a, sp, scale2, lds);
}
// both in one launch: the chunks' work-groups first, the few rows of the others where there is room (2 chunks of 509 rows among 22
// sequences of 3, 90 .. 5000 positions, 16 heads of 128: 79 us = 3.3 TB/s)
template <typename T, int HD>
__global__ __launch_bounds__(256, 2) void k_paged_mixed(stairs_paged_cache c, stairs_paged_attn a, Span chunk, Span rows, float scale2) {
  __shared__ union { ChunkLds<HD> chunk; RowsLds<HD, 2> rows; } lds;
  if ((int)blockIdx.x < rows.first_block) attend_chunk<T, HD>(c, a, chunk, scale2, lds.chunk);
  else attend_rows<T, HD, 2>(c, a, rows, scale2, lds.rows);
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

bool cache_ok(const stairs_paged_cache* c) {
  if (!c || (c->dtype != STAIRS_DTYPE_BF16 && c->dtype != STAIRS_DTYPE_FP16)) return false;
  if (c->page_size != 32 && c->page_size != 64 && c->page_size != 128 && c->page_size != 256) return false;
  if (c->head_dim != 64 && c->head_dim != 128) return false;
  if (c->n_kv_heads < 1 || c->n_kv_heads > 4096 || c->n_pages < 1 || (int64_t)c->n_pages * c->page_size > INT32_MAX) return false;
  return c->k && c->v && aligned16(c->k) && aligned16(c->v);
}

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

bool attn_sizes_ok(const stairs_paged_cache* c, const stairs_paged_attn* a) {
  if (!cache_ok(c) || !a) return false;
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
  if (!cache_ok(c) || !a || a->rows < 0 || a->rows > kMostGroups * kAppendRows || a->n_heads < 0 || a->n_heads > 4096) return STAIRS_EINVAL;
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
  by_type(c, [&](auto type, auto hd) {
    hipLaunchKernelGGL((k_paged_append<decltype(type), decltype(hd)::value>), dim3(tiles, groups, tiles * groups < 2 * kCus ? 3 : 1), dim3(256), 0, st, *c, r, log2_theta);
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
    l.chunks = Span{l.ct ? kFewCols + 1 : 1, INT32_MAX, kChunkCols, kChunkUnit, kSlots, 8, 400, 0, 0, 0};
    add(l.chunks);
  }
  if (l.ct) {
    // pieces of 4 units and more: shorter ones cost more to join than they save (8000 keys of 8 heads alone: 25 us with 2, 19 with 4)
    l.rows = Span{1, l.chunk ? kFewCols : INT32_MAX, 16 * l.ct, kRowUnit, kSlots, 4, 200, 0, most_pieces(kSlots), 0};
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
  if (!a->workspace || !aligned16(a->workspace)) return STAIRS_EINVAL;
  const Launch l = plan_attention(c, a);
  if (l.grid > kMostGroups) return STAIRS_EINVAL;
  if (a->workspace_bytes < l.work_bytes) return STAIRS_ECAPACITY;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (const int rc = check_stream(st)) return rc;
  const float scale2 = (a->scale > 0.f ? a->scale : 1.0f / sqrtf((float)c->head_dim)) * kLog2e;
  by_type(c, [&](auto type, auto hd) {
    typedef decltype(type) T;
    constexpr int HD = decltype(hd)::value;
    const dim3 grid((unsigned)l.grid), block(256);
    if (l.chunk && l.ct) hipLaunchKernelGGL((k_paged_mixed<T, HD>), grid, block, 0, st, *c, *a, l.chunks, l.rows, scale2);
    else if (l.chunk) hipLaunchKernelGGL((k_paged_chunk<T, HD>), grid, block, 0, st, *c, *a, l.chunks, scale2);
    else if (l.ct == 1) hipLaunchKernelGGL((k_paged_rows<T, HD, 1>), grid, block, 0, st, *c, *a, l.rows, scale2);
    else hipLaunchKernelGGL((k_paged_rows<T, HD, 2>), grid, block, 0, st, *c, *a, l.rows, scale2);
  });
  return launched();
}
