// Drawing tokens from rows of logits with temperature, top-k, top-p and min-p from given uniform numbers
// (stairs_sample_device), and the same cut applied to the rows of the sampled generation path (launch_truncate).
//
// Tokens are ordered by (logit, index); what the rules keep is a prefix of that order, and its end a key (the logit's bits in an
// order-preserving form) with, among equal logits, an index.  A histogram over the distance from the largest logit (1/64 of a
// temperature a bin), by count or by weight, says how far down it can be; the tokens down to there are listed and sorted, and
// the draw is made among them.  For top-k up to a work-group's threads the histogram is of each thread's largest logit
// alone: the k-th of these is not above the k-th of all.  Where the list would be too long (flat rows, equal logits by the thousand) the
// end is found in one bin, or by radix selection, and the draw goes over the row.  Weights are multiples of 2^-44 of the largest,
// held in 64-bit integers: their sums do not depend on the order of additions, so neither the histograms' atomics nor the
// split of a row over threads change a result, and equal borders are equal.  Against sums in double a border moves by 2^-45 of the largest
// weight for each token at most: about sqrt(V) of them where their roundings differ (1e-11 of the whole), all where logits are equal and round alike
// (4e-9 of 128255, 1.5e-8 of the largest vocabulary; a 24-bit random number's step is 6e-8).  Tokens below 2^-45 of the largest weigh nothing in
// the sums: they count as kept and are not drawn.
//
// A row is one work-group's, read from memory once: up to 140 KiB of it stay in LDS beside the histogram.  Bound by
// latencies (a dozen steps that wait for each other: 1 row of 32000 floats with all rules 16 .. 22 us by inputs, 320 rows of 32000
// bfloat16 with top-k and top-p 31), and with top-p alone by the exponentials in double, one a logit (64 rows of 128255 floats 95 .. 175
// us by inputs, 42 of them for a row's histogram by weight).  Without rules a row of 32000 takes 25 us and 8 of 128255 take 68, at
// temperature 0 12 and 35.  Several work-groups a row, joined over three launches, gained 14 % with top-p alone and cost 40 % where
// top-k is in front.
#include "../../include/stairs.h"
#include "stairs_device.h"

#include <type_traits>

namespace stairs {
namespace {

typedef unsigned long long u64;
constexpr int kBinBits = 11, kBins = 1 << kBinBits;
constexpr int kList = 1024;                        // tokens that are listed
constexpr int kAllListed = 16384;                  // tokens in question that a row from memory is read for once
constexpr int kRanked = 512;                       // ... and sorted by counting
constexpr int kShort = 128;                        // ... and cut by every wave for itself
constexpr double kOne = 17592186044416.0;          // 2^44: the weight of the largest logit

// Order-preserving keys: larger logit, larger key; -0 and +0 alike; NaN and -infinity are key 0 (never kept, never counted).
template <typename T> struct Logit;
template <> struct Logit<float> {
  static constexpr int kBits = 32;
  static __device__ __forceinline__ float value(float x) { return x; }
};
template <> struct Logit<uint16_t> {               // bfloat16
  static constexpr int kBits = 16;
  static __device__ __forceinline__ float value(uint16_t x) { return bf16_bits_to_float(x); }
};
template <> struct Logit<_Float16> {
  static constexpr int kBits = 32;                 // (as float: 19 bits of the key differ)
  static __device__ __forceinline__ float value(_Float16 x) { return (float)x; }
};
template <typename T>
__device__ __forceinline__ uint32_t key_of(float x) {
  if (!(x > -INFINITY)) return 0;
  const uint32_t b = __float_as_uint(x + 0.f);
  const uint32_t k = b ^ ((b >> 31) ? 0xFFFFFFFFu : 0x80000000u);
  return Logit<T>::kBits == 16 ? k >> 16 : k;
}

struct Row {
  float max;
  double inv_temp;
  float bins;                                      // bins of the distance histogram to one of the logit
};
// a logit's bin: larger logits never a later one
__device__ __forceinline__ int bin_of(float x, const Row& r) { return x == r.max ? 0 : (int)fminf((r.max - x) * r.bins, (float)(kBins - 1)); }
constexpr float kBinsPerNat = kBins / 32.f;        // weights below e^-32 are 0 in multiples of 2^-44
// logarithm of the weight: 0 for the largest logits; where those are infinite nothing else has any
__device__ __forceinline__ double exponent(float x, const Row& r) {
  if (r.max == INFINITY) return x == INFINITY ? 0.0 : -INFINITY;
  return ((double)x - (double)r.max) * r.inv_temp;
}
constexpr double kNoWeight = -745.13321910194118;  // -1075 ln 2: below it a weight is 0 in double

// exp(d) for d <= 0 in multiples of 2^-44.  d = n ln 2 + r with |r| <= ln 2 / 2; exp(r / 4) by its series up to the 8th power (the next
// term is 8e-16), squared twice; the number and the place of its last bit come from one multiply-add.
__device__ __forceinline__ u64 fixed_exp(double d) {
  d = fmax(d, -64.0);                              // (weights below 2^-45 are 0 in multiples of 2^-44; NaN is the least too)
  const double big = 6755399441055744.0;           // 1.5 * 2^52: adding it rounds to a whole number
  const double nb = fma(d, 1.4426950408889634074, big), n = nb - big;
  const double x = fma(n, -0.17328679513998632735, 0.25 * d);   // ln 2 / 4
  double p = 1.0 / 40320;
  p = fma(p, x, 1.0 / 5040);
  p = fma(p, x, 1.0 / 720);
  p = fma(p, x, 1.0 / 120);
  p = fma(p, x, 1.0 / 24);
  p = fma(p, x, 1.0 / 6);
  p = fma(p, x, 0.5);
  p = fma(p, x, 1.0);
  p = fma(p, x, 1.0);
  p *= p;
  p *= p;
  const int e = (int)(uint32_t)__double_as_longlong(nb);        // n, in the low bits
  const double scale = __longlong_as_double((long long)(1023 + 44 + e) << 52);
  return (u64)__double_as_longlong(fma(p, scale, 4503599627370496.0)) & 0xFFFFFFFFFFFFFull;   // + 2^52
}
__device__ __forceinline__ u64 weight(float x, const Row& r) { return fixed_exp(exponent(x, r)); }

__device__ __forceinline__ u64 wave_sum_u64(u64 v) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off);
  return v;
}
__device__ __forceinline__ u64 wave_scan_u64(u64 v) {              // inclusive, by lane
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const u64 o = __shfl_up(v, off);
    if (lane >= off) v += o;
  }
  return v;
}

// A work-group of NT threads; CACHE bytes of the row in LDS, or up to ALL tokens of it.  Small vocabularies take small work-groups,
// several to a CU.
template <int NT, int CACHE, int ALL>
struct Lds {
  static constexpr int kThreads = NT, kWaves = NT / 64, kCache = CACHE, kAll = ALL;
  alignas(16) unsigned char row[CACHE];
  u64 all[ALL];                                    // rows that are not in LDS: the tokens in question, unsorted
  union {
    u64 bin[kBins];                                // histogram
    struct {
      u64 order[kList], other[kRanked];            // listed tokens, (key, index from the end)
      u64 weight[kShort];
    } list;
  };
  u64 piece[64];
  u64 part[kWaves], part2[kWaves];
  u64 found[3];
  float fpart[kWaves];
  int count;
};

// the row's values, from LDS or from memory
template <typename T, typename L, bool CACHED>
struct Values {
  typedef T Type;
  typedef L Shared;
  static constexpr bool kCached = CACHED;
  const T* x;
  const L* lds;
  __device__ __forceinline__ float operator[](int v) const {
    if constexpr (CACHED) return Logit<T>::value(reinterpret_cast<const T*>(lds->row)[v]);
    else return Logit<T>::value(x[v]);
  }
};
// f(v, value) for the thread's share of the indices begin .. end, in no order; several loads at a time, more where they come from memory
template <int U, typename X, typename F>
__device__ __forceinline__ void walk(const X& x, int begin, int end, int step, F f) {
  int v = begin;
  for (; v + (U - 1) * step < end; v += U * step) {
    float a[U];
#pragma unroll
    for (int i = 0; i < U; ++i) a[i] = x[v + i * step];
#pragma unroll
    for (int i = 0; i < U; ++i) f(v + i * step, a[i]);
  }
  for (; v < end; v += step) f(v, x[v]);
}
template <int U = 8, typename X, typename F>
__device__ __forceinline__ void each(const X& x, int V, F f) {
  walk<X::kCached ? 4 : U>(x, threadIdx.x, V, X::Shared::kThreads, f);
}
__device__ __forceinline__ uint32_t index_of(u64 entry) { return 0xFFFFFFFFu - (uint32_t)entry; }
__device__ __forceinline__ float value_of_key(uint32_t k, int bits) {
  if (bits == 16) k = (k << 16) | ((k >> 15) ? 0u : 0xFFFFu);
  return __uint_as_float(k >> 31 ? k ^ 0x80000000u : ~k);
}
// ... of the n tokens in s.all
template <int B, typename L, typename F>
__device__ __forceinline__ void each_listed(int n, const L& s, F f) {
  for (int i = threadIdx.x; i < n; i += L::kThreads) {
    const u64 e = s.all[i];
    f((int)index_of(e), value_of_key((uint32_t)(e >> 32), B));
  }
}

template <typename L>
__device__ u64 block_sum(u64 v, L& s) {
  v = wave_sum_u64(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s.part[threadIdx.x >> 6] = v;
  __syncthreads();
  u64 t = 0;
  for (int w = 0; w < L::kWaves; ++w) t += s.part[w];
  return t;
}
template <typename L>
__device__ float block_max(float v, L& s) {
  v = wave_max(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s.fpart[threadIdx.x >> 6] = v;
  __syncthreads();
  for (int w = 0; w < L::kWaves; ++w) v = fmaxf(v, s.fpart[w]);
  return v;
}
// sum of the threads in front
template <typename L>
__device__ u64 block_before(u64 v, L& s) {
  const u64 to = wave_scan_u64(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 63) s.part[threadIdx.x >> 6] = to;
  __syncthreads();
  u64 before = to - v;
  for (int w = 0; w < (int)(threadIdx.x >> 6); ++w) before += s.part[w];
  return before;
}

// Of the histogram's n bins, in order (DOWN: from the last): the first at which `over` and the bins so far reach the target ->
// s.found[0], what is in front of it -> s.found[1]; s.found[0] is n if none does
template <bool DOWN, typename L>
__device__ void find_bin(int n, u64 over, u64 target, L& s) {
  const int per = (n + L::kThreads - 1) / L::kThreads, first = threadIdx.x * per;
  if (threadIdx.x == 0) s.found[0] = n;
  u64 mine = 0;
  for (int i = first; i < min(first + per, n); ++i) mine += s.bin[DOWN ? n - 1 - i : i];
  u64 before = over + block_before(mine, s);
  if (before < target && before + mine >= target) {
    for (int i = first; i < min(first + per, n); ++i) {
      const u64 b = s.bin[DOWN ? n - 1 - i : i];
      if (before < target && before + b >= target) {
        s.found[0] = (u64)(DOWN ? n - 1 - i : i);
        s.found[1] = before;
      }
      before += b;
    }
  }
  __syncthreads();
}
template <typename L>
__device__ __forceinline__ void clear_bins(int n, L& s) {
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += L::kThreads) s.bin[i] = 0;
  __syncthreads();
}

// Histogram of the keys' leading bits: all lanes of a wave in one bin (masked logits, say) are one addition
template <typename L>
__device__ __forceinline__ void add_to_bin(uint32_t bin, u64 m, L& s) {
  const uint32_t first = __builtin_amdgcn_readfirstlane(bin);
  const bool same = bin == first;
  if (__all(same)) {
    const unsigned long long lanes = __ballot(true);
    u64 sum = 0;
    if (__all(m == 1)) sum = (u64)__popcll(lanes);
    else if (lanes == ~0ull) sum = wave_sum_u64(m);
    else {
      if (m) atomicAdd(&s.bin[bin], m);
      return;
    }
    if ((threadIdx.x & 63) == (unsigned)__builtin_ctzll(lanes)) atomicAdd(&s.bin[bin], sum);
  } else if (m) {
    atomicAdd(&s.bin[bin], m);
  }
}

// The lowest index v with (measure of the indices <= v) > target, or V; measure(v) of a token.  The row is cut into a piece a wave,
// the piece found likewise, until a wave can walk it.  s.part: the waves' sums of the first cut, where the caller has them.
template <typename L, typename Measure>
__device__ int find_index(Measure measure, int V, u64 target, L& s, bool have_parts) {
  int lo = 0, n = V;
  u64 before = 0;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  while (n > 64) {
    const int piece = (n + L::kWaves - 1) / L::kWaves;
    if (!have_parts) {
      u64 m = 0;
      for (int i = lane; i < piece; i += 64) {
        const int v = wave * piece + i;
        if (v < n) m += measure(lo + v);
      }
      m = wave_sum_u64(m);
      __syncthreads();
      if (lane == 0) s.part[wave] = m;
      __syncthreads();
    }
    have_parts = false;
    int w = 0;
    for (; w < L::kWaves && before + s.part[w] <= target; ++w) before += s.part[w];
    if (w == L::kWaves) return V;
    lo += w * piece;
    n = min(piece, n - w * piece);
  }
  const u64 to = before + wave_scan_u64(lane < n ? measure(lo + lane) : 0);
  const unsigned long long over = __ballot(lane < n && to > target);
  return over ? lo + __builtin_ctzll(over) : V;
}


// The tokens of the bins first .. last among those of each_token(f) -> to, in no order, up to `most` of them; how many there are
template <typename T, typename L, typename Each>
__device__ int gather(Each each_token, const Row& r, int first, int last, u64* to, int most, L& s) {
  __syncthreads();
  if (threadIdx.x == 0) s.count = 0;
  __syncthreads();
  // Nothing below this is in those bins: a bin further than the last one's end, which outweighs the roundings of both formulas.  (One
  // comparison for nearly all tokens: 128255 gone through in 8.5 us, with every token's bin in 11.3.)
  const float least = last < kBins - 1 ? r.max - (float)(last + 2) / r.bins : -INFINITY;
  each_token([&](int v, float a) {
    if (a < least) return;                          // (not where it is NaN: temperatures without end)
    const int b = bin_of(a, r);
    if (b >= first && b <= last) {
      const uint32_t k = key_of<T>(a);
      if (k) {
        const int at = atomicAdd(&s.count, 1);
        if (at < most) to[at] = ((u64)k << 32) | (0xFFFFFFFFu - (uint32_t)v);
      }
    }
  });
  __syncthreads();
  return s.count;
}
// s.list.order[0 .. c), c <= kList, sorted, the first in front
template <typename L>
__device__ void sort_list(int c, L& s) {
  int n = 64;                                      // a power of two
  while (n < c) n *= 2;
  if (n <= kRanked && n <= L::kThreads) {
    // a token's place is the number of those in front of it, NT / n threads to a token (no two are equal); two a read
    // (320 rows of 32000, lists of up to 261: 31.6 us in all, one a read 34.4)
    if (threadIdx.x == 0) s.list.order[c] = 0;      // (for an odd one's partner)
    __syncthreads();
    const int per = L::kThreads / n, mine = threadIdx.x / per, part = threadIdx.x % per, half = (c + 1) / 2;
    const u64 a = s.list.order[mine];
    const ulonglong2* pairs = reinterpret_cast<const ulonglong2*>(s.list.order);
    int ahead = 0;
    for (int i0 = part; i0 < half; i0 += 8 * per) {   // (eight reads on their way at a time)
      ulonglong2 b[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) b[i] = pairs[min(i0 + i * per, half - 1)];
#pragma unroll
      for (int i = 0; i < 8; ++i) ahead += i0 + i * per < half ? (b[i].x > a) + (b[i].y > a) : 0;
    }
    for (int off = 1; off < per; off <<= 1) ahead += __shfl_xor(ahead, off);
    if (mine < c && part == 0) s.list.other[ahead] = a;
    __syncthreads();
    for (int i = threadIdx.x; i < c; i += L::kThreads) s.list.order[i] = s.list.other[i];
    __syncthreads();
    return;
  }
  for (int i = c + threadIdx.x; i < n; i += L::kThreads) s.list.order[i] = 0;
  __syncthreads();
  // bitonic, largest first; pairs up to 64 apart stay within the 128 entries of a wave
  for (int size = 2; size <= n; size *= 2)
    for (int gap = size / 2; gap > 0; gap /= 2) {
      for (int i = threadIdx.x; i < n / 2; i += L::kThreads) {
        const int lo = 2 * i - (i & (gap - 1)), hi = lo + gap;
        const u64 a = s.list.order[lo], b = s.list.order[hi];
        if ((a < b) == ((lo & size) == 0)) {
          s.list.order[lo] = b;
          s.list.order[hi] = a;
        }
      }
      if (gap > 64 || (gap == 1 && size >= 128)) __syncthreads();
      else asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
  __syncthreads();
}
// The largest key K with (measure of the keys >= K) >= target; *above: of the keys above it.  each_key(f): f(key, measure()) for every
// token of the row.
template <int KEYBITS, typename L, typename Each>
__device__ uint32_t select_key(Each each_key, u64 target, u64* above, L& s) {
  uint32_t prefix = 0;
  u64 over = 0;
  int below = KEYBITS;
  while (below > 0) {
    const int bits = below > 2 * kBinBits ? kBinBits : below > kBinBits ? (below + 1) / 2 : below, shift = below - bits, n = 1 << bits;
    clear_bins(n, s);
    each_key([&](uint32_t key, auto m) {
      if (below >= 32 || (key >> below) == prefix) add_to_bin((key >> shift) & (n - 1), m(), s);
    });
    __syncthreads();
    find_bin<true>(n, over, target, s);
    prefix = (below >= 32 ? 0u : prefix << bits) | (uint32_t)s.found[0];
    over = s.found[1];
    below = shift;
    __syncthreads();
  }
  *above = over;
  return prefix;
}

// What the rules keep: the tokens up to a cut, and, where they are few, the tokens themselves.
struct Cut {                       // kept: key > key, or key == key and index <= index; and exponent >= least
  uint32_t key;
  int index;
  double least;
  int listed;                      // > 0: the first so many of s.list.order; 0: not listed
  int in_all;                      // > 0: they are among the first so many of s.all
  u64 sum;                         // ... and their weight
};
__device__ __forceinline__ u64 border(float top_p, u64 z) {       // tokens with less than this in front of them stay
  const double t = ceil((double)top_p * (double)z);
  return t < 1.0 ? 1ull : (u64)t;
}

// The cut among the n listed tokens, sorted, of which the first top_k are in question; `before`: weight in front of the list; target:
// 0 to form it from the listed tokens' own weight.  Up to kShort of them every wave does it for itself.
template <int B, typename L>
__device__ Cut cut_list(int n, int top_k, float top_p, u64 before, u64 target, const Row& r, Cut c, L& s) {
  const int lane = threadIdx.x & 63, all = min(n, top_k);
  auto logit = [&](int i) { return value_of_key((uint32_t)(s.list.order[i] >> 32), B); };
  int stay;
  if (all <= kShort) {
    u64 z = 0;
    for (int i = lane; i < all; i += 64) {          // (every wave writes the same numbers, and reads its own)
      const u64 w = fixed_exp(exponent(logit(i), r));
      s.list.weight[i] = w;
      z += w;
    }
    if (top_p < 1.f && target == 0) target = border(top_p, wave_sum_u64(z));
    u64 front = before, sum = 0;
    int kept = 0;
    stay = 0;
    for (int i0 = 0; i0 < all; i0 += 64) {          // (weights do not grow along the order: what stays is a prefix)
      const int i = i0 + lane;
      const u64 w = i < all ? s.list.weight[i] : 0, to = wave_scan_u64(w);
      const bool here = i < all && (!(top_p < 1.f) || front + to - w < target), strong = here && exponent(logit(min(i, all - 1)), r) >= c.least;
      stay += __popcll(__ballot(here));
      kept += __popcll(__ballot(strong));
      if (strong) sum += w;
      front += __shfl(to, 63);
    }
    if (before == 0) {
      c.listed = kept;
      c.sum = wave_sum_u64(sum);
    }
  } else {
    constexpr int PER = kList / L::kThreads;
    u64 w[PER], mine = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int at = threadIdx.x * PER + i;
      w[i] = at < all ? fixed_exp(exponent(logit(at), r)) : 0;
      mine += w[i];
    }
    u64 front = before + block_before(mine, s), z = 0, here = 0, strong = 0, sum = 0;
    for (int k = 0; k < L::kWaves; ++k) z += s.part[k];
    if (top_p < 1.f && target == 0) target = border(top_p, z);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int at = threadIdx.x * PER + i;
      if (at < all && (!(top_p < 1.f) || front < target)) {
        ++here;
        if (exponent(logit(at), r) >= c.least) {
          ++strong;
          sum += w[i];
        }
      }
      front += w[i];
    }
    stay = (int)block_sum(here, s);
    if (before == 0) {
      c.listed = (int)block_sum(strong, s);
      c.sum = block_sum(sum, s);
    }
  }
  const u64 last = s.list.order[stay - 1];
  c.key = (uint32_t)(last >> 32);
  c.index = (int)(0xFFFFFFFFu - (uint32_t)last);
  __syncthreads();
  return c;
}

template <typename X, typename L>
__device__ Cut find_cut(const X& x, int V, const Row& r, float mine, int top_k, float top_p, float min_p, L& s) {
  typedef typename X::Type T;
  constexpr int B = Logit<T>::kBits;
  Cut c{1u, 0x7fffffff, min_p > 0.f ? fmax(kNoWeight, log((double)fminf(min_p, 1.f))) : kNoWeight, 0, 0, 0};
  // tokens that min_p may keep are in the bins up to this one
  const int weak = (int)fmin(1.0 - c.least * (double)kBinsPerNat, (double)(kBins - 1));
  const bool by_p = top_p < 1.f;                    // (not for NaN)
  // ways to list the tokens in question, one after the other until one gives a list that is short enough (one place for each step:
  // the code runs once and comes from memory)
  enum { kThreadsLargest, kCount, kWeight, kOneBin, kWeak, kNone };
  auto behind_k = [&] { return by_p ? kWeight : weak < kBins - 1 ? kWeak : kNone; };
  int way = top_k > 0 && top_k < V ? (top_k > L::kThreads ? kCount : kThreadsLargest) : behind_k();
  bool cut_k = false;                               // top_k cuts, and found no list
  int bin = weak;
  u64 before = 0, target = 0;
  while (way != kNone) {
    if (way <= kWeight) {
      clear_bins(kBins, s);
      u64 sum = 0;
      if (way == kThreadsLargest) {
        if (mine > -INFINITY) atomicAdd(&s.bin[bin_of(mine, r)], 1ull);
      } else if (way == kCount) {
        each(x, V, [&](int, float a) { if (a > -INFINITY) add_to_bin(bin_of(a, r), 1, s); });
      } else {
        each(x, V, [&](int, float a) {
          const u64 w = weight(a, r);               // (0 for NaN and -infinity)
          sum += w;
          if (w) atomicAdd(&s.bin[bin_of(a, r)], w);
        });
      }
      __syncthreads();
      if (way == kWeight) target = border(top_p, block_sum(sum, s));
      find_bin<false>(kBins, 0, way == kWeight ? target : (u64)top_k, s);
      bin = (int)s.found[0];
      before = s.found[1];
      if (bin == kBins) {                           // so many there are not: of the threads' largest, or of all
        way = way == kThreadsLargest ? kCount : behind_k();
        bin = weak;
        continue;
      }
    }
    // (under top_k with top_p all of the first top_k count, else what min_p keeps of them)
    const int first = way == kOneBin ? bin : 0, last = way == kOneBin || (way < kWeight && by_p) ? bin : min(bin, weak);
    int n;
    if (L::kAll == 0 || (way == kOneBin && !c.in_all)) {
      n = gather<T>([&](auto f) { each(x, V, f); }, r, first, last, s.list.order, kList, s);
    } else {
      // a row that is read from memory is read once for all tokens in question
      if (way != kOneBin) {
        n = gather<T>([&](auto f) { each(x, V, f); }, r, first, last, s.all, L::kAll, s);
        c.in_all = n <= L::kAll ? n : 0;
      }
      n = c.in_all ? gather<T>([&](auto f) { each_listed<B>(c.in_all, s, f); }, r, first, last, s.list.order, kList, s) : kList + 1;
    }
    if (n <= kList) {
      sort_list(n, s);
      return cut_list<B>(n, way < kWeight ? top_k : n, way == kWeak ? 1.f : top_p, way == kOneBin ? before : 0, way < kWeight ? 0 : target, r, c, s);
    }
    // (all that min_p keeps is in s.all, and top_p's border, where there is one, behind it)
    if (c.in_all && (way == kWeak || (way == kWeight && weak < bin))) return c;
    cut_k = way == kCount;
    way = way == kThreadsLargest ? kCount : way == kWeight ? kOneBin : kNone;
  }
  // flat rows: bit by bit
  c.in_all = 0;
  auto keys = [&](auto f) {
    each(x, V, [&](int, float a) {
      const uint32_t k = key_of<T>(a);
      if (k) f(k, a);
    });
  };
  u64 ties = ~0ull;                                 // kept of the tokens with key c.key, where c.index does not say it
  if (cut_k) {
    u64 above;
    c.key = select_key<B>([&](auto f) { keys([&](uint32_t k, float) { f(k, [] { return 1ull; }); }); }, (u64)top_k, &above, s);
    ties = (u64)top_k - above;
  }
  if (by_p) {
    u64 sum = 0, tie = 0;                           // weight of the first top_k; of one of the last of them
    keys([&](uint32_t k, float a) {
      if (!cut_k || k > c.key) sum += weight(a, r);
      else if (k == c.key) tie = weight(a, r);
    });
    u64 z = block_sum(sum, s);
    if (cut_k) {
      if (threadIdx.x == 0) s.found[2] = 0;
      __syncthreads();
      if (tie) s.found[2] = tie;                    // (equal logits, equal weights: whoever writes)
      __syncthreads();
      z += ties * s.found[2];
    }
    target = border(top_p, z);
    u64 above;
    const uint32_t key = select_key<B>([&](auto f) { keys([&](uint32_t k, float a) { f(k, [&] { return weight(a, r); }); }); }, target, &above, s);
    // of the equal logits at the border those with less than the target in front of them
    u64 w = 0;
    keys([&](uint32_t k, float a) { if (k == key) w = weight(a, r); });
    __syncthreads();
    if (threadIdx.x == 0) s.found[2] = 1;
    __syncthreads();
    if (w) s.found[2] = w;
    __syncthreads();
    const u64 stay = (target - above + s.found[2] - 1) / s.found[2];
    if (key > c.key || !cut_k) ties = stay;
    else ties = min(ties, stay);
    c.key = key;
  }
  if (ties != ~0ull) c.index = find_index([&](int v) { return key_of<T>(x[v]) == c.key ? 1ull : 0ull; }, V, ties - 1, s, false);
  return c;
}

template <typename T>
__device__ __forceinline__ bool is_kept(float a, int v, const Cut& c, const Row& r) {
  // (by value: 8 rows of 128255 without rules 67.4 us, by key 71.5; where nothing is cut -infinity is left out by its exponent)
  const float last = c.key > 1 ? value_of_key(c.key, Logit<T>::kBits) : -INFINITY;
  return (a > last || (a == last && v <= c.index)) && exponent(a, r) >= c.least;
}

// The same for up to 64 tokens, a lane of the first wave each, for that wave alone (0 in the others): a token's sum is formed by
// comparing its index with all (7 tokens 1.1 us, in steps of six bits of the index 3.8)
template <typename L, typename Weight>
__device__ int draw_from_wave(int n, Weight weight_of_key, u64 target, L& s) {
  const int lane = threadIdx.x;
  if (lane >= 64) return 0;
  const u64 e = lane < n ? s.list.order[lane] : 0;
  const uint32_t v = index_of(e);
  const u64 w = lane < n ? weight_of_key((uint32_t)(e >> 32)) : 0;
  u64 to = 0;
  for (int j = 0; j < n; ++j) {
    const u64 x = (u64)(uint32_t)__builtin_amdgcn_readlane((int)(w >> 32), j) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)w, j);
    if ((uint32_t)__builtin_amdgcn_readlane((int)v, j) <= v) to += x;
  }
  uint32_t found = lane < n && to > target ? v : 0xFFFFFFFFu;
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) found = min(found, (uint32_t)__shfl_xor((int)found, off));
  return (int)found;
}
// The lowest index among listed tokens at which their weights, by index, exceed the target: six bits of the index at a time, the
// weights of the tokens with the bits found so far summed by the next six.  each_weight(f): f(index, weight) for every token.
template <typename L, typename Each>
__device__ int draw_listed(Each each_weight, int V, u64 target, L& s) {
  const int lane = threadIdx.x & 63;
  uint32_t found = 0;
  u64 before = 0;
  for (int shift = (31 - __builtin_clz(V | 1)) / 6 * 6; shift >= 0; shift -= 6) {
    if (threadIdx.x < 64) s.piece[lane] = 0;
    __syncthreads();
    each_weight([&](uint32_t v, auto w) {
      if ((v >> shift >> 6) == found) {
        const u64 x = w();
        if (x) atomicAdd(&s.piece[(v >> shift) & 63], x);
      }
    });
    __syncthreads();
    const u64 p = s.piece[lane], to = before + wave_scan_u64(p);
    const int l = __builtin_ctzll(__ballot(to > target));
    before = __shfl(to, l) - __shfl(p, l);
    found = found << 6 | (uint32_t)l;
    __syncthreads();
  }
  return (int)found;
}

// the row into LDS, where it fits, its maximum and the thread's own
template <bool CACHED, typename T, typename L>
__device__ float load_row(const T* x, int V, float* mine, L& s) {
  float m = -INFINITY;
  T* row = reinterpret_cast<T*>(s.row);
  constexpr int U = 16;
  for (int v0 = threadIdx.x; v0 < V; v0 += U * L::kThreads) {
    T a[U];
#pragma unroll
    for (int i = 0; i < U; ++i) a[i] = x[min(v0 + i * L::kThreads, V - 1)];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int v = v0 + i * L::kThreads;
      if (v >= V) continue;                        // (a logit is one thread's: find_cut counts on it)
      if constexpr (CACHED) row[v] = a[i];
      m = fmaxf(m, Logit<T>::value(a[i]));
    }
  }
  *mine = m;
  return block_max(m, s);
}

template <typename T, int NT, int CACHE, bool CACHED>
__global__ __launch_bounds__(NT) void k_sample_rows(stairs_sampling a) {
  typedef Lds<NT, CACHE, CACHED ? 0 : kAllListed> L;
  __shared__ L s;
  const int row = blockIdx.x, V = a.vocab;
  const T* p = static_cast<const T*>(a.logits) + (size_t)row * a.ld;
  const Values<T, L, CACHED> x{p, &s};
  const float t = a.temperature ? a.temperature[row] : 1.f;
  const int top_k = a.top_k ? a.top_k[row] : 0;
  const float top_p = a.top_p ? a.top_p[row] : 1.f, min_p = a.min_p ? a.min_p[row] : 0.f, uniform = a.uniform ? a.uniform[row] : 0.f;
  float mine;
  Row r{load_row<CACHED>(p, V, &mine, s), fmax(1.0 / (double)t, 1e-300), kBinsPerNat / t};   // (an infinite temperature: all finite logits alike)
  int token = -1, kept = 0;
  float lp = -INFINITY;
  if (r.max == -INFINITY) {
  } else if (!(t > 0.f)) {
    token = find_index([&](int v) { return x[v] == r.max ? 1ull : 0ull; }, V, 0, s, false);
    kept = 1;
    lp = 0.f;
  } else {
    const Cut c = find_cut(x, V, r, mine, top_k, top_p, min_p, s);
    // (the lowest index whose sum exceeds u z: the sums are whole numbers, so it exceeds floor(u z) too; u below 1 by 2^-24 at
    // least, u z below z by one at least; a u outside [0, 1) or not a number is brought inside)
    const double u = fmin(fmax((double)uniform, 0.0), 1.0);
    auto target_of = [&](u64 z) { return min((u64)(u * (double)z), z - 1); };
    u64 z = 0, n = 0;
    if (c.listed > 0) {
      z = c.sum;
      kept = c.listed;
      constexpr int B = Logit<T>::kBits;
      if (c.listed <= 64) token = draw_from_wave(c.listed, [&](uint32_t key) { return weight(value_of_key(key, B), r); }, target_of(z), s);
      else token = draw_listed([&](auto f) {
        for (int i = threadIdx.x; i < c.listed; i += L::kThreads) {
          const u64 e = s.list.order[i];
          f(index_of(e), [&] { return weight(value_of_key((uint32_t)(e >> 32), B), r); });
        }
      }, V, target_of(z), s);
    } else if (L::kAll > 0 && c.in_all) {
      constexpr int B = Logit<T>::kBits;
      each_listed<B>(c.in_all, s, [&](int v, float b) {
        if (is_kept<T>(b, v, c, r)) {
          z += weight(b, r);
          ++n;
        }
      });
      z = block_sum(z, s);
      kept = (int)block_sum(n, s);
      token = draw_listed([&](auto f) {
        each_listed<B>(c.in_all, s, [&](int v, float b) {
          if (is_kept<T>(b, v, c, r)) f((uint32_t)v, [&] { return weight(b, r); });
        });
      }, V, target_of(z), s);
    } else {
      // weight and number of what is kept, a piece of the row a wave (find_index's first cut)
      const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
      const int piece = V > 64 ? (V + L::kWaves - 1) / L::kWaves : V, begin = wave * piece, end = min(V, begin + piece);
      auto add = [&](int v, float b) {
        if (is_kept<T>(b, v, c, r)) {
          z += weight(b, r);
          ++n;
        }
      };
      walk<CACHED ? 4 : 8>(x, begin + lane, end, 64, add);
      z = wave_sum_u64(z);
      n = wave_sum_u64(n);
      __syncthreads();
      if (lane == 0) {
        s.part[wave] = z;
        s.part2[wave] = n;
      }
      __syncthreads();
      z = n = 0;
      for (int w = 0; w < L::kWaves; ++w) {
        z += s.part[w];
        n += s.part2[w];
      }
      kept = (int)n;
      token = find_index([&](int v) {
        const float b = x[v];
        return is_kept<T>(b, v, c, r) ? weight(b, r) : 0ull;
      }, V, target_of(z), s, true);
    }
    double log_z = log((double)z * (1.0 / kOne));
    if ((z & ((1ull << 44) - 1)) < 1ull << 34) {
      // Perhaps little beside the largest logits (2^-10 of them): then that is summed again in multiples of 2^-44 of the largest of it
      // (2^19 tokens at most: sums stay below 2^64 however little it is), or the logarithm would be the roundings' sum.
      constexpr int B = Logit<T>::kBits;
      auto each_kept = [&](auto f) {
        if (c.listed > 0) {
          for (int i = threadIdx.x; i < c.listed; i += L::kThreads) f(value_of_key((uint32_t)(s.list.order[i] >> 32), B));
        } else if (L::kAll > 0 && c.in_all) {
          each_listed<B>(c.in_all, s, [&](int v, float b) { if (is_kept<T>(b, v, c, r)) f(b); });
        } else {
          each(x, V, [&](int v, float b) { if (is_kept<T>(b, v, c, r)) f(b); });
        }
      };
      u64 tops = 0;
      float second = -INFINITY;
      each_kept([&](float b) {
        if (b == r.max) ++tops;
        else second = fmaxf(second, b);
      });
      tops = block_sum(tops, s);
      if (z - tops * (1ull << 44) < 1ull << 34) {
        const Row low{block_max(second, s), r.inv_temp, r.bins};
        u64 rest = 0;
        each_kept([&](float b) { rest += b == r.max ? 0 : weight(b, low); });
        rest = block_sum(rest, s);
        const double share = rest ? (double)rest * (1.0 / kOne) * exp(exponent(low.max, r)) : 0.0;
        log_z = log((double)tops) + log1p(share / (double)tops);
      }
    }
    lp = (float)(exponent(x[token], r) - log_z);
  }
  if (threadIdx.x == 0) {
    a.token[row] = token;
    if (a.logprob) a.logprob[row] = lp;
    if (a.kept) a.kept[row] = kept;
  }
}

// -infinity at the tokens of rows [.., ld] of floats that the rules do not keep.  A launch a draft token and one for the main model's rows:
// with 4 draft tokens and 32000 logits an iteration is 85 .. 110 us longer (125M pair 650 -> 742 .. 749 us, 1B 1645 -> 1731 .. 1756), with top-p
// alone 215 (866, 1856).
template <int NT, int CACHE, bool CACHED>
__global__ __launch_bounds__(NT) void k_truncate(float* logits, int ld, int V, const SampleParams* sp) {
  typedef Lds<NT, CACHE, CACHED ? 0 : kAllListed> L;
  __shared__ L s;
  float* p = logits + (size_t)blockIdx.x * ld;
  const Values<float, L, CACHED> x{p, &s};
  float mine;
  const Row r{load_row<CACHED>(p, V, &mine, s), (double)sp->inv_temp, kBinsPerNat * sp->inv_temp};
  if (r.max == -INFINITY) return;
  const Cut c = find_cut(x, V, r, mine, sp->top_k, sp->top_p, sp->min_p, s);
  __syncthreads();
  each(x, V, [&](int v, float a) {
    if (!is_kept<float>(a, v, c, r)) p[v] = -INFINITY;
  });
}

// Up to 4096 logits: 256 threads, several work-groups to a CU (1, 64, 1000 rows of 4096 with top-k: 14.5, 21.4, 28.5 us, as larger ones 15.0,
// 19.8, 36.5; of 1000: 12.5, 18.9, 28.0 and 13.6, 18.6, 32.5); up to 140 KB of them: a CU's threads, or, if there are more rows than
// CUs and they take 63 KB at most, half of them for each of two work-groups (320 rows of 32000: 38 us, 44 with one); more
// is read again from L2 at every step.
constexpr int kSmallRow = 4096, kSmallThreads = 256, kSmallCache = 16384;
constexpr int kCus = 256, kHalfThreads = 512, kHalfCache = 64256;
constexpr int kLargeThreads = 1024, kLargeCache = 142848, kNoCache = 16;
static_assert(sizeof(Lds<kLargeThreads, kLargeCache, 0>) <= 160 * 1024 && sizeof(Lds<kHalfThreads, kHalfCache, 0>) <= 80 * 1024, "work-groups on a CU");

}  // namespace

// f(threads, bytes of LDS for the row, whether it fits) for rows of V logits of so many bytes; no more rows than CUs
template <typename F>
static void by_size(int V, size_t bytes, F f) {
  if (V <= kSmallRow) f(std::integral_constant<int, kSmallThreads>{}, std::integral_constant<int, kSmallCache>{}, std::true_type{});
  else if (V * bytes <= kLargeCache) f(std::integral_constant<int, kLargeThreads>{}, std::integral_constant<int, kLargeCache>{}, std::true_type{});
  else f(std::integral_constant<int, kLargeThreads>{}, std::integral_constant<int, kNoCache>{}, std::false_type{});
}
// ... any number of rows
template <typename F>
static void by_size(int rows, int V, size_t bytes, F f) {
  if (rows > kCus && V > kSmallRow && V * bytes <= kHalfCache) f(std::integral_constant<int, kHalfThreads>{}, std::integral_constant<int, kHalfCache>{}, std::true_type{});
  else by_size(V, bytes, f);
}
void launch_truncate(float* logits, int rows, int ld, int V, const SampleParams* sp, hipStream_t st) {
  by_size(V, sizeof(float), [&](auto threads, auto cache, auto cached) {
    constexpr int NT = decltype(threads)::value, C = decltype(cache)::value;
    hipLaunchKernelGGL((k_truncate<NT, C, decltype(cached)::value>), dim3(rows), dim3(NT), 0, st, logits, ld, V, sp);
  });
}

}  // namespace stairs

using namespace stairs;

static bool sampling_ok(const stairs_sampling* a) {
  if (!a || (a->dtype != STAIRS_DTYPE_FP32 && a->dtype != STAIRS_DTYPE_BF16 && a->dtype != STAIRS_DTYPE_FP16)) return false;
  return a->rows >= 0 && a->rows <= 1 << 21 && a->vocab >= 1 && a->vocab <= STAIRS_SAMPLE_MAX_VOCAB && a->ld >= a->vocab;   // (a row, 2^10 threads)
}

extern "C" int64_t stairs_sample_workspace(const stairs_sampling* a) {
  if (!sampling_ok(a)) return STAIRS_EINVAL;
  return 0;
}

extern "C" int stairs_sample_device(const stairs_sampling* a, void* hip_stream) {
  if (!sampling_ok(a)) return STAIRS_EINVAL;
  if (a->rows == 0) return STAIRS_OK;
  if (!a->logits || !a->token) return STAIRS_EINVAL;
  const size_t align = a->dtype == STAIRS_DTYPE_FP32 ? 4 : 2;
  if (reinterpret_cast<uintptr_t>(a->logits) % align) return STAIRS_EINVAL;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (const int rc = check_stream(st)) return rc;
  const dim3 grid(a->rows);
  auto launch = [&](auto type) {
    typedef decltype(type) T;
    by_size(a->rows, a->vocab, sizeof(T), [&](auto threads, auto cache, auto cached) {
      constexpr int NT = decltype(threads)::value, C = decltype(cache)::value;
      hipLaunchKernelGGL((k_sample_rows<T, NT, C, decltype(cached)::value>), grid, dim3(NT), 0, st, *a);
    });
  };
  if (a->dtype == STAIRS_DTYPE_FP32) launch(float{});
  else if (a->dtype == STAIRS_DTYPE_BF16) launch(uint16_t{});
  else launch(_Float16{});
  return hipGetLastError() == hipSuccess ? STAIRS_OK : STAIRS_EHIP;
}
