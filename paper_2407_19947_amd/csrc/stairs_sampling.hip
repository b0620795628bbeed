// Drawing tokens from rows of logits with temperature, top-k, top-p and min-p from given uniform numbers
// (stairs_sample_device), and the same cut applied to the rows of the sampled generation path (launch_truncate).
//
// Nothing is sorted.  Tokens are ordered by (logit, index); a cut is a key (the logit's bits in an order-preserving form) and,
// among equal logits, an index.  The cuts are found by radix selection: histograms of the keys' leading bits, then of the bits
// below among those with the leading bits found, by count (top-k) or by weight (top-p).  Weights are multiples of 2^-44 of the
// largest, held in 64-bit integers: their sums do not depend on the order of additions, so the atomics of the histograms and the
// split of a row over threads change no result, and equal borders are equal.  (2^-44 against sums of 1 and more: a border moves
// by about 1e-11 of the whole against sums in double; a 24-bit random number falls between the two never in practice.)
#include "../../include/stairs.h"
#include "stairs_device.h"

namespace stairs {
namespace {

typedef unsigned long long u64;
constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kBinBits = 12, kBins = 1 << kBinBits;
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

struct Shared {
  u64 bin[kBins];
  u64 part[kWaves];
  u64 found[3];
  float fpart[kWaves];
};

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
__device__ u64 block_sum(u64 v, Shared& s) {
  v = wave_sum_u64(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s.part[threadIdx.x >> 6] = v;
  __syncthreads();
  u64 t = 0;
  for (int w = 0; w < kWaves; ++w) t += s.part[w];
  return t;
}

struct Row {
  float max;
  double inv_temp;
};
__device__ __forceinline__ double weight(float x, const Row& r) {  // in double
  return x == r.max ? 1.0 : exp(((double)x - (double)r.max) * r.inv_temp);
}
__device__ __forceinline__ u64 fixed_weight(double w) { return (u64)__double2ll_rn(w * kOne); }

// The largest key K with (measure of the keys >= K) >= target, 0 < target <= measure of all; above = measure of the keys > K.
// each(f): f(key, measure) for every token of the row that takes part.
template <int KEYBITS, typename Each>
__device__ uint32_t select_key(Each each, u64 target, u64* above, Shared& s) {
  uint32_t prefix = 0;
  u64 over = 0;
  int below = KEYBITS;                              // bits of the key not decided yet
  while (below > 0) {
    const int bits = below > kBinBits ? (below - kBinBits < 8 ? (below + 1) / 2 : kBinBits) : below;
    const int shift = below - bits, n = 1 << bits;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kThreads) s.bin[i] = 0;
    __syncthreads();
    each([&](uint32_t key, u64 m) {
      if (below < 32 && (key >> below) != prefix) return;
      if (m) atomicAdd(&s.bin[(key >> shift) & (n - 1)], m);
    });
    __syncthreads();
    // bins from the top: a thread's share, then the sum in front of it
    const int per = (n + kThreads - 1) / kThreads, first = threadIdx.x * per;
    u64 mine = 0;
    for (int i = first; i < min(first + per, n); ++i) mine += s.bin[n - 1 - i];
    u64 to = wave_scan_u64(mine);
    if ((threadIdx.x & 63) == 63) s.part[threadIdx.x >> 6] = to;
    __syncthreads();
    u64 before = over + to - mine;
    for (int w = 0; w < (int)(threadIdx.x >> 6); ++w) before += s.part[w];
    if (before < target && before + mine >= target) {
      for (int i = first; i < min(first + per, n); ++i) {
        const u64 b = s.bin[n - 1 - i];
        if (before < target && before + b >= target) {
          s.found[0] = (u64)(n - 1 - i);
          s.found[1] = before;
        }
        before += b;
      }
    }
    __syncthreads();
    prefix = (below < 32 ? prefix << bits : 0u) | (uint32_t)s.found[0];
    over = s.found[1];
    below = shift;
  }
  *above = over;
  return prefix;
}

// The lowest index v with (measure of the indices <= v) > target, or V; measure(v) of a token.  The row is cut into kWaves
// pieces, the piece found into kWaves again, until a wave can walk it.
template <typename Measure>
__device__ int find_index(Measure measure, int V, u64 target, Shared& s) {
  int lo = 0, n = V;
  u64 before = 0;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  while (n > 64) {
    const int piece = (n + kWaves - 1) / kWaves;
    u64 m = 0;
    for (int i = lane; i < piece; i += 64) {
      const int v = wave * piece + i;
      if (v < n) m += measure(lo + v);
    }
    m = wave_sum_u64(m);
    __syncthreads();
    if (lane == 0) s.part[wave] = m;
    __syncthreads();
    int w = 0;
    for (; w < kWaves && before + s.part[w] <= target; ++w) before += s.part[w];
    if (w == kWaves) return V;
    lo += w * piece;
    n = min(piece, n - w * piece);
  }
  const u64 to = before + wave_scan_u64(lane < n ? measure(lo + lane) : 0);
  const unsigned long long over = __ballot(lane < n && to > target);
  return over ? lo + __builtin_ctzll(over) : V;
}

struct Cut {                       // kept: key > key, or key == key and index <= index; and weight >= min_weight, > 0
  uint32_t key;
  int index;
  double min_weight;
};

// max of the row, then the cut of its rules
template <typename T>
__device__ float row_max(const T* x, int V, Shared& s) {
  float m = -INFINITY;
  for (int v = threadIdx.x; v < V; v += kThreads) m = fmaxf(m, Logit<T>::value(x[v]));
  m = wave_max(m);
  if ((threadIdx.x & 63) == 0) s.fpart[threadIdx.x >> 6] = m;
  __syncthreads();
  for (int w = 0; w < kWaves; ++w) m = fmaxf(m, s.fpart[w]);
  return m;
}

template <typename T>
__device__ Cut find_cut(const T* x, int V, const Row& r, int top_k, float top_p, float min_p, Shared& s) {
  constexpr int B = Logit<T>::kBits;
  Cut c{1u, 0x7fffffff, min_p > 0.f ? (double)fminf(min_p, 1.f) : 0.0};
  u64 ties = ~0ull;                                 // kept of those with key c.key
  auto keys = [&](auto f) {
    for (int v = threadIdx.x; v < V; v += kThreads) {
      const float a = Logit<T>::value(x[v]);
      const uint32_t k = key_of<T>(a);
      if (k) f(k, a);
    }
  };
  if (top_k > 0 && top_k < V) {
    u64 n = 0;
    keys([&](uint32_t, float) { ++n; });
    n = block_sum(n, s);
    if ((u64)top_k < n) {
      u64 above;
      c.key = select_key<B>([&](auto f) { keys([&](uint32_t k, float) { f(k, 1ull); }); }, (u64)top_k, &above, s);
      ties = (u64)top_k - above;
    }
  }
  if (top_p < 1.f) {                                // (not for NaN)
    u64 z = 0, tie = 0;                             // weight of the first top_k; a tie's
    keys([&](uint32_t k, float a) {
      if (k > c.key || ties == ~0ull) z += fixed_weight(weight(a, r));
      else if (k == c.key) tie = fixed_weight(weight(a, r));
    });
    z = block_sum(z, s);
    if (ties != ~0ull) {
      if (tie) s.found[2] = tie;                    // (equal logits, equal weights: whoever writes)
      else if (threadIdx.x == 0) s.found[2] = 0;
      __syncthreads();
      if (tie) s.found[2] = tie;
      __syncthreads();
      z += ties * s.found[2];
    }
    const double t = ceil((double)top_p * (double)z);
    const u64 target = t < 1.0 ? 1ull : (u64)t;
    u64 above;
    const uint32_t key = select_key<B>([&](auto f) { keys([&](uint32_t k, float a) { f(k, fixed_weight(weight(a, r))); }); }, target, &above, s);
    // of the equal logits at the border those with less than the target in front of them
    u64 w = 0;
    keys([&](uint32_t k, float a) { if (k == key) w = fixed_weight(weight(a, r)); });
    __syncthreads();
    if (threadIdx.x == 0) s.found[2] = 1;
    __syncthreads();
    if (w) s.found[2] = w;
    __syncthreads();
    const u64 stay = (target - above + s.found[2] - 1) / s.found[2];
    if (key > c.key || ties == ~0ull) ties = stay;
    else ties = min(ties, stay);
    c.key = key;
  }
  if (ties != ~0ull) {
    const int v = find_index([&](int i) { return key_of<T>(Logit<T>::value(x[i])) == c.key ? 1ull : 0ull; }, V, ties - 1, s);
    c.index = v;
  }
  return c;
}

template <typename T>
__device__ __forceinline__ bool is_kept(float a, int v, const Cut& c, const Row& r, double* w) {
  const uint32_t k = key_of<T>(a);
  if (!k || k < c.key || (k == c.key && v > c.index)) return false;
  *w = weight(a, r);
  return *w > 0.0 && *w >= c.min_weight;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_sample_rows(stairs_sampling a) {
  __shared__ Shared s;
  const int row = blockIdx.x, V = a.vocab;
  const T* x = static_cast<const T*>(a.logits) + (size_t)row * a.ld;
  const float t = a.temperature ? a.temperature[row] : 1.f;
  Row r{row_max(x, V, s), fmax(1.0 / (double)t, 1e-300)};   // (an infinite temperature: all finite logits alike)
  int token = -1, kept = 0;
  float lp = -INFINITY;
  if (r.max == -INFINITY) {
  } else if (!(t > 0.f)) {
    token = find_index([&](int v) { return Logit<T>::value(x[v]) == r.max ? 1ull : 0ull; }, V, 0, s);
    kept = 1;
    lp = 0.f;
  } else {
    const Cut c = find_cut(x, V, r, a.top_k ? a.top_k[row] : 0, a.top_p ? a.top_p[row] : 1.f, a.min_p ? a.min_p[row] : 0.f, s);
    u64 z = 0, n = 0;
    for (int v = threadIdx.x; v < V; v += kThreads) {
      double w;
      if (is_kept<T>(Logit<T>::value(x[v]), v, c, r, &w)) {
        z += fixed_weight(w);
        ++n;
      }
    }
    z = block_sum(z, s);
    n = block_sum(n, s);
    kept = (int)n;
    // (the lowest index whose sum exceeds u z: the sums are whole numbers, so it exceeds floor(u z) too; u below 1 by 2^-24 at
    // least, u z below z by one at least; a u outside [0, 1) or not a number is brought inside)
    const double u = a.uniform ? fmin(fmax((double)a.uniform[row], 0.0), 1.0) : 0.0;
    const u64 target = min((u64)(u * (double)z), z - 1);
    token = find_index([&](int v) {
      double w;
      return is_kept<T>(Logit<T>::value(x[v]), v, c, r, &w) ? fixed_weight(w) : 0ull;
    }, V, target, s);
    const float xt = Logit<T>::value(x[token]);
    lp = (float)((xt == r.max ? 0.0 : ((double)xt - (double)r.max) * r.inv_temp) - log((double)z * (1.0 / kOne)));
  }
  if (threadIdx.x == 0) {
    a.token[row] = token;
    if (a.logprob) a.logprob[row] = lp;
    if (a.kept) a.kept[row] = kept;
  }
}

// -infinity at the tokens of rows [.., ld] of floats that the rules do not keep
__global__ __launch_bounds__(kThreads) void k_truncate(float* logits, int ld, int V, const SampleParams* sp) {
  __shared__ Shared s;
  float* x = logits + (size_t)blockIdx.x * ld;
  const Row r{row_max(x, V, s), (double)sp->inv_temp};
  if (r.max == -INFINITY) return;
  const Cut c = find_cut(x, V, r, sp->top_k, sp->top_p, sp->min_p, s);
  __syncthreads();
  for (int v = threadIdx.x; v < V; v += kThreads) {
    double w;
    if (!is_kept<float>(x[v], v, c, r, &w)) x[v] = -INFINITY;
  }
}

}  // namespace

void launch_truncate(float* logits, int rows, int ld, int V, const SampleParams* sp, hipStream_t st) {
  hipLaunchKernelGGL(k_truncate, dim3(rows), dim3(kThreads), 0, st, logits, ld, V, sp);
}

}  // namespace stairs

using namespace stairs;

static const char* check_sampling(const stairs_sampling* a) {
  if (!a) return "sampling is NULL";
  const int dt = a->dtype;
  if (dt != STAIRS_DTYPE_FP32 && dt != STAIRS_DTYPE_BF16 && dt != STAIRS_DTYPE_FP16) return "unknown dtype";
  if (a->rows < 0 || a->vocab < 1 || a->vocab > STAIRS_SAMPLE_MAX_VOCAB || a->ld < a->vocab) return "rows, vocab or ld out of range";
  return nullptr;
}

extern "C" int64_t stairs_sample_workspace(const stairs_sampling* a) {
  if (check_sampling(a)) return STAIRS_EINVAL;
  return 0;
}

extern "C" int stairs_sample_device(const stairs_sampling* a, void* hip_stream) {
  if (check_sampling(a)) return STAIRS_EINVAL;
  if (a->rows == 0) return STAIRS_OK;
  if (!a->logits || !a->token) return STAIRS_EINVAL;
  const size_t align = a->dtype == STAIRS_DTYPE_FP32 ? 4 : 2;
  if (reinterpret_cast<uintptr_t>(a->logits) % align) return STAIRS_EINVAL;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (const int rc = check_stream(st)) return rc;
  const dim3 grid(a->rows), block(kThreads);
  if (a->dtype == STAIRS_DTYPE_FP32)
    hipLaunchKernelGGL(k_sample_rows<float>, grid, block, 0, st, *a);
  else if (a->dtype == STAIRS_DTYPE_BF16)
    hipLaunchKernelGGL(k_sample_rows<uint16_t>, grid, block, 0, st, *a);
  else
    hipLaunchKernelGGL(k_sample_rows<_Float16>, grid, block, 0, st, *a);
  return hipGetLastError() == hipSuccess ? STAIRS_OK : STAIRS_EHIP;
}
