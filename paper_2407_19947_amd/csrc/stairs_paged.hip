// Operators over paged key/value caches: pages and slots for the requests of a step, storing the new rows, attention of the
// new rows over the pages.  The page layout is the tiled layout of the framework's own half caches (k_cache_off, v_cache_off),
// page by page.
#include "../../include/stairs.h"
#include "stairs_device.h"

#include <cmath>

namespace stairs {
namespace {

// ---------------------------------------------------------------------------------------
// pages and slots
// ---------------------------------------------------------------------------------------
constexpr int kPlanThreads = 1024;
static_assert(kPlanThreads >= STAIRS_PAGED_MAX_SEQS, "a thread per sequence");

// exclusive sum over the threads of the block
__device__ __forceinline__ long long block_scan(long long v, long long* s_part, long long* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  long long x = v;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const long long o = __shfl_up(x, off);
    if (lane >= off) x += o;
  }
  __syncthreads();
  if (lane == 63) s_part[wave] = x;
  __syncthreads();
  long long before = 0, all = 0;
  for (int w = 0; w < (int)(blockDim.x >> 6); ++w) {
    if (w < wave) before += s_part[w];
    all += s_part[w];
  }
  *total = all;
  return before + x - v;
}

// the last index b < n with first[b] <= i, first ascending, first[0] <= i
__device__ __forceinline__ int find_seq(const int* first, int n, int i) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (first[mid] <= i) lo = mid;
    else hi = mid;
  }
  return lo;
}

// position and slot of row t, from what the plan has left
__device__ __forceinline__ void row_slot(const stairs_page_plan& p, const int* row_start, int t, int total) {
  int pos = -1, slot = -1;
  if (t < total) {
    const int b = find_seq(row_start, p.n_seqs, t);
    const int len = p.seq_len[b];
    if (len > 0) {
      pos = len - (row_start[b + 1] - t);
      if (pos < 0 || pos >= len) pos = -1;          // (counts whose sum is no int)
      const int page = pos < 0 ? -1 : p.block_table[(size_t)b * p.max_blocks + pos / p.page_size];
      if ((unsigned)page < (unsigned)p.n_pages) slot = page * p.page_size + pos % p.page_size;
    }
  }
  p.position[t] = pos;
  p.slot[t] = slot;
}

// One block: a thread per sequence counts, three sums over the sequences say where everything goes, then the pages that change
// hands and the rows are spread over all threads (a sequence that ends with a thousand pages is not one thread's work).
__global__ __launch_bounds__(kPlanThreads) void k_paged_plan(stairs_page_plan p, int rows_here) {
  __shared__ long long s_part[kPlanThreads / 64];
  __shared__ int s_rows[STAIRS_PAGED_MAX_SEQS + 1], s_drop[STAIRS_PAGED_MAX_SEQS + 1], s_ask[STAIRS_PAGED_MAX_SEQS + 1];
  __shared__ int s_need[STAIRS_PAGED_MAX_SEQS], s_held[STAIRS_PAGED_MAX_SEQS];
  const int b = threadIdx.x;
  const bool here = b < p.n_seqs;
  const int cached = here ? max(p.cached[b], 0) : 0, fresh = here ? max(p.fresh[b], 0) : 0;
  const int held = here ? min(max(p.held[b], 0), p.max_blocks) : 0;
  const int n_free = min(max(p.n_free[0], 0), p.n_pages);
  const long long wants = ((long long)cached + fresh + p.page_size - 1) / p.page_size;
  const bool fits = wants <= p.max_blocks;
  const int need = fits ? (int)wants : held;
  const int ask = max(need - held, 0), drop = held - min(need, held);
  long long rows_l, asked, dropped_l, granted_l;
  const int row0 = (int)block_scan(fresh, s_part, &rows_l);
  const long long ask0 = block_scan(ask, s_part, &asked);
  const int drop0 = (int)min(block_scan(drop, s_part, &dropped_l), (long long)INT32_MAX);
  const int dropped = (int)min(dropped_l, (long long)(p.n_pages - n_free)), avail = n_free + dropped;
  const bool ok = fits && (ask == 0 || ask0 + ask <= avail);
  const int grant0 = (int)block_scan(ok ? ask : 0, s_part, &granted_l);     // (at most avail)
  const int rows = (int)rows_l, granted = (int)granted_l;
  if (here) {
    s_rows[b] = row0;
    s_drop[b] = drop0;
    s_ask[b] = grant0;
    s_need[b] = need;
    s_held[b] = held;
  }
  if (b == 0) s_rows[p.n_seqs] = rows;
  __syncthreads();
  // pages given back, behind the free ones
  for (int i = threadIdx.x; i < dropped; i += kPlanThreads) {
    const int q = find_seq(s_drop, p.n_seqs, i);
    p.free_pages[n_free + i] = p.block_table[(size_t)q * p.max_blocks + s_need[q] + (i - s_drop[q])];
  }
  __syncthreads();
  // pages taken, from the end of the stack
  for (int i = threadIdx.x; i < granted; i += kPlanThreads) {
    const int q = find_seq(s_ask, p.n_seqs, i);
    p.block_table[(size_t)q * p.max_blocks + s_held[q] + (i - s_ask[q])] = p.free_pages[avail - 1 - i];
  }
  if (here) {
    p.held_out[b] = ok ? need : held;
    p.row_start[b] = row0;
    p.seq_len[b] = ok ? cached + fresh : 0;
  }
  if (b == 0) {
    p.n_free_out[0] = avail - granted;
    p.row_start[p.n_seqs] = rows;
  }
  __syncthreads();
  for (int t = threadIdx.x; t < rows_here; t += kPlanThreads) row_slot(p, s_rows, t, rows);
}

__global__ __launch_bounds__(256) void k_paged_slots(stairs_page_plan p) {
  const int t = blockIdx.x * 256 + threadIdx.x;
  if (t < p.max_rows) row_slot(p, p.row_start, t, p.row_start[p.n_seqs]);
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

// a block per row: q and k rotated, k and v stored
template <typename T, int HD>
__global__ __launch_bounds__(256) void k_paged_append(stairs_paged_cache c, stairs_paged_rows a) {
  __shared__ float2 s_cs[HD / 2];
  const int t = blockIdx.x;
  const int slot = a.slot[t];
  const bool rotate = a.rope_theta > 0.f;
  const int pos = rotate ? a.position[t] : 0;
  if (rotate && threadIdx.x < HD / 2) {
    const double angle = (double)pos * exp2(-(2.0 * threadIdx.x / HD) * log2((double)a.rope_theta));
    double s, co;
    sincos(angle, &s, &co);
    s_cs[threadIdx.x] = make_float2((float)co, (float)s);
  }
  __syncthreads();
  const bool store = (unsigned)slot < (unsigned)c.n_pages * (unsigned)c.page_size;
  const int page = store ? slot / c.page_size : 0, p = store ? slot % c.page_size : 0;
  const size_t head_elems = (size_t)c.page_size * HD;
  const int nq = a.n_heads, nk = c.n_kv_heads;
  for (int i = threadIdx.x; i < (nq + nk) * (HD / 2); i += 256) {
    const int h = i / (HD / 2), e = i % (HD / 2);
    const bool is_q = h < nq;
    if (is_q ? pos < 0 : !store) continue;
    const T* src = is_q ? static_cast<const T*>(a.q) + (size_t)t * a.q_stride + h * HD
                        : static_cast<const T*>(a.k) + (size_t)t * a.k_stride + (h - nq) * HD;
    T lo = src[e], hi = src[e + HD / 2];
    if (rotate) {
      const float2 r = rope_rotate(Elem<T>::up(lo), Elem<T>::up(hi), s_cs[e]);
      lo = Elem<T>::down(r.x);
      hi = Elem<T>::down(r.y);
    }
    if (is_q) {
      T* dst = static_cast<T*>(a.q_out) + (size_t)t * a.q_out_stride + h * HD;
      dst[e] = lo;
      dst[e + HD / 2] = hi;
    } else {
      T* dst = static_cast<T*>(c.k) + ((size_t)page * nk + (h - nq)) * head_elems;
      dst[k_cache_off(p, e, HD)] = lo;
      dst[k_cache_off(p, e + HD / 2, HD)] = hi;
    }
  }
  if (store)
    for (int i = threadIdx.x; i < nk * HD; i += 256) {
      const int h = i / HD, e = i % HD;
      T* dst = static_cast<T*>(c.v) + ((size_t)page * nk + h) * head_elems;
      dst[v_cache_off(p, e, HD)] = static_cast<const T*>(a.v)[(size_t)t * a.v_stride + i];
    }
}

// ---------------------------------------------------------------------------------------
// attention
// ---------------------------------------------------------------------------------------
// a wave per row and head: 64 keys at a time, a lane a key; then a lane HD / 64 dims of the values
template <typename T, int HD>
__global__ __launch_bounds__(64) void k_paged_attend(stairs_paged_cache c, stairs_paged_attn a, float scale) {
  __shared__ float s_q[HD];
  __shared__ float s_p[64];
  const int t = blockIdx.x, h = blockIdx.y, lane = threadIdx.x;
  if (t < a.row_start[0] || t >= a.row_start[a.n_seqs]) return;
  const int b = find_seq(a.row_start, a.n_seqs, t);
  const int last = min(a.seq_len[b] - (a.row_start[b + 1] - t), a.max_blocks * c.page_size - 1);   // last position the row may see
  const int kvh = h / (a.n_heads / c.n_kv_heads);
  for (int e = lane; e < HD; e += 64) s_q[e] = scale * Elem<T>::up(static_cast<const T*>(a.q)[(size_t)t * a.q_stride + h * HD + e]);
  __syncthreads();
  const size_t head_elems = (size_t)c.page_size * HD, page_elems = head_elems * c.n_kv_heads;
  const T* K = static_cast<const T*>(c.k) + kvh * head_elems;
  const T* V = static_cast<const T*>(c.v) + kvh * head_elems;
  const int* table = a.block_table + (size_t)b * a.max_blocks;
  float m = -INFINITY, l = 0.f, o[HD / 64] = {};
  for (int k0 = 0; k0 <= last; k0 += 64) {
    const int key = k0 + lane, blk = key / c.page_size;
    const int page = key <= last && blk < a.max_blocks ? table[blk] : -1;
    float x = -INFINITY;
    if ((unsigned)page < (unsigned)c.n_pages) {
      const T* kp = K + page * page_elems;
      x = 0.f;
      for (int e = 0; e < HD; ++e) x += s_q[e] * Elem<T>::up(kp[k_cache_off(key % c.page_size, e, HD)]);
    }
    const float mn = fmaxf(m, wave_max(x));
    const float keep = mn == -INFINITY ? 0.f : expf(m - mn), pr = mn == -INFINITY ? 0.f : expf(x - mn);
    m = mn;
    l = l * keep + wave_sum(pr);
    __syncthreads();
    s_p[lane] = x == -INFINITY ? -1.f : Elem<T>::up(Elem<T>::down(pr));
    __syncthreads();
#pragma unroll
    for (int i = 0; i < HD / 64; ++i) o[i] *= keep;
    for (int j = 0; j < 64; ++j) {
      const float pj = s_p[j];
      if (pj < 0.f) continue;                      // not seen: its values may be anything
      const int k = k0 + j;
      const T* vp = V + table[k / c.page_size] * page_elems;
#pragma unroll
      for (int i = 0; i < HD / 64; ++i) o[i] += pj * Elem<T>::up(vp[v_cache_off(k % c.page_size, i * 64 + lane, HD)]);
    }
  }
  for (int i = 0; i < HD / 64; ++i)
    static_cast<T*>(a.out)[(size_t)t * a.out_stride + h * HD + i * 64 + lane] = Elem<T>::down(l == 0.f ? 0.f : o[i] / l);
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
  if (!one) hipLaunchKernelGGL(k_paged_slots, dim3((p->max_rows + 255) / 256), dim3(256), 0, st, *p);
  return launched();
}

extern "C" int stairs_paged_append(const stairs_paged_cache* c, const stairs_paged_rows* a, void* hip_stream) {
  if (!cache_ok(c) || !a || a->rows < 0 || a->n_heads < 0 || a->n_heads > 4096) return STAIRS_EINVAL;
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
  by_type(c, [&](auto type, auto hd) {
    hipLaunchKernelGGL((k_paged_append<decltype(type), decltype(hd)::value>), dim3(r.rows), dim3(256), 0, st, *c, r);
  });
  return launched();
}

extern "C" int64_t stairs_paged_attention_workspace(const stairs_paged_cache* c, const stairs_paged_attn* a) {
  if (!attn_sizes_ok(c, a)) return STAIRS_EINVAL;
  return 0;
}

extern "C" int stairs_paged_attention(const stairs_paged_cache* c, const stairs_paged_attn* a, void* hip_stream) {
  if (!attn_sizes_ok(c, a) || std::isnan(a->scale) || std::isinf(a->scale)) return STAIRS_EINVAL;
  if (a->n_seqs == 0 || a->rows == 0) return STAIRS_OK;
  if (!a->q || !a->out || a->q == a->out || !a->block_table || !a->row_start || !a->seq_len) return STAIRS_EINVAL;
  if (!aligned16(a->q) || !aligned16(a->out) || !stride_ok(a->q_stride, a->n_heads, c->head_dim) || !stride_ok(a->out_stride, a->n_heads, c->head_dim))
    return STAIRS_EINVAL;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (const int rc = check_stream(st)) return rc;
  const float scale = a->scale > 0.f ? a->scale : 1.0f / sqrtf((float)c->head_dim);
  by_type(c, [&](auto type, auto hd) {
    hipLaunchKernelGGL((k_paged_attend<decltype(type), decltype(hd)::value>), dim3(a->rows, a->n_heads), dim3(64), 0, st, *c, *a, scale);
  });
  return launched();
}
