// Trees of drafted tokens: what each row sees and where it stands, the path that the model's predictions follow, and the
// paged caches brought in line with it.
#include "stairs_paged.h"

#include <algorithm>
#include <cstdint>

namespace stairs {
namespace {

static_assert(STAIRS_TREE_MAX_ROWS == 64, "a lane for each row of a tree");
constexpr int kWaves = 4;                                       // of a work-group, a request each

// a request's rows: none where row_start makes no sense (lost then)
struct Rows {
  int first, count, len;
  bool lost;
};
__device__ __forceinline__ Rows rows_of(const int* row_start, const int* seq_len, int rows, int b) {
  Rows r{row_start[b], 0, seq_len[b], false};
  const int n = row_start[b + 1] - r.first;
  if (r.first >= 0 && n > 0 && n <= rows - r.first) r.count = n;
  r.lost = n != r.count;
  return r;
}
// rows behind the last request's; work-groups from `first` on
template <typename F>
__device__ __forceinline__ void rows_behind(const int* row_start, int n_seqs, int rows, F f) {
  const int first = (n_seqs + kWaves - 1) / kWaves;
  if ((int)blockIdx.x < first) return;
  const int from = n_seqs > 0 ? max(row_start[n_seqs], 0) : 0;
  for (long long t = (long long)from + (blockIdx.x - first) * 256 + threadIdx.x; t < rows; t += (gridDim.x - first) * 256) f((int)t);
}

// A wave has a request, a lane a row; ancestors by doubling: what a row's ancestors 2^i steps up see, it sees.  Bound by the latency of
// two round trips (32 trees of 61 rows 4.6 us, one of 7 rows 1.6).
__global__ __launch_bounds__(64 * kWaves) void k_tree_plan(stairs_tree t) {
  const int lane = threadIdx.x & 63, b = blockIdx.x * kWaves + (threadIdx.x >> 6);
  if (b < t.n_seqs) {
    const Rows r = rows_of(t.row_start, t.seq_len, t.rows, b);
    const bool there = r.len >= r.count;
    if (r.count <= STAIRS_TREE_MAX_ROWS) {
      int up = lane < r.count ? t.parent[r.first + lane] : -1;
      if (up >= lane) up = -1;
      unsigned long long sees = 1ull << lane;
#pragma unroll
      for (int i = 0; i < 6; ++i) {
        const int from = max(up, 0);
        const unsigned long long theirs = __shfl(sees, from);
        const int next = __shfl(up, from);
        if (up >= 0) {
          sees |= theirs;
          up = next;
        }
      }
      if (lane < r.count) {
        t.sees[r.first + lane] = there ? sees : 0;
        if (t.position) t.position[r.first + lane] = there ? r.len - r.count + __popcll(sees) - 1 : -1;
      }
    } else {
      for (int i = lane; i < r.count; i += 64) {
        t.sees[r.first + i] = 0;
        if (t.position) t.position[r.first + i] = there ? r.len - r.count + i : -1;
      }
    }
  }
  rows_behind(t.row_start, t.n_seqs, t.rows, [&](int i) {
    t.sees[i] = 0;
    if (t.position) t.position[i] = -1;
  });
}

// A wave has a request; each step of the walk is one comparison in all lanes (children are behind their parents, so it ends; 64 trees
// of 61 rows 4.7 us).
__global__ __launch_bounds__(64 * kWaves) void k_tree_walk(stairs_tree_path t) {
  const int lane = threadIdx.x & 63, b = blockIdx.x * kWaves + (threadIdx.x >> 6);
  if (b < t.n_seqs) {
    const Rows r = rows_of(t.row_start, t.seq_len, t.rows, b);
    const bool there = r.len >= r.count && !r.lost;
    int kept = 0;
    if (r.count <= STAIRS_TREE_MAX_ROWS) {
      const bool here = lane < r.count;
      const int at = r.first + lane;
      const int parent = here ? t.parent[at] : -1, token = here ? t.token[at] : 0, predicted = here ? t.predicted[at] : 0;
      int path = 0, row = 0;                                    // the path's lane-th row
      if (there && r.count > 0) {
        for (;;) {
          if (lane == kept) path = row;
          ++kept;
          const int says = __builtin_amdgcn_readlane(predicted, row);
          const unsigned long long fits = __ballot(here && parent == row && lane > row && (token == says || token < 0));
          if (!fits) break;
          row = __builtin_ctzll(fits);
        }
      }
      const int said = __shfl(predicted, path);
      if (here) {
        t.path[at] = lane < kept ? path : -1;
        t.emitted[at] = lane < kept ? said : -1;
      }
    } else {
      kept = there ? r.count : 0;
      for (int i = lane; i < r.count; i += 64) {
        t.path[r.first + i] = there ? i : -1;
        t.emitted[r.first + i] = there ? t.predicted[r.first + i] : -1;
      }
    }
    if (lane == 0) {
      t.kept[b] = kept;
      if (there) t.cached[b] = r.len - r.count + kept;
    }
  }
  rows_behind(t.row_start, t.n_seqs, t.rows, [&](int i) { t.path[i] = t.emitted[i] = -1; });
}

// ---------------------------------------------------------------------------------------
// rows of a path to their new places
// ---------------------------------------------------------------------------------------
constexpr int kLaunchCaches = 64;                               // pools of a launch: their addresses are kernel arguments
struct Pools {
  struct { void *k, *v, *scale; } of[kLaunchCaches];
};
constexpr int kMostGroups = 2048;                               // work-groups past which a wave takes several pools (1024 .. 1536 run at once, by form)
struct PoolShape { int n_pages, page_size, n_kv_heads; };

// A place of 16 bytes of a value tile: eight positions of one dim, or in 8 bits of each of two.  An aligned four of positions is one half of
// it (`high`: the four 16 behind the others): 8 bytes, in 8 bits 4 and 4 more 8 further
__device__ __forceinline__ uint32_t of_four(uint4 v, int i) {   // (i: the same in all lanes)
  const uint32_t a = i & 1 ? v.y : v.x, b = i & 1 ? v.w : v.z;
  return i & 2 ? b : a;
}
__device__ __forceinline__ uint32_t put(uint32_t there, uint32_t value, uint32_t mask) { return (there & ~mask) | (value & mask); }
// position kf of a place to position kt of a half
template <bool H8>
__device__ __forceinline__ void move_position(uint2& to, int kt, uint4 from, int kf) {
  if constexpr (H8) {
    const uint2 v = kf >> 2 ? make_uint2(from.y, from.w) : make_uint2(from.x, from.z);
    const uint32_t mask = 0xFFu << (8 * kt);
    to = make_uint2(put(to.x, v.x >> (8 * (kf & 3)) << (8 * kt), mask), put(to.y, v.y >> (8 * (kf & 3)) << (8 * kt), mask));
  } else {
    const uint32_t v = of_four(from, kf >> 1) >> (16 * (kf & 1)) << (16 * (kt & 1)), mask = 0xFFFFu << (16 * (kt & 1));
    to = make_uint2(put(to.x, v, kt >> 1 ? 0 : mask), put(to.y, v, kt >> 1 ? mask : 0));
  }
}
// (streaming hint: a launch that leaves thousands of changed lines behind in the L2s ends only when they have been written back; 31 rows of 12 heads in
// 12 pools 19.6 -> 6.8 us, 203 of 8 heads in 32 pools 92 -> 83)
__device__ __forceinline__ void st_once(void* p, uint4 v) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  __builtin_nontemporal_store(__builtin_bit_cast(u32x4, v), static_cast<u32x4*>(p));
}
template <bool H8>
__device__ __forceinline__ uint2 ld_half(const uint8_t* place, bool high) {
  if constexpr (H8) return make_uint2(*reinterpret_cast<const uint32_t*>(place + 4 * high), *reinterpret_cast<const uint32_t*>(place + 8 + 4 * high));
  else return *reinterpret_cast<const uint2*>(place + 8 * high);
}
template <bool H8>
__device__ __forceinline__ void st_half(uint8_t* place, bool high, uint2 v) {
  if constexpr (H8) {
    __builtin_nontemporal_store(v.x, reinterpret_cast<uint32_t*>(place + 4 * high));
    __builtin_nontemporal_store(v.y, reinterpret_cast<uint32_t*>(place + 8 + 4 * high));
  } else {
    __builtin_nontemporal_store(__builtin_bit_cast(uint64_t, v), reinterpret_cast<uint64_t*>(place + 8 * high));
  }
}
__device__ __forceinline__ int place_of(int pos) { return (pos & 3) + 4 * ((pos >> 4) & 1); }

// A wave has a request and a head in some of the pools: where its rows lie is found once, and the next pool's rows are requested before this one's are
// written.  Paths ascend: what moves is the path's end, to positions one behind the other, none behind its old one, so no row that is still to
// move lies where one has moved to.  Four positions at a time, aligned: all that comes there and what stays there is read before the
// first is written, and nothing beside the four is: other positions of a page may be another stream's meanwhile.  (Keys are written in runs of 64 bytes;
// of a value's places, whose other half is the four 16 further, only the half: whole places took the same time.  64 trees of 61 rows in 32 pools of 8
// heads of 128, with the walk: 87 us, in 8 bits 45.)  (Bound by the memory's granularity: a key is pieces of 16 bytes 256 apart, a value
// numbers 16 apart, so that eight times what moves is read.)
template <int HD, bool H8>
__global__ __launch_bounds__(64 * kWaves) void k_paged_compact(PoolShape c, int n_pools, stairs_paged_path p, Pools pools) {
  constexpr int U = 4;                                          // rows at a time
  constexpr int E = H8 ? 1 : 2, KL = HD * E / 16;               // bytes of a number; 16-byte parts of a key
  constexpr int PLACES = H8 ? HD / 2 : HD, NV = (PLACES + 63) / 64;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int groups = (c.n_kv_heads + kWaves - 1) / kWaves, items = p.n_seqs * groups;
  const int apart = n_pools >= 8 ? 8 : 1, i0 = blockIdx.x / apart, item = i0 % items;
  const int first_pool = blockIdx.x % apart + i0 / items * apart, step = apart * ((int)gridDim.x / (items * apart));
  const int b = item / groups, h = item % groups * kWaves + wave;
  if (h >= c.n_kv_heads || first_pool >= n_pools) return;
  const int asked = p.kept[b];
  const Rows r = rows_of(p.row_start, p.seq_len, p.rows, b);
  if (r.count == 0 || r.count > STAIRS_TREE_MAX_ROWS || r.len < r.count) return;
  const int kept = min(asked, r.count), context = r.len - r.count, shift = __builtin_ctz(c.page_size);
  // lane j: the path's j-th row, its old and new slot; the pages of all rows (three at most) in the first lanes
  const int row = lane < kept ? p.path[r.first + lane] : -1;
  const int block0 = context >> shift;
  const bool listed = lane < 4 && block0 + lane < p.max_blocks;
  int page = listed ? p.block_table[(size_t)b * p.max_blocks + block0 + lane] : -1;
  if ((unsigned)page >= (unsigned)c.n_pages) page = -1;
  auto slot = [&](int i) {                                      // of the context's position and i more
    const int pos = context + i, at = __shfl(page, min(max((pos >> shift) - block0, 0), 3));
    return at < 0 ? -1 : (at << shift) + (pos & (c.page_size - 1));
  };
  const bool moves_row = row > lane && row < r.count;
  const int from = slot(moves_row ? row : 0), to = slot(lane);
  unsigned long long left = __ballot(moves_row && from >= 0 && to >= 0);
  const size_t head_elems = (size_t)c.page_size * HD;
  auto head_of = [&](int s) { return (size_t)(s >> shift) * c.n_kv_heads + h; };
  // bytes in front of a position's part of a key, of the lane's first place of a value
  auto key_at = [&](int s, int part) {
    const int pos = s & (c.page_size - 1);
    return head_of(s) * head_elems * E + (H8 ? k_held_off(pos, part / 4 * 64 + part % 4 * 8, HD) : 2 * (int)k_cache_off(pos, part * 8, HD));
  };
  auto value_at = [&](int s) {
    const int pos = s & (c.page_size - 1) & ~19, place = lane % PLACES;   // (positions of a place: 0 .. 3 and 16 .. 19 further)
    return head_of(s) * head_elems * E + (H8 ? v_held_off(pos, place / 16 * 32 + place % 16, HD) : 2 * (int)v_cache_off(pos, place, HD));
  };
  constexpr int kNext = 4 * 1024;                               // bytes from a place to that 64 further
  auto scales_at = [&](int s) { return head_of(s) * c.page_size * 2; };
  struct Held {
    uint4 k, v[U][NV];
    uint2 place[NV];
    uint32_t s, byte[U];
  };
  while (left) {
    // the next moves whose new positions are in one aligned four
    int src[U], place[U], n = 0, last = __builtin_ctzll(left);   // (place: which of the four)
    const int first = __builtin_amdgcn_readlane(to, last) & ~3;
    int key_from = first + (lane & 3);                          // what comes to the lane's position of the four: itself
#pragma unroll
    for (int i = 0; i < U; ++i) {                               // (past the last: the last again, for nothing)
      const int next = left ? (int)__builtin_ctzll(left) : last;
      if (left && (__builtin_amdgcn_readlane(to, next) & ~3) == first) {
        last = next;
        ++n;
        left &= left - 1;
      }
      src[i] = __builtin_amdgcn_readlane(from, last);
      place[i] = __builtin_amdgcn_readlane(to, last) & 3;
      key_from = (lane & 3) == place[i] ? src[i] : key_from;
    }
    // the 16 words of powers of two that the four's lie in: the lane's, and which number of values or keys it is of (4: of others)
    const int sp = first & (c.page_size - 1);
    const bool high = sp >> 4 & 1;
    const int word = lane & 15, mine = word / 4 == (sp & 15) >> 2 && (word & 1) == (sp >> 4 & 1) ? word >> 1 & 1 : 4;
    auto load = [&](int pool, Held& x) {
      const uint8_t *K = static_cast<const uint8_t*>(pools.of[pool].k), *V = static_cast<const uint8_t*>(pools.of[pool].v), *S = static_cast<const uint8_t*>(pools.of[pool].scale);
      x.k = *reinterpret_cast<const uint4*>(K + key_at(key_from, (lane >> 2) % KL));
#pragma unroll
      for (int e = 0; e < NV; ++e) x.place[e] = ld_half<H8>(V + value_at(first) + e * kNext, high);
      if constexpr (H8) x.s = *reinterpret_cast<const uint32_t*>(S + scales_at(first) + (sp >> 5) * 64 + word * 4);
#pragma unroll
      for (int i = 0; i < U; ++i) {
        if (i >= n) break;
#pragma unroll
        for (int e = 0; e < NV; ++e) x.v[i][e] = *reinterpret_cast<const uint4*>(V + value_at(src[i]) + e * kNext);
        if constexpr (H8) x.byte[i] = S[scales_at(src[i]) + scale_off(src[i] & (c.page_size - 1)) + 8 * (mine & 1)];
      }
    };
    auto store = [&](int pool, Held& x) {
      uint8_t *K = static_cast<uint8_t*>(pools.of[pool].k), *V = static_cast<uint8_t*>(pools.of[pool].v), *S = static_cast<uint8_t*>(pools.of[pool].scale);
#pragma unroll
      for (int i = 0; i < U; ++i) {
        if (i >= n) break;
#pragma unroll
        for (int e = 0; e < NV; ++e) move_position<H8>(x.place[e], place[i], x.v[i][e], place_of(src[i]));
        if (H8 && mine < 4) x.s = put(x.s, x.byte[i] << (8 * place[i]), 0xFFu << (8 * place[i]));
      }
      // (all of it is here before the first is written)
      asm volatile("" : "+v"(x.k.x), "+v"(x.s)::"memory");
#pragma unroll
      for (int e = 0; e < NV; ++e) asm volatile("" : "+v"(x.place[e].x), "+v"(x.place[e].y)::"memory");
      if ((lane >> 2) < KL) st_once(K + key_at(first + (lane & 3), lane >> 2), x.k);
#pragma unroll
      for (int e = 0; e < NV; ++e)
        if (lane < PLACES) st_half<H8>(V + value_at(first) + e * kNext, high, x.place[e]);
      if constexpr (H8)
        if (lane < 16 && mine < 4) *reinterpret_cast<uint32_t*>(S + scales_at(first) + (sp >> 5) * 64 + word * 4) = x.s;
    };
    Held now{}, next{};
    int pool = first_pool;
    load(pool, now);
    for (;;) {
      const int then = pool + step;
      if (then < n_pools) load(then, next);
      store(pool, now);
      if (then >= n_pools) break;
      now = next;
      pool = then;
    }
    __builtin_amdgcn_s_waitcnt(0);                              // (rows that follow are read from where these were; another pool's do not meet)
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
  }
}

bool requests_ok(int n_seqs, int rows, const int32_t* row_start, const int32_t* seq_len) {
  if (n_seqs < 0 || n_seqs > STAIRS_PAGED_MAX_SEQS || rows < 0) return false;
  return n_seqs == 0 || (row_start && seq_len);
}
// a wave for each request, and work-groups for the rows behind the last
unsigned tree_grid(int n_seqs, int rows) { return (unsigned)((n_seqs + kWaves - 1) / kWaves + std::clamp((rows - 1) / 1024 + 1, 1, 64)); }
int launched() { return hipGetLastError() == hipSuccess ? STAIRS_OK : STAIRS_EHIP; }

}  // namespace
}  // namespace stairs

using namespace stairs;

extern "C" int stairs_tree_plan(const stairs_tree* t, void* hip_stream) {
  if (!t || !requests_ok(t->n_seqs, t->rows, t->row_start, t->seq_len)) return STAIRS_EINVAL;
  if (t->rows == 0) return STAIRS_OK;
  if (!t->sees || reinterpret_cast<uintptr_t>(t->sees) % 8 != 0 || (t->n_seqs > 0 && !t->parent)) return STAIRS_EINVAL;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (const int rc = check_stream(st)) return rc;
  hipLaunchKernelGGL(k_tree_plan, dim3(tree_grid(t->n_seqs, t->rows)), dim3(64 * kWaves), 0, st, *t);
  return launched();
}

extern "C" int stairs_tree_walk(const stairs_tree_path* t, void* hip_stream) {
  if (!t || !requests_ok(t->n_seqs, t->rows, t->row_start, t->seq_len)) return STAIRS_EINVAL;
  if (t->n_seqs == 0 && t->rows == 0) return STAIRS_OK;
  if (t->n_seqs > 0 && (!t->kept || !t->cached)) return STAIRS_EINVAL;
  if (t->rows > 0 && (!t->path || !t->emitted || (t->n_seqs > 0 && (!t->parent || !t->token || !t->predicted)))) return STAIRS_EINVAL;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (const int rc = check_stream(st)) return rc;
  hipLaunchKernelGGL(k_tree_walk, dim3(tree_grid(t->n_seqs, t->rows)), dim3(64 * kWaves), 0, st, *t);
  return launched();
}

extern "C" int stairs_paged_compact(const stairs_paged_cache* caches, int32_t n_caches, const stairs_paged_path* p, void* hip_stream) {
  if (n_caches < 0 || n_caches > 4096 || (n_caches > 0 && !caches) || !p || p->max_blocks < 1) return STAIRS_EINVAL;
  if (!requests_ok(p->n_seqs, p->rows, p->row_start, p->seq_len)) return STAIRS_EINVAL;
  for (int i = 0; i < n_caches; ++i) {
    const stairs_paged_cache &c = caches[i], &first = caches[0];
    for (int j = 0; j < i; ++j)                                 // (a pool twice would have its rows moved twice)
      if (caches[j].k == c.k || caches[j].v == c.v || (c.held && caches[j].scale == c.scale)) return STAIRS_EINVAL;
    if (!paged_cache_ok(&c) || c.dtype != first.dtype || c.held != first.held || c.n_pages != first.n_pages || c.page_size != first.page_size ||
        c.n_kv_heads != first.n_kv_heads || c.head_dim != first.head_dim)
      return STAIRS_EINVAL;
  }
  if (n_caches > 0 && (int64_t)p->max_blocks * caches[0].page_size > INT32_MAX) return STAIRS_EINVAL;
  if (n_caches == 0 || p->n_seqs == 0 || p->rows == 0) return STAIRS_OK;
  if (!p->block_table || !p->path || !p->kept) return STAIRS_EINVAL;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (const int rc = check_stream(st)) return rc;
  const stairs_paged_cache& c = caches[0];
  const PoolShape shape{c.n_pages, c.page_size, c.n_kv_heads};
  for (int at = 0; at < n_caches; at += kLaunchCaches) {
    const int n = std::min(kLaunchCaches, n_caches - at);
    Pools pools{};
    for (int i = 0; i < n; ++i) {
      pools.of[i].k = caches[at + i].k;
      pools.of[i].v = caches[at + i].v;
      pools.of[i].scale = caches[at + i].scale;
    }
    const int64_t items = (int64_t)p->n_seqs * ((c.n_kv_heads + kWaves - 1) / kWaves);
    const int apart = n >= 8 ? 8 : 1, turns = (n + apart - 1) / apart;
    const int spread = (int)std::clamp<int64_t>(kMostGroups / (items * apart), 1, turns);
    const dim3 grid((unsigned)(items * apart * spread)), block(64 * kWaves);
    if (c.head_dim == 64) {
      if (c.held) hipLaunchKernelGGL((k_paged_compact<64, true>), grid, block, 0, st, shape, n, *p, pools);
      else hipLaunchKernelGGL((k_paged_compact<64, false>), grid, block, 0, st, shape, n, *p, pools);
    } else {
      if (c.held) hipLaunchKernelGGL((k_paged_compact<128, true>), grid, block, 0, st, shape, n, *p, pools);
      else hipLaunchKernelGGL((k_paged_compact<128, false>), grid, block, 0, st, shape, n, *p, pools);
    }
    if (const int rc = launched()) return rc;
  }
  return STAIRS_OK;
}
