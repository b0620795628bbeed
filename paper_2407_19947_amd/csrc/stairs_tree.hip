// Trees of drafted tokens: what each row sees and where it stands, the path that the model's predictions follow, and the
// paged caches brought in line with it.
#include "stairs_paged.h"

#include <algorithm>
#include <cstdint>

namespace stairs {
namespace {

static_assert(STAIRS_TREE_MAX_ROWS == 64, "a lane for each row of a tree");
constexpr int kWaves = 4;                                       // of a work-group, a request each

// a request's rows: none where row_start makes no sense
struct Rows { int first, count, len; };
__device__ __forceinline__ Rows rows_of(const int* row_start, const int* seq_len, int rows, int b) {
  Rows r{row_start[b], 0, seq_len[b]};
  const int n = row_start[b + 1] - r.first;
  if (r.first >= 0 && n > 0 && n <= rows - r.first) r.count = n;
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

// A wave has a request, a lane a row; ancestors by doubling: what a row's ancestors 2^i steps up see, it sees.  Bound by the latency of its
// three round trips.
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

// A wave has a request; each step of the walk is one comparison in all lanes (children are behind their parents, so it ends).
__global__ __launch_bounds__(64 * kWaves) void k_tree_walk(stairs_tree_path t) {
  const int lane = threadIdx.x & 63, b = blockIdx.x * kWaves + (threadIdx.x >> 6);
  if (b < t.n_seqs) {
    const Rows r = rows_of(t.row_start, t.seq_len, t.rows, b);
    const bool there = r.len >= r.count;
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
struct PoolShape { int n_pages, page_size, n_kv_heads; };

// A wave has a request, a head and a pool.  Paths ascend, so a row's new place is never behind its old one and no row that is still to move
// lies where one has moved to: some rows at a time, all of them read before the first is written.  A value is HD single numbers 16 bytes
// apart.
template <int HD, bool H8>
__global__ __launch_bounds__(64 * kWaves) void k_paged_compact(PoolShape c, stairs_paged_path p, Pools pools) {
  constexpr int U = 4;                                          // rows at a time
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int b = blockIdx.x, h = blockIdx.y * kWaves + wave;
  if (h >= c.n_kv_heads) return;
  const Rows r = rows_of(p.row_start, p.seq_len, p.rows, b);
  if (r.count == 0 || r.count > STAIRS_TREE_MAX_ROWS || r.len < r.count) return;
  const int kept = min(p.kept[b], r.count), context = r.len - r.count;
  // lane j: the path's j-th row, its old and new slot
  const int row = lane < kept ? p.path[r.first + lane] : -1;
  const int shift = __builtin_ctz(c.page_size);
  auto slot = [&](int pos) {
    const int block = pos >> shift;
    const int page = block < p.max_blocks ? p.block_table[(size_t)b * p.max_blocks + block] : -1;
    return (unsigned)page < (unsigned)c.n_pages ? (page << shift) + (pos & (c.page_size - 1)) : -1;
  };
  int from = -1, to = -1;
  if (row > lane && row < r.count) {
    from = slot(context + row);
    to = slot(context + lane);
  }
  unsigned long long moves = __ballot(from >= 0 && to >= 0);
  const auto pool = pools.of[blockIdx.z];
  const size_t head_elems = (size_t)c.page_size * HD;
  constexpr int E = H8 ? 1 : 2;                                 // bytes of a number
  uint8_t* const K = static_cast<uint8_t*>(pool.k);
  uint8_t* const V = static_cast<uint8_t*>(pool.v);
  uint8_t* const S = static_cast<uint8_t*>(pool.scale);
  auto head_of = [&](int s) { return (size_t)(s >> shift) * c.n_kv_heads + h; };
  constexpr int KL = HD * E / 16;                               // 16-byte parts of a key
  // the lane's part of a key (parts past the last: none), its numbers of a value
  auto key_part = [&](int s) {
    const int pos = s & (c.page_size - 1), part = lane % KL;
    const int at = H8 ? k_held_off(pos, part / 4 * 64 + part % 4 * 8, HD) : 2 * (int)k_cache_off(pos, part * 8, HD);
    return K + head_of(s) * head_elems * E + at;
  };
  auto value_part = [&](int s, int e) {
    const int pos = s & (c.page_size - 1);
    return V + head_of(s) * head_elems * E + (H8 ? v_held_off(pos, e, HD) : 2 * (int)v_cache_off(pos, e, HD));
  };
  auto scale_part = [&](int s) { return S + head_of(s) * c.page_size * 2 + scale_off(s & (c.page_size - 1)) + 8 * (lane & 1); };
  while (moves) {
    int src[U], dst[U];
    bool there[U];
    int last = 0;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      there[i] = moves != 0;
      last = moves ? (int)__builtin_ctzll(moves) : last;
      src[i] = __builtin_amdgcn_readlane(from, last);
      dst[i] = __builtin_amdgcn_readlane(to, last);
      moves &= moves - 1;
    }
    uint4 k[U];
    uint16_t v[U][HD / 64];
    uint8_t s[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      k[i] = *reinterpret_cast<const uint4*>(key_part(src[i]));
#pragma unroll
      for (int e = 0; e < HD / 64; ++e) v[i][e] = H8 ? *value_part(src[i], e * 64 + lane) : *reinterpret_cast<const uint16_t*>(value_part(src[i], e * 64 + lane));
      if constexpr (H8) s[i] = *scale_part(src[i]);
    }
    __builtin_amdgcn_s_waitcnt(0);                              // (all of them are here before the first place is written)
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if (!there[i]) break;
      if (lane < KL) *reinterpret_cast<uint4*>(key_part(dst[i])) = k[i];
#pragma unroll
      for (int e = 0; e < HD / 64; ++e) {
        if constexpr (H8) *value_part(dst[i], e * 64 + lane) = (uint8_t)v[i][e];
        else *reinterpret_cast<uint16_t*>(value_part(dst[i], e * 64 + lane)) = v[i][e];
      }
      if constexpr (H8)
        if (lane < 2) *scale_part(dst[i]) = s[i];
    }
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
    const dim3 grid(p->n_seqs, (c.n_kv_heads + kWaves - 1) / kWaves, n), block(64 * kWaves);
    if (c.head_dim == 64) {
      if (c.held) hipLaunchKernelGGL((k_paged_compact<64, true>), grid, block, 0, st, shape, *p, pools);
      else hipLaunchKernelGGL((k_paged_compact<64, false>), grid, block, 0, st, shape, *p, pools);
    } else {
      if (c.held) hipLaunchKernelGGL((k_paged_compact<128, true>), grid, block, 0, st, shape, *p, pools);
      else hipLaunchKernelGGL((k_paged_compact<128, false>), grid, block, 0, st, shape, *p, pools);
    }
    if (const int rc = launched()) return rc;
  }
  return STAIRS_OK;
}
