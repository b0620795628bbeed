// What the operators over paged caches share (stairs_paged.hip, stairs_tree.hip).
#pragma once
#include "../../include/stairs.h"
#include "stairs_device.h"

namespace stairs {

// whether a pool of pages is one
bool paged_cache_ok(const stairs_paged_cache* c);

// ---- rows in 8 bits: places in bytes inside one head of a page --------------------------------------------------------
__device__ __forceinline__ int k_held_off(int pos, int e, int hd) {
  return ((pos >> 4) * (hd >> 6) + (e >> 6)) * 1024 + ((pos & 15) + 16 * ((e & 31) >> 3)) * 16 + ((e & 63) >> 5) * 8 + (e & 7);
}
__device__ __forceinline__ int v_held_off(int pos, int e, int hd) {
  return ((pos >> 5) * (hd >> 5) + (e >> 5)) * 1024 + ((e & 15) + 16 * ((pos & 15) >> 2)) * 16 + ((e & 31) >> 4) * 8 + (pos & 3) + 4 * ((pos >> 4) & 1);
}
// a position's powers of two: the keys' byte, the values' 8 further
__device__ __forceinline__ int scale_off(int pos) { return (pos >> 5) * 64 + ((pos & 15) >> 2) * 16 + ((pos >> 4) & 1) * 4 + (pos & 3); }

}  // namespace stairs
