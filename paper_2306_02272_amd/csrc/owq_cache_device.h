// Device-side access to the 4-bit cache: where a tile lies, words of eight codes.
#pragma once
#include "owq_step.h"
#include "owq_step_device.h"

namespace owq {

// Address of tile `tile` (32 tokens) of sequence b's head, nullptr where the table holds no page.
__device__ __forceinline__ uint8_t *cache_tile(const CacheView &c, int b, int head, int tile) {
  const int slot = tile >> c.page_shift;
  if (slot >= c.table_stride) return nullptr;
  const int page = c.table[(int64_t)b * c.table_stride + slot];
  if (page < 0 || page >= c.n_pages) return nullptr;
  const int in_page = tile & ((1 << c.page_shift) - 1);
  return c.pages + page * c.page_bytes + (((int64_t)head << c.page_shift) + in_page) * c.tile_bytes;
}

// The same in two steps, for a wave that walks over tiles: the page of a tile within the table (asked for a tile ahead of
// its use: a scalar load), and its address (scalar arithmetic), nullptr where it is no page.
__device__ __forceinline__ int page_of_tile(const CacheView &c, int b, int tile) {
  return c.table[(int64_t)b * c.table_stride + (tile >> c.page_shift)];
}
__device__ __forceinline__ const uint8_t *tile_in_page(const CacheView &c, int page, int head, int tile) {
  page = __builtin_amdgcn_readfirstlane(page);
  const int in_page = tile & ((1 << c.page_shift) - 1);
  const uint8_t *p = c.pages + page * c.page_bytes + (((int64_t)head << c.page_shift) + in_page) * c.tile_bytes;
  return page >= 0 && page < c.n_pages ? p : nullptr;
}

// Eight codes in bytes (elements 0..3 in a, 4..7 in b) to their word: element e at nibble e / 2 + 4 (e % 2).
__device__ __forceinline__ u32 word_of_bytes(u32 a, u32 b) {
  // even elements in the low half, odd ones in the high half
  const u32 even = (a & 15u) | ((a >> 12) & 0xf0u) | ((b & 15u) << 8) | ((b >> 4) & 0xf000u);
  const u32 odd = ((a >> 8) & 15u) | ((a >> 20) & 0xf0u) | (b & 0xf00u) | ((b >> 12) & 0xf000u);
  return even | odd << 16;
}

__device__ __forceinline__ u32x2 bytes_of_word(u32 w) {
  const u32 a = (w & 15u) | ((w >> 8) & 0xf00u) | ((w & 0xf0u) << 12) | ((w << 4) & 0x0f000000u);
  const u32 b = ((w >> 8) & 15u) | ((w >> 16) & 0xf00u) | ((w & 0xf000u) << 4) | ((w >> 4) & 0x0f000000u);
  return (u32x2){a, b};
}

}  // namespace owq
