// Geometry of the 8-bit key/value cache, shared by the kernels that write, read and attend to it.
#pragma once
#include "szo_types.h"

namespace szo {

constexpr int kKvBlock = SZO_KV_BLOCK;
constexpr int kExpMin = -32, kExpMax = 120, kExpBias = 127;

// Byte of a token within its feature's row of a block of values: bits a b c r of the token become c a b r.
__host__ __device__ __forceinline__ int value_place(int token) {
  return ((token >> 2) & 1) * 16 + (token >> 4) * 8 + ((token >> 3) & 1) * 4 + (token & 3);
}

// Block `index` of a sequence: its number among all blocks of the cache's head, or -1 where the page table names no page.
__device__ __forceinline__ int64_t block_of(const szo_kv_cache& c, int sequence, int index, int head, int blocks_per_page) {
  const int page_at = index / blocks_per_page;
  if (page_at >= c.max_pages) return -1;
  const int page = c.page_table[(int64_t)sequence * c.max_pages + page_at];
  if (page < 0 || page >= c.pages) return -1;
  return ((int64_t)page * c.kv_heads + head) * blocks_per_page + (index - page_at * blocks_per_page);
}

// 2^e for |e| <= 126.
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

__device__ __forceinline__ float finite_or_nan(float x) { return fabsf(x) < __builtin_inff() ? x : __builtin_nanf(""); }
__device__ __forceinline__ float finite_size(float x) { const float a = fabsf(x); return a < __builtin_inff() ? a : 0.f; }

int check_cache(const szo_kv_cache* c);      // szo_kvcache.hip

}  // namespace szo
