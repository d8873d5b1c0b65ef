// One layer of the paged cache as the operators that compute on it see it, and the 4-bit form of its chunks.
//
// 4-bit chunk (PTSTORE_KV_PACKED) of a block: [kv head][tile of 16 tokens], a tile = 16 x D/2 bytes of codes, then 16 x D/16 bytes of
// e4m3 scales, one per token and 16 consecutive elements; value = (code - 8) * scale * tensor scale.
//   why 16 elements and e4m3: a code has 4 significant bits and a scale 4, so a value is EXACT in bf16 and in fp16 and the
//     reader can hand it to the matrix instructions with one fused multiply-add per two elements; 4.5 bits per element;
//   why a tile is contiguous: head h of 16 tokens is one bulk copy of 9 D bytes whatever the block size;
//   codes: element i of a token is nibble i & 7 of word i >> 3.  The 16-byte chunk c of token n sits at place
//     8 (n / rho) + (((n % rho) * D/32 + c) ^ 2 (n / 4)), rho = 256 / D tokens per 128 bytes: a warp that reads the values of
//     four tokens 4t .. 4t+3 for all d (V, whose products run over the tokens) or whole rows (K) hits every bank once;
//   scales: K [token][group] - a lane needs the groups of one token; V [group][token] - it needs one group of four tokens.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/ptstore.h"

namespace ptk {

typedef long long i64;
typedef unsigned long long u64;
typedef unsigned int u32;

constexpr int TILE = 16;         // tokens of a tile
constexpr int GROUP = 16;        // elements that share a scale

struct Cache {
  unsigned char* base;
  u64 kv_stride, block_stride;
  u32 num_blocks, block_tokens, heads;
};

__host__ __device__ constexpr int tile_bytes(int D) { return 9 * D; }                    // 8 D of codes, D of scales
__host__ __device__ constexpr int code_place(int D, int n, int c) {                      // in 16-byte units
  return (n / (256 / D)) * 8 + (((n % (256 / D)) * (D / 32) + c) ^ (2 * (n >> 2)));
}
__host__ __device__ constexpr int scale_at(int D, bool is_v, int n, int g) { return 8 * D + (is_v ? g * TILE + n : n * (D / GROUP) + g); }

__device__ __forceinline__ unsigned char* tile_ptr(const Cache& c, bool is_v, u32 block, u32 head, u32 token, int D) {
  return c.base + (is_v ? c.kv_stride : 0) + (u64)block * c.block_stride + ((u64)head * (c.block_tokens / TILE) + token / TILE) * tile_bytes(D);
}
__device__ __forceinline__ unsigned char* row_ptr(const Cache& c, bool is_v, u32 block, u32 head, u32 token, int D) {   // 16-bit formats
  return c.base + (is_v ? c.kv_stride : 0) + (u64)block * c.block_stride + ((u64)token * c.heads + head) * D * 2;
}

__device__ __forceinline__ u32 e4m3_of(float x) {             // x >= 0: nearest e4m3, at most 448; NaN stays NaN
  unsigned short r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(0.0f), "f"(x));
  return r & 0xFFu;
}
__device__ __forceinline__ u32 e4m3x2_to_half2(u32 two) {
  u32 r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((unsigned short)two));
  return r;
}
__device__ __forceinline__ float e4m3_value(u32 byte) {
  const u32 h = e4m3x2_to_half2(byte);
  return __low2float(*reinterpret_cast<const __half2*>(&h));
}

// ---- host side: checks shared by the entry points ------------------------------------------------------------------------------------
inline bool power_of_two(float x) {
  int e;
  return isfinite(x) && x > 0.0f && frexpf(x, &e) == 0.5f && e >= -63 && e <= 65;
}
inline u64 chunk_bytes_of(u32 format, u64 block_tokens, u64 heads, u64 dim) {
  if (block_tokens < 1 || heads < 1 || (dim != 64 && dim != 128) || heads > 65535 || block_tokens > 65536) return 0;
  if (format == PTSTORE_KV_BF16 || format == PTSTORE_KV_FP16) return block_tokens * heads * dim * 2;
  if (format == PTSTORE_KV_PACKED) return block_tokens % TILE ? 0 : block_tokens * heads * dim * 9 / 16;
  return 0;
}
inline int check_cache(const ptstore_kv_cache_t* c) {
  if (!c || !c->base || (reinterpret_cast<uintptr_t>(c->base) & 15u) || c->num_blocks == 0 || c->num_blocks > 0x7FFFFFFFu) return PTSTORE_E_INVAL;
  const u64 chunk = chunk_bytes_of(c->format, c->block_tokens, c->num_kv_heads, c->head_dim);
  if (chunk == 0 || c->kv_stride_bytes % 16 || c->block_stride_bytes % 16 || c->block_stride_bytes < chunk) return PTSTORE_E_INVAL;
  if (c->format == PTSTORE_KV_PACKED && (!power_of_two(c->k_scale) || !power_of_two(c->v_scale))) return PTSTORE_E_INVAL;
  return PTSTORE_OK;
}
inline Cache cache_of(const ptstore_kv_cache_t* c) {
  return {static_cast<unsigned char*>(c->base), c->kv_stride_bytes, c->block_stride_bytes, c->num_blocks, c->block_tokens, c->num_kv_heads};
}
// 16-byte loads and stores of 16-bit elements; the stride of an axis of one does not matter
inline bool rows_aligned(const void* p, i64 tokens, i64 token_stride, i64 heads, i64 head_stride) {
  return !(reinterpret_cast<uintptr_t>(p) & 15u) && (tokens == 1 || token_stride % 8 == 0) && (heads == 1 || head_stride % 8 == 0);
}

}  // namespace ptk
