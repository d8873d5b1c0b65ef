// What the attention kernels share: their arguments and small pieces of PTX.
#pragma once
#include "kvcache.cuh"

namespace ptk {

constexpr u32 FULL = 0xFFFFFFFFu;
constexpr float LOG2E = 1.4426950408889634f;

struct Attend {
  Cache cache;
  const unsigned char* q;
  unsigned char* out;
  i64 q_token, q_head, o_token, o_head;       // strides in elements
  const int* offsets;                         // [R + 1] rows of q of every request
  const int* lengths;                         // [R] tokens in the cache, the new ones among them
  const int* tables;                          // [R][max_blocks]
  int R, max_blocks, heads, group, tokens;    // query heads, query heads per kv head, rows of q
  float scale2;                               // softmax scale * log2 e (* K's tensor scale and format factor for the 4-bit cache)
  float v_factor;                             // what the 4-bit values of V are multiplied by at the end (1 for 16-bit caches)
  unsigned char* work;
  u32 box_tokens;                             // tokens of a box of the cache's tensor map, 0: there is none
  u32 q_box;                                  // there is a tensor map of q
  u32 split;                                  // CTAs among which the steps of the row tiles may be cut, 0: they are not
  u32 polls;                                  // polls of a wait before its CTA gives up
  u32* status;
};
constexpr u32 POLLS = 1u << 22;               // the built-in limit (each poll may suspend for a while), and that of waits for what is in flight at the end

// rows of request r that exist, its keys, and the position of its first row (may be negative).  Rows behind `tokens` count for the
// positions although they are not there.
struct Req { int row0, fresh, keys, pos0; };
__device__ __forceinline__ Req request(const Attend& a, int r) {
  Req q;
  const int lo = a.offsets[r], end = a.offsets[r + 1], len = a.lengths[r];
  q.row0 = lo < 0 ? 0 : lo > a.tokens ? a.tokens : lo;
  const int hi = end < q.row0 ? q.row0 : end > a.tokens ? a.tokens : end;
  q.fresh = hi - q.row0;
  const i64 room = (i64)a.max_blocks * a.cache.block_tokens;
  q.keys = len < 0 ? 0 : len > room ? (int)room : len;
  // A length the table cannot hold keeps its positions; the keys it lacks are not seen.  Positions from `room` (at most 2^30) on see the same keys, so
  // 32 bits hold position + row without overflow.
  const i64 pos = (i64)len - end + q.row0;
  q.pos0 = pos > room ? (int)room : pos < -0x7FFFFFFF ? -0x7FFFFFFF : (int)pos;
  return q;
}

// What a row's sums are multiplied by.  Weights that add up to nothing: a row that sees no key is zero, one whose scores are all minus infinity has no
// softmax (NaN).  pos: the row's position.
__device__ __forceinline__ float row_factor(const Attend& a, int r, i64 pos, float sum) {
  if (sum != 0.0f) return a.v_factor / sum;
  const Req q = request(a, r);                // (read again: kept from the start it would cost the kernels registers)
  const int last = pos < q.keys ? (int)pos : q.keys - 1;
  if (last >= 0)
    for (u32 b = 0; b <= (u32)last / a.cache.block_tokens; ++b)
      if ((u32)a.tables[(i64)r * a.max_blocks + b] < a.cache.num_blocks) return NAN;
  return 0.0f;
}

__device__ __forceinline__ u32 smem_addr(const void* p) { return (u32)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void cp_async16(u32 dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async16_or_zero(u32 dst, const void* src, bool ok) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(ok ? 16 : 0) : "memory");
}
__device__ __forceinline__ void bar_init(u64* bar, u32 count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_addr(bar)), "r"(count) : "memory"); }
__device__ __forceinline__ void bar_arrive(u64* bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_addr(bar)) : "memory"); }
__device__ __forceinline__ void bar_expect(u64* bar, u32 bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_addr(bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_test(u64* bar, u32 parity) {         // never suspends
  u32 ok;
  asm volatile("{\n .reg .pred p;\n mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(ok) : "r"(smem_addr(bar)), "r"(parity) : "memory");
  return ok != 0;
}
__device__ __forceinline__ bool bar_try(u64* bar, u32 parity) {
  u32 ok;
  asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(ok) : "r"(smem_addr(bar)), "r"(parity) : "memory");
  return ok != 0;
}
// `bytes` contiguous bytes (16-byte aligned, a multiple of 16) into shared memory, counted by the barrier
__device__ __forceinline__ void bulk_load(u32 dst, const void* src, u32 bytes, u64* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(smem_addr(bar)) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
template <bool FP16>
__device__ __forceinline__ u32 pack2(float lo, float hi) {
  u32 r;
  if (FP16) asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
template <bool FP16>
__device__ __forceinline__ float2 unpack2(u32 v) {
  if (FP16) return __half22float2(*reinterpret_cast<const __half2*>(&v));
  return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&v));
}
__device__ __forceinline__ u32 hfma2(u32 a, u32 b, u32 c) {
  u32 r;
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
  return r;
}
__device__ __forceinline__ u32 hmul2(u32 a, u32 b) {
  u32 r;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// 4-bit codes to fp16.  A code n at bits p .. p+3 of 0x6400 reads as 1024 + n 2^p, and (1024 + n 2^p) * (s / 2^p) - (1024 / 2^p + 8) s
// = (n - 8) s in one fused multiply-add.  It is exact: s has 4 significant bits, so 1032 s (8 + 4 bits, at most 129 * 15 < 2^11) and 72 s fit
// fp16's 11; the codes are read at bits 0..3 and 4..7.  s is the scale times 2^-8, which keeps 1032 s inside fp16; the 2^8 is
// put back at the end.  `(x & mask) | 0x6400..` is ONE instruction only if the constants are in registers, hence Magic.
struct Magic { u32 m0, m4, one; };
__device__ __forceinline__ Magic magic() {
  Magic m;
  asm volatile("mov.b32 %0, 0x000F000F;\n mov.b32 %1, 0x00F000F0;\n mov.b32 %2, 0x64006400;" : "=r"(m.m0), "=r"(m.m4), "=r"(m.one));
  return m;
}
__device__ __forceinline__ u32 and_or(u32 a, u32 b, u32 c) {
  u32 r;
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
  return r;
}
struct Deq { u32 s0, c0, s4, c4; };
__device__ __forceinline__ Deq deq_of(u32 scale2) {          // two e4m3 scales (multiples of 2^-9) as fp16 pairs
  Deq d;
  d.s0 = hmul2(scale2, 0x1C001C00u);                         // 2^-8
  d.c0 = hmul2(d.s0, 0xE408E408u);                           // -1032
  d.s4 = hmul2(d.s0, 0x2C002C00u);                           // 2^-4 (multiples of 2^-21: exact)
  d.c4 = hmul2(d.s0, 0xD480D480u);                           // -72
  return d;
}
constexpr float DEQ_FACTOR = 256.0f;
// the four nibbles of each 16-bit half: o[j] = (nibble j of the low half, nibble j of the high half); h: x >> 8 (bits 0-7 of each half count)
__device__ __forceinline__ void deq4(u32 x, u32 h, const Deq& d, const Magic& k, u32 (&o)[4]) {
  o[0] = hfma2(and_or(x, k.m0, k.one), d.s0, d.c0);
  o[1] = hfma2(and_or(x, k.m4, k.one), d.s4, d.c4);
  o[2] = hfma2(and_or(h, k.m0, k.one), d.s0, d.c0);
  o[3] = hfma2(and_or(h, k.m4, k.one), d.s4, d.c4);
}

}  // namespace ptk
