// Attention of many new tokens per request over the paged cache (prompts, suffixes of found prefixes): bounded by the tensor cores.
//
// A CTA takes 256 rows of one (request, kv head): a row is a (new token, query head of the group) pair, so all rows share their keys and
// grouped heads fill the 128-row tensor tiles even when a request has few new tokens.  Two tiles of 128 rows alternate: while
// the softmax of one runs, the tensor cores work for the other.  Per step of 128 keys and tile:
//     S = Q K^T (tcgen05.mma, both operands in shared memory, S in tensor memory)
//     P = exp2(scale2 S - m), written over S in 16 bits     (one thread per row: no exchange between threads)
//     O += P V (A operand from tensor memory, V read as it lies: d contiguous, the "MN-major" form)
// O stays in tensor memory for the whole row of steps.  m is a running reference, not the exact maximum: it is moved (and O and the sum
// rescaled) only when a scaled score exceeds it by more than 8, so weights are at most 2^8 and the rescaling, a read and a write of all of O,
// is rare after the first steps.
//
// Warps: 0-3 and 4-7 softmax of tile 0 and 1 (and their part of Q at the start and of the output at the end), 8-11 load K and V into a ring of
// four 128-token tiles, 12 issues the tensor instructions (one thread).  13-15 only complete the warpgroup that gives its
// registers to the softmax warps; for a 4-bit cache 13 loads its tiles and 8-11 unpack them.
//
// B200, one prompt of 16384 tokens with 64 query and 8 kv heads x 128: 4.3 ms, 1.0 PFLOP/s.  A step of both tiles takes 3200 clocks, of which the tensor
// cores need 2050 to 2250 (Q K^T reads 8 KB of operands per instruction, all the shared memory can give): a tile's step is a chain, S ready, 64 + 64
// weights (975 + 740 clocks), the second half's values, the next scores, S ready.  Measured and dropped: two warpgroups per tile (4.4 to 4.7 ms);
// two S of 64 keys per tile, so that scores run ahead (4.6 ms: instructions of 64 columns are bound by their operands); a polynomial for a
// quarter of the exponentials (4.6 ms).
//
// A CTA has an SM to itself, so what a batch leaves over from whole rounds of SMs (one prompt whose prefix was found: everything) would leave
// most of them idle: the steps of those last row tiles are cut into as many chunks as there are SMs for them.  A chunk leaves
// its O, m and l in the workspace, and attend_join_kernel, one warp per row, joins them.
//
// Tensor memory (512 columns): S/P of tile 0, S/P of tile 1, O 0, O 1.  Shared memory operands are in the 128-byte swizzled form: 64
// elements of a row are 128 bytes, 16-byte chunk c of row r at c ^ (r & 7), 64-element halves one after the other.
#pragma once
#include <cuda.h>

#include "attend.cuh"

namespace ptk {

constexpr int PR_THREADS = 512;
constexpr int PR_ROWS = 256, PR_KEYS = 128;
constexpr int PR_PARTS_AT = 4096;            // where the parts begin in the workspace (behind the other kernel's counters)
constexpr int PR_SLOTS = 4;
constexpr int PR_RAW = 3;                    // 4-bit tiles on their way to being unpacked

template <int D>
struct PromptShape {
  static constexpr int TILE_BYTES = PR_KEYS * D * 2;                    // one K or V tile, one 128-row half of Q
  static constexpr int RAW_BYTES = PR_KEYS / TILE * tile_bytes(D);      // 128 keys of a 4-bit cache as they lie there
  static constexpr int SMEM = (2 + PR_SLOTS) * TILE_BYTES + 1024;       // + alignment
  static constexpr int SMEM_PACKED = SMEM + PR_RAW * RAW_BYTES;
};

// Waits, at most `polls` polls, and says whether what it waited for has come.  A wait that ran out sets *gave_up.  Its caller then issues no copy
// and no tensor instruction that needed it, the other roles see *gave_up or run out of polls themselves, and every role waits for what it has in
// flight (with the built-in limit) before it leaves.
__device__ __forceinline__ bool bar_wait(u64* bar, u32 parity, u32 polls, volatile int* gave_up) {
  if (bar_test(bar, parity)) return true;
#pragma unroll 1
  for (u32 i = 1; i < polls; ++i) {
    if (bar_try(bar, parity)) return true;
    if ((i & 1023) == 1023 && *gave_up) return false;
  }
  *gave_up = 1;
  return false;
}
__device__ __forceinline__ void bar_drain(u64* bar, u32 parity) {
  for (u32 i = 0; i < POLLS && !bar_try(bar, parity); ++i) {}
}

// barrier of the 128 loading threads, and whether the value was set in any of them
__device__ __forceinline__ bool any_of_128(int v) {
  u32 r;
  asm volatile("{\n .reg .pred p, q;\n setp.ne.s32 p, %1, 0;\n barrier.cta.red.or.pred q, 1, 128, p;\n selp.u32 %0, 1, 0, q;\n}" : "=r"(r) : "r"(v) : "memory");
  return r != 0;
}
__device__ __forceinline__ void cp_arrive(u64* bar) { asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_addr(bar)) : "memory"); }
// one box of the cache's tensor map {64 elements of a head, head, tokens of a block, block, K or V} into swizzled rows of 128 bytes
__device__ __forceinline__ void tensor_load(u32 dst, const CUtensorMap* map, int element, int head, int token, int block, int v, u64* bar) {
  asm volatile("cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];" ::"r"(dst), "l"(map), "r"(element),
               "r"(head), "r"(token), "r"(block), "r"(v), "r"(smem_addr(bar)) : "memory");
}
// one box of q's tensor map {64 elements of a head, the heads of a group, tokens}: rows in the order of a row tile
__device__ __forceinline__ void tensor_load_q(u32 dst, const CUtensorMap* map, int element, int head, int token, u64* bar) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst), "l"(map), "r"(element), "r"(head),
               "r"(token), "r"(smem_addr(bar)) : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_commit(u64* bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_addr(bar)) : "memory");
}
// 32 columns of this warp's 32 lanes, one row per thread
__device__ __forceinline__ void tc_ld32(float (&v)[32], u32 addr) {
  float* r = v;
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
               : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]), "=f"(r[8]), "=f"(r[9]), "=f"(r[10]), "=f"(r[11]), "=f"(r[12]),
                 "=f"(r[13]), "=f"(r[14]), "=f"(r[15]), "=f"(r[16]), "=f"(r[17]), "=f"(r[18]), "=f"(r[19]), "=f"(r[20]), "=f"(r[21]), "=f"(r[22]), "=f"(r[23]), "=f"(r[24]),
                 "=f"(r[25]), "=f"(r[26]), "=f"(r[27]), "=f"(r[28]), "=f"(r[29]), "=f"(r[30]), "=f"(r[31])
               : "r"(addr) : "memory");
}
// values of a load may be used from here on (after tc_wait_ld): keeps the compiler from moving their uses above the wait
__device__ __forceinline__ void tc_loaded(float (&v)[32]) {
#pragma unroll
  for (int i = 0; i < 32; i += 8)
    asm volatile("" : "+f"(v[i]), "+f"(v[i + 1]), "+f"(v[i + 2]), "+f"(v[i + 3]), "+f"(v[i + 4]), "+f"(v[i + 5]), "+f"(v[i + 6]), "+f"(v[i + 7]));
}
__device__ __forceinline__ void tc_st32(u32 addr, const u32 (&r)[32]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};"
               ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]),
                 "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]),
                 "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(addr) : "memory");
}

__device__ __forceinline__ void tc_st16(u32 addr, const u32 (&r)[16]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};"
               ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]),
                 "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(addr) : "memory");
}

// One lane of a converged warp, the same every time
__device__ __forceinline__ bool elected() {
  u32 p;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xFFFFFFFF;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(p));
  return p != 0;
}

// Shared-memory operand descriptor: 128-byte swizzle; `lead` only matters where the operand is MN-major (bytes between its 64-element
// halves), stride is 8 rows of 128 bytes.
__device__ __forceinline__ u64 operand_desc(u32 addr, u32 lead_bytes) {
  return (u64)((addr >> 4) & 0x3FFFu) | ((u64)((lead_bytes >> 4) & 0x3FFFu) << 16) | ((u64)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
// Instruction descriptor of kind::f16: 32-bit accumulator, both operands fp16 or both bf16, M = 128
__host__ __device__ constexpr u32 mma_desc(bool fp16, int N, bool b_mn_major) {
  return (1u << 4) | ((fp16 ? 0u : 1u) << 7) | ((fp16 ? 0u : 1u) << 10) | ((b_mn_major ? 1u : 0u) << 16) | ((u32)(N >> 3) << 17) | ((u32)(128 >> 4) << 24);
}
__device__ __forceinline__ void mma_ss(u32 d, u64 a, u64 b, u32 desc, bool add) {
  asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d), "l"(a), "l"(b), "r"(desc), "r"((u32)add) : "memory");
}
__device__ __forceinline__ void mma_ts(u32 d, u32 a, u64 b, u32 desc, bool add) {
  asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}" ::"r"(d), "r"(a), "l"(b), "r"(desc), "r"((u32)add) : "memory");
}
__device__ __forceinline__ u64 pair(float lo, float hi) { return (u64)__float_as_uint(lo) | ((u64)__float_as_uint(hi) << 32); }
__device__ __forceinline__ u64 fma_pair(u64 a, u64 b, u64 c) {
  u64 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ u64 add_pair(u64 a, u64 b) {
  u64 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ float lo_of(u64 v) { return __uint_as_float((u32)v); }
__device__ __forceinline__ float hi_of(u64 v) { return __uint_as_float((u32)(v >> 32)); }
template <int R>
__device__ __forceinline__ void regs_more() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(R)); }
template <int R>
__device__ __forceinline__ void regs_fewer() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(R)); }

// byte of 16-byte chunk c of row r in an operand tile of 128 rows
__device__ __forceinline__ u32 operand_at(int r, int c) { return (u32)((c >> 3) * (PR_KEYS * 128) + r * 128 + (((c & 7) ^ (r & 7)) * 16)); }

// Row tiles (of all kv heads, in CTA order) from `first` on are cut into `parts` chunks: what is left over from whole rounds of `sms` CTAs.
// With 4160 keys a row tile, cut / uncut: 16 tiles 33 / 68 us, 72 tiles 64 / 70, 148 + 20 tiles 117 / 138, 2 x 148 + 20 205 / 216, 3 x 148 + 20 297 / 308, 4 x 148 + 20
// 399 / 402; 2 x 148 + 72 231 / 227.  With 1024 keys the join costs more than it saves from 16 tiles on (27 / 26, 148 + 20 tiles 64 / 53).
struct Cut { i64 first; int parts; };
__device__ __forceinline__ Cut cut_of(i64 tiles, u32 sms) {
  const i64 rounds = tiles / sms;
  const u32 rest = (u32)(tiles - rounds * sms);
  if (rest == 0 || rounds > 3 || sms / rest < 2) return {tiles, 1};
  return {tiles - rest, (int)(sms / rest)};
}
template <int D>
__host__ __device__ constexpr int prompt_part_floats() { return PR_ROWS * (D + 2); }        // o, m, l of a tile's rows
__device__ __forceinline__ i64 prompt_tiles(const Attend& a, int r) {
  const Req q = request(a, r);
  return ((i64)q.fresh * a.group + PR_ROWS - 1) / PR_ROWS;
}

// Row tiles of all requests (of one kv head), counted by the whole CTA, consecutive requests per thread; mine, before: this thread's
// requests' and those of the requests before them.
template <int THREADS>
__device__ __forceinline__ i64 count_tiles(const Attend& a, i64* s_scan /*[THREADS / 32]*/, i64& mine, i64& before) {
  const int tid = threadIdx.x, per = (a.R + THREADS - 1) / THREADS;
  const int rb = min(tid * per, a.R), re = min(rb + per, a.R);
  mine = 0;
  for (int r = rb; r < re; ++r) mine += prompt_tiles(a, r);
  i64 x = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const i64 y = __shfl_up_sync(FULL, x, o);
    if ((tid & 31) >= o) x += y;
  }
  if ((tid & 31) == 31) s_scan[tid >> 5] = x;
  __syncthreads();
  before = x - mine;
  i64 all = 0;
  for (int w = 0; w < THREADS / 32; ++w) {
    if (w < (tid >> 5)) before += s_scan[w];
    all += s_scan[w];
  }
  return all;
}
// The thread whose requests tile `index` belongs to writes its request and its number there; a request's tiles come last to first.
template <int THREADS>
__device__ __forceinline__ void find_tile(const Attend& a, i64 index, i64 mine, i64 before, int* s_r, int* s_tile) {
  if (index < before || index >= before + mine) return;
  const int per = (a.R + THREADS - 1) / THREADS;
  int r = min((int)threadIdx.x * per, a.R);
  i64 left = index - before, n = prompt_tiles(a, r);
  for (; left >= n; n = prompt_tiles(a, ++r)) left -= n;
  *s_r = r;
  *s_tile = (int)(n - 1 - left);
}

template <int FMT, bool QFP16, int D>
__global__ void __launch_bounds__(PR_THREADS, 1) attend_prompt_kernel(const Attend a, const __grid_constant__ CUtensorMap map, const __grid_constant__ CUtensorMap q_map) {
  constexpr bool PACKED = FMT == PTSTORE_KV_PACKED;
  constexpr bool F16 = PACKED || FMT == PTSTORE_KV_FP16;
  constexpr int TB = PromptShape<D>::TILE_BYTES, CPR = D / 8;           // bytes of a tile, 16-byte chunks of a row
  extern __shared__ unsigned char smem_raw[];
  unsigned char* const smem = smem_raw + ((1024 - (smem_addr(smem_raw) & 1023)) & 1023);
  __shared__ __align__(8) u64 b_q[2], b_full[PR_SLOTS], b_empty[PR_SLOTS], b_s[2], b_pa[2], b_pb[2], b_o[2], b_end, b_raw[PR_RAW], b_raw_free[PR_RAW];
  __shared__ u32 s_tmem;
  __shared__ int s_gave_up, s_any_bad, s_r, s_tile;
  __shared__ i64 s_scan[PR_THREADS / 32];
  __shared__ i64 s_row[2][PR_KEYS];          // byte offset of a key's row (4-bit: of its tile), -1: not there
  __shared__ u32 s_valid[4][4];              // keys of a step that are there, by step & 3
  __shared__ int s_bad[3][D];                // first key whose V holds NaN, +inf, -inf in column d, among keys that some rows do not see
  __shared__ float s_qf[PR_ROWS];
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(FULL, tid >> 5, 0);

  // ---- which 256 rows: heads vary fastest; a request's tiles come last to first, the ones with most keys first
  int h, part = 0, parts = 1;                // this CTA's chunk of the tile's steps
  u32 cta = blockIdx.x, slot = 0;            // row tile; where a chunk leaves its sums
  {
    if (tid == 0) { s_gave_up = 0; s_any_bad = 0; }
    if (!PACKED && tid == 32) {               // the maps are fetched while the tile is being found
      if (a.box_tokens) asm volatile("prefetch.tensormap [%0];" ::"l"(&map) : "memory");
      if (a.q_box) asm volatile("prefetch.tensormap [%0];" ::"l"(&q_map) : "memory");
    }
    i64 mine, before;
    const i64 all = count_tiles<PR_THREADS>(a, s_scan, mine, before);
    if (a.split) {
      const Cut cut = cut_of(all * a.cache.heads, a.split);
      if (cta >= cut.first && cut.parts > 1) {
        slot = cta - (u32)cut.first;
        parts = cut.parts;
        part = slot % parts;
        cta = (u32)cut.first + slot / parts;
      }
    }
    h = cta % a.cache.heads;
    const i64 index = cta / a.cache.heads;
    if (tid == 0) s_r = -1;
    __syncthreads();
    find_tile<PR_THREADS>(a, index, mine, before, &s_r, &s_tile);
    if (tid == 0) {
      for (int i = 0; i < 2; ++i) { bar_init(&b_q[i], 128); bar_init(&b_s[i], 1); bar_init(&b_pa[i], 128); bar_init(&b_pb[i], 128); bar_init(&b_o[i], 1); }
      for (int i = 0; i < PR_SLOTS; ++i) { bar_init(&b_full[i], 128); bar_init(&b_empty[i], 1); }
      bar_init(&b_end, 1);
      for (int i = 0; i < PR_RAW; ++i) { bar_init(&b_raw[i], 1); bar_init(&b_raw_free[i], 128); }
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    for (int i = tid; i < 3 * D; i += PR_THREADS) (&s_bad[0][0])[i] = 0x7FFFFFFF;
    __syncthreads();
  }
  const int r = s_r;
  if (r < 0) return;                          // a CTA beyond the last tile
  const Req rq = request(a, r);
  const int row_base = s_tile * PR_ROWS, rows = min(PR_ROWS, rq.fresh * a.group - row_base);
  // keys the rows of each tile see (its last row), and the first row
  auto keys_of = [&](int row) {
    const i64 k = (i64)rq.pos0 + (row_base + row) / a.group + 1;
    return k < 0 ? 0 : k > rq.keys ? rq.keys : (int)k;
  };
  const int keys0 = keys_of(min(rows, 128) - 1), keys1 = rows > 128 ? keys_of(rows - 1) : 0;
  const int keys = max(keys0, keys1), all_see = keys_of(0);
  int steps[2] = {(keys0 + PR_KEYS - 1) / PR_KEYS, (keys1 + PR_KEYS - 1) / PR_KEYS};
  int key0 = 0;                               // first key of this CTA's steps
  if (parts > 1) {
    const int len = (max(steps[0], steps[1]) + parts - 1) / parts, j0 = part * len;
    steps[0] = min(max(steps[0] - j0, 0), len);
    steps[1] = min(max(steps[1] - j0, 0), len);
    key0 = j0 * PR_KEYS;
  }
  const int n_steps = max(steps[0], steps[1]);
  const u32 smem_q = smem_addr(smem), smem_kv = smem_q + 2 * TB;

  // tensor memory: allocated by warp 12 while the others load; 12 and the softmax warps meet before they use it
  auto tmem_there = [&]() {
    tc_fence_before();
    asm volatile("bar.sync 4, 288;" ::: "memory");
    tc_fence_after();
    return *reinterpret_cast<volatile u32*>(&s_tmem);
  };

  if (warp >= 12) {
    // ======== tensor instructions
    regs_fewer<40>();
    u32 tmem = 0;
    if (warp == 12) {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(&s_tmem)) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
      tmem = tmem_there();
    }
    if (warp == 12) {                         // the whole warp walks the steps, one lane issues: operands stay warp-uniform
      constexpr u32 QK = mma_desc(F16, PR_KEYS, false), PV = mma_desc(F16, D, true);
      bool quit = false;                      // a wait ran out: nothing is issued from there on
      auto wait = [&](u64* b, u32 parity) {
        if (!quit && !__all_sync(FULL, bar_wait(b, parity, a.polls, &s_gave_up))) quit = true;
      };
      auto slot_wait = [&](int op) {
        wait(&b_full[op % PR_SLOTS], (op / PR_SLOTS) & 1);
        if (!PACKED && !a.box_tokens) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");      // tiles written through the generic proxy
      };
      auto scores = [&](int w, int op) {
        const u64 qa = operand_desc(smem_q + w * TB, 0), kb = operand_desc(smem_kv + (op % PR_SLOTS) * TB, 0);
        if (!quit && elected()) {
#pragma unroll
          for (int k = 0; k < D / 16; ++k) {  // 16 elements: 32 bytes further in a row, or the next 64-element half
            const u64 off = (u64)(((k >> 2) * (PR_KEYS * 128) + (k & 3) * 32) >> 4);
            mma_ss(tmem + w * 128, qa + off, kb + off, QK, k > 0);
          }
          tc_commit(&b_s[w]);
        }
        __syncwarp();
      };
      auto values = [&](int w, int op, int half, bool add) {
        const u64 vb = operand_desc(smem_kv + (op % PR_SLOTS) * TB, PR_KEYS * 128);
        if (!quit && elected()) {
#pragma unroll
          for (int i = 0; i < PR_KEYS / 32; ++i) {   // 16 keys: 16 rows of 128 bytes; 8 columns of P
            const int k = half * (PR_KEYS / 32) + i;
            mma_ts(tmem + 256 + w * 128, tmem + w * 128 + k * 8, vb + (u64)((k * 16 * 128) >> 4), PV, add || k > 0);
          }
        }
        __syncwarp();
      };
      auto release = [&](int op) {
        if (!quit && elected()) tc_commit(&b_empty[op % PR_SLOTS]);
        __syncwarp();
      };
      for (int w = 0; w < 2; ++w)
        if (steps[w] > 0) wait(&b_q[w], 0);
      if (n_steps > 0) {
        slot_wait(0);
        tc_fence_after();
        for (int w = 0; w < 2; ++w)
          if (steps[w] > 0) scores(w, 0);
        release(0);
        slot_wait(1);
      }
      // V of step j and K of step j + 1 have been waited for by the time they are needed: the waits sit where the other tile's weights
      // would be waited for anyway
      for (int j = 0; j < n_steps && !quit && !__any_sync(FULL, *reinterpret_cast<volatile int*>(&s_gave_up)); ++j) {
        const int kop = 2 * (j + 1), vop = 2 * j + 1;
        if (j + 1 < n_steps) slot_wait(kop);
        for (int w = 0; w < 2; ++w) {
          if (j < steps[w]) {
            wait(&b_pa[w], j & 1);
            tc_fence_after();
            values(w, vop, 0, j > 0);
            wait(&b_pb[w], j & 1);
            tc_fence_after();
            values(w, vop, 1, true);
            if (j + 1 == steps[w]) { if (!quit && elected()) tc_commit(&b_o[w]); __syncwarp(); }
          }
          if (w == 1) release(vop);
          if (j + 1 < steps[w]) scores(w, kop);
          if (w == 0 && j + 1 < n_steps) slot_wait(vop + 2);
        }
        if (j + 1 < n_steps) release(kop);
      }
      // everything issued has ended before tensor and shared memory are given back (q's loads too, where their wait ran out)
      for (int w = 0; w < 2; ++w)
        if (steps[w] > 0) bar_drain(&b_q[w], 0);
      if (elected()) tc_commit(&b_end);
      __syncwarp();
      bar_drain(&b_end, 0);
    }
    if (PACKED && warp == 13) {
      // ======== 4-bit tiles as they lie in the cache: lanes 0-7 a 16-token tile each, the table entries of the next step on their way
      constexpr int RAW = PromptShape<D>::RAW_BYTES, TILES = PR_KEYS / TILE;
      const u32 raw = smem_kv + PR_SLOTS * TB, B = a.cache.block_tokens;
      const int* table = a.tables + (i64)r * a.max_blocks;
      bool bounds = false;
      int next_id = -1;
      i64 tile_off = -1;
      auto look_up = [&](int j) {
        const int key = key0 + j * PR_KEYS + lane * TILE;
        next_id = lane < TILES && key < keys ? table[(u32)key / B] : -1;
      };
      if (n_steps > 0) look_up(0);
      int op = 0;
      for (; op < 2 * n_steps && !__any_sync(FULL, *reinterpret_cast<volatile int*>(&s_gave_up)); ++op) {
        const int j = op >> 1, key = key0 + j * PR_KEYS + lane * TILE;
        if (op >= PR_RAW && !__all_sync(FULL, bar_wait(&b_raw_free[op % PR_RAW], (op / PR_RAW - 1) & 1, a.polls, &s_gave_up))) break;
        __syncwarp();
        if (!(op & 1)) {
          const bool in = lane < TILES && key < keys, have = in && (u32)next_id < a.cache.num_blocks;
          bounds |= in && !have;
          tile_off = have ? (i64)((u64)(u32)next_id * a.cache.block_stride + ((u64)h * (B / TILE) + (u32)key % B / TILE) * tile_bytes(D)) : -1;
          const u32 bits = !have ? 0 : keys - key >= TILE ? 0xFFFFu : (1u << (keys - key)) - 1u;       // keys of the tile that are there
          const u32 lo = __shfl_sync(FULL, bits, 2 * lane & 31), hi = __shfl_sync(FULL, bits, (2 * lane + 1) & 31);
          if (lane < 4) s_valid[j & 3][lane] = lo | (hi << 16);
          if (j + 1 < n_steps) look_up(j + 1);
        }
        const u32 there = __ballot_sync(FULL, tile_off >= 0);
        u64* bar = &b_raw[op % PR_RAW];
        if (lane == 0) bar_expect(bar, __popc(there) * tile_bytes(D));
        __syncwarp();
        if (tile_off >= 0) bulk_load(raw + (op % PR_RAW) * RAW + lane * tile_bytes(D), a.cache.base + (op & 1 ? a.cache.kv_stride : 0) + tile_off, tile_bytes(D), bar);
      }
      // whatever happened, what is in flight lands before the CTA gives its memory back
      for (int k = max(0, op - PR_RAW); k < op; ++k)
        bar_drain(&b_raw[k % PR_RAW], (k / PR_RAW) & 1);
      if (bounds && a.status) atomicOr(a.status, PTSTORE_S_BOUNDS);
    }
    __syncwarp();
  } else if (warp >= 8) {
    // ======== K and V into the ring
    regs_fewer<PACKED ? 88 : 72>();
    const int pt = tid - 256;
    const int* table = a.tables + (i64)r * a.max_blocks;
    const u32 B = a.cache.block_tokens;
    bool bounds = false;
    const volatile int* const gave_up = &s_gave_up;
    // where key `pt` of a step lies
    u32 id = 0;
    auto where = [&](int j) -> i64 {
      const int key = key0 + j * PR_KEYS + pt;
      if (key >= keys) return -1;
      const u32 blk = (u32)key / B, in = (u32)key % B;
      id = (u32)table[blk];
      if (id >= a.cache.num_blocks) { bounds = true; return -1; }
      const i64 base = (i64)((u64)id * a.cache.block_stride);
      if (PACKED) return base + (i64)((u64)h * (B / TILE) + in / TILE) * tile_bytes(D);
      return base + (i64)(((u64)in * a.cache.heads + h) * (D * 2));
    };
    auto wait_empty = [&](int op) { return op < PR_SLOTS || bar_wait(&b_empty[op % PR_SLOTS], ((op / PR_SLOTS) - 1) & 1, a.polls, &s_gave_up); };
    auto note_bad = [&](int d, int kind, int key) {
      atomicMin(&s_bad[kind][d], key);
      s_any_bad = 1;
    };
    if (!PACKED) {
      // chunk pt % CPR of rows pt / CPR, pt / CPR + 128 / CPR, ...
      constexpr int RPP = 128 / CPR;
      const int c = pt % CPR, r0 = pt / CPR;
      // keys that some of the rows do not see: a weight of zero would not hide an infinity or a NaN, so they are taken out here
      // and put into the rows that see them at the end
      auto mend = [&](int op) {
        unsigned char* t = smem + (2 + op % PR_SLOTS) * TB;
        constexpr u32 EX = F16 ? 0x7C00u : 0x7F80u, MANT = F16 ? 0x03FFu : 0x007Fu;
        for (int i = 0; i < CPR; ++i) {
          const int n = i * RPP + r0, key = key0 + (op >> 1) * PR_KEYS + n;
          if (key < all_see) continue;
          unsigned short* p = reinterpret_cast<unsigned short*>(t + operand_at(n, c));
          const uint4 v = *reinterpret_cast<const uint4*>(p);
          const u32 w[4] = {v.x, v.y, v.z, v.w};
          bool odd = false;
#pragma unroll
          for (int k = 0; k < 4; ++k) odd |= (w[k] & EX) == EX || ((w[k] >> 16) & EX) == EX;
          if (odd)
            for (int k = 0; k < 8; ++k)
              if ((p[k] & EX) == EX) {
                note_bad(c * 8 + k, (p[k] & MANT) ? 0 : (p[k] & 0x8000u) ? 2 : 1, key);
                p[k] = 0;
              }
        }
      };
      // A step whose keys are all there and seen by all rows comes through the tensor map where the block size allows one (blocks that
      // divide 128 tokens or are multiples of it): the first thread of every box issues it.  Other steps are copied 16 bytes at a
      // time, with zeros for keys that are not there.  (All by 16-byte copies: 4600 clocks per step of 2 x 32 KB and the tensor
      // cores waiting for them half of the time.)
      const u32 box = a.box_tokens;
      const bool leads = box && pt % box == 0;
      i64 next = n_steps > 0 ? where(0) : -1;
      int j = 0;
      for (; j < n_steps; ++j) {
        const u32 block = id;
        s_row[j & 1][pt] = next;
        const u32 present = __ballot_sync(FULL, next >= 0);
        if (lane == 0) s_valid[j & 3][warp - 8] = present;
        if (j + 1 < n_steps) next = where(j + 1);
        if (any_of_128(*gave_up)) break;      // the same in all 128 threads
        const bool plain = box && key0 + (j + 1) * PR_KEYS <= all_see && (s_valid[j & 3][0] & s_valid[j & 3][1] & s_valid[j & 3][2] & s_valid[j & 3][3]) == FULL;
        for (int is_v = 0; is_v < 2; ++is_v) {
          const int op = 2 * j + is_v;
          const bool free = wait_empty(op);
          // A slot that is not free gets no copy.  This thread arrives all the same, so that the operand's phase ends when the others' copies have landed,
          // but not before the phase of the operand that lies there has ended (all its arrivals are in, its copies may be on their way).
          if (!free) bar_drain(&b_full[op % PR_SLOTS], ((op / PR_SLOTS) - 1) & 1);
          const u32 dst = smem_kv + (op % PR_SLOTS) * TB;
          u64* full = &b_full[op % PR_SLOTS];
          if (plain) {
            if (leads && free) {
              bar_expect(full, box * D * 2);
#pragma unroll
              for (int e = 0; e < D / 64; ++e)
                tensor_load(dst + e * (PR_KEYS * 128) + pt * 128, &map, e * 64, h, (int)((u32)(key0 + j * PR_KEYS + pt) % B), (int)block, is_v, full);
            } else bar_arrive(full);
            continue;
          }
          const unsigned char* base = a.cache.base + (is_v ? a.cache.kv_stride : 0) + c * 16;
#pragma unroll 4
          for (int i = 0; i < CPR && free; ++i) {
            const int n = i * RPP + r0;
            const i64 off = s_row[j & 1][n];
            cp_async16_or_zero(dst + operand_at(n, c), base + (off < 0 ? 0 : off), off >= 0);
          }
          if (box || (is_v && key0 + (j + 1) * PR_KEYS > all_see)) {
            cp_commit();
            cp_wait<0>();
            if (free && is_v && key0 + (j + 1) * PR_KEYS > all_see) mend(op);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            bar_arrive(full);
          } else cp_arrive(full);             // arrives when this thread's copies have landed
        }
      }
      // whatever happened, what is in flight lands before the CTA gives its memory back
      for (int op = max(0, 2 * j - PR_SLOTS); op < 2 * j; ++op)
        bar_drain(&b_full[op % PR_SLOTS], (op / PR_SLOTS) & 1);
      cp_commit();
      cp_wait<0>();
    } else {
      // The tiles come as they lie in the cache, by bulk copies three operands ahead, which warp 13 issues (loaded into registers one
      // operand ahead a step took 5900 clocks, the time of two dependent loads per operand; issued by warp 8, 6000); one key per thread is unpacked and stored as fp16.  Element order
      // inside eight is 0 4 1 5 2 6 3 7, as the unpacking yields it: Q is stored likewise, and O's columns are put back at the end.
      constexpr int RAW = PromptShape<D>::RAW_BYTES;
      unsigned char* const raw = smem + (2 + PR_SLOTS) * TB;
      const Magic mg = magic();
      // a key's places: 16-byte chunk c of its codes at from ^ 16 c, chunk c of its operand row at to ^ 16 (c % 8)
      const int n = pt % TILE;
      const u32 from = (pt / TILE) * tile_bytes(D) + code_place(D, n, 0) * 16, to = (u32)operand_at(pt, 0);
      const u32 scales = (pt / TILE) * tile_bytes(D);
      for (int op = 0; op < 2 * n_steps && !__any_sync(FULL, *gave_up); ++op) {
        const int j = op >> 1, key = key0 + j * PR_KEYS + pt;
        if (!__all_sync(FULL, bar_wait(&b_raw[op % PR_RAW], (op / PR_RAW) & 1, a.polls, &s_gave_up))) break;
        const bool is_v = op & 1, has = (s_valid[j & 3][pt >> 5] >> (pt & 31)) & 1, look = is_v && has && key >= all_see;
        const unsigned char* const src = raw + (op % PR_RAW) * RAW;
        const unsigned char* const sc = src + scales + (is_v ? scale_at(D, true, n, 0) : scale_at(D, false, n, 0));
        const u32 stride = is_v ? TILE : 1;   // of a key's scales
        unsigned char* const t = smem + (2 + op % PR_SLOTS) * TB;
        if (!__all_sync(FULL, wait_empty(op))) break;
#pragma unroll 2
        for (int c = 0; c < D / 32; ++c) {    // 32 elements: two scale groups, four chunks of the operand
          const uint4 four = has ? *reinterpret_cast<const uint4*>(src + (from ^ (u32)(c * 16))) : make_uint4(0, 0, 0, 0);
          u32 b0 = has ? sc[(2 * c) * stride] : 0, b1 = has ? sc[(2 * c + 1) * stride] : 0;
          if (look) {
            if ((b0 & 0x7Fu) == 0x7Fu) {
              for (int k = 0; k < 16; ++k) note_bad(32 * c + k, 0, key);
              b0 = 0;
            }
            if ((b1 & 0x7Fu) == 0x7Fu) {
              for (int k = 0; k < 16; ++k) note_bad(32 * c + 16 + k, 0, key);
              b1 = 0;
            }
          }
          // (of a key that is not there the scale is zero, and so are its values)
          const Deq d0 = deq_of(e4m3x2_to_half2(b0 * 0x101u)), d1 = deq_of(e4m3x2_to_half2(b1 * 0x101u));
          const u32 code[4] = {four.x, four.y, four.z, four.w};
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            u32 o[4];
            deq4(code[w], code[w] >> 8, w < 2 ? d0 : d1, mg, o);
            const u32 ch = 4 * c + w;
            *reinterpret_cast<uint4*>(t + (ch >> 3) * (PR_KEYS * 128) + (to ^ ((ch & 7) * 16))) = make_uint4(o[0], o[1], o[2], o[3]);
          }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        bar_arrive(&b_full[op % PR_SLOTS]);
        bar_arrive(&b_raw_free[op % PR_RAW]);
      }
    }
    if (bounds && a.status) atomicOr(a.status, PTSTORE_S_BOUNDS);
  } else {
    // ======== softmax of tile w
    regs_more<PACKED ? 192 : 200>();
    const int w = warp >> 2, t = tid & 127, row = w * 128 + t;
    // its half of Q.  Through a tensor map where the group divides a tile (rows behind the request's last bring someone's values or
    // zeros along and are not stored); else chunk t % CPR of rows t / CPR, ..., all on their way before the first is used, with the
    // sign of the softmax scale and the changes a 4-bit cache asks for.  (Copied by the threads a CTA's first scores came 6000
    // clocks later, of 50,000 to 150,000 in all.)
    // A tile without steps loads none: nobody would wait for it, and the tile's output goes through the same memory.
    if (!PACKED && a.q_box) {
      if (steps[w] == 0) {
      } else if (t == 0) {
        bar_expect(&b_q[w], TB);
#pragma unroll
        for (int e = 0; e < D / 64; ++e)
          tensor_load_q(smem_q + w * TB + e * (PR_KEYS * 128), &q_map, e * 64, h * a.group, rq.row0 + (row_base + w * 128) / a.group, &b_q[w]);
      } else bar_arrive(&b_q[w]);
    } else {
      constexpr int RPP = 128 / CPR;
      const int c = t % CPR;
      const bool flip = a.scale2 < 0.0f;
      uint4 raw[CPR];
      const u32 first = row_base + w * 128 + t / CPR, group = a.group, step_fr = RPP / group, step_hq = RPP % group;
      u32 fr = first / group, hq = first % group;
      const unsigned char* const q0 = a.q + 2 * ((i64)rq.row0 * a.q_token + (i64)h * group * a.q_head + c * 8);
#pragma unroll
      for (int i = 0; i < CPR; ++i) {
        raw[i] = make_uint4(0, 0, 0, 0);
        if (w * 128 + i * RPP + t / CPR < rows) raw[i] = *reinterpret_cast<const uint4*>(q0 + 2 * (fr * a.q_token + hq * a.q_head));       // (out may be q)
        hq += step_hq;
        fr += step_fr;
        if (hq >= group) { hq -= group; ++fr; }
      }
#pragma unroll
      for (int i = 0; i < CPR; ++i) {
        const int n = i * RPP + t / CPR, gr = w * 128 + n;
        const uint4 v = raw[i];
        u32 x[4] = {v.x, v.y, v.z, v.w};
        float factor = 1.0f;
        if (PACKED && !QFP16) {
          // bf16 rows as fp16, scaled by a power of two so that the largest element is in [1, 2): elements below 2^-14 of it lose
          // at most 2^-25 of it, all others nothing
          float amax = 0.0f;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float2 f = unpack2<false>(x[k]);
            amax = fmaxf(amax, fmaxf(fabsf(f.x), fabsf(f.y)));
          }
#pragma unroll
          for (int o = 1; o < CPR; o <<= 1) amax = fmaxf(amax, __shfl_xor_sync(FULL, amax, o));
          int e = amax > 0.0f ? (int)(__float_as_uint(amax) >> 23) - 127 : 0;
          e = e < -126 ? -126 : e > 126 ? 126 : e;
          factor = __uint_as_float((u32)(127 + e) << 23);
          const float down = __uint_as_float((u32)(127 - e) << 23);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float2 f = unpack2<false>(x[k]);
            x[k] = pack2<true>(f.x * down, f.y * down);
          }
        }
        if (flip) {
#pragma unroll
          for (int k = 0; k < 4; ++k) x[k] ^= 0x80008000u;
        }
        if (PACKED) {                         // element order 0 4 1 5 2 6 3 7
          const u32 y[4] = {__byte_perm(x[0], x[2], 0x5410), __byte_perm(x[0], x[2], 0x7632), __byte_perm(x[1], x[3], 0x5410), __byte_perm(x[1], x[3], 0x7632)};
#pragma unroll
          for (int k = 0; k < 4; ++k) x[k] = y[k];
        }
        *reinterpret_cast<uint4*>(smem + w * TB + operand_at(n, c)) = make_uint4(x[0], x[1], x[2], x[3]);
        if (PACKED && !QFP16 && c == 0) s_qf[gr] = factor;
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      bar_arrive(&b_q[w]);
    }
    const u32 tmem = tmem_there();            // (and every row's factor is there)
    // scale2 as a positive number: of zero, the smallest that keeps masked scores at minus infinity; finite, so that scores of zero stay zero
    const float scale2 = fminf(fmaxf(fabsf(a.scale2) * (PACKED && !QFP16 ? s_qf[row] : 1.0f), 0x1p-126f), 0x1.fffffep127f);
    const int see = row < rows ? keys_of(row) : 0;
    const u32 lane_base = (u32)(32 * (warp & 3)) << 16;
    const u32 ts = tmem + lane_base + w * 128, to = tmem + lane_base + 256 + w * 128;
    float m = -INFINITY, l = 0.0f;
    bool large = false;                       // a row's reference is beyond 2^24
    for (int j = 0; j < steps[w]; ++j) {
      bar_wait(&b_s[w], j & 1, a.polls, &s_gave_up);
      if (__any_sync(FULL, *reinterpret_cast<volatile int*>(&s_gave_up))) break;
      tc_fence_after();
      float s[4][32];
#pragma unroll
      for (int c = 0; c < 4; ++c) tc_ld32(s[c], ts + 32 * c);
      tc_wait_ld();
#pragma unroll
      for (int c = 0; c < 4; ++c) tc_loaded(s[c]);
      u32 there[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) there[c] = s_valid[j & 3][c];
      const int k0 = key0 + j * PR_KEYS;
      if (k0 + PR_KEYS > all_see || (there[0] & there[1] & there[2] & there[3]) != FULL) {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const int left = see - k0 - 32 * c;             // keys of this chunk the row sees
          const u32 mask = there[c] & (left >= 32 ? FULL : left <= 0 ? 0u : (1u << left) - 1u);
#pragma unroll
          for (int i = 0; i < 32; ++i) s[c][i] = (mask >> i) & 1 ? s[c][i] : -INFINITY;
        }
      }
      // Weights of keys 64 half .. + 63 from the reference, into P.  The first half starts from the reference as it
      // stands while the maximum over all 128 keys is found in between (two keys with every weight).  All on the special function unit:
      // a quarter / a third / half of them by a polynomial on the multiply-add units cost 4 / 8 / 19 % of a 16k prompt's
      // time, since what bounds this loop is its instructions.
      float x[4] = {s[0][0], s[0][1], s[0][2], s[0][3]};
      float sum0, sum1;
      auto weights = [&](int half, bool find, u32 (&p)[32]) {
        const float ref = m == -INFINITY ? 0.0f : m;
        const u64 sc2 = pair(scale2, scale2), neg = pair(-ref, -ref);
        u64 sum[2] = {0, 0}, e[32];
        constexpr int LAG = 4;                // pairs on their way through the special function unit (8 clocks a value, some 40 to the result)
#pragma unroll
        for (int i = 0; i < 32 + LAG; ++i) {
          if (i < 32) {
            const int c = 2 * half + i / 16, k = 2 * i % 32;
            const u64 y = fma_pair(pair(s[c][k], s[c][k + 1]), sc2, neg);
            e[i] = pair(exp2_fast(lo_of(y)), exp2_fast(hi_of(y)));
            if (find) {
              const int k4 = 4 * i;
#pragma unroll
              for (int z = 0; z < 4; z += 2) x[(i & 1) * 2 + z / 2] = fmaxf(x[(i & 1) * 2 + z / 2], fmaxf(s[k4 / 32][k4 % 32 + z], s[k4 / 32][k4 % 32 + z + 1]));
            }
          }
          if (i >= LAG) {
            sum[i & 1] = add_pair(sum[i & 1], e[i - LAG]);
            p[i - LAG] = pack2<F16>(lo_of(e[i - LAG]), hi_of(e[i - LAG]));
          }
        }
        const u64 both = add_pair(sum[0], sum[1]);
        (half ? sum1 : sum0) = lo_of(both) + hi_of(both);
      };
      u32 p[32];
      if (j > 0) weights(0, true, p);
      else {                                  // there is no reference yet
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int i = 0; i < 32; ++i) x[c] = fmaxf(x[c], s[c][i]);
      }
      const float top = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])) * scale2;
      // the reference moves only when a weight would pass 2^8 (scores are in powers of two here)
      const bool move = top > m + 8.0f || (m == -INFINITY && top > m);
      if (__any_sync(FULL, move) || j == 0) {
        const float f = move ? exp2_fast(m - top) : 1.0f;
        if (move) { m = top; l *= f; }
        large = __any_sync(FULL, fabsf(m) > 0x1p24f && m != -INFINITY);
        if (j > 0) {
#pragma unroll 1
          for (int c = 0; c < D; c += 32) {
            float o[32];
            tc_ld32(o, to + c);
            tc_wait_ld();
            tc_loaded(o);
            u32 scaled[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) scaled[i] = __float_as_uint(o[i] * f);
            tc_st32(to + c, scaled);
          }
        }
        weights(0, false, p);
      }
      // A reference is a rounded product.  Beyond 2^24 its rounding is a step in the exponent or more (a largest weight that is not near 1, or out of
      // range): products are then rounded likewise before the reference is taken off.  Scores are read once more, 32 keys at a time, their weights go
      // where scores that have been read lay.
      if (large) {
        const float ref = m == -INFINITY ? 0.0f : m;
#pragma unroll 1
        for (int c = 0; c < 4; ++c) {
          float v[32];
          tc_ld32(v, ts + 32 * c);
          tc_wait_ld();
          tc_loaded(v);
          const int left = (row < rows ? keys_of(row) : 0) - key0 - j * PR_KEYS - 32 * c;
          const u32 mask = s_valid[j & 3][c] & (left >= 32 ? FULL : left <= 0 ? 0u : (1u << left) - 1u);
          u32 q[16];
#pragma unroll
          for (int i = 0; i < 32; i += 2) {
            const float e0 = (mask >> i) & 1 ? exp2_fast(__fmul_rn(v[i], scale2) - ref) : 0.0f;
            const float e1 = (mask >> (i + 1)) & 1 ? exp2_fast(__fmul_rn(v[i + 1], scale2) - ref) : 0.0f;
            l += e0 + e1;
            q[i / 2] = pack2<F16>(e0, e1);
          }
          tc_st16(ts + 16 * c, q);
          if (c & 1) {
            tc_wait_st();
            tc_fence_before();
            bar_arrive(c == 1 ? &b_pa[w] : &b_pb[w]);
          }
        }
        continue;
      }
      tc_st32(ts, p);
      tc_wait_st();
      tc_fence_before();
      bar_arrive(&b_pa[w]);                   // the tensor cores start on these while the second half is computed
      weights(1, false, p);
      tc_st32(ts + 32, p);
      l += sum0 + sum1;
      tc_wait_st();
      tc_fence_before();
      bar_arrive(&b_pb[w]);
    }
    // ---- output
    if (steps[w] > 0) {
      bar_wait(&b_o[w], 0, a.polls, &s_gave_up);
      tc_fence_after();
    }
    if (!__any_sync(FULL, *reinterpret_cast<volatile int*>(&s_gave_up))) {
      const float f = parts > 1 ? 1.0f : l == 0.0f ? 0.0f : a.v_factor / l;
      float* const sums = reinterpret_cast<float*>(a.work + PR_PARTS_AT) + (i64)slot * prompt_part_floats<D>();
      if (parts > 1) {
        sums[PR_ROWS * D + row] = m;
        sums[PR_ROWS * D + PR_ROWS + row] = l;
      }
      // through shared memory (the tile's Q is not needed any more), so that the stores are whole rows
      i64 at = -1;                            // of this thread's row, in elements
      if (row < rows) {
        const u32 flat = row_base + row, fr = flat / (u32)a.group;
        at = (i64)(rq.row0 + (int)fr) * a.o_token + (i64)(h * a.group + (int)(flat - fr * a.group)) * a.o_head;
      }
      unsigned char* const mine = smem + w * TB;
#pragma unroll
      for (int c = 0; c < D; c += 32) {
        float o[32];
        if (steps[w] > 0) {
          tc_ld32(o, to + c);
          tc_wait_ld();
          tc_loaded(o);
        }
#pragma unroll
        for (int i = 0; i < 32; ++i) o[i] = steps[w] > 0 ? o[i] * f : 0.0f;        // (weights that are all zero leave zeros)
        if (PACKED) {
#pragma unroll
          for (int i = 0; i < 32; i += 8) {
            const float v[8] = {o[i], o[i + 1], o[i + 2], o[i + 3], o[i + 4], o[i + 5], o[i + 6], o[i + 7]};
#pragma unroll
            for (int k = 0; k < 8; ++k) o[i + (k >> 1) + 4 * (k & 1)] = v[k];
          }
        }
        if (s_any_bad) {
          for (int i = 0; i < 32; ++i) {
            const bool nan = s_bad[0][c + i] < see, pos = s_bad[1][c + i] < see, neg = s_bad[2][c + i] < see;
            if (nan || (pos && neg)) o[i] = NAN;
            else if (pos) o[i] = o[i] + INFINITY;
            else if (neg) o[i] = o[i] - INFINITY;
          }
        }
        if (parts > 1) {
          if (row < rows) {
#pragma unroll
            for (int i = 0; i < 32; i += 4) *reinterpret_cast<float4*>(sums + row * D + c + i) = make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]);
          }
          continue;
        }
#pragma unroll
        for (int i = 0; i < 32; i += 8)
          *reinterpret_cast<uint4*>(mine + operand_at(t, (c + i) / 8)) =
              make_uint4(pack2<QFP16>(o[i], o[i + 1]), pack2<QFP16>(o[i + 2], o[i + 3]), pack2<QFP16>(o[i + 4], o[i + 5]), pack2<QFP16>(o[i + 6], o[i + 7]));
      }
      __syncwarp();
#pragma unroll 8
      for (int i = 0; i < CPR && parts == 1; ++i) {         // this warp's 32 rows, whole rows at a time
        const int n = i * (32 / CPR) + lane / CPR, c = lane % CPR;
        const i64 to = __shfl_sync(FULL, at, n);
        if (to >= 0) *reinterpret_cast<uint4*>(a.out + 2 * (to + c * 8)) = *reinterpret_cast<const uint4*>(mine + operand_at((warp & 3) * 32 + n, c));
      }
      // A row without weights, written as zeros, may be one whose scores are all minus infinity.  (Looked at here: chosen together with f it costs the
      // 4-bit kernel registers, and suffixes 2 to 6 %.)
      if (__any_sync(FULL, f == 0.0f && at >= 0)) {
        __syncwarp();
        if (f == 0.0f && at >= 0) {
          const int req = *reinterpret_cast<volatile int*>(&s_r), first = *reinterpret_cast<volatile int*>(&s_tile) * PR_ROWS;
          const float nan = row_factor(a, req, (i64)request(a, req).pos0 + (first + row) / a.group, 0.0f);
          if (nan != 0.0f)
            for (int c = 0; c < D; c += 8) {
              const u32 two = pack2<QFP16>(nan, nan);
              *reinterpret_cast<uint4*>(a.out + 2 * (at + c)) = make_uint4(two, two, two, two);
            }
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 12) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(s_tmem) : "memory");
    if (lane == 0 && s_gave_up && a.status) atomicOr(a.status, PTSTORE_S_TIMEOUT);
  }
}

// Joins the chunks of the row tiles that were cut: blockIdx.x the tile (behind the uncut ones), blockIdx.y some of its rows, a warp
// for K, whose loads are in flight together (K = 1 spreads few tiles over more warps).  Four CTAs an SM: the largest grid, 74 x 8, is one round.
template <bool QFP16, int D, int K>
__global__ void __launch_bounds__(256, 4) attend_join_kernel(const Attend a) {
  __shared__ i64 s_scan[8];
  __shared__ int s_r, s_tile;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  i64 mine, before;
  const i64 all = count_tiles<256>(a, s_scan, mine, before) * a.cache.heads;
  const Cut cut = cut_of(all, a.split);
  const i64 cta = cut.first + blockIdx.x;
  if (cut.parts <= 1 || cta >= all) return;
  if (threadIdx.x == 0) s_r = -1;
  __syncthreads();
  find_tile<256>(a, cta / a.cache.heads, mine, before, &s_r, &s_tile);
  __syncthreads();
  if (s_r < 0) return;
  const Req q = request(a, s_r);
  const int h = (int)(cta % a.cache.heads), parts = cut.parts, row_base = s_tile * PR_ROWS, rows = min(PR_ROWS, q.fresh * a.group - row_base);
  const float* const base = reinterpret_cast<const float*>(a.work + PR_PARTS_AT) + (i64)blockIdx.x * parts * prompt_part_floats<D>();
  constexpr int E = D / 32, PF = prompt_part_floats<D>();
  const int at0 = (blockIdx.y * 8 + warp) * K;
  if (at0 >= rows) return;
  // lane p holds m and l of part p (of 32 at a time); rows behind the last one are read, not written (the tile's memory holds 256)
  float top[K], sum[K] = {}, acc[K][E] = {};
#pragma unroll
  for (int k = 0; k < K; ++k) {
    top[k] = -INFINITY;
    for (int p = lane; p < parts; p += 32) top[k] = fmaxf(top[k], base[(i64)p * PF + PR_ROWS * D + at0 + k]);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) top[k] = fmaxf(top[k], __shfl_xor_sync(FULL, top[k], o));
  }
  for (int p0 = 0; p0 < parts; p0 += 32) {
    float f[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      f[k] = 0.0f;
      if (p0 + lane < parts) {
        const float* x = base + (i64)(p0 + lane) * PF + PR_ROWS * D + at0 + k;
        const float m = x[0];
        f[k] = m == -INFINITY ? 1.0f : exp2_fast(m - top[k]);        // a chunk that the row sees nothing of: sums of zero (or NaN)
        sum[k] += x[PR_ROWS] * f[k];
      }
    }
    const int n = min(32, parts - p0);
#pragma unroll 4
    for (int p = 0; p < n; ++p) {
      __align__(16) float v[K][E];
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const float* x = base + (i64)(p0 + p) * PF + (at0 + k) * D + lane * E;
        if (E == 4) *reinterpret_cast<float4*>(v[k]) = *reinterpret_cast<const float4*>(x);
        else *reinterpret_cast<float2*>(v[k]) = *reinterpret_cast<const float2*>(x);
      }
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const float w = __shfl_sync(FULL, f[k], p);
#pragma unroll
        for (int e = 0; e < E; ++e) acc[k][e] += v[k][e] * w;
      }
    }
  }
  u32 none = 0;
#pragma unroll
  for (int k = 0; k < K; ++k) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) sum[k] += __shfl_xor_sync(FULL, sum[k], o);
    if (at0 + k >= rows) continue;
    const u32 flat = row_base + at0 + k, fr = flat / (u32)a.group;
    const float f = sum[k] == 0.0f ? 0.0f : a.v_factor / sum[k];
    if (sum[k] == 0.0f) none |= 1u << k;
    u32* const dst = reinterpret_cast<u32*>(a.out + 2 * ((i64)(q.row0 + (int)fr) * a.o_token + (i64)(h * a.group + (int)(flat - fr * a.group)) * a.o_head + lane * E));
#pragma unroll
    for (int e = 0; e < E; e += 2) dst[e / 2] = pack2<QFP16>(acc[k][e] * f, acc[k][e + 1] * f);
  }
  // rows without weights, written as zeros: as in the other kernel
  for (; none; none &= none - 1) {
    const int row = at0 + __ffs(none) - 1;
    const u32 flat = row_base + row, fr = flat / (u32)a.group;
    const float nan = row_factor(a, s_r, (i64)q.pos0 + fr, 0.0f);
    u32* const dst = reinterpret_cast<u32*>(a.out + 2 * ((i64)(q.row0 + (int)fr) * a.o_token + (i64)(h * a.group + (int)(flat - fr * a.group)) * a.o_head + lane * E));
    for (int e = 0; e < E && nan != 0.0f; e += 2) dst[e / 2] = pack2<QFP16>(nan, nan);
  }
}

}  // namespace ptk
