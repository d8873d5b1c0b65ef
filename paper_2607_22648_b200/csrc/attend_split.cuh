// Attention of a few query rows per request over a long paged cache (decode, speculative tokens): bounded by reading K and V once.
//
// o = sum_j p_j v_j / sum_j p_j, p_j = exp2(scale2 q.k_j - m): one pass over the cache with the running maximum m and sum per row.
// Work is cut into units of 64 tokens of one (request, row tile, kv head) item.  Where cutting every item into equal chunks
// gives at most one chunk per CTA without making the longest more than a quarter longer than an even share, a CTA takes one
// chunk.  Otherwise all units stand in one line and every CTA takes the same number of them, so ragged batches load every SM
// alike; a CTA then works on parts of two or three items, each of which costs it some 5 us of start and join, which is why
// chunks come first (one 4k request: 18.5 us with the line, whose CTAs straddle two kv heads, 15.9 us with chunks).  An item
// that spans several CTAs leaves partial sums (o, m, l in 32 bits) in the workspace, and the CTA that arrives last joins them
// in CTA order: the result does not depend on who that is.  One launch; the arrival counters are left zero.
//
// A row tile is 8 or 16 (query head of the group, new token) rows.  The tensor instructions (mma.sync m16n8k16; the work is a
// twentieth of what the tensor cores could do, and tcgen05's 64 or 128 rows would be mostly empty) take TOKENS as their 16 rows and
// queries as their 8 columns: S^T = K q^T, O^T = V^T P^T, so nothing is spent on rows that do not exist, and the 4-bit
// values are unpacked straight into the A operand.  P^T changes from accumulator to operand layout by movmatrix.
//
// The four warps of a CTA run alone, each on every fourth 16-token tile through its own ring of shared-memory stages (bulk copies of
// whole tiles of a 4-bit cache, 16-byte copies of a 16-bit one, whose blocks may have any size), and meet at the end of an item.
//
// B200, 64 ragged requests of 2064 to 6256 tokens, 32 query and 8 kv heads x 128: 16-bit cache 173 us = 6.0 TB/s (bound by HBM); 4-bit cache 98 us
// = 3.1 TB/s.  The latter waits for neither memory nor issue slots (48 % and 54 % busy) but for its own results: a warp's step is one chain of unpacking, products, a
// maximum across lanes, exponentials, unpacking, products, and four warps share a scheduler.  It has 400 instructions per 16 tokens and warp, of which 184 unpack
// codes (one LOP3 and one fused multiply-add per pair).  Two accumulator chains for S, one or four tiles per softmax step, 12 or
// 20 warps an SM were each measured no better (99, 104, 161, 102, 152 us).
#pragma once
#include "attend.cuh"

namespace ptk {

constexpr int MIN_TOKENS = 256;              // a CTA takes at least this many, so that joining does not cost more than it saves
constexpr int SP_PARTS_AT = 4096;            // where the parts begin in the workspace, behind the counters of the largest grid

template <int FMT, int D>
struct SplitShape {
  static constexpr bool PACKED = FMT == PTSTORE_KV_PACKED;
  static constexpr int WARPS = 4, THREADS = 32 * WARPS;
  static constexpr int UNIT = WARPS * TILE;                                        // tokens of a unit: one tile per warp
  static constexpr int STAGE = PACKED ? 2 * tile_bytes(D) : 2 * TILE * D * 2;      // K tile, V tile
  static constexpr int STAGES = (PACKED ? 4 : 2) * (128 / D);
  static constexpr int STEP = PACKED ? 2 : 1;                                      // tiles per softmax step
  static constexpr int RING = WARPS * STAGES * STAGE;
};
// CTAs per SM, by registers: 16 warps of 128 where a row tile has 8 rows of a 4-bit cache, 12 of 168 for a 16-bit one, 8 of 255 for 16 rows
template <int FMT, int NT>
__host__ __device__ constexpr int split_ctas() { return NT == 2 ? 2 : FMT == PTSTORE_KV_PACKED ? 4 : 3; }
// shared memory: the ring, which at the end of an item holds the warps' sums and then the maxima and sums of an item's parts (at most
// one part per CTA of MAX_SMS SMs)
constexpr int MAX_SMS = 160;
template <int FMT, int D, int NT>
constexpr int split_smem() {
  const int ring = SplitShape<FMT, D>::RING, sums = SplitShape<FMT, D>::WARPS * 8 * NT * (D + 4) * 4, parts = MAX_SMS * split_ctas<FMT, NT>() * 8 * NT * 8;
  return ring > sums ? (ring > parts ? ring : parts) : (sums > parts ? sums : parts);
}

template <int NT, int D>
__host__ __device__ constexpr int part_floats() { return 8 * NT * (D + 2); }      // partial sums of one item in one CTA: o, m, l

template <bool FP16>
__device__ __forceinline__ void mma16816(float (&c)[4], const u32 (&a)[4], const u32 (&b)[2]) {
  if (FP16)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
}
__device__ __forceinline__ u32 transpose8x8(u32 v) {
  u32 r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
__device__ __forceinline__ void ldsm4(u32 (&r)[4], u32 addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ void ldsm4_t(u32 (&r)[4], u32 addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}

__device__ __forceinline__ bool bar_wait_or_give_up(u64* bar, u32 parity, u32 polls) {
  if (bar_test(bar, parity)) return true;
  for (u32 i = 1; i < polls; ++i)
    if (bar_try(bar, parity)) return true;
  return false;
}

// Rows of a kv head fit 32 bits (the host checks), unit numbers may not: a 64-bit division is a hundred instructions, so it is avoided.
__device__ __forceinline__ u32 quotient(u64 a, u64 b) { return (a | b) >> 32 ? (u32)(a / b) : (u32)a / (u32)b; }

// keys row tile rt of a request can see (of its last row), and its units (at least one: a row that sees nothing is written too)
template <int NQ>
__device__ __forceinline__ int tile_keys(const Attend& a, const Req& q, u32 rt) {
  const u32 rows = (u32)q.fresh * a.group, end = (rt + 1) * NQ;
  const int last = end >= rows ? q.fresh - 1 : (int)((end - 1) / (u32)a.group);
  const i64 k = (i64)q.pos0 + last + 1;
  return k <= 0 ? 0 : k > q.keys ? q.keys : (int)k;
}
template <int UNIT>
__device__ __forceinline__ int units_of(int keys) { return keys <= UNIT ? 1 : (int)(((u32)keys + UNIT - 1) / UNIT); }
template <int NQ>
__device__ __forceinline__ u32 row_tiles(const Attend& a, const Req& q) { return ((u32)q.fresh * a.group + NQ - 1) / NQ; }
constexpr int CUTS = 4;                      // chunk lengths that are tried: the even share, and 1/16, 1/8, 1/4 more
__device__ __forceinline__ u32 chunk_units(u64 even, int cut) { return (u32)(even + (cut ? (even >> (5 - cut)) + 1 : 0)); }
__device__ __forceinline__ u32 chunks_of(int units, u32 len) { return ((u32)units + len - 1) / len; }
template <int NQ, int UNIT>
__device__ __forceinline__ u32 request_chunks(const Attend& a, int r, u32 len) {
  const Req q = request(a, r);
  const u32 n = row_tiles<NQ>(a, q);
  u64 c = 0;
  for (u32 rt = 0; rt < n; ++rt) c += chunks_of(units_of<UNIT>(tile_keys<NQ>(a, q, rt)), len);
  return (u32)min(c * a.cache.heads, 1ull << 24);             // more than any grid
}
template <int NQ, int UNIT>
__device__ __forceinline__ u64 request_units(const Attend& a, int r) {
  const Req q = request(a, r);
  const u32 n = row_tiles<NQ>(a, q);
  u64 u = 0;
  for (u32 rt = 0; rt < n; ++rt) u += units_of<UNIT>(tile_keys<NQ>(a, q, rt));
  return u * a.cache.heads;
}

template <int FMT, bool QFP16, int D, int NT>
__global__ void __launch_bounds__(SplitShape<FMT, D>::THREADS, split_ctas<FMT, NT>()) attend_split_kernel(Attend a) {
  using Shape = SplitShape<FMT, D>;
  constexpr bool PACKED = Shape::PACKED;
  constexpr bool F16 = PACKED || FMT == PTSTORE_KV_FP16;      // type of the products' operands
  constexpr int SP_WARPS = Shape::WARPS, SP_THREADS = Shape::THREADS, UNIT = Shape::UNIT;
  constexpr int NQ = 8 * NT, STAGE = Shape::STAGE, STAGES = Shape::STAGES, STEP = Shape::STEP;
  constexpr int KS = D / 16, MT = D / 16;                     // k steps of q.k, m tiles of o
  constexpr int OS = D + 4;                                   // row stride of the joined o in shared memory (floats)
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ u64 s_scan[SP_WARPS], s_left;
  __shared__ u32 s_cuts[SP_WARPS][CUTS];
  __shared__ int s_r, s_last, s_any_bad;
  __shared__ __align__(8) u64 s_bar[SP_WARPS][STAGES];
  __shared__ int s_bad[3][D];                // first key whose V holds NaN, +inf, -inf in column d, among keys that some rows do not see
  __shared__ float s_m[SP_WARPS][NQ], s_l[SP_WARPS][NQ], s_qf[NQ];
  __shared__ __align__(16) unsigned short s_q[NQ][D + 8];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;

  // ---- which units are this CTA's: every CTA sums the units of all requests, consecutive requests per thread
  const int per_thread = (a.R + SP_THREADS - 1) / SP_THREADS;
  const int rb = tid * per_thread < a.R ? tid * per_thread : a.R, re = rb + per_thread < a.R ? rb + per_thread : a.R;
  u64 mine = 0;
  for (int r = rb; r < re; ++r) mine += request_units<NQ, UNIT>(a, r);
  u64 x = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const u64 y = __shfl_up_sync(FULL, x, o);
    if (lane >= o) x += y;
  }
  if (lane == 31) s_scan[warp] = x;
  __syncthreads();
  u64 total = 0, before = x - mine;
#pragma unroll
  for (int w = 0; w < SP_WARPS; ++w) {
    if (w < warp) before += s_scan[w];
    total += s_scan[w];
  }
  u64 per = (total + gridDim.x - 1) >> 32 ? (total + gridDim.x - 1) / gridDim.x : (u32)(total + gridDim.x - 1) / gridDim.x;
  if (per < MIN_TOKENS / UNIT) per = MIN_TOKENS / UNIT;
  const u64 u_begin = blockIdx.x * per, u_end = u_begin + per < total ? u_begin + per : total;
  u32 chunk = 0;                                              // units of a chunk, 0: an even share of the line
  if (per <= 1u << 20 && total > 0) {
    u32 cnt[CUTS], sum[CUTS];
#pragma unroll
    for (int c = 0; c < CUTS; ++c) cnt[c] = 0;
    for (int r = rb; r < re; ++r)
#pragma unroll
      for (int c = 0; c < CUTS; ++c) cnt[c] = min(cnt[c] + request_chunks<NQ, UNIT>(a, r, chunk_units(per, c)), 1u << 24);
#pragma unroll
    for (int c = 0; c < CUTS; ++c) {
      sum[c] = cnt[c];
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const u32 y = __shfl_up_sync(FULL, sum[c], o);
        if (lane >= o) sum[c] = min(sum[c] + y, 1u << 24);
      }
      if (lane == 31) s_cuts[warp][c] = sum[c];
    }
    if (tid == 0) s_r = -1;
    __syncthreads();
    u32 mine_c = 0, before_c = 0;
#pragma unroll
    for (int c = CUTS - 1; c >= 0; --c) {
      u32 all = 0, ahead = sum[c] - cnt[c];
#pragma unroll
      for (int w = 0; w < SP_WARPS; ++w) {
        if (w < warp) ahead += s_cuts[w][c];
        all += s_cuts[w][c];
      }
      if (all <= gridDim.x) { chunk = chunk_units(per, c); mine_c = cnt[c]; before_c = ahead; }
    }
    if (chunk && blockIdx.x >= before_c && blockIdx.x < before_c + mine_c) {        // at most one thread
      u32 left = blockIdx.x - before_c;
      int r = rb;
      for (; r < re - 1; ++r) {
        const u32 n = request_chunks<NQ, UNIT>(a, r, chunk);
        if (left < n) break;
        left -= n;
      }
      s_r = r;
      s_left = left;
    }
  }
  if (!chunk && u_begin >= u_end) return;
  if (!chunk && u_begin >= before && u_begin < before + mine) {         // exactly one thread
    u64 left = u_begin - before;
    int r = rb;
    for (; r < re - 1; ++r) {
      const u64 n = request_units<NQ, UNIT>(a, r);
      if (left < n) break;
      left -= n;
    }
    s_r = r;
    s_left = left;
  }
  __syncthreads();
  int r = s_r;
  if (r < 0) return;                                          // a CTA beyond the last chunk
  u64 left = s_left;
  u64 u = u_begin;

  if (PACKED && lane == 0) {
    for (int i = 0; i < STAGES; ++i) bar_init(&s_bar[warp][i], 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncwarp();
  u32 phases = 0;                            // parity of every stage's barrier
  bool gave_up = false;
  const Magic mg = magic();

  unsigned char* const ring = smem + warp * STAGES * STAGE;
  const u32 ring_addr = smem_addr(ring);
  u32 rt = 0;
  Req rq = request(a, r);
  do {
    // ---- the item under u: request r, row tile rt, kv head h, and the part [ua, ub) of its units
    int keys, n_units;
    for (;;) {
      if (rt >= row_tiles<NQ>(a, rq)) {
        if (++r >= a.R) return;                               // cannot happen while offsets and lengths hold still
        rt = 0;
        rq = request(a, r);
        continue;
      }
      keys = tile_keys<NQ>(a, rq, rt);
      n_units = units_of<UNIT>(keys);
      const u64 all = (u64)(chunk ? chunks_of(n_units, chunk) : n_units) * a.cache.heads;
      if (left < all) break;
      left -= all;
      ++rt;
    }
    int h, ua, ub;
    u32 first_cta, last_cta;                                  // CTAs that share the item
    if (chunk) {
      const u32 n = chunks_of(n_units, chunk), k = (u32)left % n;
      h = (int)((u32)left / n);
      ua = (int)(k * chunk);
      ub = min(ua + (int)chunk, n_units);
      first_cta = blockIdx.x - k;
      last_cta = first_cta + n - 1;
    } else {
      h = (int)quotient(left, n_units);
      ua = (int)(left - (u64)h * n_units);
      ub = u_end - u < (u64)(n_units - ua) ? ua + (int)(u_end - u) : n_units;
      first_cta = quotient(u - ua, per);
      last_cta = quotient(u - ua + n_units - 1, per);
    }
    const int row_base = (int)(rt * NQ), rows_left = rq.fresh * a.group - row_base, rows = rows_left < NQ ? rows_left : NQ;

    // ---- loads of this warp's tiles: tile i of the part is tokens (ua + i) * 64 + warp * 16 ..
    const int n_tiles = ub - ua;
    const int* table = a.tables + (i64)r * a.max_blocks;
    const u32 B = a.cache.block_tokens;
    u32 seen_bits = 0;                                        // bit s: stage s holds a tile (16-bit: bits of this lane's row)
    bool bounds = false;
    // 4-bit: lane l finds tile base + l, 32 tiles at a time; the table entries of the next 32 are on their way meanwhile
    i64 tile_off = -1;
    int n_id = -1;
    auto look_up32 = [&](int base) {
      const int tok = (ua + base + lane) * UNIT + warp * TILE;
      n_id = base + lane < n_tiles && tok < keys ? table[(u32)tok / B] : -1;
    };
    auto resolve32 = [&](int base) {
      const u32 tok = (u32)(ua + base + lane) * UNIT + warp * TILE;
      const bool ok = (u32)n_id < a.cache.num_blocks;
      bounds |= base + lane < n_tiles && (int)tok < keys && !ok;
      tile_off = ok ? (i64)((u64)(u32)n_id * a.cache.block_stride + ((u64)h * (B / TILE) + tok % B / TILE) * tile_bytes(D)) : -1;
      look_up32(base + 32);
    };
    // 16-bit: lane l follows row l & 15 of the tiles
    const u32 step_blk = UNIT / B, step_off = UNIT % B;
    int n_tok = ua * UNIT + warp * TILE + (lane & 15);
    u32 n_blk = (u32)n_tok / B, n_off = (u32)n_tok % B;
    if (PACKED) look_up32(0);
    else n_id = n_tiles > 0 && n_tok < keys ? table[n_blk] : -1;
    auto issue = [&](int i, int s) {
      seen_bits &= ~(1u << s);
      if (PACKED) {
        if (i < n_tiles && !gave_up) {
          if ((i & 31) == 0) resolve32(i);
          const i64 off = __shfl_sync(FULL, tile_off, i & 31);
          if (off >= 0) {
            seen_bits |= 1u << s;
            if (lane == 0) {
              u64* bar = &s_bar[warp][s];
              const unsigned char* src = a.cache.base + off;
              const u32 dst = ring_addr + s * STAGE;
              bar_expect(bar, STAGE);
              bulk_load(dst, src, tile_bytes(D), bar);
              bulk_load(dst + tile_bytes(D), src + a.cache.kv_stride, tile_bytes(D), bar);
            }
          }
        }
        return;
      }
      if (i < n_tiles) {
        const bool in_len = n_tok < keys;
        const bool ok = in_len && (u32)n_id < a.cache.num_blocks;
        bounds |= in_len && !ok;
        const u64 row_off = ok ? (u64)(u32)n_id * a.cache.block_stride + ((u64)n_off * a.cache.heads + h) * (D * 2) : 0;
        n_off += step_off;
        n_blk += step_blk;
        n_tok += UNIT;
        if (n_off >= B) { n_off -= B; ++n_blk; }
        if (i + 1 < n_tiles) n_id = n_tok < keys ? table[n_blk] : -1;
        if (ok) seen_bits |= 1u << s;
        const u32 dst = ring_addr + s * STAGE;
        // some rows per instruction; 16-byte chunk c of row n sits at c ^ (n & 7), which ldmatrix reads without conflicts
        constexpr int CPR = D / 8, RPI = 32 / CPR;            // chunks per row, rows per instruction
#pragma unroll
        for (int j = 0; j < TILE / RPI; ++j) {
          const int n = j * RPI + lane / CPR, c = lane % CPR;
          const u64 off = __shfl_sync(FULL, row_off, n);
          const bool has = __shfl_sync(FULL, ok, n);
          const unsigned char* ks = a.cache.base + off + c * 16;
          const u32 d = dst + n * (D * 2) + ((c ^ (n & 7)) * 16);
          cp_async16_or_zero(d, ks, has);
          cp_async16_or_zero(d + TILE * D * 2, ks + a.cache.kv_stride, has);
        }
      }
      cp_commit();
    };
    // The tile in stage s has landed.  After a wait that ran out no copy is issued any more; what is in flight is still waited for,
    // stage by stage, so that none lands after the CTA has ended.
    auto landed = [&](int s) {
      if (__any_sync(FULL, !bar_wait_or_give_up(&s_bar[warp][s], (phases >> s) & 1, a.polls))) {
        gave_up = true;
        bar_wait_or_give_up(&s_bar[warp][s], (phases >> s) & 1, POLLS);
      }
      phases ^= 1u << s;
    };
#pragma unroll
    for (int i = 0; i < STAGES; ++i) issue(i, i);
    if (tid == 0) s_any_bad = 0;
    if (rq.fresh > 1)
      for (int i = tid; i < 3 * D; i += SP_THREADS) (&s_bad[0][0])[i] = 0x7FFFFFFF;

    // ---- q of the item into shared memory in the products' type; rows that do not exist are zero
    {
      constexpr int TPR = SP_THREADS / NQ < D / 4 ? SP_THREADS / NQ : D / 4, E = D / TPR;       // threads per row, elements per thread
      const int row = tid / TPR, e0 = (tid % TPR) * E;
      __align__(16) u32 raw[E / 2];
      const bool live = row < rows;
      if (live) {
        const int fr = (row_base + row) / a.group, hq = h * a.group + (row_base + row) % a.group;
        const unsigned char* src = a.q + 2 * ((i64)(rq.row0 + fr) * a.q_token + (i64)hq * a.q_head + e0);
        if (E >= 8) {
#pragma unroll
          for (int i = 0; i < E / 8; ++i) *reinterpret_cast<uint4*>(raw + 4 * i) = reinterpret_cast<const uint4*>(src)[i];
        } else *reinterpret_cast<uint2*>(raw) = *reinterpret_cast<const uint2*>(src);
      } else {
#pragma unroll
        for (int i = 0; i < E / 2; ++i) raw[i] = 0;
      }
      float factor = 1.0f;
      if (PACKED && !QFP16) {
        // bf16 rows go into the products as fp16, scaled by a power of two so that the largest element is in [1, 2): exact but
        // for elements below 2^-14 of the largest, which lose at most 2^-25 of it
        float amax = 0.0f;
#pragma unroll
        for (int i = 0; i < E / 2; ++i) {
          const float2 f = unpack2<false>(raw[i]);
          amax = fmaxf(amax, fmaxf(fabsf(f.x), fabsf(f.y)));
        }
#pragma unroll
        for (int o = 1; o < TPR; o <<= 1) amax = fmaxf(amax, __shfl_xor_sync(FULL, amax, o));
        int e = amax > 0.0f ? (int)(__float_as_uint(amax) >> 23) - 127 : 0;
        e = e < -126 ? -126 : e > 126 ? 126 : e;
        factor = __uint_as_float((u32)(127 + e) << 23);
        const float down = __uint_as_float((u32)(127 - e) << 23);
#pragma unroll
        for (int i = 0; i < E / 2; ++i) {
          const float2 f = unpack2<false>(raw[i]);
          raw[i] = pack2<true>(f.x * down, f.y * down);
        }
      }
      if (row < NQ) {
        const u32 flip = a.scale2 < 0.0f ? 0x80008000u : 0;   // the sign of the softmax scale goes into q
#pragma unroll
        for (int i = 0; i < E / 2; ++i) *reinterpret_cast<u32*>(&s_q[row][e0 + 2 * i]) = raw[i] ^ flip;
        // as a positive number: of zero, the smallest that keeps masked scores at minus infinity; finite, so that scores of zero stay zero
        if (e0 == 0) s_qf[row] = fminf(fmaxf(factor * fabsf(a.scale2), 0x1p-126f), 0x1.fffffep127f);
      }
    }
    __syncthreads();
    u32 qb[NT][KS][2];
    float qs[NT][2];
    int see[NT][2];                                           // keys the lane's two query rows see
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int k = 0; k < KS; ++k)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          if (PACKED) {                                       // element order of the 4-bit rows: word w, nibbles j and j + 4
            const unsigned short* p = &s_q[8 * n + g][(D / 4) * t + 8 * (k >> 1) + 2 * (k & 1) + i];
            qb[n][k][i] = (u32)p[0] | ((u32)p[4] << 16);
          } else qb[n][k][i] = *reinterpret_cast<const u32*>(&s_q[8 * n + g][16 * k + 2 * t + 8 * i]);
        }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int row = 8 * n + 2 * t + i;
        qs[n][i] = s_qf[row];
        const i64 p = (i64)rq.pos0 + (row_base + row) / a.group + 1;
        see[n][i] = row >= rows ? 0 : p < 0 ? 0 : p > keys ? keys : (int)p;
      }
    }
    // tokens below this are seen by every row of the tile
    int all_see = rows > 0 ? rq.pos0 + row_base / a.group + 1 : 0;
    all_see = all_see < 0 ? 0 : all_see > keys ? keys : all_see;

    float o[NT][MT][4], m[NT][2], l[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int c = 0; c < 4; ++c) o[n][i][c] = 0.0f;
      m[n][0] = m[n][1] = -INFINITY;
      l[n][0] = l[n][1] = 0.0f;
    }

    // token of accumulator row (c >> 1) of tile tok0
    auto token_of = [&](int half) { return PACKED ? 4 * (g >> 1) + (g & 1) + 2 * half : g + 8 * half; };

    // o += V^T p for one tile
    auto pv = [&](const unsigned char* st, u32 st_addr, const u32 (&pb)[NT][2]) {
      if (PACKED) {
        const unsigned char* vt = st + tile_bytes(D);
        const u32 sc = *reinterpret_cast<const u32*>(vt + 8 * D + (D == 128 ? g : g >> 1) * TILE + 4 * t);
        const Deq da = deq_of(e4m3x2_to_half2(sc & 0xFFFFu)), db = deq_of(e4m3x2_to_half2(sc >> 16));
        constexpr int W = D / 64;                             // words of 8 codes of the lane's elements, per token
        u32 c[4][W];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int chunk = D == 128 ? g >> 1 : g >> 2, byte = D == 128 ? (g & 1) * 8 : (g & 3) * 4;
          // a token's place inside its tile, with n = 4 t + i written out
          const int rho = 256 / D, place = ((4 * t + i) / rho) * 8 + (((i % rho) * (D / 32) + chunk) ^ (2 * t));
          if (W == 2) {
            const uint2 two = *reinterpret_cast<const uint2*>(vt + place * 16 + byte);
            c[i][0] = two.x;
            c[i][W - 1] = two.y;
          } else c[i][0] = *reinterpret_cast<const u32*>(vt + place * 16 + byte);
        }
#pragma unroll
        for (int w = 0; w < W; ++w)
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            u32 va[4], vb[4];
            const u32 sel = half ? 0x7632u : 0x5410u, up = half ? 0x7733u : 0x5511u;      // 16 bits of either token; their upper bytes
            deq4(__byte_perm(c[0][w], c[1][w], sel), __byte_perm(c[0][w], c[1][w], up), da, mg, va);
            deq4(__byte_perm(c[2][w], c[3][w], sel), __byte_perm(c[2][w], c[3][w], up), db, mg, vb);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const u32 av[4] = {va[2 * i], va[2 * i + 1], vb[2 * i], vb[2 * i + 1]};
#pragma unroll
              for (int n = 0; n < NT; ++n) mma16816<F16>(o[n][4 * w + 2 * half + i], av, pb[n]);
            }
          }
      } else {
        const u32 vt = st_addr + TILE * D * 2;
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          // matrices of the transposing load: (d 0-7, tokens 0-7), (d 8-15, tokens 0-7), (d 0-7, tokens 8-15), (d 8-15, tokens 8-15)
          const int row = (lane & 7) + ((lane >> 4) & 1) * 8, chunk = 2 * i + ((lane >> 3) & 1);
          u32 av[4];
          ldsm4_t(av, vt + row * (D * 2) + ((chunk ^ (row & 7)) * 16));
#pragma unroll
          for (int n = 0; n < NT; ++n) mma16816<F16>(o[n][i], av, pb[n]);
        }
      }
    };
    // V of a tile that not all rows see whole.  A weight of zero does not hide an infinity or a NaN: tokens behind the last row's position
    // count as zero (a 16-bit tile has zeros there already), and what is not finite in tokens that only some rows see is taken out
    // here and put into the sums of the rows that see it when the warps are joined.
    auto mend = [&](unsigned char* st, int tok0) {
      if (PACKED) {
        unsigned char* sc = st + tile_bytes(D) + 8 * D;
        for (int i = lane; i < TILE * (D / GROUP); i += 32) {
          const int tok = tok0 + i % TILE, gr = i / TILE;
          if (tok >= keys) sc[i] = 0;
          else if (rq.fresh > 1 && (sc[i] & 0x7F) == 0x7F) {
            sc[i] = 0;
            s_any_bad = 1;
            for (int d = 0; d < GROUP; ++d) atomicMin(&s_bad[0][gr * GROUP + d], tok);
          }
        }
      } else if (rq.fresh > 1) {
        constexpr u32 EX = F16 ? 0x7C00u : 0x7F80u, MANT = F16 ? 0x03FFu : 0x007Fu;
        unsigned short* v = reinterpret_cast<unsigned short*>(st + TILE * D * 2);
        for (int i = lane; i < TILE * D; i += 32) {
          const int n = i / D, d = i % D, at = n * D + (((d >> 3) ^ (n & 7)) << 3) + (d & 7);
          const u32 x = v[at];
          if ((x & EX) == EX) {
            v[at] = 0;
            s_any_bad = 1;
            atomicMin(&s_bad[(x & MANT) ? 0 : (x & 0x8000u) ? 2 : 1][d], tok0 + n);
          }
        }
      }
      __syncwarp();
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");        // the stage's next tile comes through the async proxy
    };

    // s = q . k for one tile (not yet scaled)
    auto qk = [&](const unsigned char* st, u32 st_addr, float (&sc)[NT][4]) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int c = 0; c < 4; ++c) sc[n][c] = 0.0f;
      if (PACKED) {
        const int n0 = token_of(0), n1 = token_of(1);
        __align__(16) u32 c0[D / 32], c1[D / 32];
        u32 z0, z1;
        if (D == 128) {
          *reinterpret_cast<uint4*>(c0) = *reinterpret_cast<const uint4*>(st + code_place(D, n0, t) * 16);
          *reinterpret_cast<uint4*>(c1) = *reinterpret_cast<const uint4*>(st + code_place(D, n1, t) * 16);
          z0 = e4m3x2_to_half2(*reinterpret_cast<const unsigned short*>(st + 8 * D + n0 * 8 + 2 * t));
          z1 = e4m3x2_to_half2(*reinterpret_cast<const unsigned short*>(st + 8 * D + n1 * 8 + 2 * t));
        } else {
          *reinterpret_cast<uint2*>(c0) = *reinterpret_cast<const uint2*>(st + code_place(D, n0, t >> 1) * 16 + (t & 1) * 8);
          *reinterpret_cast<uint2*>(c1) = *reinterpret_cast<const uint2*>(st + code_place(D, n1, t >> 1) * 16 + (t & 1) * 8);
          z0 = e4m3x2_to_half2(st[8 * D + n0 * 4 + t]);
          z1 = e4m3x2_to_half2(st[8 * D + n1 * 4 + t]);
        }
#pragma unroll
        for (int gr = 0; gr < D / 64; ++gr) {                 // the lane's scale groups of 16 elements
          const u32 sel = gr ? 0x3232u : 0x1010u;
          const Deq d0 = deq_of(__byte_perm(z0, z0, sel)), d1 = deq_of(__byte_perm(z1, z1, sel));
#pragma unroll
          for (int w = 2 * gr; w < 2 * gr + 2; ++w) {
            u32 v0[4], v1[4];
            deq4(c0[w], c0[w] >> 8, d0, mg, v0);
            deq4(c1[w], c1[w] >> 8, d1, mg, v1);
#pragma unroll
            for (int b = 0; b < 2; ++b) {
              const u32 av[4] = {v0[2 * b], v1[2 * b], v0[2 * b + 1], v1[2 * b + 1]};
#pragma unroll
              for (int n = 0; n < NT; ++n) mma16816<F16>(sc[n], av, qb[n][2 * w + b]);
            }
          }
        }
      } else {
#pragma unroll
        for (int kk = 0; kk < KS; ++kk) {
          const int row = (lane & 7) + ((lane >> 3) & 1) * 8, chunk = 2 * kk + (lane >> 4);
          u32 av[4];
          ldsm4(av, st_addr + row * (D * 2) + ((chunk ^ (row & 7)) * 16));
#pragma unroll
          for (int n = 0; n < NT; ++n) mma16816<F16>(sc[n], av, qb[n][kk]);
        }
      }
    };
    // running maximum and weights of K tiles, then their values; held: tiles that are there
    auto accumulate = [&](auto& sc, int s0, auto held) {
      constexpr int K = sizeof(sc) / sizeof(sc[0]);
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          float x = fmaxf(sc[0][n][c], sc[0][n][c + 2]);
#pragma unroll
          for (int k = 1; k < K; ++k) x = fmaxf(x, fmaxf(sc[k][n][c], sc[k][n][c + 2]));
          x = fmaxf(m[n][c], x * qs[n][c]);
#pragma unroll
          for (int w = 4; w < 32; w <<= 1) x = fmaxf(x, __shfl_xor_sync(FULL, x, w));
          if (__any_sync(FULL, x != m[n][c])) {
            const float f = x == -INFINITY ? 1.0f : exp2_fast(m[n][c] - x);
            m[n][c] = x;
            l[n][c] *= f;
#pragma unroll
            for (int i2 = 0; i2 < MT; ++i2) { o[n][i2][c] *= f; o[n][i2][c + 2] *= f; }
          }
        }
      float ref[NT][2];
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int c = 0; c < 2; ++c) ref[n][c] = m[n][c] == -INFINITY ? 0.0f : m[n][c];
#pragma unroll
      for (int k = 0; k < K; ++k) {
        if (!held(k)) continue;
        u32 pb[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          float p[4];
#pragma unroll
          for (int c = 0; c < 4; ++c) {       // the product rounded as the maximum is, so that the largest weight is 1 however large the scores are
            p[c] = exp2_fast(__fmul_rn(sc[k][n][c], qs[n][c & 1]) - ref[n][c & 1]);
            l[n][c & 1] += p[c];
          }
          pb[n][0] = transpose8x8(pack2<F16>(p[0], p[1]));
          pb[n][1] = transpose8x8(pack2<F16>(p[2], p[3]));
        }
        pv(ring + (s0 + k) * STAGE, ring_addr + (s0 + k) * STAGE, pb);
      }
    };

    // ---- the tiles, STEP at a time: steps that every row sees whole, then the rest with masks
    int s0 = 0, i = 0;                                        // stage of tile i
    auto next = [&]() {
      __syncwarp();
#pragma unroll
      for (int k = 0; k < STEP; ++k) issue(i + STAGES + k, s0 + k);
      s0 += STEP;
      if (s0 == STAGES) s0 = 0;
      i += STEP;
    };
    const u32 all_held = (1u << STEP) - 1u;
    while (i < n_tiles) {
      if (!PACKED) {
        cp_wait<STAGES - STEP>();
        __syncwarp();
      }
      const int tok_end = (ua + i + STEP - 1) * UNIT + warp * TILE + TILE;
      const bool there = PACKED ? ((seen_bits >> s0) & all_held) == all_held : __all_sync(FULL, ((seen_bits >> s0) & all_held) == all_held);
      float sc[STEP][NT][4];
      if (i + STEP <= n_tiles && there && tok_end <= all_see) {
#pragma unroll
        for (int k = 0; k < STEP; ++k) {
          if (PACKED) landed(s0 + k);
          qk(ring + (s0 + k) * STAGE, ring_addr + (s0 + k) * STAGE, sc[k]);
        }
        accumulate(sc, s0, [](int) { return true; });
        next();
        continue;
      }
      u32 held = 0;
#pragma unroll
      for (int k = 0; k < STEP; ++k) {
        const int s = s0 + k, tok0 = (ua + i + k) * UNIT + warp * TILE;
        if (PACKED && ((seen_bits >> s) & 1)) landed(s);
        const u32 rows_in = PACKED ? ((seen_bits >> s) & 1 ? 0xFFFFu : 0u) : __ballot_sync(FULL, (seen_bits >> s) & 1) & 0xFFFFu;
        if (i + k < n_tiles && rows_in != 0) {
          held |= 1u << k;
          mend(ring + s * STAGE, tok0);
          qk(ring + s * STAGE, ring_addr + s * STAGE, sc[k]);
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const int in = token_of(c >> 1);
            if (!((held >> k) & 1) || tok0 + in >= see[n][c & 1] || !((rows_in >> in) & 1)) sc[k][n][c] = -INFINITY;
          }
      }
      accumulate(sc, s0, [&](int k) { return (held >> k) & 1; });
      next();
    }
    cp_wait<0>();
    if ((bounds || gave_up) && a.status) atomicOr(a.status, (bounds ? PTSTORE_S_BOUNDS : 0) | (gave_up ? PTSTORE_S_TIMEOUT : 0));

    // ---- join the four warps
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
#pragma unroll
        for (int w = 4; w < 32; w <<= 1) l[n][c] += __shfl_xor_sync(FULL, l[n][c], w);
        if (g == 0) {
          s_m[warp][8 * n + 2 * t + c] = m[n][c];
          s_l[warp][8 * n + 2 * t + c] = l[n][c];
        }
      }
    __syncthreads();                                          // the ring is idle from here on: it holds the warps' sums
    float* s_o = reinterpret_cast<float*>(smem);
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int row = 8 * n + 2 * t + c;
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < SP_WARPS; ++w) top = fmaxf(top, s_m[w][row]);
        const float f = m[n][c] == -INFINITY ? 0.0f : exp2_fast(m[n][c] - top);
        const bool none = m[n][c] == -INFINITY && l[n][c] == 0.0f;          // a NaN keeps its way through
        float* dst = s_o + (warp * NQ + row) * OS;
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          const int d0 = PACKED ? (D / 8) * g + 2 * i : 16 * i + g, d1 = PACKED ? d0 + 1 : d0 + 8;
          dst[d0] = none ? 0.0f : o[n][i][c] * (m[n][c] == -INFINITY ? 1.0f : f);
          dst[d1] = none ? 0.0f : o[n][i][c + 2] * (m[n][c] == -INFINITY ? 1.0f : f);
        }
      }
    __syncthreads();
    constexpr int TPR = SP_THREADS / NQ < D / 4 ? SP_THREADS / NQ : D / 4, E = D / TPR;         // threads per row, elements per thread
    const int row = tid / TPR, e0 = (tid % TPR) * E;
    float acc[E], top = -INFINITY, sum = 0.0f;
    const int rw = row < NQ ? row : 0;
#pragma unroll
    for (int w = 0; w < SP_WARPS; ++w) top = fmaxf(top, s_m[w][rw]);
#pragma unroll
    for (int w = 0; w < SP_WARPS; ++w) {
      const float lw = s_l[w][rw], mw = s_m[w][rw];
      sum += mw == -INFINITY ? lw : lw * exp2_fast(mw - top);
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
      acc[e] = 0.0f;
#pragma unroll
      for (int w = 0; w < SP_WARPS; ++w) acc[e] += s_o[(w * NQ + rw) * OS + e0 + e];
    }
    if (s_any_bad && row < rows) {
      const i64 p = (i64)rq.pos0 + (row_base + row) / a.group;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const bool nan = s_bad[0][e0 + e] <= p, pos = s_bad[1][e0 + e] <= p, neg = s_bad[2][e0 + e] <= p;
        if (nan || (pos && neg)) acc[e] = NAN;
        else if (pos) acc[e] += INFINITY;
        else if (neg) acc[e] -= INFINITY;
      }
    }
    bool write = true;
    if (first_cta != last_cta) {
      // partial sums: slot 1 of the CTA the item begins in, slot 0 of the others
      constexpr int PF = part_floats<NT, D>();
      u32* counters = reinterpret_cast<u32*>(a.work);
      float* parts = reinterpret_cast<float*>(a.work + SP_PARTS_AT);
      float* my = parts + (2 * (i64)blockIdx.x + (blockIdx.x == first_cta ? 1 : 0)) * PF;
      if (row < rows) {
#pragma unroll
        for (int e = 0; e < E; e += 4) *reinterpret_cast<float4*>(my + row * D + e0 + e) = make_float4(acc[e], acc[e + 1], acc[e + 2], acc[e + 3]);
        if (e0 == 0) { my[NQ * D + row] = top; my[NQ * D + NQ + row] = sum; }
      }
      __threadfence();
      __syncthreads();
      if (tid == 0) {
        const u32 n = last_cta - first_cta;
        const bool last = atomicAdd(&counters[first_cta], 1u) == n;
        if (last) counters[first_cta] = 0;
        s_last = last;
      }
      __syncthreads();
      write = false;
      if (s_last) {
        // all parts are there: maxima and sums into shared memory first, then the weighted sums with many loads in flight
        __threadfence();
        const int n_parts = (int)(last_cta - first_cta) + 1;
        float* s_pm = reinterpret_cast<float*>(smem);
        float* s_pl = s_pm + n_parts * rows;
        auto part = [&](int c) { return parts + (2 * (i64)(first_cta + c) + (c == 0 ? 1 : 0)) * PF; };
        for (int i = tid; i < n_parts * rows; i += SP_THREADS) {
          const float* p = part(i / rows) + NQ * D + i % rows;
          s_pm[i] = __ldcg(p);
          s_pl[i] = __ldcg(p + NQ);
        }
        __syncthreads();
        for (int i = tid; i < rows * (D / 4); i += SP_THREADS) {
          const int rw = i / (D / 4), e = (i % (D / 4)) * 4;
          float high = -INFINITY, all = 0.0f;
          for (int c = 0; c < n_parts; ++c) high = fmaxf(high, s_pm[c * rows + rw]);
          float4 o4 = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 8
          for (int c = 0; c < n_parts; ++c) {
            const float mc = s_pm[c * rows + rw];
            const float f = mc == -INFINITY ? 1.0f : exp2_fast(mc - high);  // nothing seen: sums of zero (or NaN)
            const float4 v = __ldcg(reinterpret_cast<const float4*>(part(c) + rw * D + e));
            all += s_pl[c * rows + rw] * f;
            o4.x += v.x * f;
            o4.y += v.y * f;
            o4.z += v.z * f;
            o4.w += v.w * f;
          }
          const float f = row_factor(a, r, (i64)rq.pos0 + (row_base + rw) / a.group, all);
          const int fr = (row_base + rw) / a.group, hq = h * a.group + (row_base + rw) % a.group;
          *reinterpret_cast<uint2*>(a.out + 2 * ((i64)(rq.row0 + fr) * a.o_token + (i64)hq * a.o_head + e)) =
              make_uint2(pack2<QFP16>(o4.x * f, o4.y * f), pack2<QFP16>(o4.z * f, o4.w * f));
        }
      }
    }
    if (write && row < rows) {
      const float f = row_factor(a, r, (i64)rq.pos0 + (row_base + row) / a.group, sum);
      const int fr = (row_base + row) / a.group, hq = h * a.group + (row_base + row) % a.group;
      unsigned char* dst = a.out + 2 * ((i64)(rq.row0 + fr) * a.o_token + (i64)hq * a.o_head + e0);
      __align__(16) u32 v[E / 2];
#pragma unroll
      for (int e = 0; e < E / 2; ++e) v[e] = pack2<QFP16>(acc[2 * e] * f, acc[2 * e + 1] * f);
      if (E >= 8) {
#pragma unroll
        for (int i = 0; i < E / 8; ++i) reinterpret_cast<uint4*>(dst)[i] = *reinterpret_cast<const uint4*>(v + 4 * i);
      } else *reinterpret_cast<uint2*>(dst) = *reinterpret_cast<const uint2*>(v);
    }
    // the joins' sums lay in the ring: they come before the next item's bulk copies, which write it through the async proxy
    if (PACKED) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncthreads();                                          // the ring and the small arrays are free again
    u += ub - ua;
    left += ub - ua;
  } while (!chunk && u < u_end);
}

}  // namespace ptk
