// Absorbed attention over a cache of latent vectors: one row c_j | r_j of L + 64 elements a token, which is the key of every query head, and its first
// L elements the value.  Bounded by reading the rows once up to some 100 rows of q a request, by the tensor cores beyond.
//
// A CTA takes 64 rows (new token, query head) of a request and walks 64 cached tokens a step; all of a step's operands are one tile of the cache in shared
// memory, which is read as keys and as values:
//     S = Q K^T          M = 64 rows, N = 64 tokens, K = L + 64
//     P = exp2(scale2 S - m)                       (one thread per row)
//     O^T += C^T P^T     M = 128 latent elements, L / 128 times; N = 64 rows, K = 64 tokens
// The output is held transposed because L columns of 64 rows would run at half the tensor cores' rate and fill tensor memory: as it is they are L / 2 of 512 columns, and S
// has two buffers beside it, so that the next step's scores are computed while this one's weights are.  m is a running reference, moved only when a scaled score exceeds it by
// more than 8 (weights are at most 2^8), since that means reading and writing all of O.
//
// Tiles come by one tensor copy per 8 tokens, {64 elements, 8 tokens, L / 64 + 1 groups of elements}: the boxes lie one behind the other as groups of 8 rows of
// 128 swizzled bytes, 1024 (L / 64 + 1) bytes apart, which both operand forms can step over, whatever the block size.
//
// Warps 0-3 softmax, and Q and the output of an item; 4 loads; 5 issues the tensor instructions.  One CTA per SM takes an even share of the line of all
// (request, row tile, 64 tokens) units.  Where requests have more than 64 rows two neighbouring CTAs walk the same units with 64 rows each, so that the second
// one finds the tiles in L2.  An item that spans several CTAs leaves sums (o, m, l in 32 bits) in the workspace, which latent_join_kernel joins in CTA order.
#pragma once
#include "attend_prompt.cuh"
#include "attend_split.cuh"

namespace ptk {

constexpr int LA_THREADS = 192, LA_ROWS = 64, LA_KEYS = 64, LA_ROPE = 64;
constexpr int LA_MIN_UNITS = 4;              // a CTA takes at least this many, so that joining does not cost more than it saves

template <int L>
struct LatentShape {
  static constexpr int BOXES = L / 64 + 1, GROUP_BYTES = BOXES * 1024;            // 8 tokens
  static constexpr int TILE_BYTES = 8 * GROUP_BYTES, Q_BYTES = BOXES * LA_ROWS * 128, P_BYTES = LA_ROWS * 128;
  static constexpr int STAGES = L == 512 ? 2 : 3;
  static constexpr int MISC = 2816;                                               // barriers, factors, the first bad token per element
  static constexpr int SMEM = Q_BYTES + STAGES * TILE_BYTES + P_BYTES + MISC;
  static constexpr int PART = LA_ROWS * (L + 2);                                  // floats of an item's sums in one CTA: o, m, l
};
struct LatentMisc {
  u64 full[3], empty[3], q, q_free, s[2], p, pv, end;
  u32 valid[3], tmem;
  int gave_up, any_bad, r;
  u64 left;
  u64 scan[6];
  float f[LA_ROWS];
  int bad[512];              // first token whose element d is not finite, among tokens that some rows do not see
};
static_assert(sizeof(LatentMisc) <= LatentShape<512>::MISC, "fits behind the operands");
static_assert(LatentShape<512>::SMEM <= 232448, "fits an SM (there is no static shared memory, so the operands begin on a multiple of 1024)");

struct Latent {
  Attend a;                  // q: q_latent; cache.heads 1, group = heads
  const unsigned char* q_rope;
  i64 qr_token, qr_head;
};
// what the join needs of an item that begins in a CTA and goes on in others
struct LatentPart { int parts, r; u32 rt; };
constexpr int LA_PARTS_AT = 8192;            // where the sums begin in the workspace, behind the descriptions of the largest grid
static_assert(MAX_SMS * sizeof(LatentPart) <= LA_PARTS_AT, "descriptions fit");

// The items of one CTA's share of the line, one after the other.  NQ rows are a row tile of the line, of which the CTA has those from `skip` on.
template <int NQ>
struct LatentLine {
  const Attend& a;
  int skip;
  u64 u, u_end, left;
  u32 per;
  int r;
  u32 rt;
  Req q;
  // the item: tokens its rows see, its units and this CTA's part of them [ua, ub), the CTAs that share it
  int keys, units, ua, ub;
  u32 first, last;
  __device__ __forceinline__ bool next() {
    for (;;) {
      if (u >= u_end) return false;
      if (rt >= row_tiles<NQ>(a, q)) {
        if (++r >= a.R) return false;                         // cannot happen while offsets and lengths hold still
        rt = 0;
        q = request(a, r);
        continue;
      }
      keys = tile_keys<NQ>(a, q, rt);
      units = units_of<LA_KEYS>(keys);
      if (left >= (u64)units) {
        left -= units;
        ++rt;
        continue;
      }
      ua = (int)left;
      ub = u_end - u < (u64)(units - ua) ? ua + (int)(u_end - u) : units;
      first = quotient(u - ua, per);
      last = quotient(u - ua + units - 1, per);
      u += ub - ua;
      left += ub - ua;
      if ((i64)rt * NQ + skip < (i64)q.fresh * a.group) return true;
    }
  }
};

__device__ __forceinline__ u64 operand_desc(u32 addr, u32 lead_bytes, u32 stride_bytes) {
  return (u64)((addr >> 4) & 0x3FFFu) | ((u64)((lead_bytes >> 4) & 0x3FFFu) << 16) | ((u64)((stride_bytes >> 4) & 0x3FFFu) << 32) | (1ull << 46) | (2ull << 61);
}
// instruction descriptor of kind::f16 for any M, A "MN-major" or not; B has its elements of one row contiguous
__host__ __device__ constexpr u32 mma_desc_m(bool fp16, int M, int N, bool a_mn_major) {
  return (1u << 4) | ((fp16 ? 0u : 1u) << 7) | ((fp16 ? 0u : 1u) << 10) | ((a_mn_major ? 1u : 0u) << 15) | ((u32)(N >> 3) << 17) | ((u32)(M >> 4) << 24);
}
// 8 tokens of a block, all their elements: box of the map {64 elements, tokens of a block, groups of 64 elements, blocks}
__device__ __forceinline__ void tensor_load_rows(u32 dst, const CUtensorMap* map, int token, int block, u64* bar) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst), "l"(map), "r"(0), "r"(token),
               "r"(0), "r"(block), "r"(smem_addr(bar)) : "memory");
}
__device__ __forceinline__ bool any_of_softmax(bool v) {      // barrier of the 128 softmax threads
  u32 r;
  asm volatile("{\n .reg .pred p, q;\n setp.ne.u32 p, %1, 0;\n barrier.cta.red.or.pred q, 2, 128, p;\n selp.u32 %0, 1, 0, q;\n}" : "=r"(r) : "r"((u32)v) : "memory");
  return r != 0;
}

template <int L, bool F16, int PAIR>
__global__ void __launch_bounds__(LA_THREADS, 1) latent_attend_kernel(const Latent la, const __grid_constant__ CUtensorMap map) {
  using Shape = LatentShape<L>;
  constexpr int NQ = LA_ROWS * PAIR, STAGES = Shape::STAGES, BOXES = Shape::BOXES, GB = Shape::GROUP_BYTES, MT = L / 128;
  extern __shared__ __align__(1024) unsigned char latent_smem[];
  unsigned char* const smem = latent_smem;
  const Attend& a = la.a;
  LatentMisc& s = *reinterpret_cast<LatentMisc*>(smem + Shape::Q_BYTES + STAGES * Shape::TILE_BYTES + Shape::P_BYTES);
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(FULL, tid >> 5, 0);
  const u32 cta = blockIdx.x / PAIR, ctas = gridDim.x / PAIR, half = blockIdx.x % PAIR;
  LatentPart* const part = reinterpret_cast<LatentPart*>(a.work) + blockIdx.x;
  float* const sums = reinterpret_cast<float*>(a.work + LA_PARTS_AT);

  // ---- this CTA's share of the line: every CTA sums the units of all requests, consecutive requests per thread
  if (tid == 0) {
    part->parts = 0;
    for (int i = 0; i < STAGES; ++i) { bar_init(&s.full[i], 1); bar_init(&s.empty[i], 1); }
    bar_init(&s.q, 128);
    bar_init(&s.q_free, 1);
    for (int i = 0; i < 2; ++i) bar_init(&s.s[i], 1);
    bar_init(&s.p, 128);
    bar_init(&s.pv, 1);
    bar_init(&s.end, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    s.gave_up = s.any_bad = 0;
    s.r = -1;
  }
  if (tid == 160) asm volatile("prefetch.tensormap [%0];" ::"l"(&map) : "memory");
  for (int i = tid; i < L; i += LA_THREADS) s.bad[i] = 0x7FFFFFFF;
  const int per_thread = (a.R + LA_THREADS - 1) / LA_THREADS;
  const int rb = min(tid * per_thread, a.R), re = min(rb + per_thread, a.R);
  u64 mine = 0;
  for (int r = rb; r < re; ++r) mine += request_units<NQ, LA_KEYS>(a, r);
  u64 x = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const u64 y = __shfl_up_sync(FULL, x, o);
    if (lane >= o) x += y;
  }
  if (lane == 31) s.scan[warp] = x;
  __syncthreads();
  u64 total = 0, before = x - mine;
#pragma unroll
  for (int w = 0; w < LA_THREADS / 32; ++w) {
    if (w < warp) before += s.scan[w];
    total += s.scan[w];
  }
  u64 even = (total + ctas - 1) / ctas;
  if (even < LA_MIN_UNITS) even = LA_MIN_UNITS;
  if (even > 0x7FFFFFFF) even = 0x7FFFFFFF;                   // (2^31 units of 64 tokens a CTA: beyond any run; what is behind them is not computed)
  const u32 per = (u32)even;
  const u64 u_begin = (u64)cta * per, u_end = u_begin + per < total ? u_begin + per : total;
  if (u_begin >= u_end) return;
  if (u_begin >= before && u_begin < before + mine) {         // exactly one thread
    u64 left = u_begin - before;
    int r = rb;
    for (; r < re - 1; ++r) {
      const u64 n = request_units<NQ, LA_KEYS>(a, r);
      if (left < n) break;
      left -= n;
    }
    s.r = r;
    s.left = left;
  }
  if (warp == 5) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(&s.tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const u32 tmem = s.tmem;
  const u32 smem_q = smem_addr(smem), smem_k = smem_q + Shape::Q_BYTES, smem_p = smem_k + STAGES * Shape::TILE_BYTES;
  LatentLine<NQ> line{a, (int)half * LA_ROWS, u_begin, u_end, s.left, per, s.r, 0, request(a, s.r)};
  const volatile int* const gave_up = &s.gave_up;

  if (warp == 5) {
    // ======== tensor instructions: S of step g + 1 before the output of step g
    constexpr u32 QK = mma_desc_m(F16, 64, LA_KEYS, false), PV = mma_desc_m(F16, 128, LA_ROWS, true);
    u32 g = 0, item = 0;
    bool quit = false;
    auto wait = [&](u64* b, u32 parity) {
      if (!quit && !__all_sync(FULL, bar_wait(b, parity, a.polls, &s.gave_up))) quit = true;
    };
    auto scores = [&](u32 n) {                // of step n, into buffer n & 1
      wait(&s.full[n % STAGES], (n / STAGES) & 1);
      tc_fence_after();
      if (!quit && elected()) {
        const u64 qa = operand_desc(smem_q, 0, 1024), kb = operand_desc(smem_k + (n % STAGES) * Shape::TILE_BYTES, 0, GB);
#pragma unroll
        for (int k = 0; k < 4 * BOXES; ++k)   // 16 elements: 32 bytes further in a row, or the next 64 elements
          mma_ss(tmem + (n & 1) * 64, qa + (u64)(((k >> 2) * (LA_ROWS * 128) + (k & 3) * 32) >> 4), kb + (u64)(((k >> 2) * 1024 + (k & 3) * 32) >> 4), QK, k > 0);
        tc_commit(&s.s[n & 1]);
      }
      __syncwarp();
    };
    while (!quit && line.next()) {
      const u32 n = line.ub - line.ua;
      wait(&s.q, item & 1);
      scores(g);
      for (u32 j = 0; j < n && !quit; ++j, ++g) {
        if (j + 1 < n) scores(g + 1);
        else if (!quit && elected()) tc_commit(&s.q_free);
        __syncwarp();
        wait(&s.p, g & 1);
        tc_fence_after();
        if (!quit && elected()) {
          const u32 tile = smem_k + (g % STAGES) * Shape::TILE_BYTES;
          const u64 pb = operand_desc(smem_p, 0, 1024);
#pragma unroll
          for (int i = 0; i < MT; ++i) {
            const u64 va = operand_desc(tile + 2 * i * 1024, 1024, GB);
#pragma unroll
            for (int k = 0; k < LA_KEYS / 16; ++k)            // 16 tokens: two groups of 8
              mma_ss(tmem + 128 + i * 64, va + (u64)((k * 2 * GB) >> 4), pb + (u64)((k * 32) >> 4), PV, j > 0 || k > 0);
          }
          tc_commit(&s.empty[g % STAGES]);
          tc_commit(&s.pv);
        }
        __syncwarp();
      }
      ++item;
    }
    // everything issued has ended before tensor and shared memory are given back
    if (elected()) tc_commit(&s.end);
    __syncwarp();
    bar_drain(&s.end, 0);
  } else if (warp == 4) {
    // ======== tiles: lane i < 8 follows tokens 8 i .. 8 i + 7 of a step
    u32 g = 0;
    const u32 B = a.cache.block_tokens;
    bool bounds = false, quit = false;
    while (!quit && line.next()) {
      const int* const table = a.tables + (i64)line.r * a.max_blocks;
      auto look_up = [&](int unit) {
        const int key = unit * LA_KEYS + 8 * lane;
        return lane < 8 && key < line.keys ? table[(u32)key / B] : -1;
      };
      int id = look_up(line.ua);
      for (int unit = line.ua; unit < line.ub; ++unit, ++g) {
        const u32 st = g % STAGES;
        const int key = unit * LA_KEYS + 8 * lane;
        const bool in = lane < 8 && key < line.keys, have = in && (u32)id < a.cache.num_blocks;
        bounds |= in && !have;
        const int block = id;
        if (unit + 1 < line.ub) id = look_up(unit + 1);
        const u32 there = __ballot_sync(FULL, have);
        if (g >= STAGES && !__all_sync(FULL, bar_wait(&s.empty[st], (g / STAGES - 1) & 1, a.polls, &s.gave_up))) { quit = true; break; }
        if (lane == 0) {
          s.valid[st] = there;
          if (there) bar_expect(&s.full[st], __popc(there) * GB);
          else bar_arrive(&s.full[st]);
        }
        __syncwarp();
        if (have) tensor_load_rows(smem_k + st * Shape::TILE_BYTES + lane * GB, &map, (int)((u32)key % B), block, &s.full[st]);
      }
    }
    // whatever happened, what is in flight lands before the CTA gives its memory back
    for (u32 k = g > STAGES ? g - STAGES : 0; k < g; ++k) bar_drain(&s.full[k % STAGES], (k / STAGES) & 1);
    if (bounds && a.status) atomicOr(a.status, PTSTORE_S_BOUNDS);
  } else {
    // ======== softmax: lanes 0-15 of warp w have rows 16 w + lane; Q before, the output behind an item
    const int row = warp * 16 + (lane & 15);
    const u32 lane_base = (u32)(32 * warp) << 16, ts = tmem + lane_base, to = tmem + lane_base + 128;
    u32 g = 0, item = 0;
    bool quit = false;
    auto wait = [&](u64* b, u32 parity) {
      const bool ok = bar_wait(b, parity, a.polls, &s.gave_up);
      if (__any_sync(FULL, !ok || *gave_up)) quit = true;
    };
    // Q of an item.  Rows that do not exist keep what lies there: their sums are never looked at, and a row's are its own.
    auto load_q = [&](const LatentLine<NQ>& it) {
      const int base = (int)(it.rt * NQ) + (int)half * LA_ROWS, rows = min(LA_ROWS, it.q.fresh * a.group - base);
      constexpr int CPR = BOXES * 8;
#pragma unroll 4
      for (int i = tid; i < rows * CPR; i += 128) {
        const int n = i / CPR, c = i % CPR, fr = (base + n) / a.group, hq = (base + n) % a.group;
        const i64 tok = it.q.row0 + fr;
        const unsigned char* src = c < L / 8 ? a.q + 2 * (tok * a.q_token + hq * a.q_head + c * 8) : la.q_rope + 2 * (tok * la.qr_token + hq * la.qr_head + (c - L / 8) * 8);
        *reinterpret_cast<uint4*>(smem + (c >> 3) * (LA_ROWS * 128) + n * 128 + (((c & 7) ^ (n & 7)) * 16)) = *reinterpret_cast<const uint4*>(src);
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      bar_arrive(&s.q);
    };
    bool more = line.next();
    if (more) load_q(line);
    while (more && !quit) {
      const Req rq = line.q;
      const int r = line.r, keys = line.keys, ua = line.ua, n = line.ub - line.ua, row_base = (int)(line.rt * NQ) + (int)half * LA_ROWS;
      const u32 rt = line.rt, first = line.first, last = line.last;
      const int rows = min(LA_ROWS, rq.fresh * a.group - row_base);
      auto seen_by = [&](int row) {
        const i64 k = (i64)rq.pos0 + (row_base + row) / a.group + 1;
        return k < 0 ? 0 : k > keys ? keys : (int)k;
      };
      const int see = lane < 16 && row < rows ? seen_by(row) : 0, all_see = seen_by(0);
      float m = -INFINITY, l = 0.0f;
      for (int j = 0; j < n; ++j, ++g) {
        const int k0 = (ua + j) * LA_KEYS;
        const u32 st = g % STAGES;
        // (a wait that ran out in one warp shows in all of them at the next barrier: until then its values are of no use, but in bounds)
        wait(&s.s[g & 1], (g >> 1) & 1);
        tc_fence_after();
        float v[2][32];
        tc_ld32(v[0], ts + (g & 1) * 64);
        tc_ld32(v[1], ts + (g & 1) * 64 + 32);
        tc_wait_ld();
        tc_loaded(v[0]);
        tc_loaded(v[1]);
        wait(&s.full[st], (g / STAGES) & 1);          // (has ended long ago: makes the tile's bytes and its valid bits this thread's too)
        const u32 valid = s.valid[st];
        const bool edge = k0 + LA_KEYS > all_see || valid != 0xFFu;
        float top = -INFINITY;
        // the products rounded as the maximum is, so that the largest weight is 1 however large the scores are
#pragma unroll
        for (int i = 0; i < 64; ++i) v[i >> 5][i & 31] = __fmul_rn(v[i >> 5][i & 31], a.scale2);
        if (edge) {
          // A weight of zero does not hide an infinity or a NaN.  Tokens that no row sees become zero; what is not finite in tokens that only some rows see is
          // taken out, and put into the sums of the rows that see it at the end.  (The scores have been computed by now.)
          unsigned char* const tile = smem + Shape::Q_BYTES + st * Shape::TILE_BYTES;
          constexpr u32 EX = F16 ? 0x7C00u : 0x7F80u;
          const int from = max(all_see - k0, 0);
          for (int i = tid; i < LA_KEYS * (L / 8); i += 128) {
            const int t = i / (L / 8), c = i % (L / 8);
            const bool there = (valid >> (t >> 3)) & 1;
            if (t < from && there) continue;
            uint4* const p = reinterpret_cast<uint4*>(tile + (t >> 3) * GB + (c >> 3) * 1024 + (t & 7) * 128 + (((c & 7) ^ (t & 7)) * 16));
            if (!there || k0 + t >= keys) { *p = make_uint4(0, 0, 0, 0); continue; }
            uint4 w = *p;
            u32 e[4] = {w.x, w.y, w.z, w.w};
            bool odd = false;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              const u32 sh = 16 * (k & 1);
              if (((e[k >> 1] >> sh) & EX) == EX) {
                e[k >> 1] &= ~(0xFFFFu << sh);
                atomicMin(&s.bad[c * 8 + k], k0 + t);
                odd = true;
              }
            }
            if (odd) {
              *p = make_uint4(e[0], e[1], e[2], e[3]);
              s.any_bad = 1;
            }
          }
#pragma unroll
          for (int i = 0; i < 64; ++i)
            if (k0 + i >= see || !((valid >> (i >> 3)) & 1)) v[i >> 5][i & 31] = -INFINITY;
        }
#pragma unroll
        for (int i = 0; i < 64; i += 4)
          top = fmaxf(fmaxf(top, fmaxf(v[i >> 5][i & 31], v[i >> 5][(i & 31) + 1])), fmaxf(v[i >> 5][(i & 31) + 2], v[i >> 5][(i & 31) + 3]));
        // the output and the weights of the step before are done with
        if (g > 0) wait(&s.pv, (g - 1) & 1);
        tc_fence_after();
        const bool live = lane < 16 && row < rows;
        const bool move = live && (top > m + 8.0f || (m == -INFINITY && top > m));
        float f = 1.0f;
        if (move) {
          f = exp2_fast(m - top);
          m = top;
          l *= f;
        }
        const bool some = any_of_softmax(move || quit);
        if (some && any_of_softmax(quit)) { quit = true; break; }
        if (some && j > 0) {
          if (lane < 16) s.f[row] = f;
          asm volatile("bar.sync 3, 128;" ::: "memory");
#pragma unroll 1
          for (int c = 0; c < MT * 64; c += 32) {
            float o[32];
            tc_ld32(o, to + c);
            tc_wait_ld();
            tc_loaded(o);
            u32 scaled[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) scaled[i] = __float_as_uint(o[i] * s.f[(c & 32) + i]);
            tc_st32(to + c, scaled);
          }
          tc_wait_st();
        }
        const float ref = m == -INFINITY ? 0.0f : m;
        float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (live) {
#pragma unroll
          for (int c = 0; c < 8; ++c) {
            u32 two[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const int i = c * 8 + 2 * k;
              const float p0 = exp2_fast(v[i >> 5][i & 31] - ref), p1 = exp2_fast(v[i >> 5][(i & 31) + 1] - ref);
              sum[k] += p0 + p1;
              two[k] = pack2<F16>(p0, p1);
            }
            *reinterpret_cast<uint4*>(smem + (smem_p - smem_q) + row * 128 + ((c ^ (row & 7)) * 16)) = make_uint4(two[0], two[1], two[2], two[3]);
          }
        }
        l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        tc_fence_before();
        bar_arrive(&s.p);
      }
      if (quit) break;
      // ---- the next item's Q while the last products run
      wait(&s.q_free, item & 1);
      more = line.next();
      if (more && !quit) load_q(line);
      ++item;
      // ---- output
      wait(&s.pv, (g - 1) & 1);
      if (any_of_softmax(quit)) break;
      tc_fence_after();
      const bool whole = first == last, live = lane < 16 && row < rows;
      float* const my = sums + ((i64)(2 * cta + (cta == first ? 1 : 0)) * PAIR + half) * Shape::PART;
      if (live) {
        const i64 pos = (i64)rq.pos0 + (row_base + row) / a.group;
        if (whole) {
          s.f[row] = row_factor(a, r, pos, l);
          if (a.lse) a.lse[(i64)(rq.row0 + (row_base + row) / a.group) * a.heads + (row_base + row) % a.group] = lse_of(m, l);
        } else {
          s.f[row] = 1.0f;
          my[LA_ROWS * L + row] = m;
          my[LA_ROWS * L + LA_ROWS + row] = l;
        }
      }
      if (tid == 0 && !whole && cta == first) { part->r = r; part->rt = rt; part->parts = (int)(last - first) + 1; }
      asm volatile("bar.sync 3, 128;" ::: "memory");
      const bool any_bad = *reinterpret_cast<volatile int*>(&s.any_bad) != 0;
#pragma unroll 1
      for (int c = 0; c < MT * 64; c += 32) {
        const int d = (c >> 6) * 128 + tid, r0 = c & 32;
        if (r0 >= rows) continue;
        float o[32];
        tc_ld32(o, to + c);
        tc_wait_ld();
        tc_loaded(o);
        const int bad = any_bad ? s.bad[d] : 0x7FFFFFFF;
        int fr = (row_base + r0) / a.group, hq = (row_base + r0) % a.group;
        unsigned char* dst = a.out + 2 * ((i64)(rq.row0 + fr) * a.o_token + (i64)hq * a.o_head + d);
#pragma unroll
        for (int i = 0; i < 32; ++i) {
          if (r0 + i < rows) {
            // weights that are all zero leave zeros (or NaN: what the factor says)
            const float f = s.f[r0 + i];
            float y = o[i] * f;
            if (bad != 0x7FFFFFFF && seen_by(r0 + i) > bad) y = NAN;
            if (whole) *reinterpret_cast<unsigned short*>(dst) = (unsigned short)pack2<F16>(y, 0.0f);
            else my[(r0 + i) * L + d] = y;
            dst += 2 * a.o_head;
            if (++hq == a.group) { hq = 0; dst += 2 * (a.o_token - (i64)a.group * a.o_head); }
          }
        }
      }
      tc_fence_before();
      asm volatile("bar.sync 3, 128;" ::: "memory");
      if (any_bad) {
        for (int i = tid; i < L; i += 128) s.bad[i] = 0x7FFFFFFF;
        if (tid == 0) s.any_bad = 0;
        asm volatile("bar.sync 3, 128;" ::: "memory");
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 5) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
    if (lane == 0 && s.gave_up && a.status) atomicOr(a.status, PTSTORE_S_TIMEOUT);
  }
}

// Joins the sums of the items that span several CTAs: blockIdx.x the CTA an item begins in, blockIdx.y four of its rows, a thread for 4 elements of a row.
template <int L, bool F16, int PAIR>
__global__ void __launch_bounds__(L / 4) latent_join_kernel(const Latent la, int grid) {
  const Attend& a = la.a;
  const LatentPart part = reinterpret_cast<const LatentPart*>(a.work)[blockIdx.x];
  if (part.parts == 0) return;
  constexpr int NQ = LA_ROWS * PAIR, PF = LatentShape<L>::PART;
  const u32 cta = blockIdx.x / PAIR, half = blockIdx.x % PAIR;
  const Req q = request(a, part.r);
  const int row_base = (int)(part.rt * NQ) + (int)half * LA_ROWS, rows = min(LA_ROWS, q.fresh * a.group - row_base);
  const float* const sums = reinterpret_cast<const float*>(a.work + LA_PARTS_AT) + (i64)half * PF;
  auto at = [&](int p) { return sums + (i64)(2 * (cta + p) + (p == 0 ? 1 : 0)) * PAIR * PF; };
  const int e = threadIdx.x * 4;
  for (int row = blockIdx.y * 4; row < min((int)blockIdx.y * 4 + 4, rows); ++row) {
    float top = -INFINITY, sum = 0.0f;
    for (int p = 0; p < part.parts; ++p) top = fmaxf(top, at(p)[LA_ROWS * L + row]);
    float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
    for (int p = 0; p < part.parts; ++p) {
      const float m = at(p)[LA_ROWS * L + row];
      const float f = m == -INFINITY ? 1.0f : exp2_fast(m - top);             // nothing seen: sums of zero (or NaN)
      const float4 v = *reinterpret_cast<const float4*>(at(p) + row * L + e);
      sum += at(p)[LA_ROWS * L + LA_ROWS + row] * f;
      o.x += v.x * f;
      o.y += v.y * f;
      o.z += v.z * f;
      o.w += v.w * f;
    }
    const int fr = (row_base + row) / a.group, hq = (row_base + row) % a.group;
    const float f = row_factor(a, part.r, (i64)q.pos0 + fr, sum);
    *reinterpret_cast<uint2*>(a.out + 2 * ((i64)(q.row0 + fr) * a.o_token + (i64)hq * a.o_head + e)) = make_uint2(pack2<F16>(o.x * f, o.y * f), pack2<F16>(o.z * f, o.w * f));
    if (a.lse && threadIdx.x == 0) a.lse[(i64)(q.row0 + fr) * a.heads + hq] = lse_of(top, sum);
  }
}

}  // namespace ptk
