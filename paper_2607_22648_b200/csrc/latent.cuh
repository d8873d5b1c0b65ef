// Absorbed attention over a cache of latent vectors: one row c_j | r_j of L + 64 elements a token, which is the key of every query head, and its first
// L elements the value.  Bounded by reading the rows once up to some 100 rows of q a request, by the tensor cores beyond.
//
// Rows of q are (new token, query head) pairs.  A step is 64 cached tokens, which lie in shared memory as boxes of 64 elements and serve as keys and as values:
//     S = Q K^T          M = 128 rows, N = 64 tokens, K = L + 64; Q in tensor memory, as far as it fits
//     P = exp2(scale2 S - m)                       (one thread per row)
//     O^T += C^T P^T     M = 128 latent elements; N = the rows, K = 64 tokens
// The output is held transposed so that few rows cost little, and so that both operands lie as the cache has them.  m is a running reference, moved only when a
// scaled score exceeds it by more than LA_MOVE, since that means reading and writing O.
//
// Up to 32 rows (NARROW): a CTA has all L elements of the output; a step's tile of 72 KB is in flight three times.  More rows (WIDE): O of 128 rows and all
// elements would fill tensor memory and Q shared memory, so two neighbouring CTAs walk the same tokens for 128 rows and have half of the output's elements each.  Both compute
// all scores, but a tile's boxes beyond a CTA's own half are free again as soon as they are: the boxes that are values too have a ring of three tiles, the others one of
// eight boxes.
//
// Warps 0-3 softmax, and Q and the output of an item; 4 and 6 load (values and other boxes); 5 issues the scores' instructions, 7 the output's.  One CTA (or pair) per SM (or two) takes an
// even share of the line of all (request, row tile, 64 tokens) units.  An item that spans several CTAs leaves sums (o, m, l in 32 bits) in the workspace,
// which latent_join_kernel joins in CTA order.
//
// B200, L = 512, bf16, ten passes behind a pause / passes for seconds at the power limit: decode of 64 x 128 heads over 4160 tokens on average 169 / 174 us (437 / 425 TFLOP/s); 16 x 64 new
// tokens of 16 heads over 4160, fp16, 249 / 268 us (592 / 550); one request of 16 heads 25 us.  A step of 128 rows has 1856 clocks of tensor instructions and moves 270 KB through shared memory (2100 clocks): 2500 clocks where its tile is there in time, 3000 to 4500
// with the waits for it: Q, P and O leave room for 1.6 tiles of the boxes that are no values, and a tensor copy takes 60 clocks + 1.75 a row of 128 bytes whatever its size, so that
// blocks of 16 tokens (36 copies a step) take 168 us where blocks of 64 take 150.  Measured and dropped: halves of the scores exchanged through distributed shared memory, each CTA
// with half of the products (324 us: remote stores go at 11 bytes a clock); rings with more room for either kind of box (180 / 282 us for the two batches).
#pragma once
#include "attend_prompt.cuh"
#include "attend_split.cuh"

namespace ptk {

constexpr int LA_THREADS = 256, LA_KEYS = 64, LA_ROPE = 64, LA_BOX = LA_KEYS * 128;      // a box: 64 tokens, 64 elements
// A reference moves when a scaled score exceeds it by more than this.  Weights are then at most 2^14 (fp16 holds 2^15): with 8, the tiles of 128 rows whose scores spread over 5
// octaves (standard deviation) were rescaled in every other step, 1400 clocks each.
constexpr float LA_MOVE = 14.0f;
constexpr int LA_AHEAD = 2;                  // units (of a pair of CTAs) that are brought into L2 before they are loaded
constexpr int LA_MIN_UNITS = 4;              // a CTA takes at least this many, so that joining does not cost more than it saves (one request of 4160 tokens, 16 heads: 1 / 2 / 4 / 8 units
                                             // 31.0 / 26.8 / 24.7 / 26.8 us)

template <int L, bool WIDE>
struct LatentShape {
  static constexpr int BOXES = L / 64 + 1, ROWS = WIDE ? 128 : 32, PAIR = WIDE ? 2 : 1;
  static constexpr int VALUES = WIDE ? L / 128 : L / 64, OTHERS = BOXES - VALUES;          // boxes of a tile that are values of this CTA, and those that are not
  static constexpr int DIMS = VALUES * 64, MT = DIMS / 128;                               // output elements, instructions' worth of them
  // tensor memory: O, S, Q
  static constexpr int S_AT = MT * ROWS, Q_AT = S_AT + LA_KEYS, Q_MOST = (512 - Q_AT) / 32, Q_TMEM = Q_MOST < BOXES ? Q_MOST : BOXES;
  // shared memory: P, the rest of Q (or a box of it on its way to tensor memory), the rings
  static constexpr int P_BYTES = ROWS * 128, Q_BYTES = (BOXES > Q_TMEM ? BOXES - Q_TMEM : 1) * ROWS * 128;
  static constexpr int STAGES = L == 512 ? 3 : WIDE ? 6 : 5, SLOTS = WIDE ? (L == 512 ? 8 : 12) : STAGES;
  static constexpr int V_AT = P_BYTES + Q_BYTES, K_AT = V_AT + STAGES * VALUES * LA_BOX, MISC_AT = K_AT + SLOTS * LA_BOX;
  static constexpr int PART = ROWS * (DIMS + 2);                                          // floats of an item's sums in one CTA: o, m, l
};
template <int L, bool WIDE>
struct LatentMisc {
  using Shape = LatentShape<L, WIDE>;
  u64 v_full[Shape::STAGES], v_empty[Shape::STAGES], k_full[Shape::SLOTS], k_empty[Shape::SLOTS], q, q_free, s, s_free, p, pv, end[2], left, scan[LA_THREADS / 32];
  u32 valid[Shape::STAGES], tmem, loaded[4];         // loaded: items whose q each warp of the other CTA has read
  int gave_up, any_bad, r;
  alignas(16) float f[Shape::ROWS];
  alignas(16) u32 moved[4];  // of each warp's rows: 1 a reference has moved, 2 a wait ran out
  int bad[Shape::DIMS];      // first token whose element d is not finite, among tokens that some rows do not see
};
template <int L, bool WIDE>
constexpr int latent_smem() { return LatentShape<L, WIDE>::MISC_AT + (int)sizeof(LatentMisc<L, WIDE>); }
static_assert(latent_smem<512, true>() <= 232448 && latent_smem<512, false>() <= 232448 && latent_smem<256, true>() <= 232448 && latent_smem<256, false>() <= 232448,
              "fits an SM (there is no static shared memory, so the operands begin on a multiple of 1024)");

struct Latent {
  Attend a;                  // q: q_latent; cache.heads 1, group = heads; box_tokens: tokens of a tensor copy
  const unsigned char* q_rope;
  i64 qr_token, qr_head;
};
// what the join needs of an item that begins in a CTA and goes on in others
struct LatentPart { int parts, r; u32 rt; };
constexpr int LA_PARTS_AT = 8192;            // where the sums begin in the workspace, behind the descriptions of the largest grid
static_assert(MAX_SMS * sizeof(LatentPart) <= LA_PARTS_AT, "descriptions fit");

// The items of one CTA's share of the line, one after the other.  NQ rows are a row tile.
template <int NQ>
struct LatentLine {
  const Attend& a;
  u64 u, u_end, left;
  u32 per;
  int r;
  u32 rt;
  Req q;
  // the item: tokens its rows see, its units and this CTA's part of them [ua, ub), the CTAs that share it
  int keys, units, ua, ub;
  u32 first, last;
  __device__ __forceinline__ bool next() {
    if (u >= u_end) return false;
    for (;;) {
      if (rt >= row_tiles<NQ>(a, q)) {
        if (++r >= a.R) return false;                         // cannot happen while offsets and lengths hold still
        rt = 0;
        q = request(a, r);
        continue;
      }
      keys = tile_keys<NQ>(a, q, rt);
      units = units_of<LA_KEYS>(keys);
      if (left < (u64)units) break;
      left -= units;
      ++rt;
    }
    ua = (int)left;
    ub = u_end - u < (u64)(units - ua) ? ua + (int)(u_end - u) : units;
    first = quotient(u - ua, per);
    last = quotient(u - ua + units - 1, per);
    u += ub - ua;
    left += ub - ua;
    return true;
  }
};

// instruction descriptor of kind::f16, M = 128, A "MN-major" or not; B has its elements of one row contiguous.  N is added at bit 17 in eights.
__host__ __device__ constexpr u32 mma_desc_a(bool fp16, bool a_mn_major) {
  return (1u << 4) | ((fp16 ? 0u : 1u) << 7) | ((fp16 ? 0u : 1u) << 10) | ((a_mn_major ? 1u : 0u) << 15) | ((u32)(128 >> 4) << 24);
}
// some tokens of a block, 64 elements: box of the map {elements, tokens of a block, blocks}
__device__ __forceinline__ void tensor_load_box(u32 dst, const CUtensorMap* map, int element, int token, int block, u64* bar) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst), "l"(map), "r"(element), "r"(token),
               "r"(block), "r"(smem_addr(bar)) : "memory");
}
__device__ __forceinline__ void bulk_prefetch(const void* src, u32 bytes) {      // into L2
  asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(src), "r"(bytes) : "memory");
}
// the other CTA of a pair: a word in its shared memory, written behind what this thread has done, and read before what it does
__device__ __forceinline__ void tell_other(const u32* word, u32 rank, u32 value) {
  u32 at;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_addr(word)), "r"(rank));
  asm volatile("st.release.cluster.shared::cluster.u32 [%0], %1;" ::"r"(at), "r"(value) : "memory");
}
__device__ __forceinline__ u32 told(const u32* word) {
  u32 v;
  asm volatile("ld.acquire.cluster.shared::cta.u32 %0, [%1];" : "=r"(v) : "r"(smem_addr(word)) : "memory");
  return v;
}
__device__ __forceinline__ void cluster_sync() { asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ bool any_of_softmax(bool v) {      // barrier of the 128 softmax threads
  u32 r;
  asm volatile("{\n .reg .pred p, q;\n setp.ne.u32 p, %1, 0;\n barrier.cta.red.or.pred q, 2, 128, p;\n selp.u32 %0, 1, 0, q;\n}" : "=r"(r) : "r"((u32)v) : "memory");
  return r != 0;
}

// ALIAS: the output is q itself.  The two CTAs of a pair are then a cluster and tell each other whose q they have read (which costs calls of many rows 5 %).
template <int L, bool F16, bool WIDE, bool ALIAS>
__global__ void __launch_bounds__(LA_THREADS, 1) latent_attend_kernel(const Latent la, const __grid_constant__ CUtensorMap map) {
  using Shape = LatentShape<L, WIDE>;
  constexpr int NQ = Shape::ROWS, STAGES = Shape::STAGES, SLOTS = Shape::SLOTS, BOXES = Shape::BOXES, VALUES = Shape::VALUES, OTHERS = Shape::OTHERS, MT = Shape::MT,
                DIMS = Shape::DIMS, PAIR = Shape::PAIR;
  extern __shared__ __align__(1024) unsigned char latent_smem_raw[];
  unsigned char* const smem = latent_smem_raw;
  const Attend& a = la.a;
  LatentMisc<L, WIDE>& s = *reinterpret_cast<LatentMisc<L, WIDE>*>(smem + Shape::MISC_AT);
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(FULL, tid >> 5, 0);
  const u32 cta = blockIdx.x / PAIR, ctas = gridDim.x / PAIR, half = blockIdx.x % PAIR;
  LatentPart* const part = reinterpret_cast<LatentPart*>(a.work) + blockIdx.x;
  float* const sums = reinterpret_cast<float*>(a.work + LA_PARTS_AT);

  // ---- this CTA's share of the line: every CTA sums the units of all requests, consecutive requests per thread
  if (tid == 0) {
    part->parts = 0;
    for (int i = 0; i < STAGES; ++i) { bar_init(&s.v_full[i], 1); bar_init(&s.v_empty[i], 1); }
    for (int i = 0; i < SLOTS; ++i) { bar_init(&s.k_full[i], 1); bar_init(&s.k_empty[i], 1); }
    bar_init(&s.q, 4);
    bar_init(&s.q_free, 1);
    bar_init(&s.s, 1);
    bar_init(&s.s_free, 4);
    bar_init(&s.p, 4);
    bar_init(&s.pv, 1);
    bar_init(&s.end[0], 1);
    bar_init(&s.end[1], 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    s.gave_up = s.any_bad = 0;
    for (int i = 0; i < 4; ++i) s.loaded[i] = 0;
    s.r = -1;
  }
  if (tid == 160) asm volatile("prefetch.tensormap [%0];" ::"l"(&map) : "memory");
  for (int i = tid; i < DIMS; i += LA_THREADS) s.bad[i] = 0x7FFFFFFF;
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
  if (WIDE && ALIAS) cluster_sync();                   // (the other CTA writes here once this one has begun)
  __syncthreads();
  tc_fence_after();
  const u32 tmem = s.tmem;
  const u32 smem_p = smem_addr(smem), smem_q = smem_p + Shape::P_BYTES, smem_v = smem_p + Shape::V_AT, smem_k = smem_p + Shape::K_AT;
  LatentLine<NQ> line{a, u_begin, u_end, s.left, per, s.r, 0, request(a, s.r)};
  // the elements of box i of a tile, in the order of the products: this CTA's values, the other half's, the rotary part
  auto element_of = [&](int i) {
    return 64 * (i < VALUES ? (int)half * VALUES + i : i < L / 64 ? (int)(1 - half) * VALUES + i - VALUES : L / 64);
  };

  if (warp == 5) {
    // ======== scores: a step's as soon as its tile is there and the ones before it have been read
    constexpr u32 QK = mma_desc_a(F16, false) | (u32)(LA_KEYS >> 3) << 17;
    u32 g = 0, item = 0, op = 0;              // step, item, box that is no value
    bool quit = false;
    auto wait = [&](u64* b, u32 parity) {     // (a lane may have a barrier of its own)
      if (!quit && !__all_sync(FULL, bar_wait(b, parity, a.polls, &s.gave_up))) quit = true;
      __syncwarp();
    };
    auto box = [&](int i, u32 at, bool first) {           // scores' part of box i, which lies at `at`
      const u64 kb = operand_desc(at, 0);
#pragma unroll
      for (int k = 0; k < 4; ++k) {           // 16 elements: 8 columns, or 32 bytes further in a row
        if (i < Shape::Q_TMEM) mma_ts(tmem + Shape::S_AT, tmem + Shape::Q_AT + i * 32 + k * 8, kb + (u64)((k * 32) >> 4), QK, !first || k > 0);
        else mma_ss(tmem + Shape::S_AT, operand_desc(smem_q + (i - Shape::Q_TMEM) * 16384, 0) + (u64)((k * 32) >> 4), kb + (u64)((k * 32) >> 4), QK, !first || k > 0);
      }
    };
    while (!quit && line.next()) {
      const int n = line.ub - line.ua;
      for (int j = 0; j < n && !quit; ++j, ++g, op += OTHERS) {
        // the tile (and Q), all at once; then the scores before these have been read
        const u32 o = op + (lane < OTHERS ? lane : 0);
        const bool first = j == 0 && lane == OTHERS + 1, value = lane == OTHERS;
        wait(first ? &s.q : value ? &s.v_full[g % STAGES] : &s.k_full[o % SLOTS], (first ? item : value ? g / STAGES : o / SLOTS) & 1);
        if (g > 0) wait(&s.s_free, (g - 1) & 1);
        tc_fence_after();
        if (!quit && elected()) {
          // boxes that are no values first: what follows them is waiting for their places
#pragma unroll
          for (int i = 0; i < OTHERS; ++i) {
            box(VALUES + i, smem_k + ((op + i) % SLOTS) * LA_BOX, i == 0);
            tc_commit(&s.k_empty[(op + i) % SLOTS]);
          }
#pragma unroll
          for (int i = 0; i < VALUES; ++i) box(i, smem_v + ((g % STAGES) * VALUES + i) * LA_BOX, false);
          tc_commit(&s.s);
          if (j + 1 == n) tc_commit(&s.q_free);
        }
        __syncwarp();
      }
      ++item;
    }
    // everything issued has ended before tensor and shared memory are given back
    if (elected()) tc_commit(&s.end[0]);
    __syncwarp();
    bar_drain(&s.end[0], 0);
  } else if (warp == 7) {
    // ======== the output, when a step's weights are there
    constexpr u32 PV = mma_desc_a(F16, true);
    u32 g = 0;
    bool quit = false;
    while (!quit && line.next()) {
      const int n = line.ub - line.ua, rows = min(NQ, line.q.fresh * a.group - (int)(line.rt * NQ));
      const u32 pv = PV | (u32)((rows + 15) / 16 * 2) << 17;
      for (int j = 0; j < n; ++j, ++g) {
        // (the tile has been there since its scores: waited for only so that its bytes are this warp's too)
        if (!__all_sync(FULL, bar_wait(&s.p, g & 1, a.polls, &s.gave_up) && bar_wait(&s.v_full[g % STAGES], (g / STAGES) & 1, a.polls, &s.gave_up))) { quit = true; break; }
        tc_fence_after();
        if (elected()) {
          const u32 tile = smem_v + (g % STAGES) * VALUES * LA_BOX;
          const u64 pb = operand_desc(smem_p, 0);
#pragma unroll
          for (int i = 0; i < MT; ++i) {
            const u64 va = operand_desc(tile + 2 * i * LA_BOX, LA_BOX);
#pragma unroll
            for (int k = 0; k < LA_KEYS / 16; ++k)            // 16 tokens: 16 rows of 128 bytes
              mma_ss(tmem + i * NQ, va + (u64)((k * 16 * 128) >> 4), pb + (u64)((k * 32) >> 4), pv, j > 0 || k > 0);
          }
          tc_commit(&s.v_empty[g % STAGES]);
          tc_commit(&s.pv);
        }
        __syncwarp();
      }
    }
    if (elected()) tc_commit(&s.end[1]);
    __syncwarp();
    bar_drain(&s.end[1], 0);
  } else if (warp >= 4) {
    // ======== tiles: warp 4 the boxes that are values, warp 6 the others.  Lane j has the tokens of copy j of a box, some tokens of a block each.
    const bool values = warp == 4;
    const u32 B = a.cache.block_tokens, bt = a.box_tokens, copies = LA_KEYS / bt;
    u32 g = 0, op = 0;
    bool bounds = false, quit = false;
    const u32 mine_at = lane % copies, team = lane / copies, teams = 32 / copies;
    while (!quit && line.next()) {
      const int* const table = a.tables + (i64)line.r * a.max_blocks;
      auto look_up = [&](int unit) {
        const int key = unit * LA_KEYS + (int)(mine_at * bt);
        return key < line.keys ? table[(u32)key / B] : -1;
      };
      const bool alone = WIDE && line.q.fresh * a.group <= NQ;               // the request's only row tile
      int id = look_up(line.ua), far_id = alone && values && line.ua + LA_AHEAD < line.ub ? look_up(line.ua + LA_AHEAD) : -1;
      for (int unit = line.ua; unit < line.ub && !quit; ++unit, ++g) {
        const int key = unit * LA_KEYS + (int)(mine_at * bt);
        const bool in = key < line.keys, have = in && (u32)id < a.cache.num_blocks;
        bounds |= values && in && !have;
        const int block = id, token = (int)((u32)key % B);
        if (unit + 1 < line.ub) id = look_up(unit + 1);
        const u32 there = __ballot_sync(FULL, have && team == 0), bytes = __popc(there) * bt * 128;
        if (values) {
          if (WIDE) {
            // Few boxes are on their way at a time, so later units' rows, which lie together in a block, are brought nearer, by the CTAs of a pair in turn: 64 requests of one row tile
            // each 170 us, without 177.  Not where a request has several row tiles, whose pairs bring them for one another (16 requests of 8: 252 us, without 240).
            const int far = unit + LA_AHEAD, fkey = far * LA_KEYS + (int)(mine_at * bt);
            if (alone && far < line.ub && team == 0 && (u32)(far & 1) == half && (u32)far_id < a.cache.num_blocks)
              bulk_prefetch(a.cache.base + (u64)(u32)far_id * a.cache.block_stride + (u64)((u32)fkey % B) * ((L + 64) * 2), bt * (L + 64) * 2);
            far_id = alone && far + 1 < line.ub ? look_up(far + 1) : -1;
          }
          const u32 st = g % STAGES;
          if (g >= STAGES && !__all_sync(FULL, bar_wait(&s.v_empty[st], (g / STAGES - 1) & 1, a.polls, &s.gave_up))) { quit = true; break; }
          // groups of 8 tokens that are there
          const u32 groups = __reduce_or_sync(FULL, have && team == 0 ? ((1u << (bt / 8)) - 1) << (mine_at * (bt / 8)) : 0u);
          if (lane == 0) {
            s.valid[st] = groups;
            if (there) bar_expect(&s.v_full[st], bytes * VALUES);
            else bar_arrive(&s.v_full[st]);
          }
          __syncwarp();
          if (have)
            for (u32 i = team; i < VALUES; i += teams)
              tensor_load_box(smem_v + (st * VALUES + i) * LA_BOX + mine_at * bt * 128, &map, element_of((int)i), token, block, &s.v_full[st]);
        } else {
          for (u32 i = 0; i < OTHERS; ++i, ++op) {
            const u32 st = op % SLOTS;
            if (op >= SLOTS && !__all_sync(FULL, bar_wait(&s.k_empty[st], (op / SLOTS - 1) & 1, a.polls, &s.gave_up))) { quit = true; break; }
            if (lane == 0) {
              if (there) bar_expect(&s.k_full[st], bytes);
              else bar_arrive(&s.k_full[st]);
            }
            __syncwarp();
            if (have && team == 0) tensor_load_box(smem_k + st * LA_BOX + mine_at * bt * 128, &map, element_of(VALUES + (int)i), token, block, &s.k_full[st]);
          }
        }
      }
    }
    // whatever happened, what is in flight lands before the CTA gives its memory back
    if (values)
      for (u32 k = g > STAGES ? g - STAGES : 0; k < g; ++k) bar_drain(&s.v_full[k % STAGES], (k / STAGES) & 1);
    else
      for (u32 k = op > SLOTS ? op - SLOTS : 0; k < op; ++k) bar_drain(&s.k_full[k % SLOTS], (k / SLOTS) & 1);
    if (bounds && a.status) atomicOr(a.status, PTSTORE_S_BOUNDS);
  } else {
    // ======== softmax: thread t has row t; Q before, the output behind an item
    const int row = tid;
    const u32 lane_base = (u32)(32 * warp) << 16, ts = tmem + lane_base + Shape::S_AT, to = tmem + lane_base;
    u32 g = 0, item = 0, loads = 0;
    bool quit = false;
    auto wait = [&](u64* b, u32 parity) {
      if (__any_sync(FULL, !bar_wait(b, parity, a.polls, &s.gave_up))) quit = true;
    };
    // Q of an item, a row a thread.  Eight lanes read 128 bytes of a row at once, and rows change into lanes through shared memory (a row a lane would touch 32 lines with each load).
    // The loop is short because its code is cold every time.  Rows that do not exist have another row's values: their sums are never looked at, and a row's are its own.
    auto load_q = [&](const LatentLine<NQ>& it) {
      const int base = (int)(it.rt * NQ), rows = min(NQ, it.q.fresh * a.group - base);
      if (warp * 32 < rows) {
        const int flat = base + min(row, rows - 1), fr = flat / a.group, hq = flat % a.group;
        const i64 tok = it.q.row0 + fr;
        const i64 latent_at = 2 * (tok * a.q_token + hq * a.q_head), rope_at = 2 * (tok * la.qr_token + hq * la.qr_head);
        constexpr int AT_ONCE = 3;            // boxes on their way
#pragma unroll 1
        for (int i0 = 0; i0 < BOXES; i0 += AT_ONCE) {
          uint4 v[AT_ONCE][8];
#pragma unroll
          for (int i = 0; i < AT_ONCE; ++i) {
            const int b = min(i0 + i, BOXES - 1);
            const i64 mine = b < L / 64 ? latent_at + 2 * element_of(b) : rope_at;
            const unsigned char* const src = (b < L / 64 ? a.q : la.q_rope) + (lane & 7) * 16;
#pragma unroll
            for (int k = 0; k < 8; ++k) v[i][k] = *reinterpret_cast<const uint4*>(src + __shfl_sync(FULL, mine, k * 4 + (lane >> 3)));
          }
#pragma unroll
          for (int i = 0; i < AT_ONCE; ++i) {
            const int b = i0 + i;
            if (b >= BOXES) continue;
            unsigned char* const z = smem + Shape::P_BYTES + max(b - Shape::Q_TMEM, 0) * (NQ * 128) + warp * 4096;
            __syncwarp();
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              const int r = k * 4 + (lane >> 3);
              *reinterpret_cast<uint4*>(z + r * 128 + (((lane ^ r) & 7) * 16)) = v[i][k];
            }
            if (b >= Shape::Q_TMEM) continue;
            __syncwarp();
            u32 w[32];
#pragma unroll
            for (int c = 0; c < 8; ++c) {
              const uint4 x = *reinterpret_cast<const uint4*>(z + lane * 128 + ((c ^ (lane & 7)) * 16));
              w[4 * c] = x.x; w[4 * c + 1] = x.y; w[4 * c + 2] = x.z; w[4 * c + 3] = x.w;
            }
            tc_st32(tmem + lane_base + Shape::Q_AT + b * 32, w);
          }
        }
        tc_wait_st();
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      }
      tc_fence_before();
      warp_arrive(&s.q);
      ++loads;
      if (WIDE && ALIAS && lane == 0) tell_other(&s.loaded[warp], 1 - half, loads);
    };
    bool more = line.next();
    if (more) load_q(line);
    while (more && !quit) {
      const Req rq = line.q;
      const int r = line.r, keys = line.keys, ua = line.ua, n = line.ub - line.ua, row_base = (int)(line.rt * NQ);
      const u32 rt = line.rt, first = line.first, last = line.last;
      const int rows = min(NQ, rq.fresh * a.group - row_base);
      const bool live = row < rows;
      auto seen_by = [&](int row) {
        const i64 k = (i64)rq.pos0 + (row_base + row) / a.group + 1;
        return k < 0 ? 0 : k > keys ? keys : (int)k;
      };
      const int see = live ? seen_by(row) : 0, all_see = seen_by(0);
      float m = -INFINITY, l = 0.0f;
      for (int j = 0; j < n; ++j, ++g) {
        const int k0 = (ua + j) * LA_KEYS;
        const u32 st = g % STAGES;
        // (a wait that ran out in one warp shows in all of them at the next barrier: until then its values are of no use, but in bounds)
        wait(&s.v_full[st], (g / STAGES) & 1);        // (there before the scores are: makes the tile's bytes and its valid bits this thread's too)
        wait(&s.s, g & 1);
        tc_fence_after();
        float v[2][32];
        const bool busy = warp * 32 < rows;           // this warp has rows
        if (busy) {
          tc_ld32(v[0], ts);
          tc_ld32(v[1], ts + 32);
          tc_wait_ld();
          tc_loaded(v[0]);
          tc_loaded(v[1]);
          tc_fence_before();
        }
        warp_arrive(&s.s_free);
        const u32 valid = s.valid[st];
        const bool edge = k0 + LA_KEYS > all_see || valid != 0xFFu;
        if (edge) {
          // A weight of zero does not hide an infinity or a NaN.  Tokens that no row sees become zero; what is not finite in tokens that only some rows see is
          // taken out, and put into the sums of the rows that see it at the end.  (The scores have been computed by now.)
          unsigned char* const tile = smem + Shape::V_AT + st * VALUES * LA_BOX;
          constexpr u32 EX = F16 ? 0x7C00u : 0x7F80u;
          const int from = max(all_see - k0, 0);
          for (int i = tid; i < LA_KEYS * (DIMS / 8); i += 128) {
            const int t = i / (DIMS / 8), c = i % (DIMS / 8);
            const bool there = (valid >> (t >> 3)) & 1;
            if (t < from && there) continue;
            uint4* const p = reinterpret_cast<uint4*>(tile + (c >> 3) * LA_BOX + t * 128 + (((c & 7) ^ (t & 7)) * 16));
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
        }
        float f = 1.0f;
        bool move = false;
        u32 p[32];
        if (busy) {
          // the products rounded as the maximum is, so that the largest weight is 1 however large the scores are
          const u64 sc2 = pair(a.scale2, a.scale2);
#pragma unroll
          for (int i = 0; i < 64; i += 2) {
            const u64 y = mul_pair(pair(v[i >> 5][i & 31], v[i >> 5][(i & 31) + 1]), sc2);
            v[i >> 5][i & 31] = lo_of(y);
            v[i >> 5][(i & 31) + 1] = hi_of(y);
          }
          if (edge) {
#pragma unroll
            for (int i = 0; i < 64; ++i)
              if (k0 + i >= see || !((valid >> (i >> 3)) & 1)) v[i >> 5][i & 31] = -INFINITY;
          }
          float x4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int i = 0; i < 64; i += 8)
#pragma unroll
            for (int k = 0; k < 4; ++k) x4[k] = fmaxf(x4[k], fmaxf(v[i >> 5][(i & 31) + 2 * k], v[i >> 5][(i & 31) + 2 * k + 1]));
          const float top = fmaxf(fmaxf(x4[0], x4[1]), fmaxf(x4[2], x4[3]));
          move = live && (top > m + LA_MOVE || (m == -INFINITY && top > m));
          if (move) {
            f = exp2_fast(m - top);
            m = top;
            l *= f;
          }
          const float ref = m == -INFINITY ? 0.0f : m;
          float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
          for (int i = 0; i < 64; i += 2) {
            const float p0 = exp2_fast(v[i >> 5][i & 31] - ref), p1 = exp2_fast(v[i >> 5][(i & 31) + 1] - ref);
            sum[(i >> 1) & 3] += p0 + p1;
            p[i >> 1] = pack2<F16>(p0, p1);
          }
          l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
        }
        // the output and the weights of the step before are done with
        if (g > 0) wait(&s.pv, (g - 1) & 1);
        tc_fence_after();
        const bool any = __any_sync(FULL, move);
        if (lane == 0) s.moved[warp] = (any ? 1u : 0u) | (quit ? 2u : 0u);
        if (row < NQ) s.f[row] = f;
        asm volatile("bar.sync 2, 128;" ::: "memory");
        const uint4 flags = *reinterpret_cast<const uint4*>(s.moved);
        const u32 moved[4] = {flags.x, flags.y, flags.z, flags.w};
        if ((moved[0] | moved[1] | moved[2] | moved[3]) & 2) { quit = true; break; }
        if (j > 0) {
#pragma unroll
          for (int w = 0; w < NQ / 32; ++w) {               // 32 rows, where one of them has moved
            if (!(moved[w] & 1)) continue;
#pragma unroll 1
            for (int c = w * 32; c < MT * NQ; c += NQ) {
              float o[32];
              tc_ld32(o, to + c);
              tc_wait_ld();
              tc_loaded(o);
              u32 scaled[32];
#pragma unroll
              for (int i = 0; i < 32; i += 4) {
                const float4 f4 = *reinterpret_cast<const float4*>(&s.f[w * 32 + i]);
                scaled[i] = __float_as_uint(o[i] * f4.x);
                scaled[i + 1] = __float_as_uint(o[i + 1] * f4.y);
                scaled[i + 2] = __float_as_uint(o[i + 2] * f4.z);
                scaled[i + 3] = __float_as_uint(o[i + 3] * f4.w);
              }
              tc_st32(to + c, scaled);
            }
          }
          tc_wait_st();
        }
        if (live) {
#pragma unroll
          for (int c = 0; c < 8; ++c)
            *reinterpret_cast<uint4*>(smem + row * 128 + ((c ^ (row & 7)) * 16)) = make_uint4(p[4 * c], p[4 * c + 1], p[4 * c + 2], p[4 * c + 3]);
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        tc_fence_before();
        warp_arrive(&s.p);
      }
      if (quit) break;
      // ---- the next item's Q while the last products run
      wait(&s.q_free, item & 1);
      tc_fence_after();
      more = line.next();
      if (more && !quit) load_q(line);
      ++item;
      // ---- output
      wait(&s.pv, (g - 1) & 1);
      if (WIDE && ALIAS) {                    // the other CTA has read all of the item's q
        bool ok = lane >= 4;
        for (u32 i = 0; !ok && i < a.polls; ++i) {
          ok = (int)(told(&s.loaded[lane]) - item) >= 0;
          if ((i & 1023) == 1023 && *reinterpret_cast<volatile int*>(&s.gave_up)) break;
        }
        if (!ok) s.gave_up = 1;
        if (!__all_sync(FULL, ok)) quit = true;
        __syncwarp();
      }
      if (any_of_softmax(quit)) break;
      tc_fence_after();
      const bool whole = first == last;
      float* const my = sums + ((i64)(2 * cta + (cta == first ? 1 : 0)) * PAIR + half) * Shape::PART;
      if (live) {
        const i64 pos = (i64)rq.pos0 + (row_base + row) / a.group;
        if (whole) {
          s.f[row] = row_factor(a, r, pos, l);
          if (a.lse && half == 0) a.lse[(i64)(rq.row0 + (row_base + row) / a.group) * a.heads + (row_base + row) % a.group] = lse_of(m, l);
        } else {
          s.f[row] = 1.0f;
          my[NQ * DIMS + row] = m;
          my[NQ * DIMS + NQ + row] = l;
        }
      }
      if (tid == 0 && !whole && cta == first) { part->r = r; part->rt = rt; part->parts = (int)(last - first) + 1; }
      asm volatile("bar.sync 3, 128;" ::: "memory");
      const bool any_bad = *reinterpret_cast<volatile int*>(&s.any_bad) != 0;
      u32 turn = 0;                           // pieces of 32 rows done: rows that are not there have none, so c does not say which place is free
#pragma unroll 1
      for (int c = 0; c < MT * NQ; c += 32) {
        const int d = c / NQ * 128 + tid, r0 = c % NQ;
        if (r0 >= rows) continue;
        float o[32];
        tc_ld32(o, to + c);
        tc_wait_ld();
        tc_loaded(o);
        // (all in registers before the first is stored: a store between the factors' loads would keep them in order, one by one)
        const int m32 = min(32, rows - r0);
#pragma unroll
        for (int i = 0; i < 32; i += 4) {
          const float4 f4 = *reinterpret_cast<const float4*>(&s.f[r0 + i]);
          o[i] *= f4.x;                       // weights that are all zero leave zeros (or NaN: what the factor says)
          o[i + 1] *= f4.y;
          o[i + 2] *= f4.z;
          o[i + 3] *= f4.w;
        }
        if (any_bad) {
          const int bad = s.bad[d];
          if (bad != 0x7FFFFFFF) {
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (seen_by(r0 + i) > bad) o[i] = NAN;
          }
        }
        if (whole) {
          // whole rows of 128 elements through shared memory (P's, which the last products have read)
          unsigned char* const z = smem + (WIDE ? (turn++ & 1) * 8192 : 0);
#pragma unroll
          for (int i = 0; i < 32; i += 2) {
            const u32 two = pack2<F16>(o[i], o[i + 1]);
            *reinterpret_cast<unsigned short*>(z + i * 256 + tid * 2) = (unsigned short)two;
            *reinterpret_cast<unsigned short*>(z + i * 256 + 256 + tid * 2) = (unsigned short)(two >> 16);
          }
          asm volatile("bar.sync 3, 128;" ::: "memory");
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int i = k * 8 + (tid >> 4), flat = row_base + r0 + i;
            if (i < m32)
              *reinterpret_cast<uint4*>(a.out + 2 * ((i64)(rq.row0 + flat / a.group) * a.o_token + (i64)(flat % a.group) * a.o_head + (int)half * DIMS + c / NQ * 128 + (tid & 15) * 8)) =
                  *reinterpret_cast<const uint4*>(z + i * 256 + (tid & 15) * 16);
          }
          // (two places take turns where there are two: a piece's writes come behind the barrier of the piece before, which the reads of the one before that precede)
          if (!WIDE) asm volatile("bar.sync 3, 128;" ::: "memory");
        } else {
          float* const dst = my + r0 * DIMS + d;
#pragma unroll
          for (int i = 0; i < 32; ++i)
            if (i < m32) dst[i * DIMS] = o[i];
        }
      }
      tc_fence_before();
      asm volatile("bar.sync 3, 128;" ::: "memory");
      if (any_bad) {
        for (int i = tid; i < DIMS; i += 128) s.bad[i] = 0x7FFFFFFF;
        if (tid == 0) s.any_bad = 0;
        asm volatile("bar.sync 3, 128;" ::: "memory");
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (WIDE && ALIAS) cluster_sync();                   // (and does not any more when this one leaves)
  if (warp == 5) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
    if (lane == 0 && s.gave_up && a.status) atomicOr(a.status, PTSTORE_S_TIMEOUT);
  }
}

// Joins the sums of the items that span several CTAs: blockIdx.x the CTA an item begins in, y eight of its rows, a warp a row, z some of its
// elements: 128 of a few rows, whose sums are many, all of many rows.
template <int L, bool F16, bool WIDE>
__global__ void __launch_bounds__(256) latent_join_kernel(const Latent la) {
  using Shape = LatentShape<L, WIDE>;
  constexpr int NQ = Shape::ROWS, DIMS = Shape::DIMS, PAIR = Shape::PAIR, PF = Shape::PART, E = WIDE ? DIMS / 128 : 1;     // float4's of a lane
  const Attend& a = la.a;
  const LatentPart part = reinterpret_cast<const LatentPart*>(a.work)[blockIdx.x];
  if (part.parts == 0) return;
  const u32 cta = blockIdx.x / PAIR, half = blockIdx.x % PAIR;
  const int lane = threadIdx.x & 31, row = blockIdx.y * 8 + (threadIdx.x >> 5);
  const float* const sums = reinterpret_cast<const float*>(a.work + LA_PARTS_AT) + (i64)half * PF;
  auto at = [&](int p) { return sums + (i64)(2 * (cta + p) + (p == 0 ? 1 : 0)) * PAIR * PF; };
  // lane p holds m and l of part p (of 32 at a time); the first 32 are on their way while the request is looked up
  const bool one = lane < part.parts;
  const float m0 = one ? at(lane)[NQ * DIMS + row] : -INFINITY, l0 = one ? at(lane)[NQ * DIMS + NQ + row] : 0.0f;
  const Req q = request(a, part.r);
  const int row_base = (int)(part.rt * NQ), rows = min(NQ, q.fresh * a.group - row_base);
  if (row >= rows) return;
  float top = m0, sum = 0.0f;
  for (int p = lane + 32; p < part.parts; p += 32) top = fmaxf(top, at(p)[NQ * DIMS + row]);
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) top = fmaxf(top, __shfl_xor_sync(FULL, top, o));
  const int mine = (int)blockIdx.z * 128 + lane * 4;
  float4 acc[E] = {};
  for (int p0 = 0; p0 < part.parts; p0 += 32) {
    float f = 0.0f;
    if (p0 + lane < part.parts) {
      const float m = p0 == 0 ? m0 : at(p0 + lane)[NQ * DIMS + row];
      f = m == -INFINITY ? 1.0f : exp2_fast(m - top);                        // nothing seen: sums of zero (or NaN)
      sum += (p0 == 0 ? l0 : at(p0 + lane)[NQ * DIMS + NQ + row]) * f;
    }
    const int n = min(32, part.parts - p0);
#pragma unroll 8
    for (int p = 0; p < n; ++p) {
      const float w = __shfl_sync(FULL, f, p);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float4 v = *reinterpret_cast<const float4*>(at(p0 + p) + row * DIMS + e * 128 + mine);
        acc[e].x += v.x * w;
        acc[e].y += v.y * w;
        acc[e].z += v.z * w;
        acc[e].w += v.w * w;
      }
    }
  }
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) sum += __shfl_xor_sync(FULL, sum, o);
  const int fr = (row_base + row) / a.group, hq = (row_base + row) % a.group;
  const float f = row_factor(a, part.r, (i64)q.pos0 + fr, sum);
#pragma unroll
  for (int e = 0; e < E; ++e)
    *reinterpret_cast<uint2*>(a.out + 2 * ((i64)(q.row0 + fr) * a.o_token + (i64)hq * a.o_head + (int)half * DIMS + e * 128 + mine)) =
        make_uint2(pack2<F16>(acc[e].x * f, acc[e].y * f), pack2<F16>(acc[e].z * f, acc[e].w * f));
  if (a.lse && half == 0 && blockIdx.z == 0 && lane == 0) a.lse[(i64)(q.row0 + fr) * a.heads + hq] = lse_of(top, sum);
}

}  // namespace ptk
