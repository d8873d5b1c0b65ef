// Attention over expanded keys and values of a latent cache (128 + 64 elements a key, 128 a value, every head its own): bounded by the tensor cores.
//
// A CTA takes 256 new tokens of one (request, head), two tiles of 128 rows that alternate: while the softmax of one runs, the tensor cores work for the other.  Per step of 128
// keys and tile:
//     S = Q K^T (192 elements), P = exp2(scale2 S - m) in 16 bits over S in tensor memory (one thread per row), O += P V
// with O in tensor memory for the whole row of steps and m a running reference that moves only when a scaled score exceeds it by more than 8.
//
// Q of both tiles takes 96 KB of shared memory, a step's K and V 80: they come through a ring of eight 16 KB slots (per step three boxes of 64 elements of K, the last one the rotary
// part that all heads share, and V in two halves of 64 keys), so that a step is on its way while another is computed with.  All by tensor copies; what they bring along from behind
// the request's keys is taken out of V where it matters (a weight of zero does not hide a NaN), for which the loading warps look at the last steps' V.
//
// B200, ten passes behind a pause / passes for seconds at the power limit: 8 whole prompts (2064 .. 6256 tokens, 16 heads, bf16) 834 / 910 us, 880 / 807 TFLOP/s; 4 suffixes of 1000 .. 2048
// tokens over 6000 .. 8192 keys, 32 heads, fp16, 678 / 794 us, 997 / 851 TFLOP/s.  A step
// of both tiles takes 4000 clocks, of which the tensor cores need 2560 and shared memory 2700 (the scores' operands are read at its full rate); the rest is the chain S, 64 + 64 weights, values,
// next scores, and waits for a ring of 1.6 steps.  One arrival a warp at the barriers and one loading thread in place of 128 each: 880 to 823 us, 790 to 665 (behind pauses).  Measured and dropped: the
// three boxes of a step's K awaited together (897 us).
//
// Warps: 0-3 and 4-7 softmax of tile 0 and 1, 8-11 load, 12 issues the tensor instructions, 13-15 only complete the warpgroup that gives its registers to the softmax warps.
#pragma once
#include "attend_prompt.cuh"

namespace ptk {

constexpr int EX_ROWS = 256, EX_SLOTS = 8, EX_SLOT = 16384, EX_Q = 3 * 128 * 128, EX_STEP = 5;      // a step's slots: 3 of K, 2 of V
constexpr int EX_SMEM = 2 * EX_Q + EX_SLOTS * EX_SLOT + 1024;                                       // + alignment

struct Expanded {
  unsigned char* out;
  i64 o_token, o_head;
  const int *offsets, *key_offsets;
  int R, heads, tokens, keys;
  u32 q_head, k_head, v_head;                // what the head's number is multiplied by in the maps: 0 where all heads share a row
  float scale2;
  u32 polls;
  u32* status;
};

// rows of request r that exist, its keys, and the position of its first row among them (may be negative)
struct ExReq { int row0, fresh, key0, keys, pos0; };
__device__ __forceinline__ ExReq request(const Expanded& a, int r) {
  ExReq q;
  const int lo = a.offsets[r], end = a.offsets[r + 1], klo = a.key_offsets[r], kend = a.key_offsets[r + 1];
  q.row0 = lo < 0 ? 0 : lo > a.tokens ? a.tokens : lo;
  const int hi = end < q.row0 ? q.row0 : end > a.tokens ? a.tokens : end;
  q.fresh = hi - q.row0;
  q.key0 = klo < 0 ? 0 : klo > a.keys ? a.keys : klo;
  const int khi = kend < q.key0 ? q.key0 : kend > a.keys ? a.keys : kend;
  q.keys = khi - q.key0;
  // rows and keys behind the arrays' ends count for the positions although they are not there
  const i64 pos = (i64)kend - q.key0 - ((i64)end - q.row0);
  q.pos0 = pos > 1 << 30 ? 1 << 30 : pos < -(1 << 30) ? -(1 << 30) : (int)pos;
  return q;
}
__device__ __forceinline__ i64 expanded_tiles(const Expanded& a, int r) { return ((i64)request(a, r).fresh + EX_ROWS - 1) / EX_ROWS; }

__device__ __forceinline__ void tensor_load_3d(u32 dst, const CUtensorMap* map, int element, int head, int token, u64* bar) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst), "l"(map), "r"(element), "r"(head),
               "r"(token), "r"(smem_addr(bar)) : "memory");
}
__device__ __forceinline__ void tensor_load_2d(u32 dst, const CUtensorMap* map, int element, int token, u64* bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst), "l"(map), "r"(element), "r"(token),
               "r"(smem_addr(bar)) : "memory");
}

template <bool F16>
__global__ void __launch_bounds__(PR_THREADS, 1) expanded_kernel(const Expanded a, const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap k_map,
                                                                 const __grid_constant__ CUtensorMap r_map, const __grid_constant__ CUtensorMap v_map) {
  extern __shared__ unsigned char smem_raw[];
  unsigned char* const smem = smem_raw + ((1024 - (smem_addr(smem_raw) & 1023)) & 1023);
  __shared__ __align__(8) u64 b_q[2], b_full[EX_SLOTS], b_empty[EX_SLOTS], b_s[2], b_pa[2], b_pb[2], b_o[2], b_end, b_raw;
  __shared__ u32 s_tmem;
  __shared__ i64 s_scan[PR_THREADS / 32];
  __shared__ int s_gave_up, s_any_bad, s_r, s_tile;
  __shared__ int s_bad[3][128];              // first key whose V holds NaN, +inf, -inf in column d, among keys that some rows do not see
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(FULL, tid >> 5, 0);

  // ---- which 256 rows: heads vary fastest; a request's tiles come last to first, the ones with most keys first
  const int h = (int)(blockIdx.x % (u32)a.heads), index = (int)(blockIdx.x / (u32)a.heads);
  {
    if (tid == 0) { s_gave_up = s_any_bad = 0; s_r = -1; }
    if (tid >= 32 && tid < 36) asm volatile("prefetch.tensormap [%0];" ::"l"(tid == 32 ? &q_map : tid == 33 ? &k_map : tid == 34 ? &r_map : &v_map) : "memory");
    const int per = (a.R + PR_THREADS - 1) / PR_THREADS, rb = min(tid * per, a.R), re = min(rb + per, a.R);
    i64 mine = 0;
    for (int r = rb; r < re; ++r) mine += expanded_tiles(a, r);
    i64 x = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const i64 y = __shfl_up_sync(FULL, x, o);
      if (lane >= o) x += y;
    }
    if (lane == 31) s_scan[warp] = x;
    if (tid == 0) {
      for (int i = 0; i < 2; ++i) { bar_init(&b_q[i], 1); bar_init(&b_s[i], 1); bar_init(&b_pa[i], 4); bar_init(&b_pb[i], 4); bar_init(&b_o[i], 1); }
      for (int i = 0; i < EX_SLOTS; ++i) { bar_init(&b_full[i], 1); bar_init(&b_empty[i], 1); }
      bar_init(&b_end, 1);
      bar_init(&b_raw, 1);
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    for (int i = tid; i < 3 * 128; i += PR_THREADS) (&s_bad[0][0])[i] = 0x7FFFFFFF;
    __syncthreads();
    i64 before = x - mine;
    for (int w = 0; w < warp; ++w) before += s_scan[w];
    if (index >= before && index < before + mine) {           // at most one thread
      int r = rb;
      i64 left = index - before, n = expanded_tiles(a, r);
      for (; left >= n; n = expanded_tiles(a, ++r)) left -= n;
      s_r = r;
      s_tile = (int)(n - 1 - left);
    }
    __syncthreads();
  }
  const int r = s_r;
  if (r < 0) return;                          // a CTA beyond the last tile
  const ExReq rq = request(a, r);
  const int row_base = s_tile * EX_ROWS, rows = min(EX_ROWS, rq.fresh - row_base);
  auto keys_of = [&](int row) {               // keys a row sees
    const int k = rq.pos0 + row_base + row + 1;
    return k < 0 ? 0 : k > rq.keys ? rq.keys : k;
  };
  const int keys0 = keys_of(min(rows, 128) - 1), keys1 = rows > 128 ? keys_of(rows - 1) : 0;
  const int all_see = keys_of(0);
  const int steps[2] = {(keys0 + PR_KEYS - 1) / PR_KEYS, (keys1 + PR_KEYS - 1) / PR_KEYS};
  const int n_steps = max(steps[0], steps[1]), keys = max(keys0, keys1);
  const u32 smem_q = smem_addr(smem), smem_kv = smem_q + 2 * EX_Q;

  // tensor memory: allocated by warp 12; 12 and the softmax warps meet before they use it
  auto tmem_there = [&]() {
    tc_fence_before();
    asm volatile("bar.sync 4, 288;" ::: "memory");
    tc_fence_after();
    return *reinterpret_cast<volatile u32*>(&s_tmem);
  };

  if (warp >= 12) {
    // ======== tensor instructions
    regs_fewer<40>();
    if (warp == 12) {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(&s_tmem)) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
      const u32 tmem = tmem_there();
      constexpr u32 QK = mma_desc(F16, PR_KEYS, false), PV = mma_desc(F16, 128, true);
      bool quit = false;                      // a wait ran out: nothing is issued from there on
      auto wait = [&](u64* b, u32 parity) {
        if (!quit && !__all_sync(FULL, bar_wait(b, parity, a.polls, &s_gave_up))) quit = true;
      };
      auto slot_wait = [&](int op) { wait(&b_full[op % EX_SLOTS], (op / EX_SLOTS) & 1); };
      auto scores = [&](int w, int j) {
#pragma unroll
        for (int i = 0; i < 3; ++i) {
          const int op = EX_STEP * j + i;
          slot_wait(op);
          tc_fence_after();
          const u64 qa = operand_desc(smem_q + w * EX_Q + i * (128 * 128), 0), kb = operand_desc(smem_kv + (op % EX_SLOTS) * EX_SLOT, 0);
          if (!quit && elected()) {
#pragma unroll
            for (int k = 0; k < 4; ++k) mma_ss(tmem + w * 128, qa + (u64)((k * 32) >> 4), kb + (u64)((k * 32) >> 4), QK, i > 0 || k > 0);
          }
          __syncwarp();
        }
        if (!quit && elected()) tc_commit(&b_s[w]);
        __syncwarp();
      };
      auto values = [&](int w, int j, int half) {
        const int op = EX_STEP * j + 3 + half;
        slot_wait(op);
        tc_fence_after();
        const u64 vb = operand_desc(smem_kv + (op % EX_SLOTS) * EX_SLOT, EX_SLOT / 2);
        if (!quit && elected()) {
#pragma unroll
          for (int k = 0; k < 4; ++k)         // 16 keys: 16 rows of 128 bytes; 8 columns of P
            mma_ts(tmem + 256 + w * 128, tmem + w * 128 + (half * 4 + k) * 8, vb + (u64)((k * 16 * 128) >> 4), PV, j > 0 || half > 0 || k > 0);
        }
        __syncwarp();
      };
      auto release = [&](int op, int n) {
        if (!quit && elected())
          for (int i = 0; i < n; ++i) tc_commit(&b_empty[(op + i) % EX_SLOTS]);
        __syncwarp();
      };
      for (int w = 0; w < 2; ++w)
        if (steps[w] > 0) wait(&b_q[w], 0);
      if (n_steps > 0) {
        for (int w = 0; w < 2; ++w)
          if (steps[w] > 0) scores(w, 0);
        release(0, 3);
      }
      for (int j = 0; j < n_steps && !quit && !__any_sync(FULL, *reinterpret_cast<volatile int*>(&s_gave_up)); ++j) {
        for (int w = 0; w < 2; ++w) {
          if (j < steps[w]) {
            wait(&b_pa[w], j & 1);
            tc_fence_after();
            values(w, j, 0);
            wait(&b_pb[w], j & 1);
            tc_fence_after();
            values(w, j, 1);
            if (j + 1 == steps[w]) { if (!quit && elected()) tc_commit(&b_o[w]); __syncwarp(); }
          }
          if (w == 1) release(EX_STEP * j + 3, 2);
          if (j + 1 < steps[w]) scores(w, j + 1);
        }
        if (j + 1 < n_steps) release(EX_STEP * (j + 1), 3);
      }
      // everything issued has ended before tensor and shared memory are given back (q's loads too, where their wait ran out)
      for (int w = 0; w < 2; ++w)
        if (steps[w] > 0) bar_drain(&b_q[w], 0);
      if (elected()) tc_commit(&b_end);
      __syncwarp();
      bar_drain(&b_end, 0);
    }
    __syncwarp();
  } else if (warp >= 8) {
    // ======== K and V into the ring.  Thread 0 loads; in the last steps all 128 look at V before it counts as there.
    regs_fewer<72>();
    const int pt = tid - 256;
    const volatile int* const gave_up = &s_gave_up;
    u32 raws = 0;
    int issued = 0;
    bool quit = false;                        // a wait ran out: nothing is loaded from there on.  Thread 0 goes on to where the others wait for it.
    for (int j = 0; j < n_steps; ++j) {
      const int k0 = j * PR_KEYS;
      const bool edge = k0 + PR_KEYS > all_see;
      if (!edge && pt != 0) continue;
#pragma unroll 1
      for (int i = 0; i < EX_STEP; ++i) {
        const int op = EX_STEP * j + i;
        const u32 dst = smem_kv + (op % EX_SLOTS) * EX_SLOT;
        u64* const full = &b_full[op % EX_SLOTS];
        const bool look = edge && i >= 3;
        if (pt == 0 && !quit) {
          if (*gave_up || (op >= EX_SLOTS && !bar_wait(&b_empty[op % EX_SLOTS], ((op / EX_SLOTS) - 1) & 1, a.polls, &s_gave_up))) quit = true;
          else {
            u64* const bar = look ? &b_raw : full;
            bar_expect(bar, EX_SLOT);
            if (i < 2) tensor_load_3d(dst, &k_map, 64 * i, (int)(a.k_head * (u32)h), rq.key0 + k0, bar);
            else if (i == 2) tensor_load_2d(dst, &r_map, 0, rq.key0 + k0, bar);
            else
#pragma unroll
              for (int e = 0; e < 2; ++e) tensor_load_3d(dst + e * (EX_SLOT / 2), &v_map, 64 * e, (int)(a.v_head * (u32)h), rq.key0 + k0 + 64 * (i - 3), bar);
            issued = op + 1;
          }
        }
        if (!look) continue;
        if (any_of_128(quit)) { quit = true; break; }         // the same in all 128 threads
        if (!bar_wait(&b_raw, raws & 1, a.polls, &s_gave_up)) bar_drain(&b_raw, raws & 1);
        ++raws;
        // keys that no row of the CTA sees become zero; what is not finite in keys that only some rows see is taken out, and put into the rows that see it at the end
        constexpr u32 EX = F16 ? 0x7C00u : 0x7F80u, MANT = F16 ? 0x03FFu : 0x007Fu;
        unsigned char* const t = smem + 2 * EX_Q + (op % EX_SLOTS) * EX_SLOT;
        for (int x = pt; x < 64 * 16; x += 128) {
          const int n = x >> 4, c = x & 15, key = k0 + 64 * (i - 3) + n;
          if (key < all_see) continue;
          uint4* const p = reinterpret_cast<uint4*>(t + (c >> 3) * (EX_SLOT / 2) + n * 128 + (((c & 7) ^ (n & 7)) * 16));
          if (key >= keys) { *p = make_uint4(0, 0, 0, 0); continue; }
          const uint4 v = *p;
          u32 e[4] = {v.x, v.y, v.z, v.w};
          bool odd = false;
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const u32 sh = 16 * (k & 1), y = e[k >> 1] >> sh;
            if ((y & EX) == EX) {
              atomicMin(&s_bad[(y & MANT) ? 0 : (y & 0x8000u) ? 2 : 1][c * 8 + k], key);
              e[k >> 1] &= ~(0xFFFFu << sh);
              odd = true;
            }
          }
          if (odd) {
            *p = make_uint4(e[0], e[1], e[2], e[3]);
            s_any_bad = 1;
          }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        any_of_128(0);
        if (pt == 0) bar_arrive(full);
      }
      if (quit && edge) break;
    }
    // whatever happened, what is in flight lands before the CTA gives its memory back
    if (pt == 0)
      for (int op = max(0, issued - EX_SLOTS); op < issued; ++op) bar_drain(&b_full[op % EX_SLOTS], (op / EX_SLOTS) & 1);
    __syncwarp();
  } else {
    // ======== softmax of tile w
    regs_more<200>();
    const int w = warp >> 2, t = tid & 127, row = w * 128 + t;
    // its half of Q; rows behind the request's last bring someone's values or zeros along and are not stored.  A tile without steps loads none: nobody would wait for it, and
    // the tile's output goes through the same memory.
    if (t == 0 && steps[w] > 0) {
      bar_expect(&b_q[w], EX_Q);
#pragma unroll
      for (int e = 0; e < 3; ++e) tensor_load_3d(smem_q + w * EX_Q + e * (128 * 128), &q_map, 64 * e, (int)(a.q_head * (u32)h), rq.row0 + row_base + w * 128, &b_q[w]);
    }
    const u32 tmem = tmem_there();
    // scale2 as a positive number (its sign goes into the scores): of zero, the smallest that keeps masked scores at minus infinity
    const float scale2 = fmaxf(fabsf(a.scale2), 0x1p-126f);
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
      const int k0 = j * PR_KEYS;
      if (a.scale2 < 0.0f) {
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int i = 0; i < 32; ++i) s[c][i] = -s[c][i];
      }
      if (k0 + PR_KEYS > all_see) {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const int left = see - k0 - 32 * c;             // keys of this chunk the row sees
          const u32 mask = left >= 32 ? FULL : left <= 0 ? 0u : (1u << left) - 1u;
#pragma unroll
          for (int i = 0; i < 32; ++i) s[c][i] = (mask >> i) & 1 ? s[c][i] : -INFINITY;
        }
      }
      // Weights of keys 64 half .. + 63 from the reference, into P.  The first half starts from the reference as it stands while the maximum over all 128 keys is found in
      // between (two keys with every weight).
      float x[4] = {s[0][0], s[0][1], s[0][2], s[0][3]};
      float sum0, sum1;
      auto weights = [&](int half, bool find, u32 (&p)[32]) {
        const float ref = m == -INFINITY ? 0.0f : m;
        const u64 sc2 = pair(scale2, scale2), neg = pair(-ref, -ref);
        u64 sum[2] = {0, 0}, e[32];
        constexpr int LAG = 4;                // pairs on their way through the special function unit
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
      const bool move = top > m + 8.0f || (m == -INFINITY && top > m);
      if (__any_sync(FULL, move) || j == 0) {
        const float f = move ? exp2_fast(m - top) : 1.0f;
        if (move) { m = top; l *= f; }
        large = __any_sync(FULL, fabsf(m) > 0x1p24f && m != -INFINITY);
        if (j > 0) {
#pragma unroll 1
          for (int c = 0; c < 128; c += 32) {
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
      // Beyond 2^24 a reference's rounding is a step in the exponent or more: products are then rounded likewise before the reference is taken off.  Scores are read once more,
      // 32 keys at a time, their weights go where scores that have been read lay.
      if (large) {
        const float ref = m == -INFINITY ? 0.0f : m;
#pragma unroll 1
        for (int c = 0; c < 4; ++c) {
          float v[32];
          tc_ld32(v, ts + 32 * c);
          tc_wait_ld();
          tc_loaded(v);
          const int left = (row < rows ? keys_of(row) : 0) - j * PR_KEYS - 32 * c;
          const u32 mask = left >= 32 ? FULL : left <= 0 ? 0u : (1u << left) - 1u;
          const float sc = a.scale2 < 0.0f ? -scale2 : scale2;
          u32 q[16];
#pragma unroll
          for (int i = 0; i < 32; i += 2) {
            const float e0 = (mask >> i) & 1 ? exp2_fast(__fmul_rn(v[i], sc) - ref) : 0.0f;
            const float e1 = (mask >> (i + 1)) & 1 ? exp2_fast(__fmul_rn(v[i + 1], sc) - ref) : 0.0f;
            l += e0 + e1;
            q[i / 2] = pack2<F16>(e0, e1);
          }
          tc_st16(ts + 16 * c, q);
          if (c & 1) {
            tc_wait_st();
            tc_fence_before();
            warp_arrive(c == 1 ? &b_pa[w] : &b_pb[w]);
          }
        }
        continue;
      }
      tc_st32(ts, p);
      tc_wait_st();
      tc_fence_before();
      warp_arrive(&b_pa[w]);                  // the tensor cores start on these while the second half is computed
      weights(1, false, p);
      tc_st32(ts + 32, p);
      l += sum0 + sum1;
      tc_wait_st();
      tc_fence_before();
      warp_arrive(&b_pb[w]);
    }
    // ---- output
    if (steps[w] > 0) {
      bar_wait(&b_o[w], 0, a.polls, &s_gave_up);
      tc_fence_after();
    }
    if (!__any_sync(FULL, *reinterpret_cast<volatile int*>(&s_gave_up))) {
      // a row that sees nothing is zero, one whose scores are all minus infinity has no softmax
      const float f = l == 0.0f ? (see > 0 ? NAN : 0.0f) : 1.0f / l;
      // through shared memory (the tile's Q is not needed any more), so that the stores are whole rows
      const i64 at = row < rows ? (i64)(rq.row0 + row_base + row) * a.o_token + (i64)h * a.o_head : -1;
      unsigned char* const mine = smem + w * EX_Q;
#pragma unroll
      for (int c = 0; c < 128; c += 32) {
        float o[32];
        if (steps[w] > 0) {
          tc_ld32(o, to + c);
          tc_wait_ld();
          tc_loaded(o);
        }
#pragma unroll
        for (int i = 0; i < 32; ++i) o[i] = steps[w] > 0 ? o[i] * f : 0.0f;
        if (s_any_bad) {
          for (int i = 0; i < 32; ++i) {
            const bool nan = s_bad[0][c + i] < see, pos = s_bad[1][c + i] < see, neg = s_bad[2][c + i] < see;
            if (nan || (pos && neg)) o[i] = NAN;
            else if (pos) o[i] = o[i] + INFINITY;
            else if (neg) o[i] = o[i] - INFINITY;
          }
        }
#pragma unroll
        for (int i = 0; i < 32; i += 8)
          *reinterpret_cast<uint4*>(mine + operand_at(t, (c + i) / 8)) =
              make_uint4(pack2<F16>(o[i], o[i + 1]), pack2<F16>(o[i + 2], o[i + 3]), pack2<F16>(o[i + 4], o[i + 5]), pack2<F16>(o[i + 6], o[i + 7]));
      }
      __syncwarp();
#pragma unroll 8
      for (int i = 0; i < 16; ++i) {          // this warp's 32 rows, whole rows at a time
        const int n = i * 2 + lane / 16, c = lane % 16;
        const i64 to2 = __shfl_sync(FULL, at, n);
        if (to2 >= 0) *reinterpret_cast<uint4*>(a.out + 2 * (to2 + c * 8)) = *reinterpret_cast<const uint4*>(mine + operand_at((warp & 3) * 32 + n, c));
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

}  // namespace ptk
