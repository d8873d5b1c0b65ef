// ptstore_attend_weights: how much attention the rows of q gave to every cached token, for eviction.
//
//     w[j] = sum over rows i that see token j of exp2(scale2 k_j.q_i - lse2_i)
//
// A CTA takes some consecutive tiles of one request's and kv head's tokens and goes over the rows in chunks: S^T = K Q^T with the TOKENS as the tensor instruction's rows, so that
// a thread has one token's scores against all rows of a chunk and adds them up by itself; no exchange, no atomics, one order of addition.  The softmax's sum is known (lse), so K is
// read once and nothing else of the cache.  The next tile is on its way while one is computed with, and Q stays where it is while its rows fit.  A decode step is bound by
// reading K, a window of many rows by its exponentials.
//
// Weights keep what 32 bits can hold of them.  The tensor cores cut off what does not fit the running sum, so every product of rows comes out small by a part of itself that grows with
// the length of the sums.  So scores are summed up in several accumulators, and the scale makes up for what is cut off on average (cut_off below).  Scale and lse, times log2 e, are kept
// as two numbers each (a rounding of an exponent of 20 is 2^-20 of the weight).
//
// B200: a decode step of 64 requests (2064 .. 6256 tokens, 32 / 8 heads x 128, bf16) 109 us, 5.3 TB/s; 32 last tokens of 16 prompts over 4160 tokens, 4-bit, 70 us: 9 exponentials a
// clock and SM of 16, since a tile's unpacking, products and sums follow one another and three CTAs an SM cover for that only in part; latent rows (8 x 16.4k, 64 heads) 59 us, 2.6 TB/s:
// one CTA an SM, whose tile of 72 KB is loaded while one is computed with.  Measured and dropped: chunks of 32 rows, one's products computed while the one before is added up (83 and
// 65 us).
#include <cfloat>
#include <type_traits>

#include "attend_prompt.cuh"
#include "launch.cuh"

using namespace ptk;

namespace {

struct Weights {
  Attend a;
  const float* lse;
  float* out;
  i64 o_request, o_head;
  double scale2;             // scale * log2 e (and the 4-bit values' factors, powers of two)
  float scale_hi, scale_lo;  // as two numbers
  int width, tiles, each;    // CTAs of a request and kv head, and tiles of a CTA
  bool add;
};

constexpr int AW_THREADS = 256;             // two warpgroups, which share the rows of a chunk
constexpr float LOG2E_REST = (float)(1.4426950408889634074 - (double)LOG2E);          // what 32 bits leave of log2 e
template <bool PACKED, int D, int NR>
struct WeightsShape {
  // tokens of a tile: all 128 rows of the instruction, but for latent rows, of which two tiles have to fit an SM beside Q
  static constexpr int KT = D > 128 ? 64 : 128;
  // instructions of 16 elements that share an accumulator, accumulators
  static constexpr int PER = NR == 16 ? 2 : D > 128 ? 6 : 4, SUMS = (D / 16 + PER - 1) / PER;
  static constexpr int HELD = NR == 16 ? 16 : D > 128 ? 64 : 128;                                                   // rows of Q that stay in shared memory
  static constexpr int STAGES = PACKED ? 1 : 2, K_BYTES = KT * D * 2, Q_BYTES = HELD * D * 2;
  static constexpr int SMEM = STAGES * K_BYTES + Q_BYTES + 1024;
  static constexpr int OTHER = 3 << 10, CTAS = 230000 / (SMEM + OTHER) < 1 ? 1 : 230000 / (SMEM + OTHER);      // static shared memory; CTAs of an SM
  static constexpr int NEED = SUMS * NR, COLS = NEED <= 32 ? 32 : NEED <= 64 ? 64 : NEED <= 128 ? 128 : NEED <= 256 ? 256 : 512;
};

__host__ __device__ constexpr u32 aw_desc(bool fp16, int M, int N) {       // both operands with a row's elements contiguous
  return (1u << 4) | ((fp16 ? 0u : 1u) << 7) | ((fp16 ? 0u : 1u) << 10) | ((u32)(N >> 3) << 17) | ((u32)(M >> 4) << 24);
}

template <bool PACKED, bool F16, bool QFP16, int D, int NR>
__global__ void __launch_bounds__(AW_THREADS, D > 128 ? 1 : 3) weights_kernel(const Weights wa) {
  using Shape = WeightsShape<PACKED, D, NR>;
  constexpr int KT = Shape::KT, CPR = D / 8, SUMS = Shape::SUMS, HELD = Shape::HELD, KB = Shape::K_BYTES;
  constexpr bool SCALED = PACKED && !QFP16;                   // bf16 rows over the 4-bit cache have a factor each
  extern __shared__ unsigned char smem_raw[];
  unsigned char* const smem = smem_raw + ((1024 - (smem_addr(smem_raw) & 1023)) & 1023);
  unsigned char* const smem_q = smem + Shape::STAGES * KB;
  __shared__ __align__(8) u64 s_bar;
  __shared__ u32 s_tmem;
  __shared__ int s_gave_up, s_min;
  __shared__ i64 s_row[2][KT];                                // where a tile's rows lie, -1: not there
  __shared__ __align__(16) float s_lse[2 * HELD];             // of two rows at a time: - lse log2 e, what 32 bits leave of it
  __shared__ __align__(8) float s_factor[SCALED ? HELD : 2];
  __shared__ float s_part[KT];
  __shared__ __align__(8) int s_see[HELD];
  const Attend& a = wa.a;
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(FULL, tid >> 5, 0);
  const u32 rh = blockIdx.x / (u32)wa.tiles, h = rh % a.cache.heads;
  const int r = (int)(rh / a.cache.heads), first = (int)(blockIdx.x % (u32)wa.tiles) * wa.each * KT;
  const Req rq = request(a, r);
  const int rows = rq.fresh * a.group;
  // tokens that count: those some row sees
  const i64 top = (i64)rq.pos0 + rq.fresh;
  const int n = rows <= 0 || top <= 0 ? 0 : (int)min((i64)min(rq.keys, wa.width), top);
  const int end = min(first + wa.each * KT, wa.width);
  float* const out = wa.out + r * wa.o_request + h * wa.o_head;
  if (!wa.add)                                                // tokens that nobody sees
    for (int j = max(first, n) + tid; j < end; j += AW_THREADS) out[j] = 0.0f;
  if (first >= n) return;
  const int tiles = (min(n, end) - first + KT - 1) / KT;
  // the thread's token; the scores of 64 tokens lie in the first 16 lanes of each warp
  const int group = warp >> 2, mine = KT == 128 ? tid & 127 : (warp & 3) * 16 + (lane & 15);
  const bool writes = KT == 128 || lane < 16;

  const u32 B = a.cache.block_tokens;
  const int* const table = a.tables + (i64)r * a.max_blocks;
  bool bounds = false;
  // where token `tid` of tile t lies
  auto look_up = [&](int t) { return tid < KT && t < tiles && first + t * KT + tid < n ? table[(u32)(first + t * KT + tid) / B] : -1; };
  auto place = [&](int t, int id) -> i64 {
    const int k = first + t * KT + tid;
    if (tid >= KT || t >= tiles || k >= n) return -1;
    if ((u32)id >= a.cache.num_blocks) { bounds = true; return -1; }
    const u32 in = (u32)k % B;
    return (i64)((u64)(u32)id * a.cache.block_stride) +
           (PACKED ? (i64)((u64)h * (B / TILE) + in / TILE) * tile_bytes(D) : (i64)((u64)in * a.cache.heads + h) * (D * 2));
  };
  // 16-bit: the tile's rows into a stage, zeros for those that are not there
  auto issue = [&](int t) {
    const u32 dst = smem_addr(smem) + (t & 1) * KB;
#pragma unroll 8
    for (int i = tid; i < KT * CPR; i += AW_THREADS) {
      const int row = i / CPR, c = i % CPR;
      const i64 at = s_row[t & 1][row];
      cp_async16_or_zero(dst + (c >> 3) * (KT * 128) + row * 128 + (((c & 7) ^ (row & 7)) * 16), a.cache.base + (at < 0 ? 0 : at) + c * 16, at >= 0);
    }
  };
  // 4-bit: half a token a thread, codes and scales on their way in registers, then unpacked to fp16 (element order 0 4 1 5 2 6 3 7 inside eight, as the unpacking yields them; Q is stored likewise)
  constexpr int HALF = PACKED ? D / 64 : 1;    // chunks of 32 elements of a thread: two threads have a token
  uint4 code[HALF];
  u32 scales;
  const Magic mg = magic();
  auto fetch = [&](int t) {
    if (!PACKED) return;
    const i64 at = s_row[t & 1][mine];
    const int m = (u32)(first + t * KT + mine) % TILE;
    const unsigned char* const src = a.cache.base + (at < 0 ? 0 : at);
#pragma unroll
    for (int c = 0; c < HALF; ++c) code[c] = at >= 0 ? *reinterpret_cast<const uint4*>(src + code_place(D, m, group * HALF + c) * 16) : make_uint4(0, 0, 0, 0);
    scales = 0;
    if (at >= 0) {
      const unsigned char* const sc = src + scale_at(D, false, m, 0);
      scales = D == 128 ? *reinterpret_cast<const u32*>(sc + 4 * group) : (u32)*reinterpret_cast<const unsigned short*>(sc + 2 * group);
    }
  };
  auto unpack = [&]() {
    if (!PACKED) return;
#pragma unroll
    for (int c = 0; c < HALF; ++c) {
      const u32 two = (scales >> (16 * c)) & 0xFFFFu;          // two scale groups of a chunk of 32 elements
      const Deq d0 = deq_of(e4m3x2_to_half2((two & 0xFFu) * 0x101u)), d1 = deq_of(e4m3x2_to_half2((two >> 8) * 0x101u));
      const u32 w[4] = {code[c].x, code[c].y, code[c].z, code[c].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        u32 o[4];
        deq4(w[i], w[i] >> 8, i < 2 ? d0 : d1, mg, o);
        *reinterpret_cast<uint4*>(smem + operand_at(mine, 4 * (group * HALF + c) + i)) = make_uint4(o[0], o[1], o[2], o[3]);
      }
    }
  };
  if (tid < KT) s_row[0][tid] = place(0, look_up(0));
  int id = look_up(1);
  if (tid == 0) {
    bar_init(&s_bar, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    s_gave_up = 0;
    s_min = 0x7FFFFFFF;
  }
  if (warp == 0) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&s_tmem)), "n"(Shape::COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const u32 tmem = s_tmem, lanes = tmem + ((u32)(32 * (warp & 3)) << 16);
  if (PACKED) fetch(0);
  else {
    issue(0);
    cp_commit();
  }
  // ---- rows row0 .. row0 + HELD - 1 of Q, in the products' type.  Rows that fill a chunk up are the last row once more, with a logarithm so large that they give nothing: rows of zeros
  // would make NaN of a key that holds an infinity, whatever the real rows' scores are.
  auto load_q = [&](int row0) {
    constexpr int TPR = D > 128 ? 32 : CPR, EACH = (CPR + TPR - 1) / TPR, PASS = AW_THREADS / TPR;
    const int m = min(HELD, rows - row0), padded = (m + NR - 1) / NR * NR;
#pragma unroll 2
    for (int p = 0; p < padded; p += PASS) {
      const int t = p + tid / TPR, c0 = tid % TPR;
      const int flat = row0 + min(t, m - 1), fr = flat / a.group, hq = (int)h * a.group + flat % a.group;
      const bool live = t < m;
      u32 x[EACH][4];
#pragma unroll
      for (int e = 0; e < EACH; ++e) {
        const int c = c0 + e * TPR;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (c < CPR) v = *reinterpret_cast<const uint4*>(a.q + 2 * ((i64)(rq.row0 + fr) * a.q_token + (i64)hq * a.q_head + c * 8));
        x[e][0] = v.x; x[e][1] = v.y; x[e][2] = v.z; x[e][3] = v.w;
      }
      float factor = 1.0f;
      if (SCALED) {
        // bf16 rows as fp16, scaled by a power of two so that the largest element is in [1, 2): elements below 2^-14 of it lose at most 2^-25 of it
        float amax = 0.0f;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float2 f = unpack2<false>(x[0][k]);
          amax = fmaxf(amax, fmaxf(fabsf(f.x), fabsf(f.y)));
        }
#pragma unroll
        for (int o = 1; o < TPR; o <<= 1) amax = fmaxf(amax, __shfl_xor_sync(FULL, amax, o));
        int e = amax > 0.0f ? (int)(__float_as_uint(amax) >> 23) - 127 : 0;
        e = e < -126 ? -126 : e > 126 ? 126 : e;
        factor = __uint_as_float((u32)(127 + e) << 23);
        const float down = __uint_as_float((u32)(127 - e) << 23);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float2 f = unpack2<false>(x[0][k]);
          x[0][k] = pack2<true>(f.x * down, f.y * down);
        }
      }
      if (PACKED) {          // element order 0 4 1 5 2 6 3 7
        const u32 y[4] = {__byte_perm(x[0][0], x[0][2], 0x5410), __byte_perm(x[0][0], x[0][2], 0x7632), __byte_perm(x[0][1], x[0][3], 0x5410),
                          __byte_perm(x[0][1], x[0][3], 0x7632)};
#pragma unroll
        for (int k = 0; k < 4; ++k) x[0][k] = y[k];
      }
      if (t >= padded) continue;
#pragma unroll
      for (int e = 0; e < EACH; ++e) {
        const int c = c0 + e * TPR;
        if (c < CPR) *reinterpret_cast<uint4*>(smem_q + (c >> 3) * (HELD * 128) + t * 128 + (((c & 7) ^ (t & 7)) * 16)) = make_uint4(x[e][0], x[e][1], x[e][2], x[e][3]);
      }
      if (c0 == 0) {
        const float l = wa.lse[(i64)(rq.row0 + fr) * a.heads + hq];
        const float hi = live ? l * LOG2E : FLT_MAX;
        // l log2 e as two numbers; an infinity is one
        s_lse[(t & ~1) * 2 + (t & 1)] = -hi;
        s_lse[(t & ~1) * 2 + 2 + (t & 1)] = live && fabsf(hi) < INFINITY ? -(fmaf(l, LOG2E, -hi) + l * LOG2E_REST) : 0.0f;
        if (SCALED) s_factor[t] = factor;
        const i64 see = (i64)rq.pos0 + fr + 1;
        const int s = l == -INFINITY || see < 0 ? 0 : see > n ? n : (int)see;          // a row that saw nothing gave nothing
        s_see[t] = s;
        atomicMin(&s_min, s);
      }
    }
  };
  load_q(0);
  const u32 smem_k = smem_addr(smem), smem_qa = smem_addr(smem_q);
  constexpr u32 QK = aw_desc(F16, KT, NR);
  const bool fits = rows <= HELD;
  bool timeout = false;
  u32 phase = 0;
  const u64 hi2 = pair(wa.scale_hi, wa.scale_hi), lo2 = pair(wa.scale_lo, wa.scale_lo);
  for (int t = 0; t < tiles; ++t) {
    if (PACKED) unpack();
    // the next tile: its rows' places, then its bytes
    const i64 next = place(t + 1, id);
    id = look_up(t + 2);
    if (tid < KT) s_row[(t + 1) & 1][tid] = next;
    if (!PACKED) {
      __syncthreads();
      if (t + 1 < tiles) issue(t + 1);
      cp_commit();
      cp_wait<1>();
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    const int key0 = first + t * KT, key = key0 + mine;
    const bool have = s_row[t & 1][mine] >= 0;
    u64 sum[2] = {0, 0};
    for (int row0 = 0; row0 < rows; row0 += HELD) {
      if (!fits && (t > 0 || row0 > 0)) {
        __syncthreads();                      // (all scores against the rows that lie there have been read)
        if (tid == 0) s_min = 0x7FFFFFFF;
        __syncthreads();
        load_q(row0);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      }
      const int chunks = (min(HELD, rows - row0) + NR - 1) / NR;
      for (int c = 0; c < chunks; ++c) {
        // operands are there, and the scores before these have been read by all
        tc_fence_before();
        __syncthreads();
        tc_fence_after();
        if (warp == 0 && elected()) {
          const u64 ka = operand_desc(smem_k + (PACKED ? 0 : t & 1) * KB, 0), qb = operand_desc(smem_qa + c * NR * 128, 0);
#pragma unroll
          for (int k = 0; k < D / 16; ++k)
            mma_ss(tmem + k / Shape::PER * NR, ka + (u64)(((k >> 2) * (KT * 128) + (k & 3) * 32) >> 4), qb + (u64)(((k >> 2) * (HELD * 128) + (k & 3) * 32) >> 4), QK, k % Shape::PER > 0);
          tc_commit(&s_bar);
        }
        __syncwarp();
        if (PACKED && row0 == 0 && c == 0 && t + 1 < tiles) fetch(t + 1);
        const bool whole = s_min >= key0 + KT;                // every row sees every token of the tile
        if (!bar_wait(&s_bar, phase, a.polls, &s_gave_up)) {  // what is in flight is awaited with the built-in limit
          timeout = true;
          bar_drain(&s_bar, phase);
        }
        phase ^= 1;
        tc_fence_after();
        // this warpgroup's rows of the chunk, W at a time
        constexpr int W = NR == 16 ? 8 : 16;
#pragma unroll
        for (int i0 = 0; i0 < NR / 2; i0 += W) {
          const int at0 = group * (NR / 2) + i0;
          u64 s[W / 2];
#pragma unroll
          for (int x0 = 0; x0 < SUMS; x0 += 2) {
            float v[2][W];
#pragma unroll
            for (int x = 0; x < 2; ++x)
              if (x0 + x < SUMS) tc_ld(v[x], lanes + (x0 + x) * NR + at0);
            tc_wait_ld();
#pragma unroll
            for (int x = 0; x < 2; ++x)
              if (x0 + x < SUMS) {
                tc_loaded(v[x]);
#pragma unroll
                for (int i = 0; i < W; i += 2) {
                  const u64 two = pair(v[x][i], v[x][i + 1]);
                  s[i / 2] = x0 + x == 0 ? two : add_pair(s[i / 2], two);
                }
              }
          }
          auto give = [&](auto all) {
#pragma unroll
            for (int i = 0; i < W; i += 2) {
              const int row = c * NR + at0 + i;
              const float4 l = *reinterpret_cast<const float4*>(&s_lse[2 * row]);
              u64 y = s[i / 2];
              if (SCALED) y = mul_pair(y, *reinterpret_cast<const u64*>(&s_factor[row]));
              const u64 e = add_pair(fma_pair(y, hi2, pair(l.x, l.y)), fma_pair(y, lo2, pair(l.z, l.w)));
              float p0 = exp2_fast(lo_of(e)), p1 = exp2_fast(hi_of(e));
              if (!decltype(all)::value) {
                const int2 see = *reinterpret_cast<const int2*>(&s_see[row]);
                p0 = key < see.x ? p0 : 0.0f;
                p1 = key < see.y ? p1 : 0.0f;
              }
              sum[(i >> 1) & 1] = add_pair(sum[(i >> 1) & 1], pair(p0, p1));
            }
          };
          if (whole) give(std::true_type{});
          else give(std::false_type{});
        }
      }
    }
    const u64 both = add_pair(sum[0], sum[1]);
    const float w = lo_of(both) + hi_of(both);
    if (group == 1 && writes) s_part[mine] = w;
    tc_fence_before();
    __syncthreads();                          // before the next tile takes the place of this one
    tc_fence_after();
    if (group == 0 && writes && key < n) {
      const float all = w + s_part[mine];
      if (!have) {
        if (!wa.add) out[key] = 0.0f;
      } else out[key] = wa.add ? out[key] + all : all;
    }
  }
  cp_wait<0>();
  if ((bounds || timeout) && a.status) atomicOr(a.status, (bounds ? PTSTORE_S_BOUNDS : 0) | (timeout ? PTSTORE_S_TIMEOUT : 0));
  if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(Shape::COLS) : "memory");
}

// What the tensor cores cut off a sum of n instructions on average, as a part of it.  They cut after every instruction instead of rounding: half a step, which is 2^-24 / (2 ln 2) of a
// number whose mantissa is as likely as numbers' are; and the running sum after j of n terms that are alike goes with j / n of the last one.  So 2^-24 / (2 ln 2) (1 + 2 + .. + n) / n.
// Measured against 64 bits with scores of 64 .. 576 elements, n = 1 / 2 / 4 / 6, in 2^-24: 0.7 .. 1.0 / 1.1 .. 1.7 / 1.6 .. 1.8 / 2.3 .. 2.6 (here 0.72 / 1.08 / 1.80 / 2.52).  A score
// whose sum is exact is off by as much instead, at most 2.6 2^-24 of it (the header says so).  Products with 4-bit keys have fewer bits, of which less
// is cut off: half of it (measured 0.3 .. 0.4 / 0.4 .. 0.7 / 0.5 .. 1.1).
// Weights against 64 bits (norm, in 1e-6) with it / without / 32-bit products of a library: a decode step 0.6 / 0.9 / 0.8, latent rows 1.4 / 2.3 / 1.3.  The loss can also be measured, by
// sums that go forth and back again (what is left of them over): 0.6 and 1.4, but three times the products, 132 and 84 us in place of 116 and 61.
constexpr double cut_off(bool packed, int n) { return 0x1p-24 / 1.3862943611198906 * (n + 1) / (packed ? 4 : 2); }

template <bool PACKED, bool F16, bool QFP16, int D, int NR>
int launch(Weights wa, const Gpu& gpu, cudaStream_t s) {
  using Shape = WeightsShape<PACKED, D, NR>;
  const double scale2 = wa.scale2 * (1.0 + cut_off(PACKED, Shape::PER));
  // towards zero, and the rest of the same sign and never zero: an infinite score then stays the infinity that it is times the scale
  wa.scale_hi = (float)scale2;
  if (fabs((double)wa.scale_hi) > fabs(scale2)) wa.scale_hi = nextafterf(wa.scale_hi, 0.0f);
  wa.scale_lo = (float)(scale2 - wa.scale_hi);
  if (wa.scale_lo == 0.0f && scale2 != 0.0) wa.scale_lo = copysignf(0x1p-126f, wa.scale_hi);
  static std::atomic<u64> devices{0};
  auto* kernel = weights_kernel<PACKED, F16, QFP16, D, NR>;
  const int rc = allow_smem(kernel, Shape::SMEM, devices, gpu.dev);
  if (rc) return rc;
  // Tiles of a CTA: one round of CTAs where that takes at most 16 each, else rounds of 8 (what a CTA does once is then a small part of its time)
  const i64 tiles = (wa.width + Shape::KT - 1) / Shape::KT, rows = (i64)wa.a.R * wa.a.cache.heads, parts = (i64)gpu.sms * Shape::CTAS / rows;
  wa.each = parts > 0 && (tiles + parts - 1) / parts <= 16 ? (int)((tiles + parts - 1) / parts) : 8;
  wa.tiles = (int)((tiles + wa.each - 1) / wa.each);
  const u64 grid = (u64)wa.tiles * wa.a.R * wa.a.cache.heads;
  if (grid > 0x7FFFFFFF) return PTSTORE_E_LIMIT;
  kernel<<<(unsigned)grid, AW_THREADS, Shape::SMEM, s>>>(wa);
  return cudaGetLastError() == cudaSuccess ? PTSTORE_OK : PTSTORE_E_CUDA;
}
template <bool PACKED, bool F16, bool QFP16, int D>
int launch_rows(const Weights& wa, i64 rows, const Gpu& gpu, cudaStream_t s) {
  return rows <= 16 ? launch<PACKED, F16, QFP16, D, 16>(wa, gpu, s) : launch<PACKED, F16, QFP16, D, 64>(wa, gpu, s);
}

}  // namespace

extern "C" int ptstore_attend_weights(const ptstore_attend_weights_t* p, const ptstore_kv_cache_t* cache, uint32_t* status, ptstore_stream_t stream) {
  if (!p || p->struct_size != sizeof(ptstore_attend_weights_t)) return PTSTORE_E_INVAL;
  const int rc = check_any_cache(cache);
  if (rc) return rc;
  if (p->requests < 0 || p->max_blocks < 1 || p->tokens < 0 || p->num_heads < 1 || p->width < 0 || p->accumulate > 1) return PTSTORE_E_INVAL;
  if (p->num_heads % (int)cache->num_kv_heads || p->num_heads > 65535) return PTSTORE_E_INVAL;
  if (p->dtype != PTSTORE_KV_BF16 && p->dtype != PTSTORE_KV_FP16) return PTSTORE_E_INVAL;
  const bool packed = cache->format == PTSTORE_KV_PACKED, half = p->dtype == PTSTORE_KV_FP16;
  if (!packed && (cache->format & 3u) != p->dtype) return PTSTORE_E_INVAL;                   // (the latent formats' lowest bits are the 16-bit types)
  const double scale2 = (double)p->scale * 1.4426950408889634074 * (packed ? (double)cache->k_scale * DEQ_FACTOR : 1.0);
  if (!(fabs(scale2) < 3.4028e38)) return PTSTORE_E_INVAL;             // finite in 32 bits
  if (p->requests == 0 || p->width == 0 || (p->accumulate && p->tokens == 0)) return PTSTORE_OK;
  if (!p->token_offsets || !p->lengths || !p->block_tables || !p->weights) return PTSTORE_E_INVAL;
  if (p->tokens > 0 && (!p->q || !p->lse || !rows_aligned(p->q, p->tokens, p->q_token_stride, p->num_heads, p->q_head_stride))) return PTSTORE_E_INVAL;
  if ((u64)p->max_blocks * cache->block_tokens > 1u << 30 || p->width > 1 << 30) return PTSTORE_E_LIMIT;
  if (p->requests > 1 << 20 || (i64)p->tokens * p->num_heads > 0x7FFFFFFF) return PTSTORE_E_LIMIT;
  Weights wa;
  Attend& a = wa.a;
  a = Attend{};
  a.cache = cache_of(cache);
  a.q = static_cast<const unsigned char*>(p->q);
  a.q_token = p->q_token_stride; a.q_head = p->q_head_stride;
  a.offsets = p->token_offsets; a.lengths = p->lengths; a.tables = p->block_tables;
  a.R = p->requests; a.max_blocks = p->max_blocks; a.heads = p->num_heads; a.tokens = p->tokens;
  a.group = p->num_heads / (int)cache->num_kv_heads;
  a.polls = p->wait_polls ? p->wait_polls : POLLS;
  a.status = status;
  wa.lse = p->lse;
  wa.out = p->weights;
  wa.o_request = p->weights_request_stride; wa.o_head = p->weights_head_stride;
  wa.width = p->width;
  wa.add = p->accumulate != 0;
  wa.scale2 = scale2;
  Gpu gpu;
  (void)cudaGetLastError();
  const int rs = current_gpu(&gpu);
  if (rs) return rs;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const i64 rows = (i64)(p->max_new < p->tokens ? p->max_new : p->tokens) * a.group;
  switch (cache->head_dim) {
    case 64:
      if (packed) return half ? launch_rows<true, true, true, 64>(wa, rows, gpu, s) : launch_rows<true, true, false, 64>(wa, rows, gpu, s);
      return half ? launch_rows<false, true, true, 64>(wa, rows, gpu, s) : launch_rows<false, false, false, 64>(wa, rows, gpu, s);
    case 128:
      if (packed) return half ? launch_rows<true, true, true, 128>(wa, rows, gpu, s) : launch_rows<true, true, false, 128>(wa, rows, gpu, s);
      return half ? launch_rows<false, true, true, 128>(wa, rows, gpu, s) : launch_rows<false, false, false, 128>(wa, rows, gpu, s);
    case 320: return half ? launch_rows<false, true, true, 320>(wa, rows, gpu, s) : launch_rows<false, false, false, 320>(wa, rows, gpu, s);
    default: return half ? launch_rows<false, true, true, 576>(wa, rows, gpu, s) : launch_rows<false, false, false, 576>(wa, rows, gpu, s);
  }
}
