// ptstore_attend_weights: how much attention the rows of q gave to every cached token, for eviction.
//
//     w[j] = sum over rows i that see token j of exp2(scale2 k_j.q_i - lse2_i)
//
// A CTA takes a tile of one request's and kv head's tokens and goes over the rows in chunks: S^T = K Q^T with the TOKENS as the tensor instruction's rows, so that a thread has
// one token's scores against all rows of a chunk and adds them up by itself; no exchange, no atomics, one order of addition.  The softmax's sum is known (lse), so K is read
// once and nothing else of the cache.  A decode step is bound by reading K (many small CTAs an SM, whose loads overlap the others' work), a window of many rows by its
// exponentials.
#include "attend_prompt.cuh"
#include "launch.cuh"

using namespace ptk;

namespace {

struct Weights {
  Attend a;
  const float* lse;
  float* out;
  i64 o_request, o_head;
  int width, tiles;          // tiles of a request
  bool add;
};

constexpr int AW_THREADS = 128;
// tokens of a tile: all 128 rows of the instruction, but for latent rows, of which twice as many CTAs fit an SM with 64
template <int D>
__host__ __device__ constexpr int aw_keys() { return D > 128 ? 64 : 128; }
// rows of a chunk: few for a decode step, more for many rows (as many as leave two CTAs an SM)
template <int D>
__host__ __device__ constexpr int aw_many() { return D > 128 ? 32 : 64; }
template <int D, int NR>
constexpr int aw_smem() { return (aw_keys<D>() + NR) * D * 2 + 1024; }

__host__ __device__ constexpr u32 aw_desc(bool fp16, int M, int N) {       // both operands with a row's elements contiguous
  return (1u << 4) | ((fp16 ? 0u : 1u) << 7) | ((fp16 ? 0u : 1u) << 10) | ((u32)(N >> 3) << 17) | ((u32)(M >> 4) << 24);
}

template <bool PACKED, bool F16, bool QFP16, int D, int NR>
__global__ void __launch_bounds__(AW_THREADS) weights_kernel(const Weights wa) {
  constexpr int KT = aw_keys<D>(), CPR = D / 8, COLS = NR < 32 ? 32 : NR;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* const smem = smem_raw + ((1024 - (smem_addr(smem_raw) & 1023)) & 1023);
  unsigned char* const smem_q = smem + KT * D * 2;
  __shared__ __align__(8) u64 s_bar;
  __shared__ u32 s_tmem;
  __shared__ int s_gave_up;
  __shared__ i64 s_row[KT];
  __shared__ float s_scale[NR], s_lse[NR];
  __shared__ int s_see[NR];
  const Attend& a = wa.a;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const u32 rh = blockIdx.x / (u32)wa.tiles, h = rh % a.cache.heads;
  const int r = (int)(rh / a.cache.heads), key0 = (int)(blockIdx.x % (u32)wa.tiles) * KT;
  const Req rq = request(a, r);
  const int n = min(rq.keys, wa.width), rows = rq.fresh * a.group;
  // thread t < KT has token key0 + t; the scores of 64 tokens lie in the first 16 lanes of each warp
  const int mine = KT == 128 ? tid : warp * 16 + (lane & 15);
  const bool writes = KT == 128 || lane < 16;
  const int key = key0 + mine;
  float* const out = wa.out + r * wa.o_request + h * wa.o_head;
  if (key0 >= n || rows <= 0 || (i64)rq.pos0 + rq.fresh - 1 < key0) {        // nothing there, or nothing seen
    if (!wa.add && writes && key < wa.width) out[key] = 0.0f;
    return;
  }
  // ---- K into shared memory
  const u32 B = a.cache.block_tokens;
  bool have = false;
  if (tid < KT) {
    const int k = key0 + tid;
    i64 at = -1;
    if (k < n) {
      const u32 id = (u32)a.tables[(i64)r * a.max_blocks + (u32)k / B], in = (u32)k % B;
      if (id < a.cache.num_blocks) {
        at = (i64)((u64)id * a.cache.block_stride);
        at += PACKED ? (i64)((u64)h * (B / TILE) + in / TILE) * tile_bytes(D) : (i64)((u64)in * a.cache.heads + h) * (D * 2);
        have = true;
      } else if (a.status) atomicOr(a.status, PTSTORE_S_BOUNDS);
    }
    s_row[tid] = at;
    if (PACKED) {            // one token a thread: codes to fp16, element order 0 4 1 5 2 6 3 7 inside eight, as the unpacking yields them (and Q is stored)
      const Magic mg = magic();
      const int m = (u32)k % TILE;
      const unsigned char* const src = a.cache.base + (have ? at : 0);
      __align__(8) unsigned char sc[D / 16] = {};
      uint4 code[D / 32];
#pragma unroll
      for (int c = 0; c < D / 32; ++c) code[c] = have ? *reinterpret_cast<const uint4*>(src + code_place(D, m, c) * 16) : make_uint4(0, 0, 0, 0);
      if (have) {
        if (D == 128) *reinterpret_cast<uint2*>(sc) = *reinterpret_cast<const uint2*>(src + scale_at(D, false, m, 0));
        else *reinterpret_cast<u32*>(sc) = *reinterpret_cast<const u32*>(src + scale_at(D, false, m, 0));
      }
#pragma unroll
      for (int c = 0; c < D / 32; ++c) {
        const Deq d0 = deq_of(e4m3x2_to_half2(sc[2 * c] * 0x101u)), d1 = deq_of(e4m3x2_to_half2(sc[2 * c + 1] * 0x101u));
        const u32 w[4] = {code[c].x, code[c].y, code[c].z, code[c].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          u32 o[4];
          deq4(w[i], w[i] >> 8, i < 2 ? d0 : d1, mg, o);
          *reinterpret_cast<uint4*>(smem + operand_at(tid, 4 * c + i)) = make_uint4(o[0], o[1], o[2], o[3]);
        }
      }
    }
  }
  if (tid == 0) {
    bar_init(&s_bar, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    s_gave_up = 0;
  }
  if (warp == 0) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&s_tmem)), "n"(COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const u32 tmem = s_tmem;
  if (!PACKED) {
#pragma unroll 8
    for (int i = tid; i < KT * CPR; i += AW_THREADS) {
      const int t = i / CPR, c = i % CPR;
      const i64 at = s_row[t];
      cp_async16_or_zero(smem_addr(smem) + (c >> 3) * (KT * 128) + t * 128 + (((c & 7) ^ (t & 7)) * 16), a.cache.base + (at < 0 ? 0 : at) + c * 16, at >= 0);
    }
    cp_commit();
  }
  have = s_row[mine] >= 0;
  // ---- rows, a chunk at a time
  const u32 smem_k = smem_addr(smem), smem_qa = smem_addr(smem_q);
  float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  bool timeout = false;
  u32 phase = 0;
  for (int row0 = 0; row0 < rows; row0 += NR) {
    const int m = min(NR, rows - row0);
    // threads of a row hold all of it, for its largest element
    constexpr int TPR = D > 128 ? 32 : CPR, EACH = (CPR + TPR - 1) / TPR, PASS = AW_THREADS / TPR;
    for (int p = 0; p < NR; p += PASS) {
      const int t = p + tid / TPR, c0 = tid % TPR;
      const int flat = row0 + t, fr = flat / a.group, hq = (int)h * a.group + flat % a.group;
      const bool live = t < m;
      u32 x[EACH][4];
#pragma unroll
      for (int e = 0; e < EACH; ++e) {
        const int c = c0 + e * TPR;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (live && c < CPR) v = *reinterpret_cast<const uint4*>(a.q + 2 * ((i64)(rq.row0 + fr) * a.q_token + (i64)hq * a.q_head + c * 8));
        x[e][0] = v.x; x[e][1] = v.y; x[e][2] = v.z; x[e][3] = v.w;
      }
      float factor = 1.0f;
      if (PACKED && !QFP16) {
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
      if (t < NR) {
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
          const int c = c0 + e * TPR;
          if (c < CPR) *reinterpret_cast<uint4*>(smem_q + (c >> 3) * (NR * 128) + t * 128 + (((c & 7) ^ (t & 7)) * 16)) = make_uint4(x[e][0], x[e][1], x[e][2], x[e][3]);
        }
        if (c0 == 0) {
          const float l = live ? wa.lse[(i64)(rq.row0 + fr) * a.heads + hq] : -INFINITY;
          const i64 see = (i64)rq.pos0 + fr + 1;
          s_scale[t] = a.scale2 * factor;
          s_lse[t] = l * LOG2E;
          s_see[t] = l == -INFINITY || see < 0 ? 0 : see > n ? n : (int)see;          // a row that saw nothing gave nothing
        }
      }
    }
    if (!PACKED) cp_wait<0>();
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 0 && elected()) {
      constexpr u32 QK = aw_desc(F16, KT, NR);
      const u64 ka = operand_desc(smem_k, 0), qb = operand_desc(smem_qa, 0);
#pragma unroll
      for (int k = 0; k < D / 16; ++k)
        mma_ss(tmem, ka + (u64)(((k >> 2) * (KT * 128) + (k & 3) * 32) >> 4), qb + (u64)(((k >> 2) * (NR * 128) + (k & 3) * 32) >> 4), QK, k > 0);
      tc_commit(&s_bar);
    }
    __syncwarp();
    const bool ok = bar_wait(&s_bar, phase, a.polls, &s_gave_up);
    if (__syncthreads_or(!ok)) {              // what is in flight is awaited with the built-in limit
      bar_drain(&s_bar, phase);
      timeout = true;
      break;
    }
    phase ^= 1;
    tc_fence_after();
    const u32 base = tmem + ((u32)(32 * warp) << 16);
#pragma unroll
    for (int c = 0; c < COLS; c += 32) {
      float v[32];
      tc_ld32(v, base + c);
      tc_wait_ld();
      tc_loaded(v);
#pragma unroll
      for (int i = 0; i < (NR < 32 ? NR : 32); ++i) {
        const float p = exp2_fast(__fmul_rn(v[i], s_scale[c + i]) - s_lse[c + i]);
        sum[i & 3] += key < s_see[c + i] ? p : 0.0f;
      }
    }
    tc_fence_before();
    __syncthreads();                          // before the next chunk takes Q's place
  }
  if (writes && key < wa.width && !timeout) {
    const float w = (sum[0] + sum[1]) + (sum[2] + sum[3]);
    if (key >= n || !have) {
      if (!wa.add) out[key] = 0.0f;
    } else out[key] = wa.add ? out[key] + w : w;
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 0) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(COLS) : "memory");
    if (lane == 0 && timeout && a.status) atomicOr(a.status, PTSTORE_S_TIMEOUT);
  }
}

template <bool PACKED, bool F16, bool QFP16, int D, int NR>
int launch(Weights wa, const Gpu& gpu, cudaStream_t s) {
  static std::atomic<u64> devices{0};
  auto* kernel = weights_kernel<PACKED, F16, QFP16, D, NR>;
  const int rc = allow_smem(kernel, aw_smem<D, NR>(), devices, gpu.dev);
  if (rc) return rc;
  wa.tiles = (wa.width + aw_keys<D>() - 1) / aw_keys<D>();
  const u64 grid = (u64)wa.tiles * wa.a.R * wa.a.cache.heads;
  if (grid > 0x7FFFFFFF) return PTSTORE_E_LIMIT;
  kernel<<<(unsigned)grid, AW_THREADS, aw_smem<D, NR>(), s>>>(wa);
  return cudaGetLastError() == cudaSuccess ? PTSTORE_OK : PTSTORE_E_CUDA;
}
template <bool PACKED, bool F16, bool QFP16, int D>
int launch_rows(const Weights& wa, i64 rows, const Gpu& gpu, cudaStream_t s) {
  return rows <= 16 ? launch<PACKED, F16, QFP16, D, 16>(wa, gpu, s) : launch<PACKED, F16, QFP16, D, aw_many<D>()>(wa, gpu, s);
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
  const float scale2 = p->scale * LOG2E * (packed ? cache->k_scale * DEQ_FACTOR : 1.0f);
  if (!isfinite(scale2)) return PTSTORE_E_INVAL;
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
  a.scale2 = scale2;
  a.polls = p->wait_polls ? p->wait_polls : POLLS;
  a.status = status;
  wa.lse = p->lse;
  wa.out = p->weights;
  wa.o_request = p->weights_request_stride; wa.o_head = p->weights_head_stride;
  wa.width = p->width;
  wa.add = p->accumulate != 0;
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
