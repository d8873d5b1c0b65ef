// ptstore_select_tokens, ptstore_kv_compact: which tokens of a cache to keep by the attention they were given, and moving them together.
#include "kvcache.cuh"
#include "launch.cuh"

using namespace ptk;

namespace {

// ---- which tokens ---------------------------------------------------------------------------------------------------------------------
// One CTA per request and head.  The smallest weight to keep is found by its bits, 11 + 11 + 10 from the top: a histogram of the candidates that agree so far in shared memory, a scan
// of its counts from the largest down.  Then one pass in index order writes the kept tokens: every warp has consecutive ones, so that a scan of the warps' counts is all they exchange.
// Rows of up to 8192 tokens (4096 where there are more rows than SMs) are read once and stay in registers.  Bound by latency, 4 x 3 barriers and the reads: one request's 8 rows of 6256 weights
// 9 us with 1024 threads, 11 with 512; 512 ragged rows 31 and 24.
constexpr int SEL_HELD = 8;                  // tokens a thread holds
constexpr int SEL_BINS = 2048;

struct SelectArgs {
  const float* weights;
  i64 w_request, w_head;
  const int* lengths;
  int heads, width, budget, first, recent;
  int *kept, *lengths_out;
  float* out;
  i64 o_request, o_head;
  u32* status;
};

// order of weights as unsigned numbers: a NaN last, zeros of both signs alike
__device__ __forceinline__ u32 order_of(float w) {
  if (w != w) return FULL;
  const u32 b = __float_as_uint(w + 0.0f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

template <int SEL_THREADS>
__global__ void __launch_bounds__(SEL_THREADS, 1024 / SEL_THREADS) select_kernel(SelectArgs a) {
  constexpr int SEL_WARPS = SEL_THREADS / 32, SEL_SEGMENT = SEL_THREADS * SEL_HELD, SEL_EACH = SEL_BINS / SEL_THREADS;
  __shared__ u32 s_bins[3][SEL_BINS];
  __shared__ u32 s_scan[2][SEL_WARPS];
  __shared__ u32 s_digit, s_want;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int r = blockIdx.x / a.heads, h = blockIdx.x % a.heads;
  const int raw = a.lengths[r], len = raw < 0 ? 0 : raw > a.width ? a.width : raw;
  const float* const w = a.weights + r * a.w_request + h * a.w_head;
  float* const out = a.out + r * a.o_request + h * a.o_head;
  int* const kept = a.kept + (i64)blockIdx.x * a.budget;
  const int n = min(len, a.budget);
  if (h == 0 && tid == 0) {
    a.lengths_out[r] = n;
    if (raw != len && a.status) atomicOr(a.status, PTSTORE_S_BOUNDS);
  }
  const int lo = len > a.budget ? a.first : 0, hi = len > a.budget ? len - a.recent : 0;      // candidates
  u32 want = (u32)(a.budget - a.first - a.recent);                                           // of them
  // thread's tokens of a segment: consecutive ones a warp, consecutive lanes
  float held[SEL_HELD];
  const int mine = warp * (32 * SEL_HELD) + lane;
  auto load = [&](int segment) {
#pragma unroll
    for (int i = 0; i < SEL_HELD; ++i) {
      const int j = segment + mine + i * 32;
      held[i] = j < len ? w[j] : 0.0f;
    }
  };
  load(0);
  const bool once = len <= SEL_SEGMENT;
  // ---- the smallest order that is kept, and how many candidates of just that order
  u32 bound = 0;
  if (hi > lo && want > 0) {
    for (int i = tid; i < 3 * SEL_BINS; i += SEL_THREADS) (&s_bins[0][0])[i] = 0;
    __syncthreads();
#pragma unroll 1
    for (int round = 0; round < 3; ++round) {
      const int shift = round == 0 ? 21 : round == 1 ? 10 : 0, above = round == 0 ? 0 : round == 1 ? 21 : 10;
      const u32 mask = round == 2 ? 1023u : 2047u;
      for (int segment = 0; segment < len; segment += SEL_SEGMENT) {
        if (!once) load(segment);
#pragma unroll
        for (int i = 0; i < SEL_HELD; ++i) {
          const int j = segment + mine + i * 32;
          const u32 o = order_of(held[i]);
          if (j >= lo && j < hi && (round == 0 || o >> above == bound >> above)) atomicAdd(&s_bins[round][(o >> shift) & mask], 1u);
        }
      }
      __syncthreads();
      // each thread has some consecutive digits, thread 0 the largest: counts from the largest digit down to its first
      u32 c[SEL_EACH], x = 0;
#pragma unroll
      for (int i = 0; i < SEL_EACH; ++i) {
        c[i] = s_bins[round][SEL_BINS - 1 - SEL_EACH * tid - i];
        x += c[i];
      }
      const u32 all = x;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const u32 y = __shfl_up_sync(FULL, x, o);
        if (lane >= o) x += y;
      }
      if (lane == 31) s_scan[0][warp] = x;
      __syncthreads();
      u32 before = __reduce_add_sync(FULL, lane < warp ? s_scan[0][lane] : 0u) + x - all;
      if (before < want && want <= before + all) {            // exactly one thread
        int i = 0;
        for (; before + c[0] < want; ++i) {
          before += c[0];
#pragma unroll
          for (int k = 1; k < SEL_EACH; ++k) c[k - 1] = c[k];
        }
        s_digit = (u32)(SEL_BINS - 1 - SEL_EACH * tid - i);
        s_want = want - before;
      }
      __syncthreads();
      bound |= s_digit << shift;
      want = s_want;
    }
  } else want = 0;
  // ---- one pass in index order: kept tokens and their weights to the front.  A segment is read whole before it is written, and a token never moves back, so weights may be their
  // own output.
  const bool inner_too = a.budget > a.first + a.recent;
  u32 done = 0, equal_done = 0;
  for (int segment = 0; segment < len; segment += SEL_SEGMENT) {
    if (!once) load(segment);
    u32 sure[SEL_HELD], eq[SEL_HELD], sures = 0, eqs = 0;     // of 32 consecutive tokens each
#pragma unroll
    for (int i = 0; i < SEL_HELD; ++i) {
      const int j = segment + mine + i * 32;
      const u32 o = order_of(held[i]);
      const bool inner = j >= lo && j < hi;
      eq[i] = __ballot_sync(FULL, inner && o == bound && want > 0);
      sure[i] = __ballot_sync(FULL, j < len && (!inner || (o > bound && inner_too)));
      sures += __popc(sure[i]);
      eqs += __popc(eq[i]);
    }
    if (lane == 0) {
      s_scan[0][warp] = sures;
      s_scan[1][warp] = eqs;
    }
    __syncthreads();
    // equal ones are taken in index order while there is room: their rank says whether
    const u32 all_sure = lane < SEL_WARPS ? s_scan[0][lane] : 0, all_eq = lane < SEL_WARPS ? s_scan[1][lane] : 0;
    u32 rank = equal_done + __reduce_add_sync(FULL, lane < warp ? all_eq : 0u);
    u32 at = done + __reduce_add_sync(FULL, lane < warp ? all_sure : 0u) + min(rank, want) - min(equal_done, want);
    const u32 below = (1u << lane) - 1u;
#pragma unroll
    for (int i = 0; i < SEL_HELD; ++i) {
      const u32 my_rank = rank + __popc(eq[i] & below);
      const bool keep = ((sure[i] >> lane) & 1) || (((eq[i] >> lane) & 1) && my_rank < want);
      const u32 to = at + __popc(sure[i] & below) + min(my_rank, want) - min(rank, want);
      if (keep) {
        kept[to] = segment + mine + i * 32;
        out[to] = held[i];
      }
      const u32 after = rank + __popc(eq[i]);
      at += __popc(sure[i]) + min(after, want) - min(rank, want);
      rank = after;
    }
    const u32 eq_after = equal_done + __reduce_add_sync(FULL, all_eq);
    done += __reduce_add_sync(FULL, all_sure) + min(eq_after, want) - min(equal_done, want);
    equal_done = eq_after;
    __syncthreads();                          // (everything of this segment has been read before the next one's counts, or the zeros, are written)
  }
  for (int i = n + tid; i < a.budget; i += SEL_THREADS) kept[i] = -1;
  for (int i = n + tid; i < a.width; i += SEL_THREADS) out[i] = 0.0f;
}

// ---- moving them ----------------------------------------------------------------------------------------------------------------------
// Pure data movement, bound by HBM.  A thread moves 16 bytes (of a 4-bit cache: 32 codes and their two scales) of CP_EACH tokens, which are all read before the first is written.
// Into other blocks, chunks of tokens are spread over CTAs.  In place one CTA takes a slice of a request's and head's rows chunk by chunk: a token never moves back, so what a
// chunk's writes cover has been read by that chunk or the ones before it.
// 64 requests cut to 2048 tokens of 8 heads x 128, K and V (1.04 GB): 166 us, 6.2 TB/s, with 8 tokens a thread and 4 CTAs an SM; 4 tokens 168 (6 CTAs) to 199 (4), 2 tokens 194 (8), 16 tokens
// 202 (3).
constexpr int CP_THREADS = 256, CP_EACH = 8;

struct CompactArgs {
  Cache cache;
  const int *kept, *lengths, *from, *to;
  int from_blocks, to_blocks, width, slices, steps;          // slices of a row; CTAs that share a row's chunks (1 in place)
  u32* status;
};

template <bool PACKED, int D, int PIECES /*16-byte pieces of a slice*/>
__global__ void __launch_bounds__(CP_THREADS, 4) compact_kernel(CompactArgs a) {
  constexpr int TOKENS = CP_THREADS / PIECES, CHUNK = TOKENS * CP_EACH;
  const u32 B = a.cache.block_tokens;
  const bool is_v = blockIdx.z != 0;
  // heads of the same tokens side by side: they write neighbouring rows
  const int r = blockIdx.y, x = blockIdx.x / a.slices, h = x % a.cache.heads, slice = blockIdx.x % a.slices, step = x / a.cache.heads;
  const int n = min(a.lengths[r], a.width);
  const int* const kept = a.kept + ((i64)r * a.cache.heads + h) * a.width;
  const int* const from = a.from + (i64)r * a.from_blocks;
  const int* const to = a.to + (i64)r * a.to_blocks;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, piece = lane % PIECES;
  constexpr int AT_ONCE = 32 / PIECES, PER = (AT_ONCE * CP_EACH + 31) / 32;        // tokens a warp moves at once, tokens a lane looks up
  bool bounds = false;
  for (int base = step * CHUNK; base < n; base += a.steps * CHUNK) {
    // Where a warp's tokens lie and go: a lane each, since the divisions by the block's size cost more than the bytes (by every thread for itself: 150 instructions a 16 bytes)
    unsigned long long from_at[PER], to_at[PER];
    u32 rows[PER];                           // 4-bit: the token's row in its tile, there and here
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      const int q = e * 32 + lane, i = base + q / AT_ONCE * TOKENS + warp * AT_ONCE + q % AT_ONCE;
      from_at[e] = to_at[e] = 0;
      rows[e] = 0;
      if (q >= AT_ONCE * CP_EACH || i >= n) continue;
      const int j = kept[i];
      const u32 ib = (u32)i / B, jb = (u32)j / B;
      const int db = ib < (u32)a.to_blocks ? to[ib] : -1, sb = j >= 0 && jb < (u32)a.from_blocks ? from[jb] : -1;
      if ((u32)sb >= a.cache.num_blocks || (u32)db >= a.cache.num_blocks) { bounds = true; continue; }
      if (a.from == a.to && i == j) continue;
      const u32 ir = (u32)i - ib * B, jr = (u32)j - jb * B;
      rows[e] = jr % TILE | ir % TILE << 8;
      from_at[e] = reinterpret_cast<unsigned long long>(PACKED ? tile_ptr(a.cache, is_v, sb, h, jr, D) : row_ptr(a.cache, is_v, sb, h, jr, D));
      to_at[e] = reinterpret_cast<unsigned long long>(PACKED ? tile_ptr(a.cache, is_v, db, h, ir, D) : row_ptr(a.cache, is_v, db, h, ir, D));
    }
    uint4 v[CP_EACH];
    u32 scale[CP_EACH];
#pragma unroll
    for (int k = 0; k < CP_EACH; ++k) {
      const int e = k * AT_ONCE / 32, who = k * AT_ONCE % 32 + lane / PIECES;
      const unsigned char* const src = reinterpret_cast<const unsigned char*>(__shfl_sync(FULL, from_at[e], who));
      const u32 m = PACKED ? __shfl_sync(FULL, rows[e], who) & 255u : 0;
      if (!src) continue;
      if (PACKED) {
        v[k] = *reinterpret_cast<const uint4*>(src + code_place(D, m, piece) * 16);
        scale[k] = src[scale_at(D, is_v, m, 2 * piece)] | (u32)src[scale_at(D, is_v, m, 2 * piece + 1)] << 8;
      } else v[k] = *reinterpret_cast<const uint4*>(src + slice * (PIECES * 16) + piece * 16);
    }
    if (a.steps == 1) __syncthreads();
#pragma unroll
    for (int k = 0; k < CP_EACH; ++k) {
      const int e = k * AT_ONCE / 32, who = k * AT_ONCE % 32 + lane / PIECES;
      unsigned char* const dst = reinterpret_cast<unsigned char*>(__shfl_sync(FULL, to_at[e], who));
      const u32 m = PACKED ? __shfl_sync(FULL, rows[e], who) >> 8 : 0;
      if (!dst) continue;
      if (PACKED) {
        *reinterpret_cast<uint4*>(dst + code_place(D, m, piece) * 16) = v[k];
        dst[scale_at(D, is_v, m, 2 * piece)] = (unsigned char)scale[k];
        dst[scale_at(D, is_v, m, 2 * piece + 1)] = (unsigned char)(scale[k] >> 8);
      } else *reinterpret_cast<uint4*>(dst + slice * (PIECES * 16) + piece * 16) = v[k];
    }
  }
  if (bounds && a.status) atomicOr(a.status, PTSTORE_S_BOUNDS);
}

template <bool PACKED, int D, int PIECES>
int launch_compact(CompactArgs a, int R, bool in_place, bool latent, cudaStream_t s) {
  constexpr int CHUNK = CP_THREADS / PIECES * CP_EACH;
  a.slices = PACKED ? 1 : D / 8 / PIECES;
  a.steps = in_place ? 1 : (a.width + CHUNK - 1) / CHUNK;
  const u64 x = (u64)a.slices * a.steps * a.cache.heads;
  if (x > 0x7FFFFFFFull) return PTSTORE_E_LIMIT;
  constexpr int most = 65535;                // requests of a launch: the grid's second axis has 16 bits
  for (int r = 0; r < R; r += most) {
    CompactArgs b = a;
    const int m = R - r < most ? R - r : most;
    b.kept += (i64)r * a.cache.heads * a.width;
    b.lengths += r;
    b.from += (i64)r * a.from_blocks;
    b.to += (i64)r * a.to_blocks;
    compact_kernel<PACKED, D, PIECES><<<dim3((unsigned)x, (unsigned)m, latent ? 1 : 2), CP_THREADS, 0, s>>>(b);
    if (cudaGetLastError() != cudaSuccess) return PTSTORE_E_CUDA;
  }
  return PTSTORE_OK;
}

}  // namespace

extern "C" int ptstore_select_tokens(const float* weights, int64_t weights_request_stride, int64_t weights_head_stride, const int32_t* lengths, int32_t R, int32_t heads,
                                     int32_t width, int32_t budget, int32_t first, int32_t recent, int32_t* kept, int32_t* lengths_out, float* weights_out,
                                     int64_t out_request_stride, int64_t out_head_stride, uint32_t* status, ptstore_stream_t stream) {
  if (R < 0 || heads < 1 || width < 1 || budget < 1 || budget > width || first < 0 || recent < 0 || first > budget || recent > budget - first) return PTSTORE_E_INVAL;
  if (R == 0) return PTSTORE_OK;
  if (!weights || !lengths || !kept || !lengths_out || !weights_out || lengths == lengths_out) return PTSTORE_E_INVAL;
  if (weights == weights_out && ((R > 1 && weights_request_stride != out_request_stride) || (heads > 1 && weights_head_stride != out_head_stride))) return PTSTORE_E_INVAL;
  if (width > 1 << 30 || (i64)R * heads > 0x7FFFFFFF) return PTSTORE_E_LIMIT;
  const SelectArgs a = {weights, weights_request_stride, weights_head_stride, lengths, heads, width, budget, first, recent, kept, lengths_out, weights_out,
                        out_request_stride, out_head_stride, status};
  (void)cudaGetLastError();
  Gpu gpu;
  const int rs = current_gpu(&gpu);
  if (rs) return rs;
  const i64 rows = (i64)R * heads;
  if (rows > gpu.sms) select_kernel<512><<<(unsigned)rows, 512, 0, static_cast<cudaStream_t>(stream)>>>(a);
  else select_kernel<1024><<<(unsigned)rows, 1024, 0, static_cast<cudaStream_t>(stream)>>>(a);
  return cudaGetLastError() == cudaSuccess ? PTSTORE_OK : PTSTORE_E_CUDA;
}

extern "C" int ptstore_kv_compact(const ptstore_kv_cache_t* cache, const int32_t* kept, const int32_t* lengths, int32_t R, int32_t width, const int32_t* from_tables,
                                  int32_t from_max_blocks, const int32_t* to_tables, int32_t to_max_blocks, uint32_t* status, ptstore_stream_t stream) {
  const int rc = check_any_cache(cache);
  if (rc) return rc;
  if (R < 0 || width < 0 || from_max_blocks < 1 || to_max_blocks < 1) return PTSTORE_E_INVAL;
  if (R == 0 || width == 0) return PTSTORE_OK;
  if (!kept || !lengths || !from_tables || !to_tables) return PTSTORE_E_INVAL;
  if (from_tables == to_tables && from_max_blocks != to_max_blocks) return PTSTORE_E_INVAL;
  if (width > 1 << 30 || R > 1 << 20) return PTSTORE_E_LIMIT;
  const CompactArgs a = {cache_of(cache), kept, lengths, from_tables, to_tables, from_max_blocks, to_max_blocks, width, 1, 1, status};
  const bool in_place = from_tables == to_tables, latent = is_latent(cache->format);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  (void)cudaGetLastError();
  if (cache->format == PTSTORE_KV_PACKED)
    return cache->head_dim == 64 ? launch_compact<true, 64, 2>(a, R, in_place, latent, s) : launch_compact<true, 128, 4>(a, R, in_place, latent, s);
  // slices of 128 bytes, or whole rows of 256, whatever the 16 bits mean
  switch (cache->head_dim) {
    case 64: return launch_compact<false, 64, 8>(a, R, in_place, latent, s);
    case 128: return launch_compact<false, 128, 16>(a, R, in_place, latent, s);
    case 320: return launch_compact<false, 320, 8>(a, R, in_place, latent, s);
    default: return launch_compact<false, 576, 8>(a, R, in_place, latent, s);
  }
}
