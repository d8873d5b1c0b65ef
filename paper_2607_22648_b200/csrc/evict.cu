// ptstore_select_tokens, ptstore_kv_compact: which tokens of a cache to keep by the attention they were given, and moving them together.
#include "kvcache.cuh"

using namespace ptk;

namespace {

constexpr u32 FULL = 0xFFFFFFFFu;

// ---- which tokens ---------------------------------------------------------------------------------------------------------------------
// One CTA per request and head.  The smallest weight to keep is found by its bits, four at a time from the top (eight rounds over the candidates, which the
// threads hold in registers or read again from L2); then one pass in index order writes the kept tokens.  Bound by latency: rounds of counting, each with
// one exchange among the warps.
constexpr int SEL_THREADS = 512, SEL_WARPS = SEL_THREADS / 32;
constexpr int SEL_HELD = 16;                 // weights a thread holds: requests of up to 8192 tokens are read once

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

__global__ void __launch_bounds__(SEL_THREADS) select_kernel(SelectArgs a) {
  __shared__ u32 s_count[2][SEL_WARPS][16];
  __shared__ u32 s_scan[2][SEL_WARPS];
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
  int want = a.budget - a.first - a.recent;                                                  // of them
  // ---- the smallest order that is kept, and how many candidates of just that order
  u32 bound = 0;
  if (hi > lo && want > 0) {
    u32 held[SEL_HELD];
    const bool fits = hi - lo <= SEL_HELD * SEL_THREADS;
    if (fits) {
#pragma unroll
      for (int i = 0; i < SEL_HELD; ++i) {
        const int j = lo + i * SEL_THREADS + tid;
        held[i] = j < hi ? order_of(w[j]) : 0;
      }
    }
    for (int round = 0; round < 8; ++round) {
      const int shift = 28 - 4 * round;
      // candidates of every next digit, among those that agree with the bound so far: 16 counts of 16 bits in 8 registers, at most 2^16 - 1 a thread and round of counting
      u32 total[16];
#pragma unroll
      for (int d = 0; d < 16; ++d) total[d] = 0;
      auto count = [&](u32 o, bool in) {
        const bool match = in && (round == 0 || (o >> (shift + 4)) == (bound >> (shift + 4)));
        const u32 digit = (o >> shift) & 15u;
#pragma unroll
        for (int d = 0; d < 16; ++d) total[d] += match && digit == (u32)d;
      };
      if (fits) {
#pragma unroll
        for (int i = 0; i < SEL_HELD; ++i)
          if (lo + i * SEL_THREADS < hi) count(held[i], lo + i * SEL_THREADS + tid < hi);
      } else {
        for (int j = lo + tid; j < hi; j += SEL_THREADS) count(order_of(w[j]), true);
      }
#pragma unroll
      for (int d = 0; d < 16; ++d) {
        const u32 t = __reduce_add_sync(FULL, total[d]);
        if (lane == d) s_count[round & 1][warp][d] = t;
      }
      __syncthreads();
      u32 mine = 0;                          // lane d: all candidates of digit d
      if (lane < 16)
        for (int x = 0; x < SEL_WARPS; ++x) mine += s_count[round & 1][x][lane];
      // candidates above digit d
      u32 above = lane < 16 ? mine : 0;
#pragma unroll
      for (int o = 1; o < 16; o <<= 1) {
        const u32 y = __shfl_down_sync(FULL, above, o);
        if (lane + o < 16) above += y;
      }
      const u32 before = above - mine;
      const u32 hit = __ballot_sync(FULL, lane < 16 && before < (u32)want && above >= (u32)want);
      const int d = hit ? __ffs(hit) - 1 : 0;
      want -= (int)__shfl_sync(FULL, before, d);
      bound |= (u32)d << shift;
    }
  } else want = 0;
  // ---- one pass in index order: kept tokens and their weights to the front.  Tokens behind the ones that are written are read before (a chunk is read whole, then written, and
  // a token never moves back), so weights may be their own output.
  u32 done = 0, equal_done = 0;
  for (int base = 0; base < len; base += SEL_THREADS) {
    const int j = base + tid;
    const float x = j < len ? w[j] : 0.0f;
    const bool inner = j >= lo && j < hi;
    const u32 o = order_of(x);
    const bool equal = inner && o == bound && want > 0;
    const u32 eq = __ballot_sync(FULL, equal);
    const u32 sure = __ballot_sync(FULL, j < len && (!inner || (o > bound && a.budget > a.first + a.recent)));
    if (lane == 0) {
      s_scan[0][warp] = __popc(eq);
      s_scan[1][warp] = __popc(sure);
    }
    __syncthreads();
    // equal ones are taken in index order while there is room: their rank says whether
    u32 eq_before = equal_done, eq_all = 0, at = done, sure_all = 0;
    for (int x2 = 0; x2 < SEL_WARPS; ++x2) {
      const u32 e = s_scan[0][x2], s = s_scan[1][x2];
      if (x2 < warp) { eq_before += e; at += s; }
      eq_all += e;
      sure_all += s;
    }
    const u32 below = (1u << lane) - 1u, w_eq = (u32)want;
    const u32 rank = eq_before + __popc(eq & below);
    // taken equals before this thread: those of rank below `want`
    const u32 taken_before = min(rank, w_eq) - min(equal_done, w_eq);
    const bool keep = ((sure >> lane) & 1) || (equal && rank < w_eq);
    at += __popc(sure & below) + taken_before;
    if (keep) {
      kept[at] = j;
      out[at] = x;
    }
    done += sure_all + (min(equal_done + eq_all, w_eq) - min(equal_done, w_eq));
    equal_done += eq_all;
    __syncthreads();
  }
  for (int i = n + tid; i < a.budget; i += SEL_THREADS) kept[i] = -1;
  for (int i = n + tid; i < a.width; i += SEL_THREADS) out[i] = 0.0f;
}

// ---- moving them ----------------------------------------------------------------------------------------------------------------------
// Pure data movement, bound by HBM.  A thread moves 16 bytes (of a 4-bit cache: 32 codes and their two scales) of CP_EACH tokens, which are all read before the first is written.
// Into other blocks, chunks of tokens are spread over CTAs.  In place one CTA takes a slice of a request's and head's rows chunk by chunk: a token never moves back, so what a
// chunk's writes cover has been read by that chunk or the ones before it.
constexpr int CP_THREADS = 256, CP_EACH = 8;

struct CompactArgs {
  Cache cache;
  const int *kept, *lengths, *from, *to;
  int from_blocks, to_blocks, width, slices, steps;          // slices of a row; CTAs that share a row's chunks (1 in place)
  u32* status;
};

template <bool PACKED, int D, int PIECES /*16-byte pieces of a slice*/>
__global__ void __launch_bounds__(CP_THREADS) compact_kernel(CompactArgs a) {
  constexpr int TOKENS = CP_THREADS / PIECES, CHUNK = TOKENS * CP_EACH;
  const u32 B = a.cache.block_tokens;
  const bool is_v = blockIdx.z != 0;
  const int r = blockIdx.y / a.cache.heads, h = blockIdx.y % a.cache.heads;
  const int slice = blockIdx.x % a.slices, step = blockIdx.x / a.slices;
  const int n = min(a.lengths[r], a.width);
  const int* const kept = a.kept + (i64)blockIdx.y * a.width;
  const int* const from = a.from + (i64)r * a.from_blocks;
  const int* const to = a.to + (i64)r * a.to_blocks;
  const int piece = threadIdx.x % PIECES, t = threadIdx.x / PIECES;
  bool bounds = false;
  for (int base = step * CHUNK; base < n; base += a.steps * CHUNK) {
    uint4 v[CP_EACH];
    u32 scale[CP_EACH];
    unsigned char* dst[CP_EACH];
    int src_tok[CP_EACH], dst_blk[CP_EACH];
#pragma unroll
    for (int k = 0; k < CP_EACH; ++k) {
      const int i = base + k * TOKENS + t;
      src_tok[k] = i < n ? kept[i] : -2;
      dst_blk[k] = i < n && (int)((u32)i / B) < a.to_blocks ? to[(u32)i / B] : -1;
    }
#pragma unroll
    for (int k = 0; k < CP_EACH; ++k) {
      const int i = base + k * TOKENS + t, j = src_tok[k];
      dst[k] = nullptr;
      if (j == -2) continue;
      const u32 jb = (u32)j / B;
      const int sb = j >= 0 && jb < (u32)a.from_blocks ? from[jb] : -1;
      if ((u32)sb >= a.cache.num_blocks || (u32)dst_blk[k] >= a.cache.num_blocks) { bounds = true; continue; }
      if (a.from == a.to && i == j) continue;
      if (PACKED) {
        const unsigned char* tile = tile_ptr(a.cache, is_v, sb, h, (u32)j % B, D);
        const int m = (u32)j % TILE;
        v[k] = *reinterpret_cast<const uint4*>(tile + code_place(D, m, piece) * 16);
        scale[k] = tile[scale_at(D, is_v, m, 2 * piece)] | (u32)tile[scale_at(D, is_v, m, 2 * piece + 1)] << 8;
        dst[k] = tile_ptr(a.cache, is_v, dst_blk[k], h, (u32)i % B, D);
      } else {
        const int at = slice * (PIECES * 16) + piece * 16;
        v[k] = *reinterpret_cast<const uint4*>(row_ptr(a.cache, is_v, sb, h, (u32)j % B, D) + at);
        dst[k] = row_ptr(a.cache, is_v, dst_blk[k], h, (u32)i % B, D) + at;
      }
    }
    if (a.steps == 1) __syncthreads();
#pragma unroll
    for (int k = 0; k < CP_EACH; ++k) {
      if (!dst[k]) continue;
      if (PACKED) {
        const int m = (u32)(base + k * TOKENS + t) % TILE;
        *reinterpret_cast<uint4*>(dst[k] + code_place(D, m, piece) * 16) = v[k];
        dst[k][scale_at(D, is_v, m, 2 * piece)] = (unsigned char)scale[k];
        dst[k][scale_at(D, is_v, m, 2 * piece + 1)] = (unsigned char)(scale[k] >> 8);
      } else *reinterpret_cast<uint4*>(dst[k]) = v[k];
    }
  }
  if (bounds && a.status) atomicOr(a.status, PTSTORE_S_BOUNDS);
}

template <bool PACKED, int D, int PIECES>
int launch_compact(CompactArgs a, int R, bool in_place, bool latent, cudaStream_t s) {
  constexpr int CHUNK = CP_THREADS / PIECES * CP_EACH;
  a.slices = PACKED ? 1 : D / 8 / PIECES;
  a.steps = in_place ? 1 : (a.width + CHUNK - 1) / CHUNK;
  const u64 x = (u64)a.slices * a.steps, y = (u64)R * a.cache.heads;
  if (x > 0x7FFFFFFFull || y > 0xFFFFull * 0x7FFFull) return PTSTORE_E_LIMIT;
  // the grid's second axis has 16 bits: a launch takes as many requests as fit
  const int most = (int)(65535 / a.cache.heads);
  for (int r = 0; r < R; r += most) {
    CompactArgs b = a;
    const int m = R - r < most ? R - r : most;
    b.kept += (i64)r * a.cache.heads * a.width;
    b.lengths += r;
    b.from += (i64)r * a.from_blocks;
    b.to += (i64)r * a.to_blocks;
    compact_kernel<PACKED, D, PIECES><<<dim3((unsigned)x, (unsigned)(m * a.cache.heads), latent ? 1 : 2), CP_THREADS, 0, s>>>(b);
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
  select_kernel<<<(unsigned)(R * heads), SEL_THREADS, 0, static_cast<cudaStream_t>(stream)>>>(a);
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
  // slices of 128 bytes, whatever the 16 bits mean
  switch (cache->head_dim) {
    case 64: return launch_compact<false, 64, 8>(a, R, in_place, latent, s);
    case 128: return launch_compact<false, 128, 8>(a, R, in_place, latent, s);
    case 320: return launch_compact<false, 320, 8>(a, R, in_place, latent, s);
    default: return launch_compact<false, 576, 8>(a, R, in_place, latent, s);
  }
}
