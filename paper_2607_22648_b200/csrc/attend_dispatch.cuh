// Host side and dispatch of the attention over the paged cache, with and without the logarithms of the rows' sums (each compiled in a file of its own).
#pragma once
#include <cstddef>

#include "attend_prompt.cuh"
#include "attend_split.cuh"
#include "launch.cuh"

namespace ptk {

// rows of an item: 8 where a request's rows of one kv head fit, else 16
inline int n_tiles_of(i64 rows) { return rows <= 8 ? 1 : 2; }

template <int FMT, bool QFP16, int D, int NT, bool LSE>
int launch_split(const Attend& a, const Gpu& gpu, cudaStream_t s) {
  constexpr int SMEM = split_smem<FMT, D, NT>();
  static std::atomic<u64> devices{0};
  auto* kernel = attend_split_kernel<FMT, QFP16, D, NT, LSE>;
  const int rc = allow_smem(kernel, SMEM, devices, gpu.dev);
  if (rc) return rc;
  kernel<<<gpu.sms * split_ctas<FMT, NT>(), SplitShape<FMT, D>::THREADS, SMEM, s>>>(a);
  return cudaGetLastError() == cudaSuccess ? PTSTORE_OK : PTSTORE_E_CUDA;
}

template <int FMT, bool QFP16, bool LSE>
int launch_split_shape(const Attend& a, int D, int nt, const Gpu& gpu, cudaStream_t s) {
  if (D == 64) return nt == 1 ? launch_split<FMT, QFP16, 64, 1, LSE>(a, gpu, s) : launch_split<FMT, QFP16, 64, 2, LSE>(a, gpu, s);
  return nt == 1 ? launch_split<FMT, QFP16, 128, 1, LSE>(a, gpu, s) : launch_split<FMT, QFP16, 128, 2, LSE>(a, gpu, s);
}

// The tensor map of one layer's 16-bit cache: {head_dim, heads, tokens of a block, blocks, K or V}, boxes of 64 elements of one head and up to 128
// tokens of one block.  Returns the tokens of a box, 0 where the block size (or the strides) allows none.
inline u32 make_tensor_map(const Attend& a, bool half, int D, CUtensorMap* map) {
  const u32 B = a.cache.block_tokens;
  if (B % 8 || (PR_KEYS % B && B % PR_KEYS)) return 0;
  const u32 box = B < PR_KEYS ? B : PR_KEYS;
  const cuuint64_t dims[5] = {(cuuint64_t)D, a.cache.heads, B, a.cache.num_blocks, 2};
  const cuuint64_t strides[4] = {(cuuint64_t)D * 2, (cuuint64_t)a.cache.heads * D * 2, a.cache.block_stride, a.cache.kv_stride};
  const cuuint32_t boxes[5] = {64, 1, box, 1, 1};
  return encode(map, half, 5, a.cache.base, dims, strides, boxes) ? box : 0;
}
// The tensor map of q: boxes of 128 rows in the order of a row tile (tokens, then the heads of a group), where the group divides 128 and the
// softmax scale is positive (its sign goes into q).
inline bool make_q_map(const Attend& a, bool half, int D, CUtensorMap* map) {
  if (128 % a.group || a.scale2 < 0.0f || a.q_token <= 0 || a.q_head <= 0) return false;
  const cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)a.heads, (cuuint64_t)a.tokens};
  const cuuint64_t strides[2] = {(cuuint64_t)a.q_head * 2, (cuuint64_t)a.q_token * 2};
  const cuuint32_t boxes[3] = {64, (cuuint32_t)a.group, 128u / a.group};
  return encode(map, half, 3, a.q, dims, strides, boxes);
}

template <int FMT, bool QFP16, int D, bool LSE>
int launch_prompt(Attend a, const Gpu& gpu, cudaStream_t s) {
  auto* kernel = attend_prompt_kernel<FMT, QFP16, D, LSE>;
  constexpr int SMEM = FMT == PTSTORE_KV_PACKED ? PromptShape<D>::SMEM_PACKED : PromptShape<D>::SMEM;
  static std::atomic<u64> devices{0};
  if (gpu.dev >= 64 || !(devices.load(std::memory_order_acquire) >> gpu.dev & 1)) {
    // the kernel's warps trade registers, which is only sound if the block is launched with all of the SM's
    cudaFuncAttributes attr;
    if (cudaFuncGetAttributes(&attr, kernel) != cudaSuccess || attr.numRegs * PR_THREADS != 65536) { (void)cudaGetLastError(); return PTSTORE_E_CUDA; }
  }
  const int rc = allow_smem(kernel, SMEM, devices, gpu.dev);
  if (rc) return rc;
  const i64 tiles = ((i64)a.tokens * a.group / PR_ROWS + a.R) * a.cache.heads;            // at most this many, wherever the requests' rows end
  if (tiles > 0x7FFFFFFF) return PTSTORE_E_LIMIT;
  a.split = tiles <= 4 * gpu.sms ? gpu.sms : 0;                        // few row tiles (by this bound): the last of them may be cut, see cut_of
  CUtensorMap map = {};
  CUtensorMap q_map = {};
  if (FMT != PTSTORE_KV_PACKED) {
    a.box_tokens = make_tensor_map(a, FMT == PTSTORE_KV_FP16, D, &map);
    a.q_box = make_q_map(a, FMT == PTSTORE_KV_FP16, D, &q_map);
  }
  kernel<<<(unsigned)(tiles + a.split), PR_THREADS, SMEM, s>>>(a, map, q_map);
  if (cudaGetLastError() != cudaSuccess) return PTSTORE_E_CUDA;
  if (a.split) {
    // At most half as many tiles are cut as there are SMs.  Whole calls with one row a warp / four rows: 4 tiles 27 / 53 us, 16 tiles 27 / 31, 32 tiles
    // 31.5 / 30, 72 tiles 43 / 35 (1024 keys each).
    const unsigned most = (unsigned)(tiles < gpu.sms / 2 ? tiles : gpu.sms / 2);
    if (most <= 32) attend_join_kernel<QFP16, D, 1, LSE><<<dim3(most, PR_ROWS / 8), 256, 0, s>>>(a);
    else attend_join_kernel<QFP16, D, 4, LSE><<<dim3(most, PR_ROWS / 32), 256, 0, s>>>(a);
    if (cudaGetLastError() != cudaSuccess) return PTSTORE_E_CUDA;
  }
  return PTSTORE_OK;
}

// Rows of one kv head from which a request's attention goes to the tensor-memory kernel: more than the split kernel's largest row tile, so that
// K and V are not read again.  4160 keys, 8 kv heads x 128, split / tensor-memory kernel: 20 rows 183 / 128 us (32 requests, 16-bit), 148 / 138 us
// (4-bit), 24.9 / 20.9 and 24.9 / 22.9 us (one request); 16 rows 95 / 128 and 80 / 138 us (32 requests).
constexpr i64 PROMPT_ROWS = 17;

// The checks and the dispatch of both entry points.
template <bool LSE>
int run_attend(const ptstore_attend_t* p, const ptstore_kv_cache_t* cache, void* workspace, uint64_t workspace_bytes, float* lse, uint32_t* status,
               ptstore_stream_t stream) {
  static_assert(offsetof(ptstore_attend_t, wait_polls) == PTSTORE_ATTEND_SIZE_1, "the first form of the struct ends here");
  if (!p || (p->struct_size != sizeof(ptstore_attend_t) && p->struct_size != PTSTORE_ATTEND_SIZE_1)) return PTSTORE_E_INVAL;
  const u32 polls = p->struct_size == PTSTORE_ATTEND_SIZE_1 ? 0 : p->wait_polls;
  const int rc = check_cache(cache);
  if (rc) return rc;
  const int D = (int)cache->head_dim;
  if (p->requests < 0 || p->max_blocks < 1 || p->tokens < 0 || p->max_new < 0 || p->num_heads < 1) return PTSTORE_E_INVAL;
  if (p->num_heads % (int)cache->num_kv_heads || p->num_heads > 65535) return PTSTORE_E_INVAL;
  if (p->dtype != PTSTORE_KV_BF16 && p->dtype != PTSTORE_KV_FP16) return PTSTORE_E_INVAL;
  if (cache->format != PTSTORE_KV_PACKED && cache->format != p->dtype) return PTSTORE_E_INVAL;
  const bool packed = cache->format == PTSTORE_KV_PACKED;
  const float scale2 = p->scale * LOG2E * (packed ? cache->k_scale * DEQ_FACTOR : 1.0f);
  if (!isfinite(scale2)) return PTSTORE_E_INVAL;             // a score of zero times it would be NaN
  if (p->requests == 0 || p->tokens == 0 || p->max_new == 0) return PTSTORE_OK;
  if (!p->q || !p->out || !p->token_offsets || !p->lengths || !p->block_tables) return PTSTORE_E_INVAL;
  if (!rows_aligned(p->q, p->tokens, p->q_token_stride, p->num_heads, p->q_head_stride) ||
      !rows_aligned(p->out, p->tokens, p->out_token_stride, p->num_heads, p->out_head_stride)) return PTSTORE_E_INVAL;
  if ((u64)p->max_blocks * cache->block_tokens > 1u << 30) return PTSTORE_E_LIMIT;                      // positions are 32 bits wide, with room for a tile
  if (p->requests > 1 << 20 || (i64)p->tokens * p->num_heads > 0x7FFFFFFF) return PTSTORE_E_LIMIT;     // row indexes of a kv head are 32 bits wide
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return PTSTORE_E_INVAL;
  if (workspace_bytes < ptstore_attend_workspace_bytes(cache->head_dim)) return PTSTORE_E_NOMEM;
  Attend a;
  a.cache = cache_of(cache);
  a.q = static_cast<const unsigned char*>(p->q);
  a.out = static_cast<unsigned char*>(p->out);
  a.q_token = p->q_token_stride; a.q_head = p->q_head_stride;
  a.o_token = p->out_token_stride; a.o_head = p->out_head_stride;
  a.offsets = p->token_offsets; a.lengths = p->lengths; a.tables = p->block_tables;
  a.R = p->requests; a.max_blocks = p->max_blocks; a.heads = p->num_heads; a.tokens = p->tokens;
  a.group = p->num_heads / (int)cache->num_kv_heads;
  a.scale2 = scale2;
  a.v_factor = packed ? cache->v_scale * DEQ_FACTOR : 1.0f;
  a.work = static_cast<unsigned char*>(workspace);
  a.polls = polls ? polls : POLLS;
  a.status = status;
  a.lse = lse;
  a.box_tokens = a.q_box = a.split = 0;
  Gpu gpu;
  (void)cudaGetLastError();
  const int rs = current_gpu(&gpu);
  if (rs) return rs;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const int most = p->max_new < p->tokens ? p->max_new : p->tokens;
  const int nt = n_tiles_of((i64)most * a.group);
  const bool half = p->dtype == PTSTORE_KV_FP16;
  if ((i64)most * a.group >= PROMPT_ROWS) {
    if (D == 64) {
      if (packed) return half ? launch_prompt<PTSTORE_KV_PACKED, true, 64, LSE>(a, gpu, s) : launch_prompt<PTSTORE_KV_PACKED, false, 64, LSE>(a, gpu, s);
      return half ? launch_prompt<PTSTORE_KV_FP16, true, 64, LSE>(a, gpu, s) : launch_prompt<PTSTORE_KV_BF16, false, 64, LSE>(a, gpu, s);
    }
    if (packed) return half ? launch_prompt<PTSTORE_KV_PACKED, true, 128, LSE>(a, gpu, s) : launch_prompt<PTSTORE_KV_PACKED, false, 128, LSE>(a, gpu, s);
    return half ? launch_prompt<PTSTORE_KV_FP16, true, 128, LSE>(a, gpu, s) : launch_prompt<PTSTORE_KV_BF16, false, 128, LSE>(a, gpu, s);
  }
  if (packed) return half ? launch_split_shape<PTSTORE_KV_PACKED, true, LSE>(a, D, nt, gpu, s) : launch_split_shape<PTSTORE_KV_PACKED, false, LSE>(a, D, nt, gpu, s);
  return half ? launch_split_shape<PTSTORE_KV_FP16, true, LSE>(a, D, nt, gpu, s) : launch_split_shape<PTSTORE_KV_BF16, false, LSE>(a, D, nt, gpu, s);
}

}  // namespace ptk
