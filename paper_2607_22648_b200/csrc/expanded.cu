// ptstore_expanded_attend: host side of the attention over expanded keys and values.
#include "expanded.cuh"
#include "launch.cuh"

using namespace ptk;

namespace {

// A tensor of rows [tokens][heads][dim]: boxes of 64 elements of one head and `box` tokens.  Heads that share a row (stride 0), or one head, are an axis of one.
bool rows_map(CUtensorMap* map, bool half, const void* base, i64 dim, i64 heads, i64 tokens, i64 head_stride, i64 token_stride, u32 box) {
  const bool shared = heads == 1 || head_stride == 0;
  const i64 token = tokens > 1 ? token_stride : dim;                   // (the stride of an axis of one may be any)
  const cuuint64_t dims[3] = {(cuuint64_t)dim, shared ? 1 : (cuuint64_t)heads, (cuuint64_t)(tokens > 0 ? tokens : 1)};
  const cuuint64_t strides[2] = {(cuuint64_t)(shared ? dim : head_stride) * 2, (cuuint64_t)token * 2};
  const cuuint32_t boxes[3] = {64, 1, box};
  return encode(map, half, 3, base, dims, strides, boxes);
}

template <bool F16>
int launch(const Expanded& a, const CUtensorMap (&maps)[4], const Gpu& gpu, cudaStream_t s) {
  static std::atomic<u64> devices{0};
  auto* kernel = expanded_kernel<F16>;
  if (gpu.dev >= 64 || !(devices.load(std::memory_order_acquire) >> gpu.dev & 1)) {
    // the kernel's warps trade registers, which is only sound if the block is launched with all of the SM's
    cudaFuncAttributes attr;
    if (cudaFuncGetAttributes(&attr, kernel) != cudaSuccess || attr.numRegs * PR_THREADS != 65536) { (void)cudaGetLastError(); return PTSTORE_E_CUDA; }
  }
  const int rc = allow_smem(kernel, EX_SMEM, devices, gpu.dev);
  if (rc) return rc;
  const i64 tiles = ((i64)a.tokens / EX_ROWS + a.R) * a.heads;         // at most this many, wherever the requests' rows end
  if (tiles > 0x7FFFFFFF) return PTSTORE_E_LIMIT;
  kernel<<<(unsigned)tiles, PR_THREADS, EX_SMEM, s>>>(a, maps[0], maps[1], maps[2], maps[3]);
  return cudaGetLastError() == cudaSuccess ? PTSTORE_OK : PTSTORE_E_CUDA;
}

bool strides_ok(const void* p, i64 tokens, i64 token_stride, i64 heads, i64 head_stride) {
  return rows_aligned(p, tokens, token_stride, heads, head_stride) && (tokens <= 1 || token_stride > 0) && (heads == 1 || head_stride >= 0) &&
         (tokens <= 1 || token_stride < 1ll << 38) && (heads == 1 || head_stride < 1ll << 38);
}

}  // namespace

extern "C" int ptstore_expanded_attend(const ptstore_expanded_attend_t* p, uint32_t* status, ptstore_stream_t stream) {
  if (!p || p->struct_size != sizeof(ptstore_expanded_attend_t)) return PTSTORE_E_INVAL;
  if (p->dtype != PTSTORE_KV_BF16 && p->dtype != PTSTORE_KV_FP16) return PTSTORE_E_INVAL;
  if (p->requests < 0 || p->heads < 1 || p->heads > 65535 || p->tokens < 0 || p->keys < 0 || p->max_new < 0) return PTSTORE_E_INVAL;
  const float scale2 = p->scale * LOG2E;
  if (!isfinite(scale2)) return PTSTORE_E_INVAL;
  if (p->requests == 0 || p->tokens == 0 || p->max_new == 0) return PTSTORE_OK;
  if (!p->q || !p->out || !p->token_offsets || !p->key_offsets || (p->keys > 0 && (!p->k || !p->k_rope || !p->v))) return PTSTORE_E_INVAL;
  if (!strides_ok(p->q, p->tokens, p->q_token_stride, p->heads, p->q_head_stride) || !strides_ok(p->k, p->keys, p->k_token_stride, p->heads, p->k_head_stride) ||
      !strides_ok(p->k_rope, p->keys, p->k_rope_token_stride, 1, 0) || !strides_ok(p->v, p->keys, p->v_token_stride, p->heads, p->v_head_stride) ||
      !rows_aligned(p->out, p->tokens, p->out_token_stride, p->heads, p->out_head_stride)) return PTSTORE_E_INVAL;
  if (p->requests > 1 << 20 || p->keys > 1 << 29 || p->tokens > 1 << 29) return PTSTORE_E_LIMIT;      // positions and rows are 32 bits wide, with room for a tile
  const bool half = p->dtype == PTSTORE_KV_FP16;
  Expanded a = {static_cast<unsigned char*>(p->out), p->out_token_stride, p->out_head_stride, p->token_offsets, p->key_offsets, p->requests, p->heads, p->tokens, p->keys,
                p->heads == 1 || p->q_head_stride == 0 ? 0u : 1u, p->heads == 1 || p->k_head_stride == 0 ? 0u : 1u, p->heads == 1 || p->v_head_stride == 0 ? 0u : 1u,
                scale2, p->wait_polls ? p->wait_polls : POLLS, status};
  Gpu gpu;
  (void)cudaGetLastError();
  const int rs = current_gpu(&gpu);
  if (rs) return rs;
  // (without keys nothing is loaded through their maps: they name q)
  const bool any = p->keys > 0;
  CUtensorMap maps[4];
  if (!rows_map(&maps[0], half, p->q, 192, p->heads, p->tokens, p->q_head_stride, p->q_token_stride, 128) ||
      !rows_map(&maps[1], half, any ? p->k : p->q, 128, p->heads, p->keys, p->k_head_stride, p->k_token_stride, 128) ||
      !rows_map(&maps[3], half, any ? p->v : p->q, 128, p->heads, p->keys, p->v_head_stride, p->v_token_stride, 64)) return PTSTORE_E_CUDA;
  const cuuint64_t dims[2] = {64, (cuuint64_t)(any ? p->keys : 1)}, strides[1] = {(cuuint64_t)(p->keys > 1 ? p->k_rope_token_stride : 64) * 2};
  const cuuint32_t boxes[2] = {64, 128};
  if (!encode(&maps[2], half, 2, any ? p->k_rope : p->q, dims, strides, boxes)) return PTSTORE_E_CUDA;
  return half ? launch<true>(a, maps, gpu, static_cast<cudaStream_t>(stream)) : launch<false>(a, maps, gpu, static_cast<cudaStream_t>(stream));
}
