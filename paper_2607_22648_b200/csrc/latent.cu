// ptstore_latent_write, ptstore_latent_read, ptstore_latent_attend: a cache of latent vectors and the absorbed attention over it.
#include "latent.cuh"
#include "launch.cuh"

using namespace ptk;

namespace {

constexpr int ROWS_THREADS = 256, ROWS_EACH = 4;             // 16-byte chunks of a thread, all on their way before the first is stored

struct RowsArgs {
  Cache cache;
  unsigned char *latent, *rope;
  i64 latent_stride, rope_stride;                            // bytes
  const i64* slots;
  i64 items;                                                 // chunks of all rows
  u32* status;
};

// Rows are copied, whatever their 16 bits mean.  Bound by HBM; a step's few rows by latency.
template <int CPR /*16-byte chunks of a row*/, bool WRITE>
__global__ void __launch_bounds__(ROWS_THREADS) latent_rows_kernel(RowsArgs a) {
  uint4 v[ROWS_EACH];
  uint4* to[ROWS_EACH];
  const i64 first = (i64)blockIdx.x * (ROWS_THREADS * ROWS_EACH) + threadIdx.x;
#pragma unroll
  for (int k = 0; k < ROWS_EACH; ++k) {
    const i64 item = first + k * ROWS_THREADS;
    to[k] = nullptr;
    if (item >= a.items) continue;
    const i64 row = item / CPR;
    const int c = (int)(item - row * CPR);
    const i64 slot = a.slots[row];
    if (slot == -1) continue;
    const u64 block = (u64)slot / a.cache.block_tokens;
    if (slot < 0 || block >= a.cache.num_blocks) {
      if (c == 0 && a.status) atomicOr(a.status, PTSTORE_S_BOUNDS);
      continue;
    }
    uint4* const in = reinterpret_cast<uint4*>(a.cache.base + block * a.cache.block_stride + ((u64)slot - block * a.cache.block_tokens) * (CPR * 16) + c * 16);
    uint4* const out = reinterpret_cast<uint4*>(c < CPR - 8 ? a.latent + row * a.latent_stride + c * 16 : a.rope + row * a.rope_stride + (c - (CPR - 8)) * 16);
    v[k] = WRITE ? *out : *in;
    to[k] = WRITE ? in : out;
  }
#pragma unroll
  for (int k = 0; k < ROWS_EACH; ++k)
    if (to[k]) *to[k] = v[k];
}

template <bool WRITE>
int run_rows(void* latent, i64 latent_stride, void* rope, i64 rope_stride, i64 tokens, const int64_t* slots, const ptstore_kv_cache_t* cache, u32* status,
             ptstore_stream_t stream) {
  const int rc = check_latent_cache(cache);
  if (rc) return rc;
  if (tokens < 0) return PTSTORE_E_INVAL;
  if (tokens == 0) return PTSTORE_OK;
  if (!latent || !rope || !slots || !rows_aligned(latent, tokens, latent_stride, 1, 0) || !rows_aligned(rope, tokens, rope_stride, 1, 0)) return PTSTORE_E_INVAL;
  const int cpr = (int)cache->head_dim / 8;
  constexpr int PER_CTA = ROWS_THREADS * ROWS_EACH;
  if ((u64)tokens > (u64)0x7FFFFFFF * PER_CTA / cpr) return PTSTORE_E_LIMIT;                 // grid of one launch
  const RowsArgs a = {cache_of(cache), static_cast<unsigned char*>(latent), static_cast<unsigned char*>(rope), 2 * latent_stride, 2 * rope_stride,
                      reinterpret_cast<const i64*>(slots), tokens * cpr, status};
  const unsigned grid = (unsigned)((a.items + PER_CTA - 1) / PER_CTA);
  (void)cudaGetLastError();
  if (cpr == 72) latent_rows_kernel<72, WRITE><<<grid, ROWS_THREADS, 0, static_cast<cudaStream_t>(stream)>>>(a);
  else latent_rows_kernel<40, WRITE><<<grid, ROWS_THREADS, 0, static_cast<cudaStream_t>(stream)>>>(a);
  return cudaGetLastError() == cudaSuccess ? PTSTORE_OK : PTSTORE_E_CUDA;
}

// The tensor map of the cache: {elements, tokens of a block, blocks}, boxes of 64 elements and the largest power of two of tokens, up to 64, that divides a block's.  Returns the
// tokens of a box, 0 if there is no map.
u32 make_rows_map(const Cache& c, bool half, int dim, CUtensorMap* map) {
  u32 box = LA_KEYS;
  while (c.block_tokens % box) box >>= 1;
  const cuuint64_t dims[3] = {(cuuint64_t)dim, c.block_tokens, c.num_blocks};
  const cuuint64_t strides[2] = {(cuuint64_t)dim * 2, c.block_stride};
  const cuuint32_t boxes[3] = {64, box, 1};
  return encode(map, half, 3, c.base, dims, strides, boxes) ? box : 0;
}

template <int L, bool F16, bool WIDE, bool ALIAS = false>
int launch_latent(const Latent& la, const CUtensorMap& map, const Gpu& gpu, cudaStream_t s) {
  using Shape = LatentShape<L, WIDE>;
  static std::atomic<u64> devices{0};
  auto* kernel = latent_attend_kernel<L, F16, WIDE, ALIAS>;
  constexpr int SMEM = latent_smem<L, WIDE>();
  const int rc = allow_smem(kernel, SMEM, devices, gpu.dev);
  if (rc) return rc;
  const int grid = gpu.sms / Shape::PAIR * Shape::PAIR;
  if (WIDE && ALIAS) {
    cudaLaunchAttribute pair;
    pair.id = cudaLaunchAttributeClusterDimension;
    pair.val.clusterDim.x = Shape::PAIR;
    pair.val.clusterDim.y = pair.val.clusterDim.z = 1;
    cudaLaunchConfig_t config = {};
    config.gridDim = grid;
    config.blockDim = LA_THREADS;
    config.dynamicSmemBytes = SMEM;
    config.stream = s;
    config.attrs = &pair;
    config.numAttrs = 1;
    (void)cudaLaunchKernelEx(&config, kernel, la, map);
  } else {
    kernel<<<grid, LA_THREADS, SMEM, s>>>(la, map);
  }
  if (cudaGetLastError() != cudaSuccess) return PTSTORE_E_CUDA;
  latent_join_kernel<L, F16, WIDE><<<dim3(grid, Shape::ROWS / 8, WIDE ? 1 : Shape::DIMS / 128), 256, 0, s>>>(la);
  return cudaGetLastError() == cudaSuccess ? PTSTORE_OK : PTSTORE_E_CUDA;
}
template <int L, bool F16>
int launch_latent_rows(const Latent& la, const CUtensorMap& map, i64 rows, const Gpu& gpu, cudaStream_t s) {
  if (rows <= LatentShape<L, false>::ROWS || gpu.sms < 2) return launch_latent<L, F16, false>(la, map, gpu, s);
  return la.a.out == la.a.q ? launch_latent<L, F16, true, true>(la, map, gpu, s) : launch_latent<L, F16, true>(la, map, gpu, s);
}

}  // namespace

extern "C" int ptstore_latent_write(const void* latent, int64_t latent_stride, const void* rope, int64_t rope_stride, int64_t tokens, const int64_t* slots,
                                    const ptstore_kv_cache_t* cache, uint32_t* status, ptstore_stream_t stream) {
  return run_rows<true>(const_cast<void*>(latent), latent_stride, const_cast<void*>(rope), rope_stride, tokens, slots, cache, status, stream);
}

extern "C" int ptstore_latent_read(const ptstore_kv_cache_t* cache, const int64_t* slots, int64_t tokens, void* latent, int64_t latent_stride, void* rope,
                                   int64_t rope_stride, uint32_t* status, ptstore_stream_t stream) {
  return run_rows<false>(latent, latent_stride, rope, rope_stride, tokens, slots, cache, status, stream);
}

extern "C" uint64_t ptstore_latent_workspace_bytes(uint32_t head_dim) {
  if (head_dim != 320 && head_dim != 576) return 0;
  // two sets of sums per CTA, of 128 rows and half of the elements or of 32 rows and all of them
  return LA_PARTS_AT + (u64)MAX_SMS * 2 * 128 * ((head_dim - LA_ROPE) / 2 + 2) * 4;
}

extern "C" int ptstore_latent_attend(const ptstore_latent_attend_t* p, const ptstore_kv_cache_t* cache, void* workspace, uint64_t workspace_bytes, uint32_t* status,
                                     ptstore_stream_t stream) {
  if (!p || p->struct_size != sizeof(ptstore_latent_attend_t)) return PTSTORE_E_INVAL;
  const int rc = check_latent_cache(cache);
  if (rc) return rc;
  if (p->requests < 0 || p->max_blocks < 1 || p->tokens < 0 || p->max_new < 0 || p->num_heads < 1 || p->num_heads > 65535) return PTSTORE_E_INVAL;
  const float scale2 = p->scale * LOG2E;
  if (!isfinite(scale2)) return PTSTORE_E_INVAL;
  if (p->requests == 0 || p->tokens == 0 || p->max_new == 0) return PTSTORE_OK;
  if (!p->q_latent || !p->q_rope || !p->out || !p->token_offsets || !p->lengths || !p->block_tables) return PTSTORE_E_INVAL;
  if (!rows_aligned(p->q_latent, p->tokens, p->q_latent_token_stride, p->num_heads, p->q_latent_head_stride) ||
      !rows_aligned(p->q_rope, p->tokens, p->q_rope_token_stride, p->num_heads, p->q_rope_head_stride) ||
      !rows_aligned(p->out, p->tokens, p->out_token_stride, p->num_heads, p->out_head_stride)) return PTSTORE_E_INVAL;
  // q itself as output: rows are written where they were read, which other strides are not
  if (p->out == p->q_latent && ((p->tokens > 1 && p->out_token_stride != p->q_latent_token_stride) || (p->num_heads > 1 && p->out_head_stride != p->q_latent_head_stride)))
    return PTSTORE_E_INVAL;
  if ((u64)p->max_blocks * cache->block_tokens > 1u << 30) return PTSTORE_E_LIMIT;
  if (p->requests > 1 << 20 || (i64)p->tokens * p->num_heads > 0x7FFFFFFF) return PTSTORE_E_LIMIT;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return PTSTORE_E_INVAL;
  if (workspace_bytes < ptstore_latent_workspace_bytes(cache->head_dim)) return PTSTORE_E_NOMEM;
  Latent la;
  Attend& a = la.a;
  a = Attend{};
  a.cache = cache_of(cache);
  a.q = static_cast<const unsigned char*>(p->q_latent);
  a.out = static_cast<unsigned char*>(p->out);
  a.q_token = p->q_latent_token_stride; a.q_head = p->q_latent_head_stride;
  a.o_token = p->out_token_stride; a.o_head = p->out_head_stride;
  a.offsets = p->token_offsets; a.lengths = p->lengths; a.tables = p->block_tables;
  a.R = p->requests; a.max_blocks = p->max_blocks; a.heads = a.group = p->num_heads; a.tokens = p->tokens;
  a.scale2 = scale2;
  a.v_factor = 1.0f;
  a.work = static_cast<unsigned char*>(workspace);
  a.polls = p->wait_polls ? p->wait_polls : POLLS;
  a.status = status;
  la.q_rope = static_cast<const unsigned char*>(p->q_rope);
  la.qr_token = p->q_rope_token_stride; la.qr_head = p->q_rope_head_stride;
  a.lse = p->lse;
  Gpu gpu;
  (void)cudaGetLastError();
  const int rs = current_gpu(&gpu);
  if (rs) return rs;
  const bool half = cache->format == PTSTORE_KV_LATENT_FP16;
  CUtensorMap map;
  a.box_tokens = make_rows_map(a.cache, half, (int)cache->head_dim, &map);
  if (!a.box_tokens) return PTSTORE_E_CUDA;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const i64 rows = (i64)(p->max_new < p->tokens ? p->max_new : p->tokens) * a.group;
  if (cache->head_dim == 576) return half ? launch_latent_rows<512, true>(la, map, rows, gpu, s) : launch_latent_rows<512, false>(la, map, rows, gpu, s);
  return half ? launch_latent_rows<256, true>(la, map, rows, gpu, s) : launch_latent_rows<256, false>(la, map, rows, gpu, s);
}
