// ptstore_kv_write / ptstore_kv_read: rows of a model's K and V into the paged cache through a slot map, and back.
//
// Bound: HBM.  A 16-bit element costs 2 bytes on the model's side and 2 or 0.5625 in the cache, nothing is read twice.  One thread
// takes 32 consecutive elements (two scale groups): four 16-byte loads, its own maxima, 16 bytes of codes and two scales, so there
// is no exchange between threads (with 16 elements finding the row and the slot was half of 327 instructions: 23.3 us for K and V of 16384 tokens of
// 8 x 128; with 32 the writer takes 20.1, the reader 19.0, their bytes 13.2.  Issue slots are 65 % busy, and scale bytes leave as parts of
// sectors.  A 16-bit cache: writer 25.4 us, reader 24.4, bytes 20.5).  What the quantiser computes is defined in exact terms (nearest code of x / (scale * tensor
// scale), ties to even); 32 bits give exactly that: x has at most 11 significant bits and the divisor 4, so a quotient that is not
// on a rounding border is at least 2^-16 away from it, and one that is comes out exactly (the division below is corrected by its residual).
#include "kvcache.cuh"

using namespace ptk;

namespace {

constexpr int WRITE_THREADS = 256;
constexpr int WRITE_SPAN = 32, READ_SPAN = 16;  // elements of a thread (a reader of 32 stores in pieces that are further apart: 21.1 us, 19.1 with 16)

struct Rows {
  unsigned char* k;
  unsigned char* v;
  i64 k_token, k_head, v_token, v_head;        // strides in elements
};

struct KvArgs {
  Cache cache;
  Rows rows;
  const i64* slots;
  i64 items;                                   // T * heads * (D / span)
  float k_scale, v_scale;
  u32* status;
};

template <bool FP16>
__device__ __forceinline__ float2 widen(u32 two) {
  if (FP16) return __half22float2(*reinterpret_cast<const __half2*>(&two));
  return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&two));
}
template <bool FP16>
__device__ __forceinline__ u32 narrow(float a, float b) {
  if (FP16) { const __half2 h = __floats2half2_rn(a, b); return *reinterpret_cast<const u32*>(&h); }
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const u32*>(&h);
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

struct Where { u32 block, token, head, span; i64 row; };
template <int D, int SPAN>
__device__ __forceinline__ void find_row(const KvArgs& a, i64 item, Where& w) {
  constexpr u32 G = D / SPAN;
  w.span = (u32)item % G;
  const u64 rest = (u64)item / G;
  if (rest <= 0xFFFFFFFFull) { w.row = (u32)rest / a.cache.heads; w.head = (u32)rest % a.cache.heads; }
  else { w.row = (i64)(rest / a.cache.heads); w.head = (u32)(rest % a.cache.heads); }
}
// cache position of a row's slot -> false if it is skipped
__device__ __forceinline__ bool find_slot(const KvArgs& a, i64 slot, Where& w) {
  if (slot == -1) return false;
  u64 block;
  if ((u64)slot <= 0xFFFFFFFFull) { block = (u32)slot / a.cache.block_tokens; w.token = (u32)slot % a.cache.block_tokens; }
  else { block = (u64)slot / a.cache.block_tokens; w.token = (u32)((u64)slot % a.cache.block_tokens); }
  if (slot < 0 || block >= a.cache.num_blocks) {
    if (a.status) atomicOr(a.status, PTSTORE_S_BOUNDS);
    return false;
  }
  w.block = (u32)block;
  return true;
}

template <int SPAN>
__device__ __forceinline__ const unsigned char* model_row(const Rows& r, bool is_v, const Where& w) {
  return is_v ? r.v + 2 * (w.row * r.v_token + w.head * r.v_head + w.span * SPAN) : r.k + 2 * (w.row * r.k_token + w.head * r.k_head + w.span * SPAN);
}

template <int D, bool FP16, bool PACKED>
__global__ void __launch_bounds__(WRITE_THREADS) kv_write_kernel(KvArgs a) {
  const i64 item = (i64)blockIdx.x * WRITE_THREADS + threadIdx.x;
  if (item >= a.items) return;
  const bool is_v = blockIdx.y != 0;
  Where w;
  find_row<D, WRITE_SPAN>(a, item, w);
  const i64 slot = a.slots[w.row];
  const uint4* src = reinterpret_cast<const uint4*>(model_row<WRITE_SPAN>(a.rows, is_v, w));
  const uint4 in[4] = {src[0], src[1], src[2], src[3]};       // on their way together with the slot
  if (!find_slot(a, slot, w)) return;
  if (!PACKED) {
    uint4* dst = reinterpret_cast<uint4*>(row_ptr(a.cache, is_v, w.block, w.head, w.token, D) + w.span * WRITE_SPAN * 2);
#pragma unroll
    for (int i = 0; i < 4; ++i) dst[i] = in[i];
    return;
  }
  const float t = is_v ? a.v_scale : a.k_scale;
  u32 code[4], sb[2];
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    const u32 raw[8] = {in[2 * g].x, in[2 * g].y, in[2 * g].z, in[2 * g].w, in[2 * g + 1].x, in[2 * g + 1].y, in[2 * g + 1].z, in[2 * g + 1].w};
    float x[16], amax = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float2 f = widen<FP16>(raw[i]);
      x[2 * i] = f.x;
      x[2 * i + 1] = f.y;
      amax = max_nan(amax, max_nan(fabsf(f.x), fabsf(f.y)));
    }
    sb[g] = e4m3_of(__fdiv_rn(amax, 7.0f * t));
    const float e = e4m3_value(sb[g]) * t;             // exact: 4 significant bits times a power of two
    code[2 * g] = code[2 * g + 1] = 0x88888888u;       // code 8 is zero
    if (e > 0.0f) {
      const float inv = __frcp_rn(e);
      if (amax > 8.4f * e) {                           // the scale is far too small for the largest (at most 448, or next to zero): an infinity
        const float most = 8.0f * e;                   // becomes finite, and codes stay above -9
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = fminf(fmaxf(x[i], -most), most);
      }
      u32 sum[2] = {0, 0};
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float y = x[i] * inv;
        const float q = fmaf(fmaf(-y, e, x[i]), inv, y);       // the quotient, exact where it is representable; at least -8.4
        // adding 1.5 * 2^23 + 8 rounds to an integer, ties to even, and leaves the code in the low bits: the words are sums of
        // these bit patterns times powers of 16, less what the constant's bits add up to
        sum[i >> 3] += __float_as_uint(fminf(q, 7.0f) + 12582920.0f) << (4 * (i & 7));
      }
      constexpr u32 B = 0x4B400000u, REST = B + (B << 4) + (B << 8) + (B << 12) + (B << 16) + (B << 20) + (B << 24) + (B << 28);
      code[2 * g] = sum[0] - REST;
      code[2 * g + 1] = sum[1] - REST;
    }
  }
  unsigned char* tile = tile_ptr(a.cache, is_v, w.block, w.head, w.token, D);
  const int n = w.token % TILE;
  *reinterpret_cast<uint4*>(tile + code_place(D, n, w.span) * 16) = make_uint4(code[0], code[1], code[2], code[3]);
  if (is_v) {
    tile[scale_at(D, true, n, 2 * w.span)] = (unsigned char)sb[0];
    tile[scale_at(D, true, n, 2 * w.span + 1)] = (unsigned char)sb[1];
  } else *reinterpret_cast<unsigned short*>(tile + scale_at(D, false, n, 2 * w.span)) = (unsigned short)(sb[0] | (sb[1] << 8));
}

template <int D, bool FP16, bool PACKED>
__global__ void __launch_bounds__(WRITE_THREADS) kv_read_kernel(KvArgs a) {
  const i64 item = (i64)blockIdx.x * WRITE_THREADS + threadIdx.x;
  if (item >= a.items) return;
  const bool is_v = blockIdx.y != 0;
  Where w;
  find_row<D, READ_SPAN>(a, item, w);
  if (!find_slot(a, a.slots[w.row], w)) return;
  uint4* dst = reinterpret_cast<uint4*>(const_cast<unsigned char*>(model_row<READ_SPAN>(a.rows, is_v, w)));
  if (!PACKED) {
    const uint4* src = reinterpret_cast<const uint4*>(row_ptr(a.cache, is_v, w.block, w.head, w.token, D) + w.span * READ_SPAN * 2);
    const uint4 lo = src[0], hi = src[1];
    dst[0] = lo;
    dst[1] = hi;
    return;
  }
  const unsigned char* tile = tile_ptr(a.cache, is_v, w.block, w.head, w.token, D);
  const int n = w.token % TILE;
  const uint2 two = *reinterpret_cast<const uint2*>(tile + code_place(D, n, w.span >> 1) * 16 + (w.span & 1) * 8);
  const u32 code[2] = {two.x, two.y};
  const float e = e4m3_value(tile[scale_at(D, is_v, n, w.span)]) * (is_v ? a.v_scale : a.k_scale);
  // code n at bits p .. p+3 of 2^23 reads as 2^23 + n 2^p: less 2^23 + 8 2^p it is (n - 8) 2^p, exactly (p <= 16)
#pragma unroll
  for (int o = 0; o < 2; ++o) {                        // eight elements: a word of codes
    u32 out[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const u32 c = code[o] >> (16 * (i >> 1));
      const int p = 8 * (i & 1);
      float v[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const float f = __uint_as_float((c & (15u << (p + 4 * k))) | 0x4B000000u) - (8388608.0f + 8.0f * (float)(1 << (p + 4 * k)));
        v[k] = f * (e * (1.0f / (float)(1 << (p + 4 * k))));
      }
      out[i] = narrow<FP16>(v[0], v[1]);
    }
    dst[o] = make_uint4(out[0], out[1], out[2], out[3]);
  }
}

// shared checks and launch; WRITE picks the kernel
template <bool WRITE>
int run(const void* k, const void* v, i64 k_token, i64 k_head, i64 v_token, i64 v_head, i64 tokens, u32 dtype, const int64_t* slots,
        const ptstore_kv_cache_t* cache, u32* status, ptstore_stream_t stream) {
  const int rc = check_cache(cache);
  if (rc) return rc;
  if (tokens < 0 || (dtype != PTSTORE_KV_BF16 && dtype != PTSTORE_KV_FP16)) return PTSTORE_E_INVAL;
  if (cache->format != PTSTORE_KV_PACKED && cache->format != dtype) return PTSTORE_E_INVAL;
  if (tokens == 0) return PTSTORE_OK;
  if (!k || !v || !slots || !rows_aligned(k, tokens, k_token, cache->num_kv_heads, k_head) ||
      !rows_aligned(v, tokens, v_token, cache->num_kv_heads, v_head)) return PTSTORE_E_INVAL;
  const int D = (int)cache->head_dim;
  KvArgs a = {cache_of(cache), {(unsigned char*)k, (unsigned char*)v, k_token, k_head, v_token, v_head}, reinterpret_cast<const i64*>(slots), 0,
              cache->k_scale, cache->v_scale, status};
  const u64 per_token = (u64)a.cache.heads * (D / (WRITE ? WRITE_SPAN : READ_SPAN));
  if ((u64)tokens > (u64)0x7FFFFFFF * WRITE_THREADS / per_token) return PTSTORE_E_LIMIT;       // grid of one launch
  a.items = (i64)((u64)tokens * per_token);
  const dim3 grid((unsigned)((a.items + WRITE_THREADS - 1) / WRITE_THREADS), 2);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const bool half = dtype == PTSTORE_KV_FP16, packed = cache->format == PTSTORE_KV_PACKED;
  (void)cudaGetLastError();
#define PTK_LAUNCH(D_, H_, P_) \
  if (D == D_ && half == H_ && packed == P_) { \
    if (WRITE) kv_write_kernel<D_, H_, P_><<<grid, WRITE_THREADS, 0, s>>>(a); \
    else kv_read_kernel<D_, H_, P_><<<grid, WRITE_THREADS, 0, s>>>(a); \
  }
  PTK_LAUNCH(64, false, false) PTK_LAUNCH(64, false, true) PTK_LAUNCH(64, true, true)
  PTK_LAUNCH(128, false, false) PTK_LAUNCH(128, false, true) PTK_LAUNCH(128, true, true)
  // a 16-bit cache is copied, whatever the 16 bits mean: the kernels compiled for bf16 serve fp16 too
  if (half && !packed) {
    if (D == 64) { if (WRITE) kv_write_kernel<64, false, false><<<grid, WRITE_THREADS, 0, s>>>(a); else kv_read_kernel<64, false, false><<<grid, WRITE_THREADS, 0, s>>>(a); }
    else { if (WRITE) kv_write_kernel<128, false, false><<<grid, WRITE_THREADS, 0, s>>>(a); else kv_read_kernel<128, false, false><<<grid, WRITE_THREADS, 0, s>>>(a); }
  }
#undef PTK_LAUNCH
  return cudaGetLastError() == cudaSuccess ? PTSTORE_OK : PTSTORE_E_CUDA;
}

}  // namespace

extern "C" uint64_t ptstore_kv_chunk_bytes(uint32_t format, uint32_t block_tokens, uint32_t num_kv_heads, uint32_t head_dim) {
  return chunk_bytes_of(format, block_tokens, num_kv_heads, head_dim);
}

extern "C" int ptstore_kv_write(const void* k, int64_t k_token_stride, int64_t k_head_stride, const void* v, int64_t v_token_stride,
                                int64_t v_head_stride, int64_t tokens, uint32_t dtype, const int64_t* slots, const ptstore_kv_cache_t* cache,
                                uint32_t* status, ptstore_stream_t stream) {
  return run<true>(k, v, k_token_stride, k_head_stride, v_token_stride, v_head_stride, tokens, dtype, slots, cache, status, stream);
}

extern "C" int ptstore_kv_read(const ptstore_kv_cache_t* cache, const int64_t* slots, int64_t tokens, uint32_t dtype, void* k,
                               int64_t k_token_stride, int64_t k_head_stride, void* v, int64_t v_token_stride, int64_t v_head_stride,
                               uint32_t* status, ptstore_stream_t stream) {
  return run<false>(k, v, k_token_stride, k_head_stride, v_token_stride, v_head_stride, tokens, dtype, slots, cache, status, stream);
}
