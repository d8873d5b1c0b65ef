// ptstore_assign_blocks / ptstore_map_slots: the paged cache's bookkeeping on the device.  The matched lengths of a
// lookup are on the GPU; so block tables grow and shrink, and new tokens get their slots, without the host seeing a length.
//
// Both are prefix sums over the requests followed by a flat pass over what moves (blocks, tokens), and both are latency bound:
// a few kilobytes to a few megabytes against a launch, two or three dependent memory round trips and a block-wide scan.  So
// each is ONE launch in which every CTA scans all requests for itself (16,384 of them per step, 16 consecutive ones per
// thread), and the entries that move are dealt out evenly and find their request by a binary search in shared memory.
// B200, plan of one decode step of 64 requests / of 16,384 requests with 0.5 M new tokens: see the table of measurements.
#include <cuda_runtime.h>
#include <limits.h>

#include "../../include/ptstore.h"

namespace {

typedef long long i64;

constexpr int THREADS = 1024;
constexpr int ITEMS = 16;                    // consecutive requests of one thread
constexpr int CHUNK = THREADS * ITEMS;       // requests scanned per step
constexpr int CLUSTER = 8;                   // CTAs of an assignment (the portable cluster size)

__device__ __forceinline__ void cluster_sync() {     // orders global memory between the CTAs of the cluster too
  asm volatile("barrier.cluster.arrive.release;\n barrier.cluster.wait.acquire;" ::: "memory");
}

__device__ __forceinline__ void raise_status(uint32_t* status, uint32_t bits) {
  if (status) atomicOr(status, bits);
}

// Exclusive prefix sum of one value per thread over the CTA; total in every thread.  Called by all threads.
__device__ __forceinline__ i64 block_scan(i64 v, i64* s_warp, i64& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  i64 x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const i64 y = __shfl_up_sync(0xFFFFFFFFu, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();                           // the previous scan's readers are done with s_warp
  if (lane == 31) s_warp[warp] = x;
  __syncthreads();
  const i64 w = s_warp[lane];                // 32 warps: one total per lane
  i64 z = w;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const i64 y = __shfl_up_sync(0xFFFFFFFFu, z, o);
    if (lane >= o) z += y;
  }
  total = __shfl_sync(0xFFFFFFFFu, z, 31);
  const i64 before = __shfl_sync(0xFFFFFFFFu, z - w, warp);
  return before + x - v;
}

// last index i in [0, n) with first[i] <= k; first is non-decreasing, first[0] <= k
__device__ __forceinline__ int owner_of(const uint32_t* first, int n, uint32_t k) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (first[mid] <= k) lo = mid; else hi = mid;
  }
  return lo;
}

struct Assign {
  const int* lengths;
  const int* held;
  int R, block_tokens, max_blocks, capacity;
  int* tables;
  int* free_ids;
  const int* free_count;
  int* held_out;
  int* free_count_out;
  uint32_t* status;
};

// blocks a request holds and needs; a length its row cannot hold leaves the row as it is
__device__ __forceinline__ void want(const Assign& a, int r, int& held, int& need, uint32_t& bad) {
  const int h = a.held ? a.held[r] : 0, len = a.lengths[r];
  held = h < 0 ? 0 : h > a.max_blocks ? a.max_blocks : h;
  if (held != h || len < 0) bad = PTSTORE_S_BOUNDS;
  const i64 n = len <= 0 ? 0 : ((i64)len + a.block_tokens - 1) / a.block_tokens;
  if (n > a.max_blocks) { need = held; bad = PTSTORE_S_BOUNDS; } else need = (int)n;
}

__global__ void __cluster_dims__(CLUSTER, 1, 1) __launch_bounds__(THREADS) assign_blocks_kernel(Assign a) {
  extern __shared__ uint32_t s_dyn[];
  __shared__ i64 s_warp[32];
  __shared__ unsigned long long s_taken;
  const int cap_items = a.R < CHUNK ? a.R : CHUNK;
  uint32_t* s_grow = s_dyn;                  // exclusive prefix sums inside the chunk
  uint32_t* s_back = s_dyn + cap_items;
  const int items = (cap_items + THREADS - 1) / THREADS;
  const int gtid = blockIdx.x * THREADS + threadIdx.x, gthreads = CLUSTER * THREADS;
  uint32_t bad = 0;
  const int c0 = *a.free_count;
  const int count = c0 < 0 ? 0 : c0 > a.capacity ? a.capacity : c0;
  if (count != c0) bad = PTSTORE_S_BOUNDS;
  if (threadIdx.x == 0) s_taken = 0;

  auto scan_chunk = [&](int base, int n, i64& grow_total, i64& back_total) {
    i64 g = 0, b = 0;
    const int i0 = threadIdx.x * items;
    uint32_t gi[ITEMS], bi[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      gi[i] = bi[i] = 0;
      if (i < items && i0 + i < n) {
        int held, need;
        want(a, base + i0 + i, held, need, bad);
        gi[i] = need > held ? need - held : 0;
        bi[i] = need < held ? held - need : 0;
      }
      g += gi[i];
      b += bi[i];
    }
    i64 ge = block_scan(g, s_warp, grow_total), be = block_scan(b, s_warp, back_total);
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
      if (i < items && i0 + i < n) {
        s_grow[i0 + i] = (uint32_t)ge;
        s_back[i0 + i] = (uint32_t)be;
        ge += gi[i];
        be += bi[i];
      }
    __syncthreads();
  };

  // surplus blocks of shrinking rows go onto the stack, in (request, block) order
  i64 pushed = 0, grow_total = 0, back_total = 0;
  for (int base = 0; base < a.R; base += CHUNK) {
    const int n = a.R - base < CHUNK ? a.R - base : CHUNK;
    scan_chunk(base, n, grow_total, back_total);
    for (i64 k = gtid; k < back_total; k += gthreads) {
      const int i = owner_of(s_back, n, (uint32_t)k), r = base + i;
      int held, need;
      want(a, r, held, need, bad);
      const i64 to = count + pushed + k;
      if (to < a.capacity) a.free_ids[to] = a.tables[(i64)r * a.max_blocks + need + (k - s_back[i])];
      else bad = PTSTORE_S_BOUNDS;           // more ids than the stack has room for: the surplus ones are lost
    }
    pushed += back_total;
    __syncthreads();
  }
  i64 top = count + pushed;
  if (top > a.capacity) top = a.capacity;
  cluster_sync();                            // the pushed ids are visible; nothing has been popped yet

  // growing rows pop from the top; a request is granted its blocks iff all growth up to and including it fits
  i64 wanted = 0;
  for (int base = 0; base < a.R; base += CHUNK) {
    const int n = a.R - base < CHUNK ? a.R - base : CHUNK;
    if (a.R > CHUNK) {                       // a single chunk's sums are still in shared memory
      scan_chunk(base, n, grow_total, back_total);
      cluster_sync();                        // every CTA has read held of this chunk before one overwrites it
    }
    i64 fits = top - wanted;                 // pops of this chunk that the stack can serve
    const int i0 = threadIdx.x * items;
    for (int i = 0; i < items; ++i)
      if (i0 + i < n) {
        const int r = base + i0 + i;
        int held, need;
        want(a, r, held, need, bad);
        const i64 upto = (i64)s_grow[i0 + i] + (need - held);
        if (need > held) {
          if (upto <= fits) atomicMax(&s_taken, (unsigned long long)(wanted + upto));
          else { bad |= PTSTORE_S_NOSPACE; need = held; }
        }
      }
    __syncthreads();
    const i64 end = (i64)s_taken - wanted;   // pops granted in this chunk: the first `end` of them
    for (i64 k = gtid; k < end; k += gthreads) {
      const int i = owner_of(s_grow, n, (uint32_t)k), r = base + i;
      int held, need;
      want(a, r, held, need, bad);
      a.tables[(i64)r * a.max_blocks + held + (k - s_grow[i])] = a.free_ids[top - 1 - (wanted + k)];
    }
    // held is read by every CTA above, so one CTA's writes wait for all of them
    cluster_sync();
    for (int i = gtid; i < n; i += gthreads) {
      int held, need;
      want(a, base + i, held, need, bad);
      a.held_out[base + i] = need <= held || (i64)s_grow[i] + (need - held) <= fits ? need : held;
    }
    wanted += grow_total;
    __syncthreads();
  }
  if (gtid == 0) *a.free_count_out = (int)(top - (i64)s_taken);
  if (bad) raise_status(a.status, bad);
}

struct MapSlots {
  const int* lengths;
  const int* done;
  int done_unit, min_new, R, block_tokens, max_blocks;
  const int* tables;
  i64 max_tokens, per_cta;
  int* offsets;
  i64* slots;
  int* positions;
  uint32_t* status;
};

// tokens of the request that are in the cache already, and new ones
__device__ __forceinline__ void done_new(const MapSlots& m, int r, int& done, int& fresh, uint32_t& bad) {
  int len = m.lengths[r];
  if (len < 0) { len = 0; bad = PTSTORE_S_BOUNDS; }
  i64 d = m.done ? (i64)m.done[r] * m.done_unit : 0;
  const i64 most = (i64)len - m.min_new;
  if (d > most) d = most;
  if (d < 0) d = 0;
  done = (int)d;
  fresh = len - done;
}

__global__ void __launch_bounds__(THREADS) map_slots_kernel(MapSlots m) {
  extern __shared__ uint32_t s_first[];      // exclusive prefix sums inside the chunk
  __shared__ i64 s_warp[32];
  const int cap_items = m.R < CHUNK ? m.R : CHUNK;
  const int items = (cap_items + THREADS - 1) / THREADS;
  const i64 t0 = blockIdx.x * m.per_cta, t1 = t0 + m.per_cta < m.max_tokens ? t0 + m.per_cta : m.max_tokens;
  uint32_t bad = 0;
  i64 base_tok = 0;
  for (int base = 0; base < m.R; base += CHUNK) {
    const int n = m.R - base < CHUNK ? m.R - base : CHUNK;
    const int i0 = threadIdx.x * items;
    i64 sum = 0;
    int f[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      f[i] = 0;
      int done;
      if (i < items && i0 + i < n) done_new(m, base + i0 + i, done, f[i], bad);
      sum += f[i];
    }
    i64 total;
    i64 e = block_scan(sum, s_warp, total);
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
      if (i < items && i0 + i < n) {
        // a chunk's sums can pass 32 bits only where they pass max_tokens too; those are never searched for
        s_first[i0 + i] = e > UINT_MAX ? UINT_MAX : (uint32_t)e;
        if (blockIdx.x == 0) {
          const i64 at = base_tok + e;
          m.offsets[base + i0 + i] = at > INT_MAX ? INT_MAX : (int)at;
        }
        e += f[i];
      }
    __syncthreads();
    const i64 lo = t0 > base_tok ? t0 : base_tok, hi = t1 < base_tok + total ? t1 : base_tok + total;
    for (i64 t = lo + threadIdx.x; t < hi; t += THREADS) {
      const uint32_t k = (uint32_t)(t - base_tok);
      const int i = owner_of(s_first, n, k), r = base + i;
      int done, fresh;
      done_new(m, r, done, fresh, bad);
      const int pos = done + (int)(k - s_first[i]);
      const int j = pos / m.block_tokens;
      i64 slot = -1;
      if (j < m.max_blocks) {
        const int b = m.tables[(i64)r * m.max_blocks + j];
        if (b >= 0) slot = (i64)b * m.block_tokens + (pos - j * m.block_tokens);
      } else bad = PTSTORE_S_BOUNDS;
      m.slots[t] = slot;
      if (m.positions) m.positions[t] = pos;
    }
    base_tok += total;
    __syncthreads();
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    m.offsets[m.R] = base_tok > INT_MAX ? INT_MAX : (int)base_tok;
    if (base_tok > m.max_tokens) bad = PTSTORE_S_BOUNDS;
  }
  // entries behind the last token are empty slots, so a write of a padded batch skips them
  for (i64 t = (t0 > base_tok ? t0 : base_tok) + threadIdx.x; t < t1; t += THREADS) {
    m.slots[t] = -1;
    if (m.positions) m.positions[t] = -1;
  }
  if (bad) raise_status(m.status, bad);
}

int launch_ok() { return cudaGetLastError() == cudaSuccess ? PTSTORE_OK : PTSTORE_E_CUDA; }

// More dynamic shared memory than 48 KB has to be allowed per function; set on every call that needs it, since the setting
// belongs to the current device.
template <typename F>
int allow_smem(F* kernel, size_t bytes) {
  if (bytes <= 48 * 1024) return PTSTORE_OK;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) == cudaSuccess) return PTSTORE_OK;
  (void)cudaGetLastError();
  return PTSTORE_E_CUDA;
}

}  // namespace

extern "C" int ptstore_assign_blocks(const int32_t* lengths, const int32_t* held, int32_t R, int32_t block_tokens, int32_t* block_tables,
                                     int32_t max_blocks, int32_t* free_ids, int32_t free_capacity, const int32_t* free_count,
                                     int32_t* held_out, int32_t* free_count_out, uint32_t* status, ptstore_stream_t stream) {
  if (R < 0 || block_tokens < 1 || max_blocks < 1 || free_capacity < 0) return PTSTORE_E_INVAL;
  if (!free_count || !free_count_out || (free_capacity > 0 && !free_ids)) return PTSTORE_E_INVAL;
  if (R > 0 && (!lengths || !block_tables || !held_out)) return PTSTORE_E_INVAL;
  if (R > 1 << 30) return PTSTORE_E_LIMIT;
  if ((i64)(R < CHUNK ? R : CHUNK) * max_blocks > (i64)UINT_MAX) return PTSTORE_E_LIMIT;      // sums inside a chunk are 32 bits wide
  const Assign a = {lengths, held, R, block_tokens, max_blocks, free_capacity, block_tables, free_ids, free_count, held_out, free_count_out, status};
  const size_t smem = 8 * (size_t)(R < CHUNK ? R : CHUNK);
  (void)cudaGetLastError();
  const int rc = allow_smem(assign_blocks_kernel, smem);
  if (rc) return rc;
  assign_blocks_kernel<<<CLUSTER, THREADS, smem, static_cast<cudaStream_t>(stream)>>>(a);
  return launch_ok();
}

extern "C" int ptstore_map_slots(const int32_t* lengths, const int32_t* done, int32_t done_unit, int32_t min_new, int32_t R,
                                 const int32_t* block_tables, int32_t max_blocks, int32_t block_tokens, int64_t max_tokens,
                                 int32_t* token_offsets, int64_t* slots, int32_t* positions, uint32_t* status, ptstore_stream_t stream) {
  if (R < 0 || block_tokens < 1 || max_blocks < 1 || max_tokens < 0 || max_tokens > INT_MAX || done_unit < 1 || min_new < 0) return PTSTORE_E_INVAL;
  if (!token_offsets || (max_tokens > 0 && !slots) || (R > 0 && (!lengths || !block_tables))) return PTSTORE_E_INVAL;
  if (R > 1 << 30) return PTSTORE_E_LIMIT;
  MapSlots m = {lengths, done, done_unit, min_new, R, block_tokens, max_blocks, block_tables, max_tokens, 0, token_offsets,
                reinterpret_cast<i64*>(slots), positions, status};
  // at most one CTA per SM (148): every CTA scans all requests, so more of them would only repeat that
  i64 per = (max_tokens + 147) / 148;
  per = (per + THREADS - 1) / THREADS * THREADS;
  if (per < THREADS) per = THREADS;
  m.per_cta = per;
  i64 grid = (max_tokens + per - 1) / per;
  if (grid < 1) grid = 1;
  const size_t smem = 4 * (size_t)(R < CHUNK ? R : CHUNK);
  (void)cudaGetLastError();
  const int rc = allow_smem(map_slots_kernel, smem);
  if (rc) return rc;
  map_slots_kernel<<<(unsigned)grid, THREADS, smem, static_cast<cudaStream_t>(stream)>>>(m);
  return launch_ok();
}
