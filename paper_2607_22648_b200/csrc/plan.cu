// ptstore_assign_blocks / ptstore_map_slots: the paged cache's bookkeeping on the device.  The matched lengths of a
// lookup are on the GPU; so block tables grow and shrink, and new tokens get their slots, without the host seeing a length.
//
// Both are prefix sums over the requests followed by a flat pass over what moves (blocks, tokens), and both are latency bound:
// a few kilobytes to a few megabytes against a launch, two or three dependent memory round trips and a block-wide scan.  So
// each is ONE launch in which every CTA scans all requests for itself (16,384 of them per step, up to 16 per
// thread, both sums of an assignment in one 64-bit value), and the entries that move are dealt out evenly and find their request by a binary search in shared memory.
// B200, plan of one decode step of 64 requests / of 16,384 requests with 0.5 M new tokens: see the table of measurements.
#include <cuda_runtime.h>
#include <limits.h>

#include "../../include/ptstore.h"

namespace {

typedef long long i64;
typedef unsigned long long u64;

constexpr int THREADS = 1024;
constexpr int ITEMS = 16;                    // requests of one thread
constexpr int CHUNK = THREADS * ITEMS;       // requests scanned per step
constexpr int CLUSTER = 8;                   // CTAs of an assignment (the portable cluster size)

__device__ __forceinline__ void cluster_sync() {     // orders global memory between the CTAs of the cluster too
  asm volatile("barrier.cluster.arrive.release;\n barrier.cluster.wait.acquire;" ::: "memory");
}

__device__ __forceinline__ void raise_status(uint32_t* status, uint32_t bits) {
  if (status) atomicOr(status, bits);
}

__device__ __forceinline__ u64 plus(u64 a, u64 b) { return a + b; }
__device__ __forceinline__ uint32_t plus(uint32_t a, uint32_t b) {        // saturates
  const uint32_t s = a + b;
  return s < a ? UINT_MAX : s;
}

// Exclusive prefix sums over a chunk: v[i] belongs to request i * THREADS + threadIdx.x of it (so that loads are coalesced and the
// warps' scans of the rows are independent), rows of them are in use.  total in every thread.  Called by all threads.
template <typename T>
__device__ __forceinline__ void scan_chunk(T (&v)[ITEMS], int rows, T* s_tot /*[ITEMS * 32 + 1]*/, T& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  __syncthreads();                           // the previous scan's readers are done with s_tot
#pragma unroll
  for (int i = 0; i < ITEMS; ++i)
    if (i < rows) {
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const T y = __shfl_up_sync(0xFFFFFFFFu, v[i], o);
        if (lane >= o) v[i] = plus(v[i], y);
      }
      if (lane == 31) s_tot[i * 32 + warp] = v[i];
      v[i] = __shfl_up_sync(0xFFFFFFFFu, v[i], 1);
      if (lane == 0) v[i] = 0;
    }
  __syncthreads();
  if (warp == 0) {                           // lane l: the totals l * rows .. of the rows * 32 in order
    T sum = 0;
    for (int k = 0; k < rows; ++k) sum = plus(sum, s_tot[lane * rows + k]);
    T x = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const T y = __shfl_up_sync(0xFFFFFFFFu, x, o);
      if (lane >= o) x = plus(x, y);
    }
    if (lane == 31) s_tot[ITEMS * 32] = x;
    T run = __shfl_up_sync(0xFFFFFFFFu, x, 1);
    if (lane == 0) run = 0;
    for (int k = 0; k < rows; ++k) {
      const T t = s_tot[lane * rows + k];
      s_tot[lane * rows + k] = run;
      run = plus(run, t);
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < ITEMS; ++i)
    if (i < rows) v[i] = plus(v[i], s_tot[i * 32 + warp]);
  total = s_tot[ITEMS * 32];
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
  const uint32_t n = len <= 0 ? 0 : (uint32_t)(len - 1) / (uint32_t)a.block_tokens + 1;
  if (n > (uint32_t)a.max_blocks) { need = held; bad = PTSTORE_S_BOUNDS; } else need = (int)n;
}

__global__ void __cluster_dims__(CLUSTER, 1, 1) __launch_bounds__(THREADS) assign_blocks_kernel(Assign a) {
  extern __shared__ uint32_t s_dyn[];
  __shared__ u64 s_tot[ITEMS * 32 + 1];
  __shared__ u64 s_taken;
  const int cap_items = a.R < CHUNK ? a.R : CHUNK;
  uint32_t* s_grow = s_dyn;                  // exclusive prefix sums inside the chunk
  uint32_t* s_back = s_dyn + cap_items;
  uint32_t* s_held = s_dyn + 2 * cap_items;
  const int rows = (cap_items + THREADS - 1) / THREADS;
  const int gtid = blockIdx.x * THREADS + threadIdx.x, gthreads = CLUSTER * THREADS;
  uint32_t bad = 0;
  const int c0 = *a.free_count;
  const int count = c0 < 0 ? 0 : c0 > a.capacity ? a.capacity : c0;
  if (count != c0) bad = PTSTORE_S_BOUNDS;
  if (threadIdx.x == 0) s_taken = 0;

  u64 moves = 0;                             // growth of the chunk, and in the upper half what it gives back
  auto scan = [&](int base, int n) {
    u64 v[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      v[i] = 0;
      const int k = i * THREADS + threadIdx.x;
      if (i < rows && k < n) {
        int held, need;
        want(a, base + k, held, need, bad);
        s_held[k] = held;
        v[i] = need > held ? (u64)(need - held) : (u64)(held - need) << 32;
      }
    }
    scan_chunk(v, rows, s_tot, moves);
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int k = i * THREADS + threadIdx.x;
      if (i < rows && k < n) {
        s_grow[k] = (uint32_t)v[i];
        s_back[k] = (uint32_t)(v[i] >> 32);
      }
    }
    __syncthreads();
  };
  auto after = [&](const uint32_t* s, int k, int n, uint32_t end) { return k + 1 < n ? s[k + 1] : end; };

  // surplus blocks of shrinking rows go onto the stack, in (request, block) order
  i64 pushed = 0;
  for (int base = 0; base < a.R; base += CHUNK) {
    const int n = a.R - base < CHUNK ? a.R - base : CHUNK;
    scan(base, n);
    const uint32_t back = (uint32_t)(moves >> 32);
    for (u64 k = gtid; k < back; k += gthreads) {
      const int i = owner_of(s_back, n, (uint32_t)k);
      const uint32_t first = s_back[i], need = s_held[i] - (after(s_back, i, n, back) - first);
      const i64 to = count + pushed + (i64)k;
      if (to < a.capacity) a.free_ids[to] = a.tables[(i64)(base + i) * a.max_blocks + need + ((uint32_t)k - first)];
      else bad |= PTSTORE_S_BOUNDS;          // more ids than the stack has room for: the surplus ones are lost
    }
    pushed += back;
  }
  i64 top = count + pushed;
  if (top > a.capacity) top = a.capacity;
  cluster_sync();                            // the pushed ids are visible, and every CTA has read held and free_count

  // growing rows pop from the top; a request is granted its blocks iff all growth up to and including it fits
  i64 wanted = 0;
  for (int base = 0; base < a.R; base += CHUNK) {
    const int n = a.R - base < CHUNK ? a.R - base : CHUNK;
    if (a.R > CHUNK) {                       // a single chunk's sums are still in shared memory
      scan(base, n);
      cluster_sync();                        // every CTA has read held of this chunk before one overwrites it
    }
    const uint32_t grow = (uint32_t)moves, back = (uint32_t)(moves >> 32);
    const i64 fits = top - wanted;           // pops of this chunk that the stack can serve
    uint32_t best = 0;                       // grants are a prefix of the pops: the largest granted end is their number
    for (int k = threadIdx.x; k < n; k += THREADS) {
      const uint32_t g0 = s_grow[k], g = after(s_grow, k, n, grow) - g0, held = s_held[k];
      const bool granted = (i64)g0 + g <= fits;
      if (g > 0) {
        if (granted) best = g0 + g;
        else bad |= PTSTORE_S_NOSPACE;
      }
      if (k / (THREADS / CLUSTER) % CLUSTER == blockIdx.x)       // each CTA writes its share
        a.held_out[base + k] = held + (granted ? g : 0) - (after(s_back, k, n, back) - s_back[k]);
    }
    best = __reduce_max_sync(0xFFFFFFFFu, best);
    if ((threadIdx.x & 31) == 0 && best > 0) atomicMax(&s_taken, (u64)(wanted + best));
    __syncthreads();
    const i64 end = (i64)s_taken - wanted;   // pops granted in this chunk: the first `end` of them
    for (i64 k = gtid; k < end; k += gthreads) {
      const int i = owner_of(s_grow, n, (uint32_t)k);
      a.tables[(i64)(base + i) * a.max_blocks + s_held[i] + ((uint32_t)k - s_grow[i])] = a.free_ids[top - 1 - (wanted + k)];
    }
    wanted += grow;
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
  extern __shared__ uint32_t s_dyn[];
  __shared__ uint32_t s_tot[ITEMS * 32 + 1];
  const int cap_items = m.R < CHUNK ? m.R : CHUNK;
  uint32_t* s_first = s_dyn;                 // exclusive prefix sums inside the chunk
  int* s_done = reinterpret_cast<int*>(s_dyn + cap_items);
  const int rows = (cap_items + THREADS - 1) / THREADS;
  const i64 t0 = blockIdx.x * m.per_cta, t1 = t0 + m.per_cta < m.max_tokens ? t0 + m.per_cta : m.max_tokens;
  uint32_t bad = 0;
  i64 base_tok = 0;
  for (int base = 0; base < m.R; base += CHUNK) {
    const int n = m.R - base < CHUNK ? m.R - base : CHUNK;
    uint32_t v[ITEMS], sum;                  // sums saturate at 2^32 - 1: no token beyond max_tokens < 2^31 is listed
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      v[i] = 0;
      const int k = i * THREADS + threadIdx.x;
      if (i < rows && k < n) {
        int done, fresh;
        done_new(m, base + k, done, fresh, bad);
        s_done[k] = done;
        v[i] = (uint32_t)fresh;
      }
    }
    scan_chunk(v, rows, s_tot, sum);
    const i64 total = sum;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int k = i * THREADS + threadIdx.x;
      if (i < rows && k < n) {
        s_first[k] = v[i];
        if (blockIdx.x == 0) {
          const i64 at = base_tok + v[i];
          m.offsets[base + k] = at > INT_MAX ? INT_MAX : (int)at;
        }
      }
    }
    __syncthreads();
    const i64 lo = t0 > base_tok ? t0 : base_tok, hi = t1 < base_tok + total ? t1 : base_tok + total;
    for (i64 t = lo + threadIdx.x; t < hi; t += THREADS) {
      const uint32_t k = (uint32_t)(t - base_tok);
      const int i = owner_of(s_first, n, k);
      const int pos = s_done[i] + (int)(k - s_first[i]);
      const int j = pos / m.block_tokens;
      i64 slot = -1;
      if (j < m.max_blocks) {
        const int b = m.tables[(i64)(base + i) * m.max_blocks + j];
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
  const size_t smem = 12 * (size_t)(R < CHUNK ? R : CHUNK);
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
  const size_t smem = 8 * (size_t)(R < CHUNK ? R : CHUNK);
  (void)cudaGetLastError();
  const int rc = allow_smem(map_slots_kernel, smem);
  if (rc) return rc;
  map_slots_kernel<<<(unsigned)grid, THREADS, smem, static_cast<cudaStream_t>(stream)>>>(m);
  return launch_ok();
}
