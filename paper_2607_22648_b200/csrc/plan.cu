// ptstore_assign_blocks / ptstore_map_slots: the paged cache's bookkeeping on the device.  The matched lengths of a
// lookup are on the GPU; so block tables grow and shrink, and new tokens get their slots, without the host seeing a length.
//
// Both are prefix sums over the requests followed by a flat pass over what moves (blocks, tokens), and both are latency bound:
// a few kilobytes to a few megabytes against a launch, two or three dependent memory round trips and a block-wide scan.  So
// each is ONE launch in which every CTA scans all requests for itself (16,384 of them per step, up to 16 per thread, both
// sums of an assignment in one value), and the entries that move are dealt out evenly and find their request by a binary
// search in shared memory.  An assignment is one cluster of eight CTAs: its pops read ids that pushes of other CTAs have written,
// and a cluster's barrier orders the two.  (A pop could find such an id in the tables itself; not done.)  Time on a B200,
// assignment + slots: a decode step of 64 requests 4.5 + 2.8 us; 16,384 requests that push 53,000 blocks, pop 30,000 and list 476,000 tokens
// 32 + 14 us, of which the assignment's scan takes a quarter and its searches in two to eight SMs most of the rest.
#include <cuda_runtime.h>
#include <limits.h>

#include <type_traits>

#include "../../include/ptstore.h"

namespace {

typedef long long i64;
typedef unsigned long long u64;

constexpr int THREADS = 1024;
constexpr int ITEMS = 16;                    // requests of one thread in a batch of more than THREADS (one otherwise)
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

// Exclusive prefix sum inside a warp; the warp's sum in every lane.
template <typename W>
__device__ __forceinline__ W warp_scan(W v, W& sum) {
  const int lane = threadIdx.x & 31;
  W x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const W y = __shfl_up_sync(0xFFFFFFFFu, x, o);
    if (lane >= o) x = plus(x, y);
  }
  sum = __shfl_sync(0xFFFFFFFFu, x, 31);
  x = __shfl_up_sync(0xFFFFFFFFu, x, 1);
  return lane == 0 ? (W)0 : x;
}

// Turns the sums of a chunk's ROWS x 32 warps (row by row) into exclusive prefix sums.  Called by all threads.
template <int ROWS, typename T>
__device__ __forceinline__ void scan_totals(T* s_tot /*[ROWS * 32]*/, T& total, T* s_all) {
  const int lane = threadIdx.x & 31;
  __syncthreads();
  if (threadIdx.x < 32) {                    // lane l: the totals l * ROWS ..
    T sum = 0;
#pragma unroll 4
    for (int k = 0; k < ROWS; ++k) sum = plus(sum, s_tot[lane * ROWS + k]);
    T all, run = warp_scan(sum, all);
    if (lane == 0) *s_all = all;
#pragma unroll 4
    for (int k = 0; k < ROWS; ++k) {
      const T t = s_tot[lane * ROWS + k];
      s_tot[lane * ROWS + k] = run;
      run = plus(run, t);
    }
  }
  __syncthreads();
  total = *s_all;
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
  int R, block_tokens, shift, max_blocks, capacity;           // shift: block_tokens is 2^shift, or -1
  int* tables;
  int* free_ids;
  const int* free_count;
  int* held_out;
  int* free_count_out;
  uint32_t* status;
};

// blocks a request holds and needs; a length its row cannot hold leaves the row as it is
__device__ __forceinline__ void want(const Assign& a, int h, int len, int& held, int& need, uint32_t& bad) {
  held = h < 0 ? 0 : h > a.max_blocks ? a.max_blocks : h;
  if (held != h || len < 0) bad |= PTSTORE_S_BOUNDS;
  const uint32_t n = len <= 0 ? 0 : a.shift >= 0 ? ((uint32_t)(len - 1) >> a.shift) + 1 : (uint32_t)(len - 1) / (uint32_t)a.block_tokens + 1;
  if (n > (uint32_t)a.max_blocks) { need = held; bad |= PTSTORE_S_BOUNDS; } else need = (int)n;
}

// NARROW: 32 requests' blocks fit 16 bits, so a warp scans growth and give-back in one 32-bit value
template <int ROWS, bool NARROW>
__global__ void __cluster_dims__(CLUSTER, 1, 1) __launch_bounds__(THREADS) assign_blocks_kernel(const Assign a) {
  extern __shared__ uint32_t s_dyn[];
  __shared__ u64 s_tot[ROWS * 32], s_all, s_taken;
  constexpr int RUN = ROWS == 1 ? 1 : 8;     // consecutive entries a thread moves: one search, their loads in flight together
  const int cap_items = a.R < ROWS * THREADS ? a.R : ROWS * THREADS;
  uint32_t* s_grow = s_dyn;                  // exclusive prefix sums inside the chunk
  uint32_t* s_back = s_dyn + cap_items;
  uint32_t* s_held = s_dyn + 2 * cap_items;
  const int gtid = blockIdx.x * THREADS + threadIdx.x, gthreads = CLUSTER * THREADS;
  uint32_t bad = 0;
  if (threadIdx.x == 0) s_taken = 0;

  u64 moves = 0;                             // growth of the chunk, and in the upper half what it gives back
  auto scan = [&](int base, int n) {
    using W = typename std::conditional<NARROW, uint32_t, u64>::type;
    constexpr int HALF = NARROW ? 16 : 32, BATCH = ROWS < 4 ? ROWS : 4;
    __syncthreads();                         // nobody moves the last chunk's entries any more
    // four rows' loads at a time; loops stay rolled, since the code of a launch this short comes from afar
#pragma unroll 1
    for (int row = 0; row < ROWS; row += BATCH) {
      int len[BATCH], h[BATCH];
#pragma unroll
      for (int i = 0; i < BATCH; ++i) {      // a request beyond the end reads the last one
        const int k = (row + i) * THREADS + threadIdx.x, r = base + (k < n ? k : n - 1);
        len[i] = a.lengths[r];
        h[i] = a.held ? a.held[r] : 0;
      }
#pragma unroll
      for (int i = 0; i < BATCH; ++i) {
        const int k = (row + i) * THREADS + threadIdx.x;
        int held, need;
        want(a, h[i], len[i], held, need, bad);
        const W v = k >= n ? 0 : need > held ? (W)(need - held) : (W)(held - need) << HALF;
        W sum;
        const W first = warp_scan(v, sum);
        auto wide = [](W x) { return NARROW ? (u64)(x & 0xFFFFu) | (u64)((u64)x >> 16) << 32 : (u64)x; };
        if ((threadIdx.x & 31) == 0) s_tot[(row + i) * 32 + (threadIdx.x >> 5)] = wide(sum);
        if (k < n) {
          s_held[k] = held;
          s_grow[k] = (uint32_t)wide(first);
          s_back[k] = (uint32_t)(wide(first) >> 32);
        }
      }
    }
    scan_totals<ROWS>(s_tot, moves, &s_all);
#pragma unroll 4
    for (int k = threadIdx.x; k < n; k += THREADS) {
      const u64 before = s_tot[k >> 5];
      s_grow[k] += (uint32_t)before;
      s_back[k] += (uint32_t)(before >> 32);
    }
    __syncthreads();
  };
  auto after = [&](const uint32_t* s, int k, int n, uint32_t end) { return k + 1 < n ? s[k + 1] : end; };

  const int c0 = *a.free_count;
  const int count = c0 < 0 ? 0 : c0 > a.capacity ? a.capacity : c0;
  if (count != c0) bad |= PTSTORE_S_BOUNDS;
  // surplus blocks of shrinking rows go onto the stack, in (request, block) order
  i64 pushed = 0;
  for (int base = 0; base < a.R; base += ROWS * THREADS) {
    const int n = a.R - base < ROWS * THREADS ? a.R - base : ROWS * THREADS;
    scan(base, n);
    const uint32_t back = (uint32_t)(moves >> 32);
    for (u64 k = (u64)gtid * RUN; k < back; k += (u64)gthreads * RUN) {
      int i = owner_of(s_back, n, (uint32_t)k), id[RUN];
#pragma unroll
      for (int e = 0; e < RUN; ++e) {
        id[e] = -1;
        if (k + e < back) {
          if (after(s_back, i, n, back) <= (uint32_t)k + e) i = owner_of(s_back, n, (uint32_t)k + e);        // few requests shrink: the next may be far
          const uint32_t first = s_back[i], need = s_held[i] - (after(s_back, i, n, back) - first);
          id[e] = a.tables[(i64)(base + i) * a.max_blocks + need + ((uint32_t)k + e - first)];
        }
      }
#pragma unroll
      for (int e = 0; e < RUN; ++e) {
        const i64 to = count + pushed + (i64)k + e;
        if (k + e < back) {
          if (to < a.capacity) a.free_ids[to] = id[e];
          else bad |= PTSTORE_S_BOUNDS;      // more ids than the stack has room for: the surplus ones are lost
        }
      }
    }
    pushed += back;
  }
  i64 top = count + pushed;
  if (top > a.capacity) top = a.capacity;
  cluster_sync();                            // the pushed ids are visible, and every CTA has read held and free_count

  // growing rows pop from the top; a request is granted its blocks iff all growth up to and including it fits
  i64 wanted = 0;
  for (int base = 0; base < a.R; base += ROWS * THREADS) {
    const int n = a.R - base < ROWS * THREADS ? a.R - base : ROWS * THREADS;
    if (a.R > ROWS * THREADS) {              // a single chunk's sums are still in shared memory
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
    for (i64 k = (i64)gtid * RUN; k < end; k += (i64)gthreads * RUN) {
      int i = owner_of(s_grow, n, (uint32_t)k), id[RUN];
#pragma unroll
      for (int e = 0; e < RUN; ++e) id[e] = k + e < end ? a.free_ids[top - 1 - (wanted + k + e)] : -1;
#pragma unroll
      for (int e = 0; e < RUN; ++e)
        if (k + e < end) {
          while (after(s_grow, i, n, grow) <= (uint32_t)k + e) ++i;         // most requests grow; ends: the last that does reaches `grow`
          a.tables[(i64)(base + i) * a.max_blocks + s_held[i] + ((uint32_t)k + e - s_grow[i])] = id[e];
        }
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
  int done_unit, min_new, R, block_tokens, shift, max_blocks;
  const int* tables;
  i64 max_tokens, per_cta;
  int* offsets;
  i64* slots;
  int* positions;
  uint32_t* status;
};

// tokens of a request that are in the cache already, and new ones
__device__ __forceinline__ void done_new(const MapSlots& m, int len, int d0, int& done, int& fresh, uint32_t& bad) {
  if (len < 0) { len = 0; bad |= PTSTORE_S_BOUNDS; }
  i64 d = (i64)d0 * m.done_unit;
  const i64 most = (i64)len - m.min_new;
  if (d > most) d = most;
  if (d < 0) d = 0;
  done = (int)d;
  fresh = len - done;
}

template <int ROWS>
__global__ void __launch_bounds__(THREADS) map_slots_kernel(const MapSlots m) {
  extern __shared__ uint32_t s_dyn[];
  __shared__ uint32_t s_tot[ROWS * 32], s_all;
  const int cap_items = m.R < ROWS * THREADS ? m.R : ROWS * THREADS;
  uint32_t* s_first = s_dyn;                 // exclusive prefix sums inside the chunk
  int* s_done = reinterpret_cast<int*>(s_dyn + cap_items);
  const i64 t0 = blockIdx.x * m.per_cta, t1 = t0 + m.per_cta < m.max_tokens ? t0 + m.per_cta : m.max_tokens;
  uint32_t bad = 0;
  i64 base_tok = 0;
  for (int base = 0; base < m.R; base += ROWS * THREADS) {
    const int n = m.R - base < ROWS * THREADS ? m.R - base : ROWS * THREADS;
    constexpr int BATCH = ROWS < 4 ? ROWS : 4;
    uint32_t sum;                            // sums saturate at 2^32 - 1: no token beyond max_tokens < 2^31 is listed
#pragma unroll 1
    for (int row = 0; row < ROWS; row += BATCH) {
      int len[BATCH], d[BATCH];
#pragma unroll
      for (int i = 0; i < BATCH; ++i) {      // a request beyond the end reads the last one
        const int k = (row + i) * THREADS + threadIdx.x, r = base + (k < n ? k : n - 1);
        len[i] = m.lengths[r];
        d[i] = m.done ? m.done[r] : 0;
      }
#pragma unroll
      for (int i = 0; i < BATCH; ++i) {
        const int k = (row + i) * THREADS + threadIdx.x;
        int done, fresh;
        done_new(m, len[i], d[i], done, fresh, bad);
        uint32_t all;
        const uint32_t first = warp_scan(k < n ? (uint32_t)fresh : 0u, all);
        if ((threadIdx.x & 31) == 0) s_tot[(row + i) * 32 + (threadIdx.x >> 5)] = all;
        if (k < n) {
          s_done[k] = done;
          s_first[k] = first;
        }
      }
    }
    scan_totals<ROWS>(s_tot, sum, &s_all);
    const i64 total = sum;
#pragma unroll 4
    for (int k = threadIdx.x; k < n; k += THREADS) {
      const uint32_t first = plus(s_first[k], s_tot[k >> 5]);
      s_first[k] = first;
      if (blockIdx.x == 0) {
        const i64 at = base_tok + first;
        m.offsets[base + k] = at > INT_MAX ? INT_MAX : (int)at;
      }
    }
    __syncthreads();
    const i64 lo = t0 > base_tok ? t0 : base_tok, hi = t1 < base_tok + total ? t1 : base_tok + total;
    // four tokens of a thread at a time, THREADS apart: their table loads are in flight together and stores stay coalesced
    constexpr int E = 4;
    for (i64 t = lo + threadIdx.x; t < hi; t += E * THREADS) {
      int pos[E], b[E];
#pragma unroll
      for (int e = 0; e < E; ++e) {
        b[e] = -1;
        if (t + e * THREADS < hi) {
          const uint32_t k = (uint32_t)(t + e * THREADS - base_tok);
          const int i = owner_of(s_first, n, k);
          pos[e] = s_done[i] + (int)(k - s_first[i]);
          const int j = m.shift >= 0 ? pos[e] >> m.shift : pos[e] / m.block_tokens;
          if (j < m.max_blocks) b[e] = m.tables[(i64)(base + i) * m.max_blocks + j];
          else bad |= PTSTORE_S_BOUNDS;
        }
      }
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (t + e * THREADS < hi) {
          const int in = m.shift >= 0 ? pos[e] & (m.block_tokens - 1) : pos[e] % m.block_tokens;
          m.slots[t + e * THREADS] = b[e] >= 0 ? (i64)b[e] * m.block_tokens + in : -1;
          if (m.positions) m.positions[t + e * THREADS] = pos[e];
        }
    }
    base_tok += total;
    __syncthreads();
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    m.offsets[m.R] = base_tok > INT_MAX ? INT_MAX : (int)base_tok;
    if (base_tok > m.max_tokens) bad |= PTSTORE_S_BOUNDS;
  }
  // entries behind the last token are empty slots, so a write of a padded batch skips them
  for (i64 t = (t0 > base_tok ? t0 : base_tok) + threadIdx.x; t < t1; t += THREADS) {
    m.slots[t] = -1;
    if (m.positions) m.positions[t] = -1;
  }
  if (bad) raise_status(m.status, bad);
}

int shift_of(int block_tokens) {             // block_tokens = 2^shift, or -1
  for (int s = 0; s < 31; ++s)
    if (block_tokens == 1 << s) return s;
  return -1;
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
  const Assign a = {lengths, held, R, block_tokens, shift_of(block_tokens), max_blocks, free_capacity, block_tables, free_ids, free_count, held_out, free_count_out, status};
  const size_t smem = 12 * (size_t)(R < CHUNK ? R : CHUNK);
  (void)cudaGetLastError();
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (R <= THREADS) assign_blocks_kernel<1, false><<<CLUSTER, THREADS, smem, st>>>(a);
  else if (max_blocks < 2048) {
    const int rc = allow_smem(assign_blocks_kernel<ITEMS, true>, smem);
    if (rc) return rc;
    assign_blocks_kernel<ITEMS, true><<<CLUSTER, THREADS, smem, st>>>(a);
  } else {
    const int rc = allow_smem(assign_blocks_kernel<ITEMS, false>, smem);
    if (rc) return rc;
    assign_blocks_kernel<ITEMS, false><<<CLUSTER, THREADS, smem, st>>>(a);
  }
  return launch_ok();
}

extern "C" int ptstore_map_slots(const int32_t* lengths, const int32_t* done, int32_t done_unit, int32_t min_new, int32_t R,
                                 const int32_t* block_tables, int32_t max_blocks, int32_t block_tokens, int64_t max_tokens,
                                 int32_t* token_offsets, int64_t* slots, int32_t* positions, uint32_t* status, ptstore_stream_t stream) {
  if (R < 0 || block_tokens < 1 || max_blocks < 1 || max_tokens < 0 || max_tokens > INT_MAX || done_unit < 1 || min_new < 0) return PTSTORE_E_INVAL;
  if (!token_offsets || (max_tokens > 0 && !slots) || (R > 0 && (!lengths || !block_tables))) return PTSTORE_E_INVAL;
  if (R > 1 << 30) return PTSTORE_E_LIMIT;
  MapSlots m = {lengths, done, done_unit, min_new, R, block_tokens, shift_of(block_tokens), max_blocks, block_tables, max_tokens, 0, token_offsets,
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
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (R <= THREADS) map_slots_kernel<1><<<(unsigned)grid, THREADS, smem, st>>>(m);
  else {
    const int rc = allow_smem(map_slots_kernel<ITEMS>, smem);
    if (rc) return rc;
    map_slots_kernel<ITEMS><<<(unsigned)grid, THREADS, smem, st>>>(m);
  }
  return launch_ok();
}
