// ptstore_attend_lse: attention over the paged cache that also writes the logarithm of every row's sum.
#include "attend_dispatch.cuh"

using namespace ptk;

extern "C" int ptstore_attend_lse(const ptstore_attend_t* p, const ptstore_kv_cache_t* cache, void* workspace, uint64_t workspace_bytes, float* lse,
                                  uint32_t* status, ptstore_stream_t stream) {
  if (!lse) return ptstore_attend(p, cache, workspace, workspace_bytes, status, stream);
  return run_attend<true>(p, cache, workspace, workspace_bytes, lse, status, stream);
}
