// ptstore_attend: attention over the paged cache.
#include "attend_dispatch.cuh"

using namespace ptk;

extern "C" uint64_t ptstore_attend_workspace_bytes(uint32_t head_dim) {
  if (head_dim != 64 && head_dim != 128) return 0;
  // counters, then two parts per CTA of the split kernel (of 8 rows where 4 CTAs share an SM, of 16 where 2 do), or one of 256 rows per SM
  static_assert(MAX_SMS * 4 * 4 <= PR_PARTS_AT && MAX_SMS * 4 * 4 <= SP_PARTS_AT, "parts lie behind the counters of any grid");
  const u64 split = SP_PARTS_AT + (u64)MAX_SMS * 4 * 2 * 8 * (head_dim + 2) * 4;
  const u64 prompt = PR_PARTS_AT + (u64)MAX_SMS * PR_ROWS * (head_dim + 2) * 4;
  return split > prompt ? split : prompt;
}

extern "C" int ptstore_attend(const ptstore_attend_t* p, const ptstore_kv_cache_t* cache, void* workspace, uint64_t workspace_bytes,
                              uint32_t* status, ptstore_stream_t stream) {
  return run_attend<false>(p, cache, workspace, workspace_bytes, nullptr, status, stream);
}
