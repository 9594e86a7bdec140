// Stand-ins for the launchers of the token-level cache: a call that reaches one has passed the argument checks of
// csrc/wk_paged_api.cu.
#include "wk_internal.cuh"

extern "C" {
int launched = 0;
int last_max_pages = 0, last_window = 0, last_sink = 0;
float last_scale = 0.f;
}

namespace wk {
wk_status launch_page_plan(wk_ctx*, const PlanArgs&, cudaStream_t) { return ++launched, WK_OK; }
wk_status launch_page_store(wk_ctx*, const wk_paged_kv&, const void*, const void*, int, int, int64_t, const int32_t*, cudaStream_t) {
  return ++launched, WK_OK;
}
wk_status launch_paged_attention(wk_ctx*, const PagedArgs& a, cudaStream_t) {
  last_max_pages = a.max_pages;
  last_window = a.window;
  last_sink = a.sink;
  last_scale = a.scale;
  return ++launched, WK_OK;
}
size_t paged_scratch_bytes(int) { return 512; }
}  // namespace wk
