// C-ABI entry points of the token-level cache in pages: argument checks.  Every device-side step lives in wk_pages.cu and
// wk_paged_attention.cu; nothing here computes.
#include <math.h>

#include "wk_internal.cuh"

namespace wk {

// Whether a cache description is one that the kernels can read and write anywhere in bounds of what it describes.
static wk_status check_cache(const wk_paged_kv* c) {
  if (!c || !c->K || !c->V || !aligned16(c->K) || !aligned16(c->V)) return WK_ERR_ARG;
  if (c->type != WK_BF16 && c->type != WK_F16 && c->type != WK_E4M3) return WK_ERR_ARG;
  if (c->head_dim != 64 && c->head_dim != 128) return WK_ERR_ARG;
  if (c->n_pages < 1 || c->page_tokens < 1 || c->n_kv_heads < 1 || c->reserved != 0) return WK_ERR_ARG;
  if ((c->type == WK_E4M3) != (c->K_exp != nullptr) || (c->type == WK_E4M3) != (c->V_exp != nullptr)) return WK_ERR_ARG;
  if ((reinterpret_cast<uintptr_t>(c->K_exp) & 3u) || (reinterpret_cast<uintptr_t>(c->V_exp) & 3u)) return WK_ERR_ARG;
  const int64_t unit = c->type == WK_E4M3 ? 16 : 8;   // elements in 16 bytes
  // From the innermost axis out, each stride steps over all of what the axis inside it covers: no two rows share a byte.
  struct { int64_t stride, n; } ax[3] = {{c->page_stride, c->n_pages}, {c->token_stride, c->page_tokens}, {c->head_stride, c->n_kv_heads}};
  for (const auto& x : ax)
    if (x.n > 1 && (x.stride < 0 || x.stride % unit)) return WK_ERR_ARG;
  double covered = c->head_dim;
  for (int pass = 0; pass < 3; ++pass) {
    int best = -1;
    for (int i = 0; i < 3; ++i)
      if (ax[i].n > 1 && (best < 0 || ax[i].stride < ax[best].stride)) best = i;
    if (best < 0) break;
    if (ax[best].stride < covered) return WK_ERR_ARG;
    covered = static_cast<double>(ax[best].stride) * ax[best].n;
    ax[best].n = 1;
  }
  // the kernels count places of tokens in 16-byte units of 32 bits, a head's beside them
  const double most = 4294967295.0 * 16 / (c->type == WK_E4M3 ? 1 : 2);   // elements
  if (static_cast<double>(c->n_pages - 1) * c->page_stride + static_cast<double>(c->page_tokens - 1) * c->token_stride >= most) return WK_ERR_SHAPE;
  if (c->n_kv_heads > 1 && c->head_stride >= most) return WK_ERR_SHAPE;
  const int64_t tokens = static_cast<int64_t>(c->n_pages) * c->page_tokens;
  if (tokens > 0x7fffffffLL || (c->type == WK_E4M3 && tokens * c->n_kv_heads > 0xffffffffLL)) return WK_ERR_SHAPE;
  return WK_OK;
}

static bool source_fits(const wk_paged_kv* c, int32_t type) {
  return c->type == WK_E4M3 ? type == WK_BF16 || type == WK_F16 : type == c->type;
}

}  // namespace wk

using namespace wk;

extern "C" {

wk_status wk_page_plan(wk_ctx* ctx, int32_t n_pages, int32_t page_tokens, int32_t n_req, const int32_t* lens,
                       const int32_t* new_tokens, int32_t* lens_out, int32_t* tables, int32_t max_pages,
                       int64_t table_stride, int32_t* ring, int32_t* state, int32_t* state_out, int32_t max_tokens,
                       int32_t* slots_out, int32_t* starts_out, void* stream) {
  if (!ctx || !lens || !new_tokens || !lens_out || !tables || !ring || !state || !state_out || !starts_out) return WK_ERR_ARG;
  if (n_pages < 1 || page_tokens < 1 || n_req < 1 || max_pages < 1 || max_tokens < 0) return WK_ERR_ARG;
  if ((max_tokens > 0 && !slots_out) || (n_req > 1 && table_stride < max_pages)) return WK_ERR_ARG;
  if (n_req > kPlanMaxReq || static_cast<int64_t>(n_req) * max_pages > 0x7fffffffLL) return WK_ERR_SHAPE;
  if (static_cast<int64_t>(n_pages) * page_tokens > 0x7fffffffLL) return WK_ERR_SHAPE;
  WK_USE_DEVICE(ctx);
  const PlanArgs a{n_pages, page_tokens, n_req, lens, new_tokens, lens_out, tables, max_pages, table_stride, ring, state,
                   state_out, max_tokens, slots_out, starts_out, ctx->bound ? ctx->status_dev : nullptr};
  return launch_page_plan(ctx, a, static_cast<cudaStream_t>(stream));
}

wk_status wk_page_store(wk_ctx* ctx, const wk_paged_kv* cache, const void* K_new, const void* V_new, int32_t src_type,
                        int32_t n_tokens, int64_t row_stride, const int32_t* slots, void* stream) {
  if (!ctx || n_tokens < 0) return WK_ERR_ARG;
  const wk_status st = check_cache(cache);
  if (st != WK_OK) return st;
  if (!source_fits(cache, src_type)) return WK_ERR_ARG;
  if (n_tokens == 0) return WK_OK;
  if (!K_new || !V_new || !slots || !aligned16(K_new) || !aligned16(V_new)) return WK_ERR_ARG;
  if (n_tokens > 1 && (row_stride % 8 || row_stride < static_cast<int64_t>(cache->n_kv_heads) * cache->head_dim))
    return WK_ERR_ARG;
  if (static_cast<int64_t>(n_tokens) * cache->n_kv_heads > 0x7fffffffLL || row_stride / 8 > 0x7fffffffLL) return WK_ERR_SHAPE;
  WK_USE_DEVICE(ctx);
  return launch_page_store(ctx, *cache, K_new, V_new, src_type, n_tokens, row_stride, slots,
                           static_cast<cudaStream_t>(stream));
}

size_t wk_paged_scratch_bytes(const wk_ctx* ctx) { return ctx ? paged_scratch_bytes(ctx->sm_count) : 0; }

wk_status wk_paged_attention(wk_ctx* ctx, const wk_paged_kv* cache, const void* Q, int32_t q_type, int64_t q_stride,
                             int32_t n_req, int32_t n_heads, const int32_t* tables, int32_t max_pages,
                             int64_t table_stride, const int32_t* lens, int32_t window, int32_t sink,
                             float softmax_scale, void* O, float* lse_out, void* scratch, size_t scratch_bytes,
                             void* stream) {
  if (!ctx || !Q || !O || !tables || !lens || !scratch) return WK_ERR_ARG;
  const wk_status st = check_cache(cache);
  if (st != WK_OK) return st;
  if (!source_fits(cache, q_type) || n_req < 1 || n_heads < 1 || max_pages < 1 || window < 0 || sink < 0) return WK_ERR_ARG;
  if (!(softmax_scale >= 0.f) || isinf(softmax_scale)) return WK_ERR_ARG;
  if (!aligned16(Q) || !aligned16(O) || (reinterpret_cast<uintptr_t>(scratch) & 255u)) return WK_ERR_ARG;
  if (n_req > 1 && (q_stride % 8 || q_stride < static_cast<int64_t>(n_heads) * cache->head_dim)) return WK_ERR_ARG;
  if (n_req > 1 && table_stride < max_pages) return WK_ERR_ARG;
  if (n_heads % cache->n_kv_heads) return WK_ERR_SHAPE;
  if (scratch_bytes < paged_scratch_bytes(ctx->sm_count)) return WK_ERR_SHAPE;
  // positions are 32-bit; a table longer than that cannot be used to its end
  const int64_t room = 0x7fffffffLL / cache->page_tokens;
  WK_USE_DEVICE(ctx);
  PagedArgs a;
  a.c = *cache;
  a.Q = Q;
  a.q_stride = q_stride;
  a.q_type = q_type;
  a.n_req = n_req;
  a.n_heads = n_heads;
  a.tables = tables;
  a.max_pages = max_pages < room ? max_pages : static_cast<int32_t>(room);
  a.table_stride = table_stride;
  a.lens = lens;
  const bool all = window == 0 || static_cast<int64_t>(window) + sink > 0x7fffffffLL;
  a.window = all ? 0 : window;
  a.sink = all ? 0 : sink;
  a.scale = softmax_scale > 0.f ? softmax_scale : 1.f / sqrtf(static_cast<float>(cache->head_dim));
  a.O = O;
  a.lse = lse_out;
  a.scratch = static_cast<uint8_t*>(scratch);
  a.status = ctx->bound ? ctx->status_dev : nullptr;
  return launch_paged_attention(ctx, a, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
