// Token-level cache in pages: handing out pages and slots on the GPU (page_plan), and writing rows into their slots, as they
// are (store_rows) or in 8 bits (store_rows_e4m3).
#include <cuda_fp16.h>

#include "wk_internal.cuh"

namespace wk {
namespace {

// ---------------------------------------------------------------- page_plan
constexpr int kPlanThreads = 1024;
constexpr int kPlanPer = kPlanMaxReq / kPlanThreads;   // requests per thread, consecutive
constexpr int kPlanTokens = 4 * kPlanThreads;          // new tokens per block and round

__device__ __forceinline__ void report(uint32_t* status, uint32_t bits) {
  if (status) atomicOr(status, bits);
}

// Exclusive prefix of v over the block (all threads call it); the sum of all goes to *total.
__device__ int64_t block_prefix(int64_t v, int64_t* total) {
  __shared__ int64_t part[kPlanThreads / 32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int64_t up = v;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int64_t o = __shfl_up_sync(0xffffffffu, up, d);
    if (lane >= d) up += o;
  }
  __syncthreads();   // `part` may still be read from the call before
  if (lane == 31) part[warp] = up;
  __syncthreads();
  int64_t w = part[lane];
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int64_t o = __shfl_up_sync(0xffffffffu, w, d);
    if (lane >= d) w += o;
  }
  *total = __shfl_sync(0xffffffffu, w, 31);
  return up - v + (warp ? __shfl_sync(0xffffffffu, w, warp - 1) : 0);
}

// Pages that hold so many tokens (a negative count stands for no request and has none).
__device__ __forceinline__ int64_t pages_of(int64_t tokens, int page) {
  return tokens > 0 ? static_cast<int64_t>((static_cast<uint32_t>(tokens) - 1u) / static_cast<uint32_t>(page)) + 1 : 0;
}

// Last index i of a[0 .. n) (ascending, a[0] <= x) with a[i] <= x.
__device__ __forceinline__ int last_at_most(const int32_t* a, int n, int32_t x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a[mid] <= x) lo = mid; else hi = mid;
  }
  return lo;
}

// Every block computes the prefix sums over all requests (a few thousand at most: one read of two short arrays, two
// scans) and then fills its share of the new tokens' slots, each on its own: whose token it is by a search in the prefix, its page from
// the table or straight from the ring.  What is read that this call also changes (lengths, ring state) is changed by the block
// that finishes last; ring places given out and ring places filled never coincide, because free and returned pages together are at most
// n_pages.  Block 0 also puts the pages of ended requests back.  Bound by latency: one launch, two dependent loads, two scans.
__global__ void __launch_bounds__(kPlanThreads)
page_plan(const __grid_constant__ PlanArgs a) {
  __shared__ int32_t start[kPlanMaxReq + 1];   // first row; later: the ended requests' first returned entry
  __shared__ int32_t place[kPlanMaxReq];       // ring offset of the request's table column 0, or kRefused; later: ended requests
  __shared__ int32_t n_ended, last;
  constexpr int32_t kRefused = INT32_MIN;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int B = a.n_req, page = a.page_tokens;
  int32_t head = a.state[0], count = a.state[1];
  uint32_t bad = 0;
  if (head < 0 || head >= a.n_pages || count < 0 || count > a.n_pages) {
    head = count = 0;
    bad = WK_DEV_BAD_SLOT;
  }
  const int per = (B + kPlanThreads - 1) / kPlanThreads, r0 = tid * per;
  int32_t len[kPlanPer], more[kPlanPer];
  int64_t sum = 0;
#pragma unroll
  for (int i = 0; i < kPlanPer; ++i) {
    const bool on = i < per && r0 + i < B;
    len[i] = on ? a.lens[r0 + i] : -1;
    more[i] = on ? a.more[r0 + i] : 0;
    sum += max(more[i], 0);
  }
  int64_t rows;
  int64_t at = block_prefix(sum, &rows);
  int64_t need[kPlanPer], needs = 0;
  bool fits[kPlanPer];
#pragma unroll
  for (int i = 0; i < kPlanPer; ++i) {
    if (i < per && r0 + i < B) start[r0 + i] = static_cast<int32_t>(min(at, static_cast<int64_t>(INT32_MAX)));
    const int64_t n = max(more[i], 0);
    at += n;
    const int64_t after = pages_of(len[i] + n, page);
    fits[i] = len[i] >= 0 && n > 0 && len[i] + n <= INT32_MAX && after <= a.max_pages && at <= a.max_tokens;
    need[i] = fits[i] ? after - pages_of(len[i], page) : 0;
    needs += need[i];
  }
  if (tid == 0) start[B] = static_cast<int32_t>(min(rows, static_cast<int64_t>(INT32_MAX)));
  int64_t asked;
  int64_t upto = block_prefix(needs, &asked);
  int64_t taken = 0;
  bool ended = false;
#pragma unroll
  for (int i = 0; i < kPlanPer; ++i) {
    if (i >= per || r0 + i >= B) continue;
    const bool granted = fits[i] && (need[i] == 0 || upto + need[i] <= count);
    // (granted: upto and the columns are below 2^31, so is their difference)
    place[r0 + i] = granted ? static_cast<int32_t>(need[i] ? upto - pages_of(len[i], page) : 0) : kRefused;
    if (granted) taken += need[i];
    else if (more[i] > 0) bad |= WK_DEV_POOL_FULL;
    if (more[i] < 0 && len[i] >= 0) ended = true;
    upto += need[i];
    fits[i] = granted;
  }
  int64_t popped;
  block_prefix(taken, &popped);
  __syncthreads();

  // slots of the new tokens
  for (int64_t t0 = static_cast<int64_t>(blockIdx.x) * kPlanTokens; t0 < a.max_tokens; t0 += static_cast<int64_t>(gridDim.x) * kPlanTokens) {
#pragma unroll
    for (int i = 0; i < kPlanTokens / kPlanThreads; ++i) {
      const int64_t t = t0 + i * kPlanThreads + tid;
      if (t >= a.max_tokens) break;
      int32_t slot = -1;
      if (t < rows) {
        // (rows before t are rows of requests that have some: the last start that is at most t is that of t's own)
        const int r = last_at_most(start, B, static_cast<int32_t>(t));
        if (place[r] != kRefused) {
          const int64_t held = a.lens[r], pos = held + t - start[r];
          const int32_t col = static_cast<int32_t>(static_cast<uint32_t>(pos) / static_cast<uint32_t>(page));
          int32_t* entry = a.tables + r * a.table_stride + col;
          int32_t id;
          if (col >= pages_of(held, page)) {
            const int64_t ix = static_cast<int64_t>(head) + place[r] + col;
            id = a.ring[ix < a.n_pages ? ix : ix - a.n_pages];
            if (pos == static_cast<int64_t>(col) * page) *entry = id;   // the page's first token enters it
          } else {
            id = *entry;
          }
          if (id >= 0 && id < a.n_pages) slot = static_cast<int32_t>(static_cast<int64_t>(id) * page + pos - static_cast<int64_t>(col) * page);
          else bad |= WK_DEV_BAD_SLOT;
        }
      }
      a.slots[t] = slot;
    }
  }
  for (int64_t r = blockIdx.x * static_cast<int64_t>(kPlanThreads) + tid; r <= B; r += static_cast<int64_t>(gridDim.x) * kPlanThreads)
    a.starts[r] = start[r];

  // pages of ended requests go behind the ring's last free page
  int64_t pushed = 0;
  if (blockIdx.x == 0 && __syncthreads_or(ended)) {   // (also: nobody reads start and place any more)
    int64_t mine = 0, entries = 0, n_list, n_entries;
#pragma unroll
    for (int i = 0; i < kPlanPer; ++i)
      if (more[i] < 0 && len[i] >= 0) {
        ++mine;
        entries += min(pages_of(len[i], page), static_cast<int64_t>(a.max_pages));
      }
    int64_t li = block_prefix(mine, &n_list), e0 = block_prefix(entries, &n_entries);
#pragma unroll
    for (int i = 0; i < kPlanPer; ++i)
      if (more[i] < 0 && len[i] >= 0) {
        place[li] = r0 + i;
        start[li] = static_cast<int32_t>(e0);   // fewer than 2^31: n_req * max_pages is
        ++li;
        e0 += min(pages_of(len[i], page), static_cast<int64_t>(a.max_pages));
      }
    __syncthreads();
    const int list = static_cast<int>(n_list);
    // each warp takes a run of the entries: counts those that are pages, then writes them behind those of the warps before it
    const int64_t run = (n_entries + 32 * 32 - 1) / (32 * 32) * 32, w0 = warp * run, w1 = min(w0 + run, n_entries);
    auto entry_at = [&](int64_t e) -> int32_t {
      if (e >= w1) return -1;
      const int k = last_at_most(start, list, static_cast<int32_t>(e));
      return a.tables[place[k] * a.table_stride + (e - start[k])];
    };
    int64_t found = 0;
    for (int64_t e = w0; e < w1; e += 128) {
      int32_t id[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) id[u] = entry_at(e + 32 * u + lane);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const bool ok = id[u] >= 0 && id[u] < a.n_pages;
        if (!ok && id[u] != -1) bad |= WK_DEV_BAD_SLOT;
        found += __popc(__ballot_sync(0xffffffffu, ok));
      }
    }
    int64_t k0 = block_prefix(lane == 0 ? found : 0, &pushed);
    k0 = __shfl_sync(0xffffffffu, k0, 0);
    const int64_t room = a.n_pages - count;   // ring places behind the free pages
    if (pushed > room) bad |= WK_DEV_BAD_SLOT;
    pushed = min(pushed, room);
    for (int64_t e = w0; e < w1; e += 128) {
      int32_t id[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) id[u] = entry_at(e + 32 * u + lane);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const bool ok = id[u] >= 0 && id[u] < a.n_pages;
        const uint32_t all = __ballot_sync(0xffffffffu, ok);
        const int64_t k = k0 + __popc(all & ((1u << lane) - 1));
        if (ok && k < room) a.ring[(static_cast<int64_t>(head) + count + k) % a.n_pages] = id[u];
        k0 += __popc(all);
      }
    }
  }
  if (bad) report(a.status, bad);

  // The block that arrives last writes lengths and ring state: all others have read them.
  if (gridDim.x > 1) {
    if (blockIdx.x == 0 && tid == 0) {
      *reinterpret_cast<volatile int32_t*>(a.state + 3) = static_cast<int32_t>(pushed);
      __threadfence();
    }
    __syncthreads();
    if (tid == 0) {
      __threadfence();
      last = atomicInc(reinterpret_cast<uint32_t*>(a.state + 2), gridDim.x - 1) == gridDim.x - 1;
      __threadfence();
    }
    __syncthreads();
    if (!last) return;
    pushed = *reinterpret_cast<volatile int32_t*>(a.state + 3);
    __syncthreads();
  } else {
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < kPlanPer; ++i)
    if (i < per && r0 + i < B) a.lens_out[r0 + i] = more[i] < 0 && len[i] >= 0 ? 0 : fits[i] ? len[i] + more[i] : len[i];
  if (tid == 0) {
    const int64_t h = static_cast<int64_t>(head) + popped;
    a.state[2] = a.state[3] = 0;
    a.state_out[0] = static_cast<int32_t>(h < a.n_pages ? h : h - a.n_pages);
    a.state_out[1] = static_cast<int32_t>(count - popped + pushed);
    a.state_out[2] = a.state_out[3] = 0;
  }
}

// ---------------------------------------------------------------- page_store
constexpr int kStoreThreads = 256;
constexpr int kStoreLoads = 4;   // 16-byte loads in flight per thread

struct StoreArgs {
  wk_paged_kv c;
  const uint8_t *src[2];
  int64_t row_bytes;      // from one source row to the next
  int32_t n_tokens, rows; // rows per block
  const int32_t* slots;
  uint32_t* status;
};

// The slot's page and place in it; false: nothing to write.
__device__ __forceinline__ bool slot_place(const StoreArgs& a, int32_t token, int64_t* page, int64_t* off) {
  const int32_t slot = a.slots[token];
  const int32_t id = slot / a.c.page_tokens;
  if (slot < 0 || id >= a.c.n_pages) {
    if (slot != -1) report(a.status, WK_DEV_BAD_SLOT);
    return false;
  }
  *page = id;
  *off = slot - id * a.c.page_tokens;
  return true;
}

// Copies rows: bound by memory.  A block takes K or V of a few rows; each thread moves four 16-byte vectors, all loads before the
// first store.  head_dim is 64 or 128, so a head is 8 or 16 vectors.
__global__ void __launch_bounds__(kStoreThreads)
store_rows(const __grid_constant__ StoreArgs a) {
  const int side = blockIdx.y;
  const int head_shift = a.c.head_dim == 128 ? 4 : 3;
  const int vecs = a.c.n_kv_heads << head_shift;
  const int32_t t0 = blockIdx.x * a.rows, n = min(a.rows, a.n_tokens - t0);
  uint8_t* dst = static_cast<uint8_t*>(side ? a.c.V : a.c.K);
  const int64_t total = static_cast<int64_t>(n) * vecs;
  for (int64_t i0 = threadIdx.x; i0 < total; i0 += kStoreLoads * kStoreThreads) {
    uint4 q[kStoreLoads];
    uint4* to[kStoreLoads];
#pragma unroll
    for (int u = 0; u < kStoreLoads; ++u) {
      const int64_t i = i0 + u * kStoreThreads;
      to[u] = nullptr;
      if (i >= total) continue;
      const int r = a.rows == 1 ? 0 : static_cast<int>(static_cast<uint32_t>(i) / static_cast<uint32_t>(vecs));
      const int v = static_cast<int>(i - static_cast<int64_t>(r) * vecs);
      int64_t page, off;
      if (!slot_place(a, t0 + r, &page, &off)) continue;
      const int h = v >> head_shift, w = v & ((1 << head_shift) - 1);
      to[u] = reinterpret_cast<uint4*>(dst + 2 * (page * a.c.page_stride + off * a.c.token_stride + h * a.c.head_stride)) + w;
      q[u] = __ldcs(reinterpret_cast<const uint4*>(a.src[side] + static_cast<int64_t>(t0 + r) * a.row_bytes) + v);
    }
#pragma unroll
    for (int u = 0; u < kStoreLoads; ++u)
      if (to[u]) *to[u] = q[u];
  }
}

__device__ __forceinline__ void unpack2(uint32_t w, bool bf16, float* lo, float* hi) {
  if (bf16) {
    *lo = __uint_as_float(w << 16);
    *hi = __uint_as_float(w & 0xffff0000u);
  } else {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
    *lo = f.x;
    *hi = f.y;
  }
}

// Rows in 8 bits: a row (one token, one head) belongs to head_dim / 8 neighbouring lanes, 16 bytes each.  The exponent is read off the
// bits of the largest magnitude: amax = m * 2^x with 1 <= m < 2 fits 448 * 2^e = 1.75 * 2^(e + 8) for e = x - 8 if m <= 1.75, else
// for x - 7.  A power of two keeps the scaling exact (the one rounding is that to the code) and costs a byte per row; codes of 17
// binades leave no accuracy to be won from a finer scale.
template <bool BF16>
__global__ void __launch_bounds__(kStoreThreads)
store_rows_e4m3(const __grid_constant__ StoreArgs a) {
  const int side = blockIdx.y;
  const int head_shift = a.c.head_dim == 128 ? 4 : 3;
  const int vecs = a.c.n_kv_heads << head_shift;
  const int32_t t0 = blockIdx.x * a.rows, n = min(a.rows, a.n_tokens - t0);
  uint8_t* dst = static_cast<uint8_t*>(side ? a.c.V : a.c.K);
  uint8_t* exps = side ? a.c.V_exp : a.c.K_exp;
  const int64_t total = static_cast<int64_t>(n) * vecs;   // a multiple of the lanes that share a row
  const int64_t rounds = (total + kStoreLoads * kStoreThreads - 1) / (kStoreLoads * kStoreThreads);
  for (int64_t k = 0; k < rounds; ++k) {   // the same number for all lanes: they exchange values
    uint4 q[kStoreLoads];
#pragma unroll
    for (int u = 0; u < kStoreLoads; ++u) {
      const int64_t i = (k * kStoreLoads + u) * kStoreThreads + threadIdx.x;
      q[u] = make_uint4(0, 0, 0, 0);
      if (i >= total) continue;
      const int r = a.rows == 1 ? 0 : static_cast<int>(static_cast<uint32_t>(i) / static_cast<uint32_t>(vecs));
      q[u] = __ldcs(reinterpret_cast<const uint4*>(a.src[side] + static_cast<int64_t>(t0 + r) * a.row_bytes) + (i - static_cast<int64_t>(r) * vecs));
    }
#pragma unroll
    for (int u = 0; u < kStoreLoads; ++u) {
      const int64_t i = (k * kStoreLoads + u) * kStoreThreads + threadIdx.x;
      const uint32_t w[4] = {q[u].x, q[u].y, q[u].z, q[u].w};
      float x[8], top = 0.f;
      bool odd = false;
#pragma unroll
      for (int j = 0; j < 4; ++j) unpack2(w[j], BF16, &x[2 * j], &x[2 * j + 1]);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const bool fine = fabsf(x[j]) <= 3.402823466e38f;
        if (fine) top = fmaxf(top, fabsf(x[j]));
        else { x[j] = __int_as_float(0x7fffffff); odd = true; }
      }
      for (int d = 1; d < (1 << head_shift); d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
      // byte = e + 127; a bf16 below the normal numbers reads x = -127 here and ends at the least exponent, as it should
      const uint32_t bits = __float_as_uint(top);
      const int byte = top == 0.f ? 127 : max(1, static_cast<int>(bits >> 23) - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0));
      if (i >= total) continue;
      const int r = a.rows == 1 ? 0 : static_cast<int>(static_cast<uint32_t>(i) / static_cast<uint32_t>(vecs));
      const int v = static_cast<int>(i - static_cast<int64_t>(r) * vecs);
      int64_t page, off;
      if (!slot_place(a, t0 + r, &page, &off)) continue;
      if (odd) report(a.status, WK_DEV_NONFINITE);
      const float scale = __uint_as_float(static_cast<uint32_t>(254 - byte) << 23);   // 2^-e; byte is at most 247
      uint32_t code[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        uint16_t lo, hi;
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(x[4 * j + 1] * scale), "f"(x[4 * j] * scale));
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(x[4 * j + 3] * scale), "f"(x[4 * j + 2] * scale));
        code[j] = lo | static_cast<uint32_t>(hi) << 16;
      }
      const int h = v >> head_shift, l = v & ((1 << head_shift) - 1);
      *reinterpret_cast<uint2*>(dst + page * a.c.page_stride + off * a.c.token_stride + h * a.c.head_stride + 8 * l) =
          make_uint2(code[0], code[1]);
      if (l == 0) exps[(page * a.c.n_kv_heads + h) * a.c.page_tokens + off] = static_cast<uint8_t>(byte);
    }
  }
}

}  // namespace

wk_status launch_page_plan(wk_ctx* ctx, const PlanArgs& a, cudaStream_t s) {
  // Up to 4,096 new tokens one block does it all; more are spread.
  const int64_t blocks = (static_cast<int64_t>(a.max_tokens) + kPlanTokens - 1) / kPlanTokens;
  const int grid = blocks < 1 ? 1 : blocks < ctx->sm_count ? static_cast<int>(blocks) : ctx->sm_count;
  page_plan<<<grid, kPlanThreads, 0, s>>>(a);
  return after_launch(ctx);
}

wk_status launch_page_store(wk_ctx* ctx, const wk_paged_kv& c, const void* K_new, const void* V_new, int src_type, int n_tokens,
                            int64_t row_stride, const int32_t* slots, cudaStream_t s) {
  StoreArgs a;
  a.c = c;
  a.src[0] = static_cast<const uint8_t*>(K_new);
  a.src[1] = static_cast<const uint8_t*>(V_new);
  a.row_bytes = row_stride * 2;
  a.n_tokens = n_tokens;
  a.slots = slots;
  a.status = ctx->bound ? ctx->status_dev : nullptr;
  const int64_t vecs = static_cast<int64_t>(c.n_kv_heads) * c.head_dim / 8;
  const int64_t rows = kStoreLoads * kStoreThreads / vecs;
  a.rows = rows > 1 ? static_cast<int>(rows) : 1;
  const dim3 grid(static_cast<unsigned>((n_tokens + a.rows - 1) / a.rows), 2);
  if (c.type != WK_E4M3) store_rows<<<grid, kStoreThreads, 0, s>>>(a);
  else if (src_type == WK_BF16) store_rows_e4m3<true><<<grid, kStoreThreads, 0, s>>>(a);
  else store_rows_e4m3<false><<<grid, kStoreThreads, 0, s>>>(a);
  return after_launch(ctx);
}

}  // namespace wk
