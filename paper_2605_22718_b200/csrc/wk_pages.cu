// Token-level cache in pages: handing out pages and slots on the GPU (page_plan), and writing rows into their slots, as they
// are (store_rows) or in 8 bits (store_rows_e4m3).
#include <cuda_fp16.h>

#include "wk_internal.cuh"

namespace wk {
namespace {

// ---------------------------------------------------------------- page_plan
constexpr int kPlanPer = 4;      // requests per thread, consecutive

__device__ __forceinline__ void report(uint32_t* status, uint32_t bits) {
  if (status) atomicOr(status, bits);
}

// Pages that hold so many tokens (a negative count stands for no request and has none).
__device__ __forceinline__ uint32_t pages_of(int64_t tokens, int page) {
  return tokens > 0 ? (static_cast<uint32_t>(tokens) - 1u) / static_cast<uint32_t>(page) + 1 : 0;
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

// What is summed over the requests.
struct Sums {
  int64_t rows;       // new tokens
  uint32_t need;      // pages asked for (n_req * max_pages at most)
  uint32_t ended, entries;   // ended requests and the table entries that they give back
  __device__ __forceinline__ void add(const Sums& o) { rows += o.rows; need += o.need; ended += o.ended; entries += o.entries; }
};
__device__ __forceinline__ Sums warp_inclusive(Sums v, int lane) {
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const Sums o{__shfl_up_sync(0xffffffffu, v.rows, d), __shfl_up_sync(0xffffffffu, v.need, d),
                 __shfl_up_sync(0xffffffffu, v.ended, d), __shfl_up_sync(0xffffffffu, v.entries, d)};
    if (lane >= d) v.add(o);
  }
  return v;
}

// Every block computes the prefix sums over all requests (one read of two short arrays, one scan) and then fills its share of
// the new tokens' slots, each on its own: whose token it is by a search in the prefix, its page from the table or straight from
// the ring.  What is read that this call also changes (lengths, ring state) is changed by the block that finishes last; ring
// places given out and ring places filled never coincide, because free and returned pages together are at most n_pages.  Block 0
// also puts the pages of ended requests back.  Bound by latency: one launch, a scan, two or three dependent loads.
template <int THREADS>
__global__ void __launch_bounds__(THREADS)
page_plan(const __grid_constant__ PlanArgs a) {
  constexpr int kReq = kPlanPer * THREADS, kWarps = THREADS / 32, kTokens = 4 * THREADS;
  constexpr int32_t kRefused = INT32_MIN;
  __shared__ int32_t start[kReq + 1];   // first row; later: the ended requests' first returned entry
  __shared__ int32_t place[kReq];       // ring offset of the request's table column 0, or kRefused; later: ended requests
  __shared__ Sums part[kWarps];
  __shared__ uint32_t popped, found_by[kWarps];
  __shared__ int32_t last;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  dep_release();
  dep_wait();   // nothing is read or written before the kernel in front has ended
  const int B = a.n_req, page = a.page_tokens;
  int32_t head = a.state[0], count = a.state[1];
  uint32_t bad = 0;
  if (head < 0 || head >= a.n_pages || count < 0 || count > a.n_pages) {
    head = count = 0;
    bad = WK_DEV_BAD_SLOT;
  }
  const int per = (B + THREADS - 1) / THREADS, r0 = tid * per;
  int32_t len[kPlanPer], more[kPlanPer];
#pragma unroll
  for (int i = 0; i < kPlanPer; ++i) {
    const bool on = i < per && r0 + i < B;
    len[i] = on ? a.lens[r0 + i] : -1;
    more[i] = on ? a.more[r0 + i] : 0;
  }
  // Rows past max_tokens are those of the last requests that bring any, so that these may be counted among the ones that ask for
  // pages: they come behind all that are granted.
  uint32_t have[kPlanPer], need[kPlanPer];
  bool fits[kPlanPer];
  Sums mine{0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < kPlanPer; ++i) {
    const int64_t n = max(more[i], 0);
    have[i] = pages_of(len[i], page);
    const uint32_t after = pages_of(len[i] + n, page);
    fits[i] = len[i] >= 0 && n > 0 && len[i] + n <= INT32_MAX && after <= static_cast<uint32_t>(a.max_pages);
    need[i] = fits[i] ? after - have[i] : 0;
    const bool ended = more[i] < 0 && len[i] >= 0;
    mine.add(Sums{n, need[i], ended ? 1u : 0u, ended ? min(have[i], static_cast<uint32_t>(a.max_pages)) : 0u});
  }
  const Sums upto = warp_inclusive(mine, lane);
  if (lane == 31) part[warp] = upto;
  if (tid == 0) popped = 0;
  __syncthreads();
  Sums others = lane < kWarps ? part[lane] : Sums{0, 0, 0, 0};
  others = warp_inclusive(others, lane);
  const Sums all{__shfl_sync(0xffffffffu, others.rows, 31), __shfl_sync(0xffffffffu, others.need, 31),
                 __shfl_sync(0xffffffffu, others.ended, 31), __shfl_sync(0xffffffffu, others.entries, 31)};
  Sums at{upto.rows - mine.rows, upto.need - mine.need, upto.ended - mine.ended, upto.entries - mine.entries};
  {
    const int w = max(warp - 1, 0);
    const Sums before{__shfl_sync(0xffffffffu, others.rows, w), __shfl_sync(0xffffffffu, others.need, w),
                      __shfl_sync(0xffffffffu, others.ended, w), __shfl_sync(0xffffffffu, others.entries, w)};
    if (warp) at.add(before);
  }
  const int64_t rows = all.rows;
  const Sums begin = at;
  uint32_t taken = 0;   // pages given out up to and with this thread's requests
#pragma unroll
  for (int i = 0; i < kPlanPer; ++i) {
    const int64_t first = at.rows;
    at.rows += max(more[i], 0);
    fits[i] = fits[i] && at.rows <= a.max_tokens && (need[i] == 0 || at.need + need[i] <= static_cast<uint32_t>(count));
    if (i < per && r0 + i < B) {
      start[r0 + i] = static_cast<int32_t>(min(first, static_cast<int64_t>(INT32_MAX)));
      // (granted: both are below 2^31, so is their difference)
      place[r0 + i] = fits[i] ? static_cast<int32_t>(at.need) - static_cast<int32_t>(have[i]) : kRefused;
      if (!fits[i] && more[i] > 0) bad |= WK_DEV_POOL_FULL;
    }
    at.need += need[i];
    if (fits[i] && need[i]) taken = at.need;
  }
  if (tid == 0) start[B] = static_cast<int32_t>(min(rows, static_cast<int64_t>(INT32_MAX)));
  taken = __reduce_max_sync(0xffffffffu, taken);
  if (lane == 0 && taken) atomicMax(&popped, taken);
  __syncthreads();

  // slots of the new tokens
  for (int64_t t0 = static_cast<int64_t>(blockIdx.x) * kTokens; t0 < a.max_tokens; t0 += static_cast<int64_t>(gridDim.x) * kTokens) {
#pragma unroll
    for (int i = 0; i < kTokens / THREADS; ++i) {
      const int64_t t = t0 + i * THREADS + tid;
      if (t >= a.max_tokens) break;
      int32_t slot = -1;
      if (t < rows) {
        // (rows before t are rows of requests that have some: the last start that is at most t is that of t's own)
        const int r = last_at_most(start, B, static_cast<int32_t>(t));
        if (place[r] != kRefused) {
          const int32_t held = a.lens[r];
          const uint32_t pos = static_cast<uint32_t>(held + static_cast<int32_t>(t) - start[r]);
          const uint32_t col = pos / static_cast<uint32_t>(page);
          int32_t* entry = a.tables + r * a.table_stride + col;
          int32_t id;
          if (col >= pages_of(held, page)) {
            const int64_t ix = static_cast<int64_t>(head) + place[r] + col;
            id = a.ring[ix < a.n_pages ? ix : ix - a.n_pages];
            if (pos == col * page) *entry = id;   // the page's first token enters it
          } else {
            id = *entry;
          }
          if (id >= 0 && id < a.n_pages) slot = id * page + static_cast<int32_t>(pos - col * page);
          else bad |= WK_DEV_BAD_SLOT;
        }
      }
      a.slots[t] = slot;
    }
  }
  for (int r = blockIdx.x * THREADS + tid; r <= B; r += gridDim.x * THREADS) a.starts[r] = start[r];

  // pages of ended requests go behind the ring's last free page
  uint32_t pushed = 0;
  if (blockIdx.x == 0 && all.ended) {
    __syncthreads();   // nobody reads start and place any more
    uint32_t li = begin.ended, e0 = begin.entries;
#pragma unroll
    for (int i = 0; i < kPlanPer; ++i)
      if (more[i] < 0 && len[i] >= 0) {
        place[li] = r0 + i;
        start[li] = static_cast<int32_t>(e0);   // fewer than 2^31: n_req * max_pages is
        ++li;
        e0 += min(have[i], static_cast<uint32_t>(a.max_pages));
      }
    __syncthreads();
    // Each warp takes a run of the entries: counts those that are pages, then writes them behind those of the warps before it.  It
    // keeps the first 128 in registers in between.
    const int list = static_cast<int>(all.ended);
    const int64_t run = (static_cast<int64_t>(all.entries) + THREADS - 1) / THREADS * 32, w0 = warp * run;
    const int64_t w1 = min(w0 + run, static_cast<int64_t>(all.entries));
    auto entry_at = [&](int64_t e) -> int32_t {
      if (e >= w1) return -1;
      const int k = last_at_most(start, list, static_cast<int32_t>(e));
      return a.tables[place[k] * a.table_stride + (e - start[k])];
    };
    uint32_t found = 0;
    int32_t id[4] = {-1, -1, -1, -1};
#pragma unroll 1
    for (int64_t e = w0; e < w1; e += 128) {
#pragma unroll
      for (int u = 0; u < 4; ++u) id[u] = entry_at(e + 32 * u + lane);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const bool ok = id[u] >= 0 && id[u] < a.n_pages;
        if (!ok && id[u] != -1) bad |= WK_DEV_BAD_SLOT;
        found += __popc(__ballot_sync(0xffffffffu, ok));
      }
    }
    if (lane == 0) found_by[warp] = found;
    __syncthreads();
    uint32_t behind = 0;
    for (int w = 0; w < kWarps; ++w) {
      if (w < warp) behind += found_by[w];
      pushed += found_by[w];
    }
    const uint32_t room = static_cast<uint32_t>(a.n_pages - count);   // ring places behind the free pages
    if (pushed > room) {
      bad |= WK_DEV_BAD_SLOT;
      pushed = room;
    }
    const bool again = run > 128;
#pragma unroll 1
    for (int64_t e = w0; e < w1; e += 128) {
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (again) id[u] = entry_at(e + 32 * u + lane);
        const bool ok = id[u] >= 0 && id[u] < a.n_pages;
        const uint32_t mask = __ballot_sync(0xffffffffu, ok);
        const uint32_t k = behind + __popc(mask & ((1u << lane) - 1));
        if (ok && k < room) {   // head, count + k: each at most n_pages
          const uint32_t to = static_cast<uint32_t>(head) + count + k;
          a.ring[to < static_cast<uint32_t>(a.n_pages) ? to : to - a.n_pages] = id[u];
        }
        behind += __popc(mask);
      }
    }
  }
  if (bad) report(a.status, bad);

  // The block that arrives last writes lengths and ring state: all others have read them.
  if (gridDim.x > 1) {
    if (blockIdx.x == 0 && tid == 0) *reinterpret_cast<volatile int32_t*>(a.state + 3) = static_cast<int32_t>(pushed);
    __syncthreads();
    if (tid == 0) {
      __threadfence();
      last = atomicInc(reinterpret_cast<uint32_t*>(a.state + 2), gridDim.x - 1) == gridDim.x - 1;
      __threadfence();
    }
    __syncthreads();
    if (!last) return;
    pushed = *reinterpret_cast<volatile int32_t*>(a.state + 3);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kPlanPer; ++i)
    if (i < per && r0 + i < B) a.lens_out[r0 + i] = more[i] < 0 && len[i] >= 0 ? 0 : fits[i] ? len[i] + more[i] : len[i];
  if (tid == 0) {
    const uint32_t h = static_cast<uint32_t>(head) + popped;
    a.state[2] = a.state[3] = 0;
    a.state_out[0] = static_cast<int32_t>(h < static_cast<uint32_t>(a.n_pages) ? h : h - a.n_pages);
    a.state_out[1] = static_cast<int32_t>(count - popped + pushed);
    a.state_out[2] = a.state_out[3] = 0;
  }
}

// ---------------------------------------------------------------- page_store
constexpr int kStoreThreads = 128;
constexpr int kStoreLoads = 4;   // 16-byte loads in flight per thread

struct StoreArgs {
  wk_paged_kv c;
  const uint8_t *src[2];
  int64_t row_bytes;      // from one source row to the next
  int32_t n_tokens, rows; // rows per block
  const int32_t* slots;
  uint32_t* status;
  Divisor by_page, by_heads;
};

// The slot's page and place in it; false: nothing to write.
__device__ __forceinline__ bool slot_place(const StoreArgs& a, int32_t slot, int64_t* page, int64_t* off) {
  const uint32_t id = a.by_page.quotient(static_cast<uint32_t>(slot));
  if (slot < 0 || id >= static_cast<uint32_t>(a.c.n_pages)) {
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
  dep_release();
  dep_wait();
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
      if (!slot_place(a, a.slots[t0 + r], &page, &off)) continue;
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
// The larger of two magnitudes of 16 bits each: without the sign, both types' bits grow with the magnitude.
__device__ __forceinline__ uint32_t larger2(uint32_t x, uint32_t y) { return __vmaxu2(x & 0x7fff7fffu, y & 0x7fff7fffu); }

// Rows in 8 bits: a row (one token, one head) belongs to head_dim / 8 neighbouring lanes, 16 bytes each.  The exponent is read off
// the bits of the largest magnitude: amax = m * 2^x with 1 <= m < 2 fits 448 * 2^e = 1.75 * 2^(e + 8) for e = x - 8 if m <= 1.75,
// else for x - 7.  A power of two keeps the scaling exact (the one rounding is that to the code) and costs a byte per row; codes of
// 17 binades leave no accuracy to be won from a finer scale.  The largest magnitude is found on the 16-bit patterns; a row in
// which that is Inf or NaN looks again among its finite values.
template <bool BF16, int D>
__global__ void __launch_bounds__(kStoreThreads)
store_rows_e4m3(const __grid_constant__ StoreArgs a) {
  constexpr int LANES = D / 8, ROWS = kStoreThreads / LANES;   // lanes per row, rows at a time
  constexpr uint32_t kInf = BF16 ? 0x7f80u : 0x7c00u;
  dep_release();
  dep_wait();
  const int side = blockIdx.y, l = threadIdx.x % LANES;
  uint8_t* dst = static_cast<uint8_t*>(side ? a.c.V : a.c.K);
  uint8_t* exps = side ? a.c.V_exp : a.c.K_exp;
  const int32_t t0 = blockIdx.x * a.rows, n = min(a.rows, a.n_tokens - t0) * a.c.n_kv_heads;   // this block's rows
#pragma unroll 1
  for (int32_t k = 0; k < n; k += kStoreLoads * ROWS) {   // the same number for all lanes: they exchange values
    uint4 q[kStoreLoads];
    int32_t slot[kStoreLoads], head[kStoreLoads];
#pragma unroll
    for (int u = 0; u < kStoreLoads; ++u) {
      const int32_t i = k + u * ROWS + threadIdx.x / LANES;
      q[u] = make_uint4(0, 0, 0, 0);
      slot[u] = -1;
      head[u] = 0;
      if (i < n) {
        const int32_t t = a.by_heads.quotient(i);
        head[u] = i - t * a.c.n_kv_heads;
        slot[u] = a.slots[t0 + t];
        q[u] = __ldcs(reinterpret_cast<const uint4*>(a.src[side] + static_cast<int64_t>(t0 + t) * a.row_bytes) + head[u] * LANES + l);
      }
    }
#pragma unroll
    for (int u = 0; u < kStoreLoads; ++u) {
      const uint32_t w[4] = {q[u].x, q[u].y, q[u].z, q[u].w};
      uint32_t m = larger2(larger2(w[0], w[1]), larger2(w[2], w[3]));
#pragma unroll
      for (int d = 1; d < LANES; d <<= 1) m = __vmaxu2(m, __shfl_xor_sync(0xffffffffu, m, d));
      uint32_t top16 = max(m & 0xffffu, m >> 16);
      const bool odd = top16 >= kInf;
      if (__any_sync(0xffffffffu, odd)) {
        uint32_t fine = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t lo = w[j] & 0x7fffu, hi = w[j] >> 16 & 0x7fffu;
          fine = max(fine, max(lo < kInf ? lo : 0u, hi < kInf ? hi : 0u));
        }
#pragma unroll
        for (int d = 1; d < LANES; d <<= 1) fine = max(fine, __shfl_xor_sync(0xffffffffu, fine, d));
        if (odd) top16 = fine;
      }
      // byte = e + 127; a bf16 below the normal numbers reads x = -127 here and ends at the least exponent, as it should
      const uint32_t bits = BF16 ? top16 << 16 : __float_as_uint(__half2float(__ushort_as_half(static_cast<uint16_t>(top16))));
      const int byte = top16 == 0 ? 127 : max(1, static_cast<int>(bits >> 23) - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0));
      int64_t page, off;
      if (!slot_place(a, slot[u], &page, &off)) continue;
      const float scale = __uint_as_float(static_cast<uint32_t>(254 - byte) << 23);   // 2^-e; byte is at most 247
      float x[8];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        unpack2(w[j], BF16, &x[2 * j], &x[2 * j + 1]);
        x[2 * j] *= scale;
        x[2 * j + 1] *= scale;
      }
      if (odd) {   // infinities, too, become NaN; the conversion would make them the largest code
        if (l == 0) report(a.status, WK_DEV_NONFINITE);
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (!(fabsf(x[j]) <= 3.402823466e38f)) x[j] = __int_as_float(0x7fffffff);
      }
      uint32_t code[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        uint16_t lo, hi;
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(x[4 * j + 1]), "f"(x[4 * j]));
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(x[4 * j + 3]), "f"(x[4 * j + 2]));
        code[j] = lo | static_cast<uint32_t>(hi) << 16;
      }
      *reinterpret_cast<uint2*>(dst + page * a.c.page_stride + off * a.c.token_stride + head[u] * a.c.head_stride + 8 * l) =
          make_uint2(code[0], code[1]);
      if (l == 0) exps[(page * a.c.n_kv_heads + head[u]) * a.c.page_tokens + off] = static_cast<uint8_t>(byte);
    }
  }
}

}  // namespace

wk_status launch_page_plan(wk_ctx* ctx, const PlanArgs& a, cudaStream_t s) {
  // Blocks of 256 threads scan up to 1,024 requests in half the time that blocks of 1,024 threads take (3.0 us a call against 6.3,
  // without new tokens); four new tokens per thread.
  const auto blocks = [&](int64_t threads) {
    const int64_t n = (static_cast<int64_t>(a.max_tokens) + 4 * threads - 1) / (4 * threads);
    return static_cast<int>(n < 1 ? 1 : n < ctx->sm_count ? n : ctx->sm_count);
  };
  if (a.n_req <= kPlanPer * 256) launch_chained(page_plan<256>, dim3(blocks(256)), dim3(256), 0, s, a);
  else launch_chained(page_plan<1024>, dim3(blocks(1024)), dim3(1024), 0, s, a);
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
  a.by_page = divisor(c.page_tokens);
  a.by_heads = divisor(c.n_kv_heads);
  const int64_t vecs = static_cast<int64_t>(c.n_kv_heads) * c.head_dim / 8;
  const int64_t rows = kStoreLoads * kStoreThreads / vecs;
  a.rows = rows > 1 ? static_cast<int>(rows) : 1;
  const dim3 grid(static_cast<unsigned>((n_tokens + a.rows - 1) / a.rows), 2);
  const bool wide = c.head_dim == 128;
  void (*kernel)(const StoreArgs) = store_rows;
  if (c.type == WK_E4M3 && src_type == WK_BF16) kernel = wide ? store_rows_e4m3<true, 128> : store_rows_e4m3<true, 64>;
  else if (c.type == WK_E4M3) kernel = wide ? store_rows_e4m3<false, 128> : store_rows_e4m3<false, 64>;
  launch_chained(kernel, grid, dim3(kStoreThreads), 0, s, a);
  return after_launch(ctx);
}

}  // namespace wk
