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

  // slots of the new tokens.  Where there are several blocks, the first has the pages of ended requests to see to instead.
  const int fillers = max(gridDim.x - 1, 1), filler = gridDim.x > 1 ? static_cast<int>(blockIdx.x) - 1 : 0;
  for (int64_t t0 = filler < 0 ? a.max_tokens : static_cast<int64_t>(filler) * kTokens; t0 < a.max_tokens; t0 += static_cast<int64_t>(fillers) * kTokens) {
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
  uint8_t *dst[2], *exps[2];
  const uint8_t *src[2];
  uint32_t page16, token16, head16, row16;   // strides in units of 16 bytes: of the cache, of the source's rows
  uint32_t n_rows;                           // rows of K (one token, one head): of V as many
  int32_t n_pages, page_tokens, n_heads;
  const int32_t* slots;
  uint32_t* status;
  Divisor by_page, by_heads;
};

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
// The larger of two magnitudes of 16 bits each (no signs): both types' bits grow with the magnitude.
__device__ __forceinline__ uint32_t larger2(uint32_t x, uint32_t y) { return __vmaxs2(x, y); }

// Eight values of a row, which belongs to LANES neighbouring lanes, in 8 bits; *byte: the row's exponent + 127.  The exponent is read
// off the bits of the row's largest magnitude: amax = m * 2^x with 1 <= m < 2 fits 448 * 2^e = 1.75 * 2^(e + 8) for e = x - 8 if
// m <= 1.75, else for x - 7.  A power of two keeps the scaling exact (the one rounding is that to the code) and costs a byte per
// row; codes of 17 binades leave no accuracy to be won from a finer scale.  The largest magnitude is found on the 16-bit patterns;
// a row in which that is Inf or NaN looks again among its finite values.
template <bool BF16, int LANES>
__device__ __forceinline__ uint2 to_codes(uint4 q, int* byte, bool* odd) {
  constexpr uint32_t kInf = BF16 ? 0x7f80u : 0x7c00u;
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
  uint32_t m = larger2(larger2(w[0] & 0x7fff7fffu, w[1] & 0x7fff7fffu), larger2(w[2] & 0x7fff7fffu, w[3] & 0x7fff7fffu));
#pragma unroll
  for (int d = 1; d < LANES; d <<= 1) m = larger2(m, __shfl_xor_sync(0xffffffffu, m, d));
  uint32_t top16 = max(m & 0xffffu, m >> 16);
  *odd = top16 >= kInf;
  if (__any_sync(0xffffffffu, *odd)) {
    uint32_t fine = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t lo = w[j] & 0x7fffu, hi = w[j] >> 16 & 0x7fffu;
      fine = max(fine, max(lo < kInf ? lo : 0u, hi < kInf ? hi : 0u));
    }
#pragma unroll
    for (int d = 1; d < LANES; d <<= 1) fine = max(fine, __shfl_xor_sync(0xffffffffu, fine, d));
    if (*odd) top16 = fine;
  }
  // a bf16 below the normal numbers reads x = -127 here and ends at the least exponent, as it should
  const uint32_t bits = BF16 ? top16 << 16 : __float_as_uint(__half2float(__ushort_as_half(static_cast<uint16_t>(top16))));
  *byte = top16 == 0 ? 127 : max(1, static_cast<int>((bits + 0x1fffffu) >> 23) - 8);   // (a mantissa above 0.75 carries)
  const float scale = __uint_as_float(static_cast<uint32_t>(254 - *byte) << 23);          // 2^-e; byte is at most 247
  float x[8];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    unpack2(w[j], BF16, &x[2 * j], &x[2 * j + 1]);
    x[2 * j] *= scale;
    x[2 * j + 1] *= scale;
  }
  if (*odd) {   // infinities, too, become NaN; the conversion would make them the largest code
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (!(fabsf(x[j]) <= 3.402823466e38f)) x[j] = __int_as_float(0x7fffffff);
  }
  uint32_t code[2];
#pragma unroll
  for (int j = 0; j < 2; ++j)
    asm("{\n\t.reg .b16 l, h;\n\tcvt.rn.satfinite.e4m3x2.f32 l, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 h, %4, %3;\n\tmov.b32 %0, {l, h};\n\t}"
        : "=r"(code[j]) : "f"(x[4 * j]), "f"(x[4 * j + 1]), "f"(x[4 * j + 2]), "f"(x[4 * j + 3]));
  return make_uint2(code[0], code[1]);
}

// SRC: the type of the source where the cache is in 8 bits, -1 where rows are copied.  A row belongs to D / 8 neighbouring lanes,
// 16 bytes each; a thread has four rows, whose loads are all under way before the first is worked on.  Strides and divisions in 32
// bits matter: with 64 the copies filled 68 % of the issue slots and the rows in 8 bits 79 %.  8,937 tokens of 12 heads (110 MB): 19.5
// us -> 18.3 = 6.0 TB/s; 40,001 tokens of 8 heads to 8 bits (247 MB): 52.9 -> 45.5 = 5.4 TB/s, the scattered exponent bytes 5 of them.
template <int SRC, int D>
__global__ void __launch_bounds__(kStoreThreads)
store_rows(const __grid_constant__ StoreArgs a) {
  constexpr int LANES = D / 8, ROWS = kStoreThreads / LANES;
  dep_release();
  dep_wait();
  const int side = blockIdx.y;
  const uint32_t l = threadIdx.x % LANES;
  uint4 q[kStoreLoads];
  int32_t slot[kStoreLoads];
  uint32_t head[kStoreLoads];
#pragma unroll
  for (int u = 0; u < kStoreLoads; ++u) {
    const uint32_t i = (blockIdx.x * kStoreLoads + u) * ROWS + threadIdx.x / LANES;
    q[u] = make_uint4(0, 0, 0, 0);
    slot[u] = -1;
    head[u] = 0;
    if (i < a.n_rows) {
      const uint32_t t = a.by_heads.quotient(i);
      head[u] = i - t * a.n_heads;
      slot[u] = a.slots[t];
      q[u] = __ldcs(reinterpret_cast<const uint4*>(a.src[side]) + static_cast<uint64_t>(t) * a.row16 + (head[u] * LANES + l));
    }
  }
#pragma unroll
  for (int u = 0; u < kStoreLoads; ++u) {
    int byte = 0;
    bool odd = false;
    uint2 code;
    if constexpr (SRC >= 0) code = to_codes<SRC == WK_BF16, LANES>(q[u], &byte, &odd);   // (all lanes: they exchange values)
    const uint32_t id = a.by_page.quotient(static_cast<uint32_t>(slot[u]));
    if (slot[u] < 0 || id >= static_cast<uint32_t>(a.n_pages)) {
      if (slot[u] != -1) report(a.status, WK_DEV_BAD_SLOT);
      continue;
    }
    const uint32_t off = slot[u] - id * a.page_tokens;
    uint4* const row = reinterpret_cast<uint4*>(a.dst[side]) + (static_cast<uint64_t>(head[u]) * a.head16 + (id * a.page16 + off * a.token16));
    if constexpr (SRC < 0) {
      row[l] = q[u];
    } else {
      reinterpret_cast<uint2*>(row)[l] = code;
      if (l == 0) {
        a.exps[side][(id * a.n_heads + head[u]) * a.page_tokens + off] = static_cast<uint8_t>(byte);
        if (odd) report(a.status, WK_DEV_NONFINITE);
      }
    }
  }
}

}  // namespace

wk_status launch_page_plan(wk_ctx* ctx, const PlanArgs& a, cudaStream_t s) {
  // Blocks of 256 threads scan up to 1,024 requests in half the time that blocks of 1,024 threads take (3.0 us a call against 6.3,
  // without new tokens); four new tokens per thread.
  const auto blocks = [&](int64_t threads) {
    const int64_t n = (static_cast<int64_t>(a.max_tokens) + 4 * threads - 1) / (4 * threads);
    return static_cast<int>(n <= 1 ? 1 : n + 1 < ctx->sm_count ? n + 1 : ctx->sm_count);
  };
  if (a.n_req <= kPlanPer * 256) launch_chained(page_plan<256>, dim3(blocks(256)), dim3(256), 0, s, a);
  else launch_chained(page_plan<1024>, dim3(blocks(1024)), dim3(1024), 0, s, a);
  return after_launch(ctx);
}

wk_status launch_page_store(wk_ctx* ctx, const wk_paged_kv& c, const void* K_new, const void* V_new, int src_type, int n_tokens,
                            int64_t row_stride, const int32_t* slots, cudaStream_t s) {
  const int es = c.type == WK_E4M3 ? 1 : 2;
  StoreArgs a;
  a.dst[0] = static_cast<uint8_t*>(c.K);
  a.dst[1] = static_cast<uint8_t*>(c.V);
  a.exps[0] = c.K_exp;
  a.exps[1] = c.V_exp;
  a.src[0] = static_cast<const uint8_t*>(K_new);
  a.src[1] = static_cast<const uint8_t*>(V_new);
  a.page16 = static_cast<uint32_t>(c.page_stride * es / 16);
  a.token16 = static_cast<uint32_t>(c.token_stride * es / 16);
  a.head16 = static_cast<uint32_t>(c.head_stride * es / 16);
  a.row16 = static_cast<uint32_t>(row_stride * 2 / 16);
  a.n_rows = static_cast<uint32_t>(n_tokens) * c.n_kv_heads;
  a.n_pages = c.n_pages;
  a.page_tokens = c.page_tokens;
  a.n_heads = c.n_kv_heads;
  a.slots = slots;
  a.status = ctx->bound ? ctx->status_dev : nullptr;
  a.by_page = divisor(c.page_tokens);
  a.by_heads = divisor(c.n_kv_heads);
  const bool wide = c.head_dim == 128;
  const uint32_t rows = kStoreThreads / (c.head_dim / 8) * kStoreLoads;
  void (*kernel)(const StoreArgs) = wide ? store_rows<-1, 128> : store_rows<-1, 64>;
  if (c.type == WK_E4M3 && src_type == WK_BF16) kernel = wide ? store_rows<WK_BF16, 128> : store_rows<WK_BF16, 64>;
  else if (c.type == WK_E4M3) kernel = wide ? store_rows<WK_F16, 128> : store_rows<WK_F16, 64>;
  launch_chained(kernel, dim3((a.n_rows - 1) / rows + 1, 2), dim3(kStoreThreads), 0, s, a);
  return after_launch(ctx);
}

}  // namespace wk
