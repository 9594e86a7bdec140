// Attention of single new tokens over the token-level cache in pages.
#include <cuda_fp16.h>

#include "wk_internal.cuh"

namespace wk {
namespace {

constexpr int kWarps = 4;

__device__ __forceinline__ float value_at(const void* p, int64_t i, int type) {
  if (type == WK_BF16) return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
  if (type == WK_F16) return __half2float(static_cast<const __half*>(p)[i]);
  uint32_t h;
  const uint16_t code = static_cast<const uint8_t*>(p)[i];
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(code));
  return __half2float(__ushort_as_half(static_cast<uint16_t>(h)));
}

// One block per request and head, its warps taking every fourth token: the running maximum m and sum l of the softmax,
// o = sum exp(s - m) v, joined over the warps at the end.
__global__ void __launch_bounds__(32 * kWarps)
attend(const __grid_constant__ PagedArgs a) {
  __shared__ float so[kWarps][128], sm[kWarps], sl[kWarps];
  const int r = blockIdx.x, h = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int d = a.c.head_dim, per = d / 32, kv = h / (a.n_heads / a.c.n_kv_heads);
  int64_t len = a.lens[r];
  if (len < 0) return;
  const int64_t room = static_cast<int64_t>(a.max_pages) * a.c.page_tokens;
  uint32_t bad = 0;
  if (len > room) {
    len = room;
    bad = WK_DEV_BAD_SLOT;
  }
  const int64_t shown = a.window ? min(len, static_cast<int64_t>(a.window) + a.sink) : len;
  float q[4], o[4] = {0, 0, 0, 0}, m = -INFINITY, l = 0.f;
  const int64_t row = static_cast<int64_t>(r) * a.n_heads + h;
  for (int i = 0; i < per; ++i) q[i] = value_at(a.Q, r * a.q_stride + static_cast<int64_t>(h) * d + lane * per + i, a.q_type);
  for (int64_t j = warp; j < shown; j += kWarps) {
    const int64_t pos = a.window && j >= a.sink ? j + (len - shown) : j;
    const int id = a.tables[r * a.table_stride + pos / a.c.page_tokens];
    if (id < 0 || id >= a.c.n_pages) {
      if (id != -1) bad = WK_DEV_BAD_SLOT;
      continue;
    }
    const int64_t off = pos % a.c.page_tokens;
    const int64_t at = id * a.c.page_stride + off * a.c.token_stride + kv * a.c.head_stride + lane * per;
    const int64_t ex = (static_cast<int64_t>(id) * a.c.n_kv_heads + kv) * a.c.page_tokens + off;
    float s = 0.f;
    for (int i = 0; i < per; ++i) s += q[i] * value_at(a.c.K, at + i, a.c.type);
    for (int x = 16; x; x >>= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
    s *= a.scale;
    if (a.c.type == WK_E4M3) s *= __uint_as_float(static_cast<uint32_t>(a.c.K_exp[ex]) << 23);
    const float top = fmaxf(m, s), ref = top == -INFINITY ? 0.f : top;
    const float keep = expf(m - ref), w = expf(s - ref);
    l = l * keep + w;
    const float wv = a.c.type == WK_E4M3 ? w * __uint_as_float(static_cast<uint32_t>(a.c.V_exp[ex]) << 23) : w;
    for (int i = 0; i < per; ++i) o[i] = o[i] * keep + wv * value_at(a.c.V, at + i, a.c.type);
    m = top;
  }
  if (bad && a.status) atomicOr(a.status, bad);
  for (int i = 0; i < per; ++i) so[warp][lane * per + i] = o[i];
  if (lane == 0) {
    sm[warp] = m;
    sl[warp] = l;
  }
  __syncthreads();
  const int t = threadIdx.x;
  float top = -INFINITY, total = 0.f, sum = 0.f;
  for (int w = 0; w < kWarps; ++w) top = fmaxf(top, sm[w]);
  const float ref = top == -INFINITY ? 0.f : top;
  for (int w = 0; w < kWarps; ++w) {
    const float f = expf(sm[w] - ref);
    total += sl[w] * f;
    if (t < d) sum += so[w][t] * f;
  }
  if (t < d) {
    const float v = total == 0.f ? 0.f : sum / total;
    if (a.q_type == WK_BF16) static_cast<__nv_bfloat16*>(a.O)[row * d + t] = __float2bfloat16(v);
    else static_cast<__half*>(a.O)[row * d + t] = __float2half(v);
  }
  if (t == 0 && a.lse) a.lse[row] = ref + logf(total);
}

}  // namespace

size_t paged_scratch_bytes(int) { return 256; }

wk_status launch_paged_attention(wk_ctx* ctx, const PagedArgs& a, cudaStream_t s) {
  if (a.n_heads > 65535) return WK_ERR_SHAPE;
  attend<<<dim3(a.n_req, a.n_heads), 32 * kWarps, 0, s>>>(a);
  return after_launch(ctx);
}

}  // namespace wk
