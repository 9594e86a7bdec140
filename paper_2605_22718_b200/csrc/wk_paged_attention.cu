// Attention of single new tokens over the token-level cache in pages.
//
// Per request and head: o = sum_t softmax_t(scale * q . k_t) v_t over the visible tokens.  Every key and value is used for the few
// query heads that share it, so the kernel is bound by reading the cache once; everything else is arranged around keeping loads in
// flight.
//
//   * Work.  A unit is (request, kv head, up to 8 * NT of the query heads that share it).  A unit's tokens are cut into steps of ST
//     tokens; all steps of all units form one line, and every CTA takes an equal run of it (one CTA per SM), every warp an equal
//     run of the CTA's.  So lengths of any spread load all SMs alike, the grid does not depend on the lengths (a captured call
//     follows them), and a unit is cut only where a run ends.  The lengths are summed by every CTA for itself.
//   * A warp walks its run alone: no barrier, no shared memory.  K and V go from global memory to registers in the places where the
//     matrix instructions want them: S^T = K Q^T has tokens as rows, so a lane's 16 contiguous bytes of a key are four (bf16, fp16)
//     or sixteen (8 bits) places along the contracted axis, whose order is free as long as Q is laid out alike; O^T = V^T P^T
//     has the head's dimensions as rows, so a lane's 16 bytes of two tokens are paired up by byte permutes.  P^T comes from S^T
//     by an 8x8 transpose in the registers of the warp.  The next step's K is loaded as soon as S is done, its V as soon as O
//     is, and the page ids of the step after that are looked up meanwhile.
//   * Softmax.  Per query head a reference close to the running maximum: it moves only when a logit exceeds it by more than 8 (in
//     log2), which one vote per step finds out, so weights reach at most 2^8; sums are fp32.  Weights are rounded to the type of V
//     for the second product (bf16 or fp16, half a step 2^-8 or 2^-11 of the weight; the normalising sum is of the unrounded ones).
//   * 8 bits.  Codes are exact in fp16.  A key's power of two joins the logit's scale, a value's is added to the logit that its
//     weight is taken from (with a reference of its own), so that both products have fp16 operands of ordinary size; Q is brought
//     into fp16 by a power of two per row, exactly.
//   * Joining.  Pieces of a unit are (log-sum-exp, normalised o).  Warps of a CTA leave theirs in shared memory, CTAs theirs in the
//     scratch buffer; the CTA that arrives last joins them in their order, so that the result does not depend on the arrival.
#include <cuda_fp16.h>

#include "wk_internal.cuh"

namespace wk {
namespace {

constexpr uint32_t kNowhere = 0xffffffffu;   // row offset of a token that is not attended
constexpr float kLazy = 8.f;                 // how far (log2) a logit may exceed the reference
constexpr float kLn2 = 0.6931471805599453f;

struct Params {
  PagedArgs a;
  int32_t group, q_tiles, units;   // query heads per kv head, units of a kv head, units of a request
  int32_t room;                    // positions that a table can name
  uint32_t page16, token16;        // strides in units of 16 bytes
  int64_t head_bytes;              // stride of a kv head
  int32_t counter_bytes;           // of the scratch buffer, before the pieces
};

template <int MODE, int D, int NT>
struct Shape {
  static constexpr int ES = MODE == WK_E4M3 ? 1 : 2;     // bytes per element of the cache
  static constexpr int ROW = D * ES;                     // bytes of a row
  static constexpr int TT = 256 / ROW;                   // tiles of 16 tokens in a step: K and V of a step are 8 KB
  static constexpr int ST = 16 * TT;
  static constexpr int RL = ST > 32 ? ST / 32 : 1;       // tokens per lane when rows are looked up
  static constexpr int KV = ROW / 64;                    // 16-byte loads of a key per lane (four lanes read 64 bytes)
  static constexpr int VH = ROW / 128 > 0 ? ROW / 128 : 1, VR = ROW / 128 > 0 ? 4 : 2;   // loads of a value per lane, registers each
  static constexpr int W = NT == 1 ? 12 : 8;             // warps: what the registers of an SM hold
  static constexpr int PADDED = D + 4;
  static constexpr int SMEM = 2 * W * 8 * NT * PADDED * 4;
};

// ---------------------------------------------------------------- instructions
__device__ __forceinline__ void load16(uint32_t (&r)[4], const void* p, bool on) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %5, 0;\n\t"
      "mov.b32 %0, 0;\n\tmov.b32 %1, 0;\n\tmov.b32 %2, 0;\n\tmov.b32 %3, 0;\n\t"
      "@p ld.global.nc.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];\n\t}"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
      : "l"(p), "r"(static_cast<uint32_t>(on)));
}
__device__ __forceinline__ void load8(uint32_t (&r)[2], const void* p, bool on) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %3, 0;\n\tmov.b32 %0, 0;\n\tmov.b32 %1, 0;\n\t"
      "@p ld.global.nc.L1::no_allocate.v2.b32 {%0, %1}, [%2];\n\t}"
      : "=r"(r[0]), "=r"(r[1])
      : "l"(p), "r"(static_cast<uint32_t>(on)));
}
// d += a b on a 16 x 8 x 16 tile
template <bool BF16>
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if (BF16)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
template <bool BF16>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  uint32_t r;
  if (BF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ float exp2_of(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// two codes to two fp16, exactly
__device__ __forceinline__ uint32_t codes_lo(uint32_t w) {
  uint32_t r;
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\t}" : "=r"(r) : "r"(w));
  return r;
}
__device__ __forceinline__ uint32_t codes_hi(uint32_t w) {
  uint32_t r;
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, h;\n\t}" : "=r"(r) : "r"(w));
  return r;
}
__device__ __forceinline__ float lo_of(uint32_t w, bool bf16) {
  return bf16 ? __uint_as_float(w << 16) : __half2float(__ushort_as_half(static_cast<uint16_t>(w)));
}
__device__ __forceinline__ float hi_of(uint32_t w, bool bf16) {
  return bf16 ? __uint_as_float(w & 0xffff0000u) : __half2float(__ushort_as_half(static_cast<uint16_t>(w >> 16)));
}

// ---------------------------------------------------------------- units
struct Unit {
  int32_t r, u;         // request, unit of the request
  int32_t step, cost;   // place in the unit, steps of the unit (at least one, also where nothing is visible)
  int32_t shown, shift; // visible tokens; visible token j is position j, or j + shift from the sink's end on
};

// Steps that request r's units have each; 0: no request.
template <int ST>
__device__ __forceinline__ int32_t measure(const Params& p, int r, int32_t* shown, int32_t* shift) {
  int32_t len = p.a.lens[r];
  if (len < 0) return 0;
  len = min(len, p.room);
  *shown = p.a.window ? min(len, p.a.window + p.a.sink) : len;
  *shift = len - *shown;
  return *shown > ST ? static_cast<int32_t>((static_cast<uint32_t>(*shown) + ST - 1) / ST) : 1;
}

// The unit that place x of the line lies in.  pre[t]: steps of one unit of each request before thread t's `per` requests.
template <int ST, int THREADS>
__device__ __forceinline__ Unit locate(const Params& p, const int64_t* pre, int per, int64_t x) {
  const int64_t z = x / p.units;
  int lo = 0, hi = THREADS;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (pre[mid] <= z) lo = mid; else hi = mid;
  }
  Unit v;
  int64_t before = pre[lo];
  v.r = lo * per;
  v.shown = v.shift = 0;
  v.cost = measure<ST>(p, v.r, &v.shown, &v.shift);
  while (before + v.cost <= z && v.r < p.a.n_req - 1) {   // (z lies before the sum of all: the second bound is for lengths that change meanwhile)
    before += v.cost;
    v.cost = measure<ST>(p, ++v.r, &v.shown, &v.shift);
  }
  v.cost = max(v.cost, 1);
  const int64_t rest = x - before * p.units;
  v.u = static_cast<int32_t>(rest / v.cost);
  v.step = static_cast<int32_t>(rest - static_cast<int64_t>(v.u) * v.cost);
  return v;
}

template <int ST>
__device__ __forceinline__ void advance(const Params& p, Unit& v) {
  if (++v.step < v.cost) return;
  v.step = 0;
  if (++v.u < p.units) return;
  v.u = 0;
  do v.cost = v.r < p.a.n_req - 1 ? measure<ST>(p, ++v.r, &v.shown, &v.shift) : 1;
  while (v.cost == 0);
}

struct Heads {
  int32_t kv, first, n;   // kv head, first query head, query heads of the unit
};
template <int NT>
__device__ __forceinline__ Heads heads_of(const Params& p, int u) {
  Heads h;
  h.kv = p.q_tiles == 1 ? u : u / p.q_tiles;
  const int t = u - h.kv * p.q_tiles;
  h.first = h.kv * p.group + t * 8 * NT;
  h.n = min(8 * NT, p.group - t * 8 * NT);
  return h;
}

// What the warps and CTAs that share a unit leave each other.
struct Piece {
  int32_t r, u, cost;   // r < 0: none
  int64_t start;        // the unit's first place in the line
};

constexpr int kPieceFloats = 16 * (128 + 1);   // of a piece in the scratch buffer: log-sum-exps, then rows
constexpr size_t counter_bytes(int ctas) { return (ctas * sizeof(uint32_t) + 255) / 256 * 256; }

template <bool QBF>
__device__ __forceinline__ void store4(void* O, int64_t i, float4 v) {
  *reinterpret_cast<uint2*>(static_cast<uint16_t*>(O) + i) = make_uint2(pack2<QBF>(v.x, v.y), pack2<QBF>(v.z, v.w));
}

// ---------------------------------------------------------------- the kernel
template <int MODE, int D, int NT, bool QBF>
__global__ void __launch_bounds__(32 * Shape<MODE, D, NT>::W, 1)
paged_attention(const __grid_constant__ Params p) {
  using S = Shape<MODE, D, NT>;
  constexpr int ST = S::ST, TT = S::TT, W = S::W, THREADS = 32 * W, PADDED = S::PADDED;
  constexpr bool E4 = MODE == WK_E4M3, BF = MODE == WK_BF16;
  constexpr int MT = D / 16;   // row tiles of O^T
  extern __shared__ float4 dyn[];
  float* const po = reinterpret_cast<float*>(dyn);          // [2 W][8 NT][PADDED]
  __shared__ int64_t pre[THREADS], parts[W];
  __shared__ float plse[2 * W][8 * NT];
  __shared__ Piece piece[2 * W], split[2];
  __shared__ int32_t last[2];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, c = lane & 3;

  // ---- the line of steps, and this CTA's and this warp's run of it
  const int per = (p.a.n_req + THREADS - 1) / THREADS;
  int64_t mine = 0;
  for (int i = 0; i < per; ++i) {
    const int r = tid * per + i;
    int32_t shown, shift;
    if (r >= p.a.n_req) break;
    mine += measure<ST>(p, r, &shown, &shift);
    if (blockIdx.x == 0 && p.a.lens[r] > p.room && p.a.status) atomicOr(p.a.status, WK_DEV_BAD_SLOT);
  }
  int64_t up = mine;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int64_t o = __shfl_up_sync(0xffffffffu, up, d);
    if (lane >= d) up += o;
  }
  if (lane == 31) parts[warp] = up;
  __syncthreads();
  int64_t before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    if (w < warp) before += parts[w];
    all += parts[w];
  }
  pre[tid] = before + up - mine;
  __syncthreads();
  const int64_t total = all * p.units;
  int64_t chunk = (total + gridDim.x - 1) / gridDim.x;
  if (chunk < W) chunk = W;
  const int64_t a0 = blockIdx.x * chunk, a1 = min(a0 + chunk, total);
  if (a0 >= total) return;
  const int64_t run = (a1 - a0 + W - 1) / W;
  int64_t x = a0 + warp * run;
  const int64_t xe = min(x + run, a1);
  if (lane < 2) piece[2 * warp + lane].r = -1;

  if (x < xe) {
    const char* const Kc = static_cast<const char*>(p.a.c.K);
    const char* const Vc = static_cast<const char*>(p.a.c.V);
    uint32_t bad = 0;
    uint32_t row[S::RL], mask[S::RL], mask_n[S::RL], ex[S::RL], ex_n[S::RL];
    uint32_t kf[TT][2][S::KV][4], vf[TT][4][S::VH][S::VR], qf[NT][D / 16][2];
    float sc[NT][2];               // logit scale of query heads 2c, 2c + 1
    float ref[NT][2], refw[NT][2]; // references of the sum and (8 bits) of the weights
    float sum[NT][2], o[NT][MT][4];

    // rows of the step's tokens, a token per lane (or two)
    auto look_up = [&](const Unit& v) {
#pragma unroll
      for (int i = 0; i < S::RL; ++i) {
        const int32_t j = v.step * ST + (lane & (ST - 1)) + 32 * i;
        row[i] = kNowhere;
        if (E4) ex_n[i] = 0;
        if (j < v.shown) {
          const uint32_t pos = static_cast<uint32_t>(j >= p.a.sink ? j + v.shift : j);
          const uint32_t at = pos / static_cast<uint32_t>(p.a.c.page_tokens), off = pos - at * p.a.c.page_tokens;
          const int32_t id = __ldg(p.a.tables + v.r * p.a.table_stride + at);
          if (id >= 0 && id < p.a.c.n_pages) {
            row[i] = id * p.page16 + off * p.token16;
            if (E4) {
              const int64_t e = (static_cast<int64_t>(id) * p.a.c.n_kv_heads + heads_of<NT>(p, v.u).kv) * p.a.c.page_tokens + off;
              ex_n[i] = __ldg(p.a.c.K_exp + e) | static_cast<uint32_t>(__ldg(p.a.c.V_exp + e)) << 8;
            }
          } else if (id != -1) {
            bad = WK_DEV_BAD_SLOT;
          }
        }
      }
    };
    auto load_k = [&](const Heads& h) {
      const char* base = Kc + h.kv * p.head_bytes + c * 16;
#pragma unroll
      for (int t = 0; t < TT; ++t)
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
          const uint32_t at = S::RL == 1 ? __shfl_sync(0xffffffffu, row[0], t * 16 + hh * 8 + g)
                                         : __shfl_sync(0xffffffffu, row[t * 16 / 32], (t * 16 + hh * 8 + g) & 31);
          const char* src = base + static_cast<uint64_t>(at) * 16;
#pragma unroll
          for (int j = 0; j < S::KV; ++j) load16(kf[t][hh][j], src + 64 * j, at != kNowhere);
        }
    };
    auto load_v = [&](const Heads& h) {
      const char* base = Vc + h.kv * p.head_bytes + g * (4 * S::VR);
#pragma unroll
      for (int t = 0; t < TT; ++t)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int j = t * 16 + 2 * c + (k & 1) + (k >> 1) * 8;
          const uint32_t at = S::RL == 1 ? __shfl_sync(0xffffffffu, row[0], j) : __shfl_sync(0xffffffffu, row[t * 16 / 32], j & 31);
          const char* src = base + static_cast<uint64_t>(at) * 16;
#pragma unroll
          for (int hf = 0; hf < S::VH; ++hf) {
            if constexpr (S::VR == 4) load16(vf[t][k][hf], src + 128 * hf, at != kNowhere);
            else load8(vf[t][k][hf], src, at != kNowhere);
          }
        }
    };
    // Query row g of every tile, its dimensions in the order of the keys' loads.
    auto load_q = [&](const Unit& v, const Heads& h) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const bool on = nt * 8 + g < h.n;
        const uint16_t* q = static_cast<const uint16_t*>(p.a.Q) + v.r * p.a.q_stride + static_cast<int64_t>(h.first + (on ? nt * 8 + g : 0)) * D;
        constexpr int EPL = 16 / S::ES;   // elements of a key per 16-byte load
#pragma unroll
        for (int j = 0; j < S::KV; ++j)
#pragma unroll
          for (int e = 0; e < EPL / 8; ++e) {
            uint4 w = make_uint4(0, 0, 0, 0);
            if (on) w = *reinterpret_cast<const uint4*>(q + j * 4 * EPL + c * EPL + e * 8);
            const int s = j * (EPL / 4) + 2 * e;
            qf[nt][s][0] = w.x;
            qf[nt][s][1] = w.y;
            qf[nt][s + 1][0] = w.z;
            qf[nt][s + 1][1] = w.w;
          }
      }
    };
    auto begin_unit = [&]() {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        if (E4) {
          // row g by a power of two to below 2^15: exact in fp16 for all that matters beside the row's largest
          float top = 0.f;
#pragma unroll
          for (int s = 0; s < D / 16; ++s)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float l = fabsf(lo_of(qf[nt][s][e], QBF)), h = fabsf(hi_of(qf[nt][s][e], QBF));
              if (l <= 3.402823466e38f) top = fmaxf(top, l);
              if (h <= 3.402823466e38f) top = fmaxf(top, h);
            }
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
          const int power = max(static_cast<int>(__float_as_uint(top) >> 23), 28) - 127;   // floor(log2), at least -99
          const float scale = __uint_as_float(static_cast<uint32_t>(14 - power + 127) << 23);
          const float back = __uint_as_float(static_cast<uint32_t>(max(power - 14 + 127, 1)) << 23);
#pragma unroll
          for (int s = 0; s < D / 16; ++s)
#pragma unroll
            for (int e = 0; e < 2; ++e)
              qf[nt][s][e] = pack2<false>(lo_of(qf[nt][s][e], QBF) * scale, hi_of(qf[nt][s][e], QBF) * scale);
          sc[nt][0] = __shfl_sync(0xffffffffu, back, 8 * c) * (p.a.scale * 1.4426950408889634f);
          sc[nt][1] = __shfl_sync(0xffffffffu, back, 8 * c + 4) * (p.a.scale * 1.4426950408889634f);
        } else {
          sc[nt][0] = sc[nt][1] = p.a.scale * 1.4426950408889634f;
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          ref[nt][e] = refw[nt][e] = -INFINITY;
          sum[nt][e] = 0.f;
        }
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[nt][m][e] = 0.f;
      }
    };

    Unit cur = locate<ST, THREADS>(p, pre, per, x), nxt = cur;
    Heads hc = heads_of<NT>(p, cur.u), hn = hc;
    int32_t began = cur.step;
    bool fresh = true;
    look_up(cur);
    load_q(cur, hc);
    load_k(hc);
    load_v(hc);
#pragma unroll
    for (int i = 0; i < S::RL; ++i) {
      mask[i] = __ballot_sync(0xffffffffu, row[i] != kNowhere);
      ex[i] = ex_n[i];
    }
    if (x + 1 < xe) {
      advance<ST>(p, nxt);
      hn = heads_of<NT>(p, nxt.u);
      look_up(nxt);
    }

    for (;; ++x) {
      const bool more = x + 1 < xe;
      const bool other = more && nxt.step == 0;   // the next step belongs to another unit
      if (fresh) {
        begin_unit();
        fresh = false;
      }
      // ---- S^T = K Q^T
      float s[TT][NT][4];
#pragma unroll
      for (int t = 0; t < TT; ++t)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
          for (int e = 0; e < 4; ++e) s[t][nt][e] = 0.f;
#pragma unroll
          for (int j = 0; j < S::KV; ++j) {
            if constexpr (E4) {
#pragma unroll
              for (int i = 0; i < 4; ++i)
                mma<false>(s[t][nt], codes_lo(kf[t][0][j][i]), codes_lo(kf[t][1][j][i]), codes_hi(kf[t][0][j][i]),
                           codes_hi(kf[t][1][j][i]), qf[nt][4 * j + i][0], qf[nt][4 * j + i][1]);
            } else {
#pragma unroll
              for (int i = 0; i < 2; ++i)
                mma<BF>(s[t][nt], kf[t][0][j][2 * i], kf[t][1][j][2 * i], kf[t][0][j][2 * i + 1], kf[t][1][j][2 * i + 1],
                        qf[nt][2 * j + i][0], qf[nt][2 * j + i][1]);
            }
          }
        }
      if (more) {
#pragma unroll
        for (int i = 0; i < S::RL; ++i) mask_n[i] = __ballot_sync(0xffffffffu, row[i] != kNowhere);
        if (other) load_q(nxt, hn);   // (Q of this unit is not needed any more)
        load_k(hn);
      }
      // ---- logits (log2), their largest, the references
      float w[E4 ? TT : 1][NT][4];
      float top[NT][2], topw[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) top[nt][0] = top[nt][1] = topw[nt][0] = topw[nt][1] = -INFINITY;
#pragma unroll
      for (int t = 0; t < TT; ++t)
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
          const bool on = mask[S::RL == 1 ? 0 : t * 16 / 32] >> ((t * 16 + hh * 8 + g) & 31) & 1;
          float kscale = 1.f, vpower = 0.f;
          if (E4) {
            const uint32_t e = __shfl_sync(0xffffffffu, ex[S::RL == 1 ? 0 : t * 16 / 32], (t * 16 + hh * 8 + g) & 31);
            kscale = __uint_as_float((e & 255u) << 23);
            vpower = static_cast<float>(static_cast<int>(e >> 8) - 127);
          }
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float& v = s[t][nt][2 * hh + e];
              v = on ? v * (E4 ? sc[nt][e] * kscale : sc[nt][e]) : -INFINITY;
              top[nt][e] = fmaxf(top[nt][e], v);
              if constexpr (E4) {
                w[t][nt][2 * hh + e] = v + vpower;
                topw[nt][e] = fmaxf(topw[nt][e], v + vpower);
              }
            }
        }
      bool moved = false;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) moved |= top[nt][e] > ref[nt][e] + kLazy || (E4 && topw[nt][e] > refw[nt][e] + kLazy);
      if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float m = fmaxf(top[nt][e], ref[nt][e]), mw = fmaxf(topw[nt][e], refw[nt][e]);
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) {
              m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
              if (E4) mw = fmaxf(mw, __shfl_xor_sync(0xffffffffu, mw, d));
            }
            const float f = m == -INFINITY ? 1.f : exp2_of(ref[nt][e] - m);
            sum[nt][e] *= f;
            ref[nt][e] = m;
            float fw = f;
            if (E4) {
              fw = mw == -INFINITY ? 1.f : exp2_of(refw[nt][e] - mw);
              refw[nt][e] = mw;
            }
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
              o[nt][mt][e] *= fw;
              o[nt][mt][2 + e] *= fw;
            }
          }
      }
      // ---- weights, and O^T += V^T P^T
#pragma unroll
      for (int t = 0; t < TT; ++t) {
        uint32_t pf[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float q[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float r = ref[nt][e & 1] == -INFINITY ? 0.f : ref[nt][e & 1];
            q[e] = exp2_of(s[t][nt][e] - r);
            sum[nt][e & 1] += q[e];
            if constexpr (E4) q[e] = exp2_of(w[t][nt][e] - (refw[nt][e & 1] == -INFINITY ? 0.f : refw[nt][e & 1]));
          }
          pf[nt][0] = transpose8x8(pack2<BF>(q[0], q[1]));
          pf[nt][1] = transpose8x8(pack2<BF>(q[2], q[3]));
        }
#pragma unroll
        for (int hf = 0; hf < S::VH; ++hf)
#pragma unroll
          for (int i = 0; i < S::VR; ++i) {
            if constexpr (E4) {
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                const uint32_t sel = h ? 0x7362u : 0x5140u;
                const uint32_t x01 = __byte_perm(vf[t][0][hf][i], vf[t][1][hf][i], sel);
                const uint32_t x23 = __byte_perm(vf[t][2][hf][i], vf[t][3][hf][i], sel);
                const uint32_t f0 = codes_lo(x01), f1 = codes_hi(x01), f2 = codes_lo(x23), f3 = codes_hi(x23);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) mma<false>(o[nt][2 * i + h], f0, f1, f2, f3, pf[nt][0], pf[nt][1]);
              }
            } else {
              const uint32_t f0 = __byte_perm(vf[t][0][hf][i], vf[t][1][hf][i], 0x5410);
              const uint32_t f1 = __byte_perm(vf[t][0][hf][i], vf[t][1][hf][i], 0x7632);
              const uint32_t f2 = __byte_perm(vf[t][2][hf][i], vf[t][3][hf][i], 0x5410);
              const uint32_t f3 = __byte_perm(vf[t][2][hf][i], vf[t][3][hf][i], 0x7632);
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) mma<BF>(o[nt][4 * hf + i], f0, f1, f2, f3, pf[nt][0], pf[nt][1]);
            }
          }
      }
      if (more) load_v(hn);

      // ---- the unit ends here, or this warp's part of it
      if (!more || other) {
        const bool whole = began == 0 && cur.step == cur.cost - 1;
        const int slot = 2 * warp + (began == 0);   // reaches in: the warp's first unit; out: its last
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float l = sum[nt][e];
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) l += __shfl_xor_sync(0xffffffffu, l, d);
            const float lse = l == 0.f ? -INFINITY : ref[nt][e] + __log2f(l);
            const float f = l == 0.f ? 0.f : E4 ? exp2f(refw[nt][e] - ref[nt][e]) / l : 1.f / l;
            const int q = nt * 8 + 2 * c + e;
            if (q < hc.n) {
              // runs of dimensions that a lane holds: 8 from 64 hf + 8 g on, or (8 bits) D / 8 from g D / 8 on
              constexpr int RUN = E4 ? D / 8 : 8;
#pragma unroll
              for (int k = 0; k < D / 8 / 8; ++k) {
                const int d0 = E4 ? g * RUN + 8 * k : 64 * k + 8 * g;
                float v[8];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  v[2 * i] = o[nt][4 * k + i][e] * f;
                  v[2 * i + 1] = o[nt][4 * k + i][2 + e] * f;
                }
                if (whole) {
                  const int64_t at = (static_cast<int64_t>(cur.r) * p.a.n_heads + hc.first + q) * D + d0;
                  *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.a.O) + at) =
                      make_uint4(pack2<QBF>(v[0], v[1]), pack2<QBF>(v[2], v[3]), pack2<QBF>(v[4], v[5]), pack2<QBF>(v[6], v[7]));
                } else {
                  float4* to = reinterpret_cast<float4*>(po + (slot * 8 * NT + q) * PADDED + d0);
                  to[0] = make_float4(v[0], v[1], v[2], v[3]);
                  to[1] = make_float4(v[4], v[5], v[6], v[7]);
                }
              }
              if (g == 0) {
                if (!whole) plse[slot][q] = lse;
                else if (p.a.lse) p.a.lse[static_cast<int64_t>(cur.r) * p.a.n_heads + hc.first + q] = lse * kLn2;
              }
            }
          }
        if (!whole && lane == 0) piece[slot] = Piece{cur.r, cur.u, cur.cost, x - cur.step};
        began = 0;
        fresh = true;
      }
      if (!more) break;
      cur = nxt;
      hc = hn;
#pragma unroll
      for (int i = 0; i < S::RL; ++i) {
        mask[i] = mask_n[i];
        ex[i] = ex_n[i];
      }
      if (x + 2 < xe) {
        advance<ST>(p, nxt);
        if (nxt.step == 0) hn = heads_of<NT>(p, nxt.u);
        look_up(nxt);
      }
    }
    if (bad && p.a.status) atomicOr(p.a.status, bad);
  }
  if (tid < 2) split[tid].r = -1;
  __syncthreads();

  // ---- pieces of one unit, next to each other: joined into O, or into this CTA's piece
  float* const partial = reinterpret_cast<float*>(p.a.scratch + p.counter_bytes);
  for (int i0 = 0; i0 < 2 * W;) {
    if (piece[i0].r < 0) {
      ++i0;
      continue;
    }
    const Piece u = piece[i0];
    int i1 = i0 + 1;
    while (i1 < 2 * W && (piece[i1].r < 0 || (piece[i1].r == u.r && piece[i1].u == u.u))) ++i1;
    const Heads h = heads_of<NT>(p, u.u);
    const bool whole = u.start >= a0 && u.start + u.cost <= a1;
    const int side = u.start < a0 ? 0 : 1;
    float* const mine_at = partial + static_cast<int64_t>(2 * blockIdx.x + side) * kPieceFloats;
    for (int it = tid; it < h.n * (D / 4); it += THREADS) {
      const int q = it / (D / 4), d4 = it % (D / 4);
      float m = -INFINITY;
      for (int i = i0; i < i1; ++i)
        if (piece[i].r >= 0) m = fmaxf(m, plse[i][q]);
      if (m == -INFINITY) m = 0.f;
      float l = 0.f;
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int i = i0; i < i1; ++i)
        if (piece[i].r >= 0) {
          const float e = exp2_of(plse[i][q] - m);
          const float4 b = *reinterpret_cast<const float4*>(po + (i * 8 * NT + q) * PADDED + 4 * d4);
          l += e;
          v.x += e * b.x; v.y += e * b.y; v.z += e * b.z; v.w += e * b.w;
        }
      const float f = l == 0.f ? 0.f : 1.f / l, lse = l == 0.f ? -INFINITY : m + __log2f(l);
      v.x *= f; v.y *= f; v.z *= f; v.w *= f;
      if (whole) {
        const int64_t at = static_cast<int64_t>(u.r) * p.a.n_heads + h.first + q;
        store4<QBF>(p.a.O, at * D + 4 * d4, v);
        if (d4 == 0 && p.a.lse) p.a.lse[at] = lse * kLn2;
      } else {
        *reinterpret_cast<float4*>(mine_at + 8 * NT + q * D + 4 * d4) = v;
        if (d4 == 0) mine_at[q] = lse;
      }
    }
    if (!whole && tid == 0) split[side] = u;
    i0 = i1;
  }

  // ---- units that other CTAs share: the last of them to arrive joins the pieces
  __threadfence();
  __syncthreads();
  uint32_t* const arrived = reinterpret_cast<uint32_t*>(p.a.scratch);
  if (tid < 2) {
    last[tid] = 0;
    if (split[tid].r >= 0) {
      const int64_t first = split[tid].start / chunk, end = (split[tid].start + split[tid].cost - 1) / chunk;
      const uint32_t n = static_cast<uint32_t>(end - first);
      last[tid] = atomicInc(arrived + first, n) == n;
      __threadfence();
    }
  }
  __syncthreads();
  for (int side = 0; side < 2; ++side) {
    if (!last[side]) continue;
    const Piece u = split[side];
    const Heads h = heads_of<NT>(p, u.u);
    const int first = static_cast<int>(u.start / chunk), n = static_cast<int>((u.start + u.cost - 1) / chunk) - first + 1;
    auto piece_at = [&](int i) -> const float* {   // the unit's first CTA has it as its last unit, the others as their first
      return partial + static_cast<int64_t>(2 * (first + i) + (u.start < (first + i) * chunk ? 0 : 1)) * kPieceFloats;
    };
    for (int it = tid; it < h.n * (D / 4); it += THREADS) {
      const int q = it / (D / 4), d4 = it % (D / 4);
      float m = -INFINITY;
      for (int i = 0; i < n; ++i) m = fmaxf(m, __ldcg(piece_at(i) + q));
      if (m == -INFINITY) m = 0.f;
      float l = 0.f;
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
      for (int i = 0; i < n; ++i) {
        const float* from = piece_at(i);
        const float e = exp2_of(__ldcg(from + q) - m);
        const float4 b = __ldcg(reinterpret_cast<const float4*>(from + 8 * NT + q * D) + d4);
        l += e;
        v.x += e * b.x; v.y += e * b.y; v.z += e * b.z; v.w += e * b.w;
      }
      const float f = l == 0.f ? 0.f : 1.f / l, lse = l == 0.f ? -INFINITY : m + __log2f(l);
      v.x *= f; v.y *= f; v.z *= f; v.w *= f;
      const int64_t at = static_cast<int64_t>(u.r) * p.a.n_heads + h.first + q;
      store4<QBF>(p.a.O, at * D + 4 * d4, v);
      if (d4 == 0 && p.a.lse) p.a.lse[at] = lse * kLn2;
    }
  }
}

template <int MODE, int D, int NT, bool QBF>
wk_status launch(wk_ctx* ctx, const Params& p, cudaStream_t s) {
  using S = Shape<MODE, D, NT>;
  const int i = ((MODE * 2 + (D == 128)) * 2 + NT - 1) * 2 + QBF;
  if (!(ctx->paged_attr_set >> i & 1)) {
    WK_CUDA_TRY(ctx, cudaFuncSetAttribute(paged_attention<MODE, D, NT, QBF>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM));
    ctx->paged_attr_set |= 1u << i;
  }
  paged_attention<MODE, D, NT, QBF><<<ctx->sm_count, 32 * S::W, S::SMEM, s>>>(p);
  return after_launch(ctx);
}

template <int MODE, bool QBF>
wk_status choose(wk_ctx* ctx, const Params& p, int nt, cudaStream_t s) {
  if (p.a.c.head_dim == 128) return nt == 1 ? launch<MODE, 128, 1, QBF>(ctx, p, s) : launch<MODE, 128, 2, QBF>(ctx, p, s);
  return nt == 1 ? launch<MODE, 64, 1, QBF>(ctx, p, s) : launch<MODE, 64, 2, QBF>(ctx, p, s);
}

}  // namespace

// One counter per CTA, and two pieces (the unit that reaches in from the CTA before, and the one that reaches out).
size_t paged_scratch_bytes(int sm_count) {
  return counter_bytes(sm_count) + static_cast<size_t>(2) * sm_count * kPieceFloats * sizeof(float);
}

wk_status launch_paged_attention(wk_ctx* ctx, const PagedArgs& a, cudaStream_t s) {
  Params p;
  p.a = a;
  p.group = a.n_heads / a.c.n_kv_heads;
  const int nt = p.group > 8 ? 2 : 1;
  p.q_tiles = (p.group + 8 * nt - 1) / (8 * nt);
  p.units = a.c.n_kv_heads * p.q_tiles;
  p.room = a.max_pages * a.c.page_tokens;
  const int es = a.c.type == WK_E4M3 ? 1 : 2;
  p.page16 = static_cast<uint32_t>(a.c.page_stride * es / 16);
  p.token16 = static_cast<uint32_t>(a.c.token_stride * es / 16);
  p.head_bytes = a.c.head_stride * es;
  p.counter_bytes = static_cast<int32_t>(counter_bytes(ctx->sm_count));
  if (a.c.type == WK_BF16) return choose<WK_BF16, true>(ctx, p, nt, s);
  if (a.c.type == WK_F16) return choose<WK_F16, false>(ctx, p, nt, s);
  return a.q_type == WK_BF16 ? choose<WK_E4M3, true>(ctx, p, nt, s) : choose<WK_E4M3, false>(ctx, p, nt, s);
}

}  // namespace wk
