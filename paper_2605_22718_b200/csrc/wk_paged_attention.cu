// Attention of single new tokens over the token-level cache in pages.
//
// Per request and head: o = sum_t softmax_t(scale * q . k_t) v_t over the visible tokens.  Every key and value is used for the few
// query heads that share it, so the kernel is bound by reading the cache once; everything else is arranged around keeping loads in
// flight.
//
//   * Work.  A unit is (request, kv head, up to 8 * NT of the query heads that share it).  A unit's tokens are cut into steps of ST
//     tokens (8 KB of K and V); all steps of all units form one line (or several of the same length), and every CTA takes an equal
//     run of it (one CTA per SM), every warp an equal run of the CTA's.  So lengths of any spread load all SMs alike, the grid does
//     not depend on the lengths (a captured call follows them), and a unit is cut only where a run ends.  The lengths are summed by
//     every CTA for itself.
//   * A warp walks its run alone, without barriers: it copies the rows of coming steps into its own ring in shared memory
//     (16-byte asynchronous copies, tokens that are not attended become zeros) and multiplies out of it.  Page ids are looked up
//     a step before their rows are asked for.
//   * S^T = K Q^T and O^T = V^T P^T: tokens, then dimensions are the rows of the 16 x 8 x 16 matrix instructions, query heads their
//     columns.  (With one token per request there are at most a few columns: the instructions of the SM's large matrix unit
//     work on 64 rows at least and would be filled no better, and the time goes into the copies.)  P^T comes from S^T by an
//     8 x 8 transpose in the warp's registers.
//   * Softmax.  Per query head a reference close to the running maximum: it moves only when a logit exceeds it by more than 8 (in
//     log2), which one vote per step finds out, so weights reach at most 2^8; sums are fp32.  Weights are rounded to the type of V
//     for the second product (bf16 or fp16, half a step 2^-8 or 2^-11 of the weight; the normalising sum is of the unrounded ones).
//     fp16 has steps of 2^-24 at its lower end, and a long tail of small weights may add up to all that a row has: there the
//     weights are taken 2^7 times as large (at most 2^15), so that one is off by 2^-32 of the largest at most.  Exponentials,
//     logarithms and quotients are the SM's approximations (2^-22 or so of the value, 2^-21 of a logarithm): small beside that.
//   * 8 bits.  Codes are exact in fp16.  A key's power of two joins the logit's scale, a value's is added to the logit that its
//     weight is taken from (with a reference of its own), so that both products have fp16 operands of ordinary size; Q is brought
//     into fp16 by a power of two per row, exactly.
//   * Joining.  Pieces of a unit are (log-sum-exp, normalised o).  Warps of a CTA leave theirs in shared memory, CTAs theirs in the
//     scratch buffer; the CTA that arrives last joins them in their order, so that the result does not depend on the arrival.
#include <cuda_fp16.h>

#include <algorithm>

#include "ptx_sm100.cuh"
#include "wk_internal.cuh"

namespace wk {
namespace {

constexpr uint32_t kNowhere = 0xffffffffu;   // row offset of a token that is not attended
constexpr float kLazy = 8.f;                 // how far (log2) a logit may exceed the largest that the reference was taken from
constexpr float kUp = 7.f;                   // how far (log2) below that the reference of weights in fp16 lies
constexpr float kLn2 = 0.6931471805599453f, kLog2e = 1.4426950408889634f;
constexpr int kShortRun = 4, kWhole = 8;     // where runs are that short, CTAs go round units of up to so many steps
constexpr int kLongRun = 24;                 // steps per warp from which on heads are walked side by side

struct Params {
  PagedArgs a;
  int32_t group, q_tiles, units;   // query heads per kv head, units of a kv head, units of a request
  int32_t lines;                   // lines that CTAs walk side by side (where runs are long): a divisor of `units`
  int32_t room;                    // positions that a table can name
  uint32_t page16, token16;        // strides in units of 16 bytes
  int64_t head_bytes;              // stride of a kv head
  int32_t counter_bytes;           // of the scratch buffer, before the pieces
  uint32_t n_exps;                 // bytes of an array of exponents
  Divisor by_page, by_workers[2];  // by the warps that share a line: of one, of `lines`
};

template <int MODE, int D, int NT>
struct Shape {
  // As measured, warps x steps in a warp's ring (us for 1.35 GB in bf16 / 0.92 GB in 8 bits): 6 x 2 210 / 187, 7 x 2 207 / 172, 8 x 2
  // 207 / 165, 9 x 2 214 / 177, 10 x 2 216 / 168, 6 x 3 212 / 188, 7 x 3 221 / 175 (8 x 3 has no room).
  static constexpr int W = 8;
  static constexpr int STAGES = 2;
  static constexpr int ES = MODE == WK_E4M3 ? 1 : 2;     // bytes per element of the cache
  static constexpr int ROW = D * ES;                     // bytes of a row
  static constexpr int STEP = 8192;                      // bytes of K and V in a step
  static constexpr int COPIES = STEP / 1024;             // copy instructions for a step's K, as many for its V
  static constexpr int ST = STEP / 2 / ROW;              // tokens of a step: 16, 32 or 64
  static constexpr int RL = ST > 32 ? ST / 32 : 1;       // tokens per lane when rows are looked up
  static constexpr int LPR = ROW / 16;                   // lanes (16-byte chunks) per row
  static constexpr int RPI = 32 / LPR;                   // rows per copy instruction
  static constexpr int PADDED = D + 4;
  static constexpr int PIECE = 8 * NT * PADDED * 4;      // bytes of a piece in shared memory
  static constexpr int META = MODE == WK_E4M3 ? 8 * ST : 0;   // bytes of a step's exponents: the word with K's, the word with V's
};

// ---------------------------------------------------------------- instructions
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, uint32_t skip) {   // zeros, and nothing read, where skip is not 0
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %2, 0;\n\tcp.async.cg.shared.global [%0], [%1], 16, p;\n\t}"
               ::"r"(dst), "l"(src), "r"(skip) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t dst, const void* src, uint32_t bytes) {   // so many of the four are read
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
template <bool TRANS>
__device__ __forceinline__ void load_matrices(uint32_t (&r)[4], uint32_t addr) {
  if (TRANS)
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
  else
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
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
using ptx::ex2_approx;
__device__ __forceinline__ float warp_max(float x) {   // NaN counts for nothing
  float y;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(x));
  return y;
}

// ---------------------------------------------------------------- units
// A line: for one unit of a request (kv heads first) the steps of all requests, one after the other, then the same for another unit.
// Units are dealt to the lines in turn: line i of n has units i, i + n, ...  A place of the line before every unit's first step stands
// for what a unit costs by itself (about a step's time).
struct Unit {
  int32_t r, u;         // request, unit of the request
  int32_t steps, left;  // of the unit (at least one, also where nothing is visible), those from the one at hand on
  int32_t shown, shift; // visible tokens; visible token j is position j, or j + shift from the sink's end on
};

// Steps that the units of a request of that length have each; 0: no request.
template <int ST>
__device__ __forceinline__ int32_t measure(const Params& p, int32_t len, int32_t* shown, int32_t* shift) {
  if (len < 0) return 0;
  len = min(len, p.room);
  *shown = p.a.window ? min(len, p.a.window + p.a.sink) : len;
  *shift = len - *shown;
  return *shown > ST ? static_cast<int32_t>((static_cast<uint32_t>(*shown) + ST - 1) / ST) : 1;
}

__device__ __forceinline__ uint32_t places(int32_t steps) { return steps ? steps + 1u : 0u; }

__device__ __forceinline__ int32_t request_after(const Params& p, int32_t r) { return r + 1 == p.a.n_req ? 0 : r + 1; }

// The unit behind v on its line.  `ahead` is the length of the request behind v's, loaded a unit early.
template <int ST>
__device__ __forceinline__ void next_unit(const Params& p, Unit& v, int32_t& ahead, int32_t lines) {
  int32_t skipped = 0;
#pragma unroll 1
  do {
    v.r = request_after(p, v.r);
    if (v.r == 0) v.u += lines;
    v.steps = measure<ST>(p, ahead, &v.shown, &v.shift);
    ahead = p.a.lens[request_after(p, v.r)];
  } while (v.steps == 0 && ++skipped < p.a.n_req);   // (some request has steps: the bound is for lengths that change meanwhile)
  v.left = v.steps = max(v.steps, 1);
}

// What a run that begins at place x of a line begins with: the step at x or the first one behind it; with `uncut`, inside a unit of few
// steps, the unit's first step or the next unit's, whichever is nearer (only the place is told then).
// *at: that step's place.  u: counted in the line.  pre[t]: places of the requests before thread t's `per` requests, of all: `all`.
template <int ST, int THREADS>
__device__ __forceinline__ Unit locate(const Params& p, const uint32_t* pre, int per, uint32_t all, uint32_t x, bool uncut, int32_t* at) {
  Unit v;
  v.u = x < all ? 0 : x / all;
  const uint32_t z = x - v.u * all;
  int lo = -1;   // (the whole warp is here)
#pragma unroll
  for (int k = 0; k < THREADS; k += 32) lo += __popc(__ballot_sync(0xffffffffu, pre[k + (threadIdx.x & 31)] <= z));
  uint32_t before = pre[lo];
  v.r = lo * per;
  v.shown = v.shift = 0;
  v.steps = measure<ST>(p, p.a.lens[v.r], &v.shown, &v.shift);
#pragma unroll 1
  while (before + places(v.steps) <= z && v.r < p.a.n_req - 1) {   // (z is less than the sum of all: the second bound is for lengths that change meanwhile)
    before += places(v.steps);
    v.steps = measure<ST>(p, p.a.lens[++v.r], &v.shown, &v.shift);
  }
  v.steps = max(v.steps, 1);
  int32_t step = max(static_cast<int32_t>(z - before) - 1, 0);
  if (uncut && v.steps <= kWhole) step = 2 * (z - before) >= places(v.steps) ? v.steps + 1 : 0;
  *at = v.u * all + before + 1 + step;
  v.left = v.steps - step;
  return v;
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
  int32_t r, u, steps;  // r < 0: none
  int32_t start;        // place of the unit's first step
};
constexpr int kPieceFloats = 16 * (128 + 1);   // of a piece in the scratch buffer: log-sum-exps, then rows
constexpr size_t counter_bytes(int ctas) { return (ctas * sizeof(uint32_t) + 255) / 256 * 256; }

// A row of D values over the lanes of a warp.
template <int D>
struct Lane;
template <>
struct Lane<128> {
  using Vec = float4;
  static __device__ __forceinline__ void scale(Vec& v, float f) { v.x *= f; v.y *= f; v.z *= f; v.w *= f; }
  static __device__ __forceinline__ void add(Vec& v, float e, const Vec& b) { v.x += e * b.x; v.y += e * b.y; v.z += e * b.z; v.w += e * b.w; }
  template <bool BF16>
  static __device__ __forceinline__ void store(void* O, int64_t i, int lane, const Vec& v) {
    reinterpret_cast<uint2*>(static_cast<uint16_t*>(O) + i)[lane] = make_uint2(pack2<BF16>(v.x, v.y), pack2<BF16>(v.z, v.w));
  }
};
template <>
struct Lane<64> {
  using Vec = float2;
  static __device__ __forceinline__ void scale(Vec& v, float f) { v.x *= f; v.y *= f; }
  static __device__ __forceinline__ void add(Vec& v, float e, const Vec& b) { v.x += e * b.x; v.y += e * b.y; }
  template <bool BF16>
  static __device__ __forceinline__ void store(void* O, int64_t i, int lane, const Vec& v) {
    reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(O) + i)[lane] = pack2<BF16>(v.x, v.y);
  }
};
// ---------------------------------------------------------------- the kernel
// Shared memory: a ring of STAGES steps per warp (at a warp's end also its last piece), the warps' first pieces, the steps' masks
// and exponents.
template <int MODE, int D, int NT, bool QBF>
__global__ void __launch_bounds__(32 * Shape<MODE, D, NT>::W, 1)
paged_attention(const __grid_constant__ Params p) {
  using S = Shape<MODE, D, NT>;
  constexpr int ST = S::ST, PADDED = S::PADDED, ROW = S::ROW, W = S::W, THREADS = 32 * W, STAGES = S::STAGES;
  constexpr bool E4 = MODE == WK_E4M3, BF = MODE == WK_BF16;
  constexpr int MT = D / 16;   // row tiles of O^T, and steps along the dimensions in S
  constexpr float UP = MODE == WK_F16 ? kUp : 0.f;   // (in 8 bits the sum has a reference of its own, and the weights' lies kUp below)
  extern __shared__ __align__(1024) uint8_t dyn[];
  __shared__ uint32_t pre[THREADS], parts[W];
  __shared__ float plse[2 * W][8 * NT];
  __shared__ Piece piece[2 * W], split[2];
  __shared__ uint32_t masks[W][STAGES][E4 ? 3 * S::RL : S::RL];   // which tokens there are; (8 bits) which byte of a word is theirs
  __shared__ int32_t to_come[W][4][3];   // units that the walk ahead has entered: request, unit, steps
  __shared__ int32_t first[2], count[2], n_groups, group_at[2 * W + 1], order[2 * W];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, c = lane & 3;
  uint8_t* const ring = dyn + warp * (STAGES * S::STEP);
  uint8_t* const firsts = dyn + W * (STAGES * S::STEP);
  uint8_t* const exps = firsts + W * S::PIECE + warp * (STAGES * S::META);
  // piece i of the CTA (warp i / 2's first or last)
  auto piece_rows = [&](int i) -> float* {
    return reinterpret_cast<float*>(i & 1 ? dyn + (i >> 1) * (STAGES * S::STEP) : firsts + (i >> 1) * S::PIECE);
  };

  // (launched while the kernel before it drains, and the one behind it likewise: nothing is read or written before this)
  dep_release();
  dep_wait();

  // ---- the line of steps, and this warp's run of it
  const int per = (p.a.n_req + THREADS - 1) / THREADS;
  uint32_t mine = 0;
#pragma unroll 1
  for (int i = 0; i < per; ++i) {
    const int r = tid * per + i;
    int32_t shown, shift;
    if (r >= p.a.n_req) break;
    const int32_t len = p.a.lens[r];
    mine += places(measure<ST>(p, len, &shown, &shift));
    if (blockIdx.x == 0 && len > p.room && p.a.status) atomicOr(p.a.status, WK_DEV_BAD_SLOT);
  }
  uint32_t up = mine;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const uint32_t o = __shfl_up_sync(0xffffffffu, up, d);
    if (lane >= d) up += o;
  }
  if (lane == 31) parts[warp] = up;
  __syncthreads();
  uint32_t before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    if (w < warp) before += parts[w];
    all += parts[w];
  }
  pre[tid] = before + up - mine;
  __syncthreads();
  // CTA k * lines + line takes the k-th run of a line; for short runs side by side is not worth the SMs that are left over.
  const uint32_t total = all * p.units;   // (the host has seen to it that places have 31 bits)
  const int lines = p.lines > 1 && total >= kLongRun * gridDim.x * W ? p.lines : 1;
  const int line = lines == 1 ? 0 : blockIdx.x % lines, column = lines == 1 ? blockIdx.x : blockIdx.x / lines;
  const int32_t length = lines == 1 ? total : total / lines, line0 = line * length;
  const Divisor by_workers = p.by_workers[lines > 1];
  const uint32_t workers = (lines == 1 ? gridDim.x : gridDim.x / lines) * W;
  int32_t run = by_workers.quotient(length + workers - 1);
  const int32_t chunk = run * W;
  if (column * chunk >= length) return;
  if (lane < 2) piece[2 * warp + lane].r = -1;
  // Short runs of short units: a CTA's run begins and ends with a unit, for a join of CTAs costs more than a few steps (20 requests of 55 tokens,
  // 8 heads of 64: 8.7 us -> 7.0; where runs are longer, cuts anywhere balance them: 256 requests of up to 300 tokens, 16 heads of 64, 21.2 us,
  // 23.2 if they went round units).
  int32_t a0 = column * chunk, a1 = min(a0 + chunk, length);
  if (run <= kShortRun && all <= 2u * kWhole * p.a.n_req) {
    const int32_t from = a0, to = a1;
    if (from > 0) locate<ST, THREADS>(p, pre, per, all, from, true, &a0);
    if (to < length) locate<ST, THREADS>(p, pre, per, all, to, true, &a1);
    run = max(a1 - a0 + W - 1, 0) / W;
  }
  const int32_t x = a0 + warp * run, xe = min(x + run, a1);
  a0 += line0;
  a1 += line0;

  if (x < xe) {
    uint32_t bad = 0;
    int32_t id[S::RL];             // page ids of the step after the next one to ask for, and places in the page
    uint32_t off[S::RL], row[S::RL], ex[S::RL];   // ex: place of the row's exponent bytes
    uint32_t qf[NT][MT][2];
    float sc[NT][2];               // logit scale of query heads 2c, 2c + 1
    float ref[NT][2], refw[NT][2]; // references of the sum and (8 bits) of the weights
    float sum[NT][2], o[NT][MT][4];
    int32_t place;                 // of the step at hand
    Unit nxt = locate<ST, THREADS>(p, pre, per, all, x, false, &place);   // of the step to look up; it is STAGES + 1 ahead
    nxt.u = nxt.u * lines + line;
    int32_t ahead = p.a.lens[request_after(p, nxt.r)];
    int32_t togo = xe - place;   // places from the step to look up to the end of this run
    int32_t steps = 0;             // of this run, as far as they have been looked up
    place += line0;
    int32_t cur_r = nxt.r, cur_u = nxt.u, of_unit = nxt.steps, left = nxt.left;   // of the step at hand
    Heads hc = heads_of<NT>(p, cur_u);
    int32_t kv_up = hc.kv, kv_ask = hc.kv;   // kv heads of the step to look up, of the one to ask for
    int32_t j_up = (of_unit - left) * ST + (lane & (ST - 1));   // this lane's token of the step to look up
    const int32_t* table = p.a.tables + nxt.r * p.a.table_stride;
    int in = 0, out = 0;                     // places in to_come
    bool whole = left == of_unit;            // the unit at hand began in this run
    bool fresh = true;
    // Where this lane's chunks go: token k * RPI + lane / LPR, swizzled so that eight rows' chunks lie in different banks.
    const uint32_t ring_at = ptx::smem_u32(ring), chunk_l = lane % S::LPR, hi = lane / S::LPR;
    const uint32_t to_l = hi * ROW + ((chunk_l ^ (ROW == 64 ? hi >> 1 & 3 : hi)) << 4);
    const int64_t v_minus_k = static_cast<const char*>(p.a.c.V) - static_cast<const char*>(p.a.c.K);
    int slot = 0;

#pragma unroll 1
    for (int32_t i = -STAGES - 1; i < steps || i < 0; ++i) {
      // ---- step i + STAGES: its page ids have come; rows of its tokens, a token per lane (or two)
      const bool ask = i >= -STAGES && i + STAGES < steps;
      if (ask) {
        kv_ask = kv_up;
#pragma unroll
        for (int k = 0; k < S::RL; ++k) {
          const bool there = static_cast<uint32_t>(id[k]) < static_cast<uint32_t>(p.a.c.n_pages);
          if (!there && id[k] != -1) bad = WK_DEV_BAD_SLOT;
          row[k] = there ? id[k] * p.page16 + off[k] * p.token16 : kNowhere;
          if constexpr (E4) ex[k] = there ? (static_cast<uint32_t>(id[k]) * p.a.c.n_kv_heads + kv_ask) * p.a.c.page_tokens + off[k] : 0;
        }
      }
      // ---- step i + STAGES + 1: look up the page ids
      if (i > -STAGES - 1 && togo > 0) {
        j_up += ST;
        --togo;
        if (--nxt.left == 0) {
          --togo;
          next_unit<ST>(p, nxt, ahead, lines);
          if (lane < 3) to_come[warp][in][lane] = lane == 0 ? nxt.r : lane == 1 ? nxt.u : nxt.steps;
          in = (in + 1) & 3;   // (at most STAGES + 1 of them are waiting)
          kv_up = heads_of<NT>(p, nxt.u).kv;
          j_up = lane & (ST - 1);
          table = p.a.tables + nxt.r * p.a.table_stride;
        }
      }
      if (togo > 0) {
        ++steps;
#pragma unroll
        for (int k = 0; k < S::RL; ++k) {
          const int32_t j = j_up + 32 * k;
          id[k] = -1;
          if (j < nxt.shown) {
            const uint32_t pos = static_cast<uint32_t>(j >= p.a.sink ? j + nxt.shift : j);
            const uint32_t at = p.by_page.quotient(pos);
            off[k] = pos - at * p.a.c.page_tokens;
            id[k] = table[at];   // (not through the read-only path: the kernel in front may have written it)
          }
        }
      }

      if (i >= 0) {
        copies_wait<STAGES - 1>();
        __syncwarp();
        const uint32_t k_at = ring_at + slot * S::STEP, v_at = k_at + S::STEP / 2;
        if (fresh) {   // a unit begins: Q has been asked for
          fresh = false;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            if (E4) {
              // row g by a power of two to below 2^15: exact in fp16 for all that matters beside the row's largest
              float top = 0.f;
#pragma unroll
              for (int s = 0; s < MT; ++s)
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
              for (int s = 0; s < MT; ++s)
#pragma unroll
                for (int e = 0; e < 2; ++e)
                  qf[nt][s][e] = pack2<false>(lo_of(qf[nt][s][e], QBF) * scale, hi_of(qf[nt][s][e], QBF) * scale);
              sc[nt][0] = __shfl_sync(0xffffffffu, back, 8 * c) * (p.a.scale * kLog2e);
              sc[nt][1] = __shfl_sync(0xffffffffu, back, 8 * c + 4) * (p.a.scale * kLog2e);
            } else {
              sc[nt][0] = sc[nt][1] = p.a.scale * kLog2e;
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
        }
        // ---- S^T = K Q^T.  A lane's place in the matrices that it points to: rows 0-7 and 8-15 of the left, then of the right 16 bytes
        float s[ST / 16][NT][4];
        {
          const int r8 = lane & 7, sw = ROW == 64 ? r8 >> 1 : r8;
          const uint32_t at = k_at + ((lane >> 3 & 1) * 8 + r8) * ROW + (((lane >> 4) ^ sw) << 4);
          constexpr int CHAINS = ST == 16 ? 2 : 1;   // sums that do not wait for one another (steps of several tiles have them anyway)
          float more[ST / 16][NT][4];
#pragma unroll
          for (int t = 0; t < ST / 16; ++t)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int e = 0; e < 4; ++e) s[t][nt][e] = more[t][nt][e] = 0.f;
#pragma unroll
          for (int j = 0; j < ROW / 32; ++j)
#pragma unroll
            for (int t = 0; t < ST / 16; ++t) {
              uint32_t f[4];
              load_matrices<false>(f, (at + t * 16 * ROW) ^ (j << 5));
              if constexpr (E4) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                  const uint32_t f0 = codes_lo(f[2 * h]), f1 = codes_lo(f[2 * h + 1]), f2 = codes_hi(f[2 * h]), f3 = codes_hi(f[2 * h + 1]);
#pragma unroll
                  for (int nt = 0; nt < NT; ++nt) mma<false>(s[t][nt], f0, f1, f2, f3, qf[nt][2 * j + h][0], qf[nt][2 * j + h][1]);
                }
              } else {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
                  mma<BF>(CHAINS == 2 && j % 2 ? more[t][nt] : s[t][nt], f[0], f[1], f[2], f[3], qf[nt][j][0], qf[nt][j][1]);
              }
            }
          if (CHAINS == 2) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int e = 0; e < 4; ++e) s[0][nt][e] += more[0][nt][e];
          }
        }
        // ---- logits (log2), their largest, the references
        float w[E4 ? ST / 16 : 1][NT][4];
        float top[NT][2], topw[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) top[nt][0] = top[nt][1] = topw[nt][0] = topw[nt][1] = -INFINITY;
        float vpower[E4 ? ST / 16 : 1][2], k_of[S::RL], v_of[S::RL];
        if constexpr (E4) {   // a lane for each token: its key's power of two, its value's exponent
#pragma unroll
          for (int k = 0; k < S::RL; ++k) {
            const uint2 w2 = *reinterpret_cast<const uint2*>(exps + slot * S::META + 8 * ((lane & (ST - 1)) + 32 * k));
            const uint32_t byte = (masks[warp][slot][S::RL + 2 * k] >> lane & 1) * 8 + (masks[warp][slot][S::RL + 2 * k + 1] >> lane & 1) * 16;
            k_of[k] = __uint_as_float((w2.x >> byte & 255u) << 23);
            v_of[k] = static_cast<float>(static_cast<int>(w2.y >> byte & 255u) - 127);
          }
        }
#pragma unroll
        for (int t = 0; t < ST / 16; ++t)
#pragma unroll
          for (int hh = 0; hh < 2; ++hh) {
            float kscale = 1.f;
            if constexpr (E4) {
              kscale = __shfl_sync(0xffffffffu, k_of[t / 2 % S::RL], t % 2 * 16 + hh * 8 + g);
              vpower[t][hh] = __shfl_sync(0xffffffffu, v_of[t / 2 % S::RL], t % 2 * 16 + hh * 8 + g);
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int e = 0; e < 2; ++e) s[t][nt][2 * hh + e] *= E4 ? sc[nt][e] * kscale : sc[nt][e];
          }
#pragma unroll
        for (int k = 0; k < S::RL; ++k) {
          const uint32_t mask = masks[warp][slot][k];
          if (mask != 0xffffffffu) {
#pragma unroll
            for (int t = 2 * k; t < (ST == 16 ? 1 : 2 * k + 2); ++t)
#pragma unroll
              for (int hh = 0; hh < 2; ++hh)
                if (!(mask >> (t % 2 * 16 + hh * 8 + g) & 1)) {
#pragma unroll
                  for (int nt = 0; nt < NT; ++nt) s[t][nt][2 * hh] = s[t][nt][2 * hh + 1] = -INFINITY;
                }
          }
        }
#pragma unroll
        for (int t = 0; t < ST / 16; ++t)
#pragma unroll
          for (int hh = 0; hh < 2; ++hh) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const float v = s[t][nt][2 * hh + e];
                top[nt][e] = fmaxf(top[nt][e], v);
                if constexpr (E4) {
                  w[t][nt][2 * hh + e] = v + vpower[t][hh];
                  topw[nt][e] = fmaxf(topw[nt][e], v + vpower[t][hh]);
                }
              }
          }
        bool moved = false;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 2; ++e)   // (differences: they are exact where it matters, so no weight passes 2^15, however large logits are)
            moved |= top[nt][e] - ref[nt][e] > UP + kLazy || (E4 && topw[nt][e] - refw[nt][e] > kUp + kLazy);
        if (__any_sync(0xffffffffu, moved)) {
          if constexpr (E4) {
            // A row of zeros is stored with power 1, which may lie far above the other rows', and would take the weights' reference
            // along: it gets no weight.  (Below the reference it does no harm, so that rows are looked at here only.)
            bool none = false;
#pragma unroll
            for (int k = 0; k < S::RL; ++k) {
              if (!__any_sync(0xffffffffu, v_of[k] == 0.f)) continue;
              const uint4* const x = reinterpret_cast<const uint4*>(ring + slot * S::STEP + S::STEP / 2 + ((lane & (ST - 1)) + 32 * k) * ROW);
              uint32_t bits = 0;
#pragma unroll 1
              for (int j = 0; j < ROW / 16; ++j) bits |= x[j].x | x[j].y | x[j].z | x[j].w;   // (all of the row, in whichever order)
              const uint32_t zero = __ballot_sync(0xffffffffu, v_of[k] == 0.f && !(bits & 0x7f7f7f7fu));
              none |= zero != 0;
#pragma unroll
              for (int t = 2 * k; t < 2 * k + 2; ++t)
#pragma unroll
                for (int hh = 0; hh < 2; ++hh)
                  if (zero >> (t % 2 * 16 + hh * 8 + g) & 1) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) w[t][nt][2 * hh] = w[t][nt][2 * hh + 1] = -INFINITY;
                  }
            }
            if (none) {
#pragma unroll
              for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                  topw[nt][e] = -INFINITY;
#pragma unroll
                  for (int t = 0; t < ST / 16; ++t) topw[nt][e] = fmaxf(topw[nt][e], fmaxf(w[t][nt][e], w[t][nt][2 + e]));
                }
            }
          }
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float m = fmaxf(top[nt][e], ref[nt][e] + UP), mw = fmaxf(topw[nt][e], refw[nt][e] + kUp);
#pragma unroll
              for (int d = 4; d < 32; d <<= 1) {
                m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
                if (E4) mw = fmaxf(mw, __shfl_xor_sync(0xffffffffu, mw, d));
              }
              m -= UP;
              const float f = m == -INFINITY ? 1.f : ex2_approx(ref[nt][e] - m);
              sum[nt][e] *= f;
              ref[nt][e] = m;
              float fw = f;
              if (E4) {
                mw -= kUp;
                fw = mw == -INFINITY ? 1.f : ex2_approx(refw[nt][e] - mw);
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
        const int r8 = lane & 7, sw = ROW == 64 ? r8 >> 1 : r8;
        const uint32_t at = v_at + ((lane >> 4) * 8 + r8) * ROW + (((lane >> 3 & 1) ^ sw) << 4);
        float at_sum[NT][2], at_w[NT][2];   // the references, 0 where no key has had weight
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            at_sum[nt][e] = ref[nt][e] == -INFINITY ? 0.f : ref[nt][e];
            at_w[nt][e] = refw[nt][e] == -INFINITY ? 0.f : refw[nt][e];
          }
#pragma unroll
        for (int t = 0; t < ST / 16; ++t) {
          uint32_t pf[NT][2];
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            float q[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              q[e] = ex2_approx(s[t][nt][e] - at_sum[nt][e & 1]);
              sum[nt][e & 1] += q[e];
              if constexpr (E4) q[e] = ex2_approx(w[t][nt][e] - at_w[nt][e & 1]);
            }
            pf[nt][0] = transpose8x8(pack2<BF>(q[0], q[1]));
            pf[nt][1] = transpose8x8(pack2<BF>(q[2], q[3]));
          }
#pragma unroll
          for (int j = 0; j < ROW / 32; ++j) {
            uint32_t f[4];
            load_matrices<true>(f, (at + t * 16 * ROW) ^ (j << 5));
            if constexpr (E4) {   // pairs of neighbouring dimensions of two tokens: to pairs of tokens
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                const uint32_t x0 = __byte_perm(f[h], 0, 0x3120), x1 = __byte_perm(f[2 + h], 0, 0x3120);
                const uint32_t f0 = codes_lo(x0), f1 = codes_hi(x0), f2 = codes_lo(x1), f3 = codes_hi(x1);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) mma<false>(o[nt][2 * j + h], f0, f1, f2, f3, pf[nt][0], pf[nt][1]);
              }
            } else {
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) mma<BF>(o[nt][j], f[0], f[1], f[2], f[3], pf[nt][0], pf[nt][1]);
            }
          }
        }
      }

      // ---- ask for the rows just looked up, in the place of the step just used
      __syncwarp();
      if (ask) {
        const uint32_t to = ring_at + slot * S::STEP + to_l;
        const char* const from = static_cast<const char*>(p.a.c.K) + kv_ask * p.head_bytes + chunk_l * 16;
#pragma unroll
        for (int k = 0; k < S::COPIES; ++k) {
          const uint32_t at = __shfl_sync(0xffffffffu, row[k * S::RPI / 32], (k * S::RPI + hi) & 31);
          const bool skip = at == kNowhere;
          const char* const src = from + static_cast<uint64_t>(skip ? 0 : at) * 16;
          const uint32_t dst = (ROW == 64 ? to : to ^ ((k * S::RPI & 7) << 4)) + k * 512;
          copy16(dst, src, skip);
          copy16(dst + S::STEP / 2, src + v_minus_k, skip);
        }
#pragma unroll
        for (int k = 0; k < S::RL; ++k) {
          const uint32_t mask = __ballot_sync(0xffffffffu, row[k] != kNowhere);
          if (lane == 0) masks[warp][slot][k] = mask;
          if constexpr (E4) {   // aligned words are what can be copied asynchronously: the one with the byte, up to the array's end
            const uint32_t to_ex = ptx::smem_u32(exps) + slot * S::META + 8 * ((lane & (ST - 1)) + 32 * k);
            const ByteWord word = word_of_byte(ex[k], p.n_exps);
            copy4(to_ex, p.a.c.K_exp + word.at, word.bytes);
            copy4(to_ex + 4, p.a.c.V_exp + word.at, word.bytes);
            const uint32_t lo = __ballot_sync(0xffffffffu, ex[k] & 1), hi2 = __ballot_sync(0xffffffffu, ex[k] & 2);
            if (lane == 0) {
              masks[warp][slot][S::RL + 2 * k] = lo;
              masks[warp][slot][S::RL + 2 * k + 1] = hi2;
            }
          }
        }
      }
      copies_commit();
      if (++slot == STAGES) slot = 0;

      // ---- does the unit end here, or this warp's part of it?  (What will be looked up has been: that is ahead.)
      if (i < -1) continue;
      const bool over = i >= 0 && --left == 0, ends = i >= 0 && (over || i + 1 == steps);
      if (!ends && i >= 0) {
        ++place;
        continue;
      }
      const int32_t was_r = cur_r, was_u = cur_u, was_steps = of_unit;
      const int32_t was_start = place - (of_unit - left - 1);
      const Heads hw = hc;
      if (over && i + 1 < steps) {
        place += 2;
        cur_r = to_come[warp][out][0];
        cur_u = to_come[warp][out][1];
        of_unit = left = to_come[warp][out][2];
        out = (out + 1) & 3;
        hc = heads_of<NT>(p, cur_u);
      }
      float f[NT][2];
      if (ends) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float l = sum[nt][e];
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) l += __shfl_xor_sync(0xffffffffu, l, d);
            sum[nt][e] = l == 0.f ? -INFINITY : ref[nt][e] + __log2f(l);   // log-sum-exp (log2)
            // (8 bits: the power in two parts, for values up to bf16's largest)
            f[nt][e] = l == 0.f ? 0.f : E4 ? __fdividef(ex2_approx(refw[nt][e] - ref[nt][e] + 4.f), 16.f * l) : __fdividef(1.f, l);
          }
      }
      if (i + 1 < steps) {   // Q of the unit that comes next: row g of every tile
        fresh = true;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const bool on = nt * 8 + g < hc.n;
          const uint16_t* q = static_cast<const uint16_t*>(p.a.Q) + cur_r * p.a.q_stride + static_cast<int64_t>(hc.first + (on ? nt * 8 + g : 0)) * D;
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            if (E4) {
              const uint2 v = on ? *reinterpret_cast<const uint2*>(q + m * 16 + 4 * c) : make_uint2(0, 0);
              qf[nt][m][0] = v.x;
              qf[nt][m][1] = v.y;
            } else {
#pragma unroll
              for (int e = 0; e < 2; ++e) qf[nt][m][e] = on ? *reinterpret_cast<const uint32_t*>(q + m * 16 + 8 * e + 2 * c) : 0u;
            }
          }
        }
      }
      if (ends) {
        const int which = 2 * warp + whole;   // reaches in: the warp's first unit; out: its last
        if (whole && over) {
          // transposed in registers: lane (g, c) then has head g's dimensions 2c, 2c + 1 of every 8 (8 bits: 4c .. 4c + 3 of 16)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            const int64_t head = static_cast<int64_t>(was_r) * p.a.n_heads + hw.first + nt * 8;
            uint16_t* const to = static_cast<uint16_t*>(p.a.O) + (head + g) * D;
#pragma unroll
            for (int m = 0; m < MT; ++m) {
              const uint32_t y0 = transpose8x8(pack2<QBF>(o[nt][m][0] * f[nt][0], o[nt][m][1] * f[nt][1]));
              const uint32_t y1 = transpose8x8(pack2<QBF>(o[nt][m][2] * f[nt][0], o[nt][m][3] * f[nt][1]));
              if (nt * 8 + g < hw.n) {
                if (E4) {
                  *reinterpret_cast<uint2*>(to + m * 16 + 4 * c) = make_uint2(__byte_perm(y0, y1, 0x5410), __byte_perm(y0, y1, 0x7632));
                } else {
                  *reinterpret_cast<uint32_t*>(to + m * 16 + 2 * c) = y0;
                  *reinterpret_cast<uint32_t*>(to + m * 16 + 8 + 2 * c) = y1;
                }
              }
            }
            if (g == 0 && p.a.lse) {
#pragma unroll
              for (int e = 0; e < 2; ++e)
                if (nt * 8 + 2 * c + e < hw.n) p.a.lse[head + 2 * c + e] = sum[nt][e] * kLn2;
            }
          }
        } else {
          float* const rows = piece_rows(which);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int q = nt * 8 + 2 * c + e;
              if (q >= hw.n) continue;
#pragma unroll
              for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int h = 0; h < 2; ++h)
                  rows[q * PADDED + m * 16 + (E4 ? 2 * g + h : 8 * h + g)] = o[nt][m][2 * h + e] * f[nt][e];
              if (g == 0) plse[which][q] = sum[nt][e];
            }
          if (lane == 0) piece[which] = Piece{was_r, was_u, was_steps, was_start};
        }
        whole = true;
      }
    }
    if (bad && p.a.status) atomicOr(p.a.status, bad);
  }
  __syncthreads();

  // ---- pieces of one unit lie next to each other: joined into O, or into this CTA's piece.  A warp takes a row at a time.
  float* const partial = reinterpret_cast<float*>(p.a.scratch + p.counter_bytes);
  if (warp == 0) {
    static_assert(2 * W <= 32, "a lane per piece");
    const bool there = lane < 2 * W && piece[lane].r >= 0;
    const uint32_t all_there = __ballot_sync(0xffffffffu, there), below = all_there & ((1u << lane) - 1);
    const int prev = below ? 31 - __clz(below) : lane;
    const bool start = there && (prev == lane || piece[prev].r != piece[lane].r || piece[prev].u != piece[lane].u);
    const uint32_t starts = __ballot_sync(0xffffffffu, start);
    if (lane < 2) split[lane].r = -1;
    __syncwarp();
    if (there) order[__popc(below)] = lane;
    if (start) {
      const Piece u = piece[lane];
      group_at[__popc(starts & ((1u << lane) - 1))] = __popc(below);
      if (u.start < a0 || u.start + u.steps > a1) {
        const int side = u.start < a0 ? 0 : 1;
        split[side] = u;
        const int k = static_cast<uint32_t>(u.start - line0) / static_cast<uint32_t>(chunk);
        first[side] = k * lines + line;   // the CTA that the unit begins in
        count[side] = static_cast<uint32_t>(u.start + u.steps - 1 - line0) / static_cast<uint32_t>(chunk) - k + 1;
      }
    }
    if (lane == 0) {
      n_groups = __popc(starts);
      group_at[__popc(starts)] = __popc(all_there);
    }
  }
  __syncthreads();
  using Vec = typename Lane<D>::Vec;       // a lane's part of a row
  const int rows = min(8 * NT, p.group);   // query heads of a full unit
#pragma unroll 1
  for (int it = warp; it < n_groups * rows; it += W) {
    const int k = it / rows, q = it - k * rows;
    const int i0 = group_at[k], n = group_at[k + 1] - i0;
    const Piece u = piece[order[i0]];
    const Heads h = heads_of<NT>(p, u.u);
    if (q >= h.n) continue;
    const float lse = lane < n ? plse[order[i0 + lane]][q] : -INFINITY;
    float m = warp_max(lse), l = 0.f;
    if (m == -INFINITY) m = 0.f;
    const float e = ex2_approx(lse - m);
    Vec v = {};
#pragma unroll 4
    for (int i = 0; i < n; ++i) {
      const float w = __shfl_sync(0xffffffffu, e, i);
      l += w;
      Lane<D>::add(v, w, reinterpret_cast<const Vec*>(piece_rows(order[i0 + i]) + q * PADDED)[lane]);
    }
    Lane<D>::scale(v, l == 0.f ? 0.f : __fdividef(1.f, l));
    l = l == 0.f ? -INFINITY : m + __log2f(l);
    if (u.start >= a0 && u.start + u.steps <= a1) {
      const int64_t at = static_cast<int64_t>(u.r) * p.a.n_heads + h.first + q;
      Lane<D>::template store<QBF>(p.a.O, at * D, lane, v);
      if (lane == 0 && p.a.lse) p.a.lse[at] = l * kLn2;
    } else {
      float* const to = partial + static_cast<int64_t>(2 * blockIdx.x + (u.start < a0 ? 0 : 1)) * kPieceFloats;
      reinterpret_cast<Vec*>(to + 8 * NT + q * D)[lane] = v;
      if (lane == 0) to[q] = l;
    }
  }
  if (split[0].r < 0 && split[1].r < 0) return;

  // ---- units that other CTAs share: the last of them to arrive joins the pieces
  __syncthreads();
  if (tid < 2) {
    const uint32_t n = split[tid].r < 0 ? 0 : count[tid] - 1;
    bool mine = false;
    if (n) {
      __threadfence();   // the barrier has ordered the CTA's pieces before this
      mine = atomicInc(reinterpret_cast<uint32_t*>(p.a.scratch) + first[tid], n) == n;
      if (mine) __threadfence();
    }
    if (!mine) count[tid] = 0;
  }
  __syncthreads();
  Vec* const part = reinterpret_cast<Vec*>(dyn);                              // [W][32]
  float* const sums = reinterpret_cast<float*>(dyn + W * 32 * sizeof(Vec));   // [W][2]: reference and sum of a part
  const int n0 = count[0] ? heads_of<NT>(p, split[0].u).n : 0, tasks = n0 + (count[1] ? heads_of<NT>(p, split[1].u).n : 0);
  int lg = 0;   // 2^lg warps share a row, taking the pieces in turn (as many whoever arrives last: the order of the sums is fixed)
  while (rows << (lg + 2) <= W) ++lg;
#pragma unroll 1
  for (int t0 = 0; t0 < tasks; t0 += W >> lg) {
    const int task = t0 + (warp >> lg), set = warp & ((1 << lg) - 1);
    const int side = task >= n0;
    const bool on = task < tasks;
    const int n = on ? count[side] : 0, q = task - (side ? n0 : 0);
    float top = -INFINITY, l = 0.f;   // of this warp's pieces
    Vec v = {};
    // the unit's first CTA has it as its last unit, the others as their first
    const float* const from = partial + (2 * first[side] + 1) * static_cast<int64_t>(kPieceFloats) + q;
    auto piece_at = [&](int i) { return from + (2 * i * lines - (i != 0)) * static_cast<int64_t>(kPieceFloats); };
#pragma unroll 1
    for (int i0 = set; i0 < n; i0 += 32 << lg) {   // 32 of the pieces at a time
      const int mine = i0 + (lane << lg), some = min((n - i0 + (1 << lg) - 1) >> lg, 32);
      const float lse = mine < n ? __ldcg(piece_at(mine)) : -INFINITY;
      Vec b[4];
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (k < some) b[k] = __ldcg(reinterpret_cast<const Vec*>(piece_at(i0 + (k << lg)) - q + 8 * NT + q * D) + lane);
      const float m = fmaxf(warp_max(lse), top), keep = m == -INFINITY ? 1.f : ex2_approx(top - m);
      const float e = ex2_approx(lse - (m == -INFINITY ? 0.f : m));
      top = m;
      l *= keep;
      Lane<D>::scale(v, keep);
#pragma unroll 1
      for (int k0 = 0; k0 < some; k0 += 4) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (k0 + k < some) {
            const float w = __shfl_sync(0xffffffffu, e, k0 + k);
            l += w;
            Lane<D>::add(v, w, b[k]);
          }
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (k0 + 4 + k < some) b[k] = __ldcg(reinterpret_cast<const Vec*>(piece_at(i0 + ((k0 + 4 + k) << lg)) - q + 8 * NT + q * D) + lane);
      }
    }
    if (lg) {
      part[warp * 32 + lane] = v;
      if (lane == 0) {
        sums[2 * warp] = top;
        sums[2 * warp + 1] = l;
      }
      __syncthreads();
      if (set == 0) {
        const float t = lane < 1 << lg ? sums[2 * (warp + lane)] : -INFINITY, s = lane < 1 << lg ? sums[2 * (warp + lane) + 1] : 0.f;
        top = warp_max(t);
        const float e = ex2_approx(t - (top == -INFINITY ? 0.f : top));
        l = 0.f;
        v = {};
#pragma unroll 1
        for (int k = 0; k < 1 << lg; ++k) {
          const float w = __shfl_sync(0xffffffffu, e, k);
          l += w * __shfl_sync(0xffffffffu, s, k);
          Lane<D>::add(v, w, part[(warp + k) * 32 + lane]);
        }
      }
    }
    if (on && set == 0) {
      Lane<D>::scale(v, l == 0.f ? 0.f : __fdividef(1.f, l));
      const int64_t to = static_cast<int64_t>(split[side].r) * p.a.n_heads + heads_of<NT>(p, split[side].u).first + q;
      Lane<D>::template store<QBF>(p.a.O, to * D, lane, v);
      if (lane == 0 && p.a.lse) p.a.lse[to] = l == 0.f ? -INFINITY : (top + __log2f(l)) * kLn2;
    }
    if (lg) __syncthreads();
  }
}

template <int MODE, int D, int NT, bool QBF>
wk_status launch(wk_ctx* ctx, const Params& p, cudaStream_t s) {
  using S = Shape<MODE, D, NT>;
  constexpr int smem = S::W * (S::STAGES * (S::STEP + S::META) + S::PIECE);
  const int i = ((MODE * 2 + (D == 128)) * 2 + NT - 1) * 2 + QBF;
  if (!(ctx->paged_attr_set >> i & 1)) {
    WK_CUDA_TRY(ctx, cudaFuncSetAttribute(paged_attention<MODE, D, NT, QBF>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
    ctx->paged_attr_set |= 1u << i;
  }
  launch_chained(paged_attention<MODE, D, NT, QBF>, dim3(ctx->sm_count), dim3(32 * S::W), smem, s, p);
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

static wk_status launch_requests(wk_ctx* ctx, const PagedArgs& a, int32_t room, cudaStream_t s) {
  Params p;
  p.a = a;
  p.group = a.n_heads / a.c.n_kv_heads;
  const int nt = p.group > 8 ? 2 : 1;
  p.q_tiles = paged_query_tiles(p.group);
  p.units = a.c.n_kv_heads * p.q_tiles;
  const int es = a.c.type == WK_E4M3 ? 1 : 2;
  // Units of long requests are walked side by side, so that rows of neighbouring heads, neighbours in memory as a rule, are read at
  // about the same time, and the rows of a kv head with more than 16 query heads once.  Rows of 128 bytes (8 bits), 16 x 20,000
  // tokens of 8 heads: 121 us -> 107, of 16 heads 124 -> 107; of 64 bytes 112 -> 69; rows of 256 bytes gain nothing (197 -> 196).
  // As many lines as leave hardly any SM over.
  p.lines = 1;
  if (a.c.head_dim * es < 256 || p.q_tiles > 1)
    for (int d = 2; d <= 16; ++d)
      if (p.units % d == 0 && ctx->sm_count / d * d >= ctx->sm_count - ctx->sm_count / 32) p.lines = d;
  p.room = room;
  p.page16 = static_cast<uint32_t>(a.c.page_stride * es / 16);
  p.token16 = static_cast<uint32_t>(a.c.token_stride * es / 16);
  p.head_bytes = a.c.head_stride * es;
  p.n_exps = static_cast<uint32_t>(a.c.n_pages) * a.c.page_tokens * a.c.n_kv_heads;   // (8 bits: less than 2^32)
  p.by_page = divisor(a.c.page_tokens);
  using S = Shape<WK_BF16, 128, 1>;   // (all shapes have as many warps)
  p.by_workers[0] = divisor(ctx->sm_count * S::W);
  p.by_workers[1] = divisor(ctx->sm_count / p.lines * S::W);
  p.counter_bytes = static_cast<int32_t>(counter_bytes(ctx->sm_count));
  if (a.c.type == WK_BF16) return choose<WK_BF16, true>(ctx, p, nt, s);
  if (a.c.type == WK_F16) return choose<WK_F16, false>(ctx, p, nt, s);
  return a.q_type == WK_BF16 ? choose<WK_E4M3, true>(ctx, p, nt, s) : choose<WK_E4M3, false>(ctx, p, nt, s);
}

wk_status launch_paged_attention(wk_ctx* ctx, const PagedArgs& a, cudaStream_t s) {
  // The kernel counts places of its line in 31 bits.  What the lengths are only the GPU knows; where the tables have room for more
  // than that, the requests are taken in several launches.  (For a single request it is 2^35 tokens over its kv heads, more than a
  // cache of less than 64 GB holds.)
  const int64_t units = static_cast<int64_t>(a.c.n_kv_heads) * paged_query_tiles(a.n_heads / a.c.n_kv_heads);
  const int64_t most = 0x7fff0000LL / units;   // places of the requests of a launch, per unit
  const int64_t room = std::min<int64_t>(static_cast<int64_t>(a.max_pages) * a.c.page_tokens, (most - 2) * 16);
  const int64_t each = room / 16 + 2, some = std::max<int64_t>(std::min<int64_t>(a.n_req, most / each), 1);
  for (int64_t r = 0; r < a.n_req; r += some) {
    PagedArgs b = a;
    b.n_req = static_cast<int32_t>(std::min<int64_t>(some, a.n_req - r));
    b.Q = static_cast<const uint16_t*>(a.Q) + r * a.q_stride;
    b.O = static_cast<uint16_t*>(a.O) + r * a.n_heads * a.c.head_dim;
    b.lse = a.lse ? a.lse + r * a.n_heads : nullptr;
    b.tables = a.tables + r * a.table_stride;
    b.lens = a.lens + r;
    const wk_status st = launch_requests(ctx, b, static_cast<int32_t>(room), s);
    if (st != WK_OK) return st;
  }
  return WK_OK;
}

}  // namespace wk
