// Attention of a chunk on the 5th-generation tensor cores: forward, and the two kernels of the backward.
//
// Every product is a chain of 128 x N x 16 tcgen05 MMAs into TMEM.  The softmax weights go from registers straight back
// into TMEM (over the scores they came from) and are the next product's first operand from there, so no score ever
// touches shared or global memory.  Tiles come in by TMA as 64-column, 128-byte-swizzled boxes of 128 rows of one head;
// the same box serves as a K-contiguous operand (contraction over head_dim) and as an M/N-contiguous one (contraction
// over its rows).  Head dims up to 64 and up to 128 have a kernel each; the columns behind head_dim read as zero.
#include "attention.cuh"
#include "tc_device.cuh"
#include "tc_host.h"

#include <algorithm>
#include <cfloat>

namespace templora {
namespace {

constexpr int kRows = 128;               // rows of a tile
constexpr int kBox = kRows * 64 * 2;     // bytes of one 64-column box

// ------------------------------------------------------------------ instruction wrappers beyond tc_device.cuh
// Before the CTA may exit its stores must have left shared memory; before a row is written again they must be complete.
__device__ __forceinline__ void finish_stores(bool rewritten) {
  bulk_commit_group();
  if (rewritten) bulk_wait_group_all(); else bulk_wait_group_read<0>();
}
__device__ __forceinline__ void prefetch_map(const CUtensorMap *map) {
  asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}
__device__ __forceinline__ void tma_store_3d(const CUtensorMap *map, uint32_t src, int c0, int c1, int c2) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];"
               ::"l"(map), "r"(src), "r"(c0), "r"(c1), "r"(c2) : "memory");
}
// D += A B with A (bf16, 128 rows, 8 columns of TMEM per 16 contraction steps) in TMEM
__device__ __forceinline__ void tc_mma_bf16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc,
                                               uint32_t accumulate) {
  asm volatile(
      "{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\n"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}"
      ::"r"(d_tmem), "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t *v) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};"
      ::"r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
        "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rcp(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  const __nv_bfloat162 t = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t *>(&t);
}

// mbar_wait, inline: a call would force the many values that are live across a wait into memory
__device__ __forceinline__ bool wait_inline(uint32_t bar, uint32_t parity, volatile int *abort_flag, DeviceStatus *st, int where) {
  if (mbar_try(bar, parity)) return true;
  unsigned long long t0 = 0;
  for (unsigned n = 1;; ++n) {
    if (mbar_try(bar, parity)) return true;
    if ((n & 255u) == 0) {
      if (*abort_flag) return false;
      const unsigned long long t = globaltimer_ns();
      if (t0 == 0) t0 = t;
      if (t - t0 > kWaitLimitNs) {
        *abort_flag = 1;
        if (atomicCAS(&st->code, 0, (int)TEMPLORA_ERR_TIMEOUT) == 0) st->where = where;
        __threadfence();
        return false;
      }
    }
  }
}

// K-contiguous operand tile: descriptor of contraction steps [16 k, 16 k + 16); boxes of 64 columns follow one another
__device__ __forceinline__ uint64_t desc_k(uint64_t tmpl, uint32_t tile, int k) {
  return tmpl | (uint64_t)(((tile + (k >> 2) * kBox + (k & 3) * 32) & 0x3FFFFu) >> 4);
}
// the same tile contracted over its rows: steps are 16 rows, boxes are the chunks along N
__device__ __forceinline__ uint64_t desc_mn(uint64_t tmpl, uint32_t tile, int k) {
  return tmpl | (uint64_t)(((tile + k * 2048) & 0x3FFFFu) >> 4);
}

// ------------------------------------------------------------------ pairs of fp32 values
// sm_100 multiplies and adds two fp32 values per lane and instruction.
__device__ __forceinline__ uint64_t f2(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ uint64_t f2u(uint32_t a, uint32_t b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ float2 un2(uint64_t v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// ------------------------------------------------------------------ score modifications, in units of log2
// z = tanh(s * cap_in) * cap_out - slope * |p - j|, or s * cap_out - slope * |p - j| without a cap.
struct ScoreMod {
  float cap_in, cap_out;   // scale / softcap and softcap * log2(e); without a cap 0 and scale * log2(e)
};

// tanh(x) = 1 - 2 / (1 + exp(2 x)): absolute error about 1e-7, two special-function instructions
__device__ __forceinline__ float tanh_of_scaled(float x2log2e) { return fmaf(-2.f, rcp(1.f + ex2(x2log2e)), 1.f); }

// The polynomial of two values: scores rarely come near their cap, and seven multiply-adds on a pipe with eight times the
// special-function unit's rate replace its two instructions.
__device__ __forceinline__ uint64_t tanh_poly2(uint64_t x) {
  const uint64_t u = mul2(x, x);
  uint64_t f = fma2(u, f2(kTanh5, kTanh5), f2(kTanh4, kTanh4));
  f = fma2(u, f, f2(kTanh3, kTanh3));
  f = fma2(u, f, f2(kTanh2, kTanh2));
  f = fma2(u, f, f2(kTanh1, kTanh1));
  f = fma2(u, f, f2(kTanh0, kTanh0));
  return mul2(x, f);
}

// 32 scores of a row (columns j0 ...; back = position - j0) to z in place; with KEEP_T, t receives their tanh.
template <bool KEEP_T>
__device__ __forceinline__ void modify_scores(const ScoreMod &mod, bool slopes, float slope, float back, uint32_t (&v)[32],
                                              float *t) {
  if (mod.cap_in != 0.f) {
    float big = 0.f;
#pragma unroll
    for (int i = 0; i < 32; i += 2) big = fmaxf(fmaxf(big, fabsf(__uint_as_float(v[i]))), fabsf(__uint_as_float(v[i + 1])));
    const uint64_t out = f2(mod.cap_out, mod.cap_out);
    if (__all_sync(0xffffffffu, big * fabsf(mod.cap_in) <= kTanhPolyMax)) {
      const uint64_t in = f2(mod.cap_in, mod.cap_in);
#pragma unroll
      for (int i = 0; i < 32; i += 2) {
        const uint64_t th = tanh_poly2(mul2(f2u(v[i], v[i + 1]), in));
        const float2 z = un2(mul2(th, out));
        v[i] = __float_as_uint(z.x); v[i + 1] = __float_as_uint(z.y);
        if (KEEP_T) { const float2 w = un2(th); t[i] = w.x; t[i + 1] = w.y; }
      }
    } else {
      const float in = mod.cap_in * (2.f * kLog2e);
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        const float th = tanh_of_scaled(__uint_as_float(v[i]) * in);
        v[i] = __float_as_uint(th * mod.cap_out);
        if (KEEP_T) t[i] = th;
      }
    }
  } else if (KEEP_T) {
#pragma unroll
    for (int i = 0; i < 32; ++i) t[i] = 0.f;
  }
  const float c = mod.cap_in != 0.f ? 1.f : mod.cap_out;
  const bool ahead = back >= 31.f, behind = back <= 0.f;
  if (slopes && (__all_sync(0xffffffffu, ahead) || __all_sync(0xffffffffu, behind))) {
    // all keys on one side of all rows: the distance is linear, two multiply-adds a score instead of three instructions
    const float up = ahead ? slope : -slope, from = -up * back;
    const uint64_t c2 = f2(c, c), up2 = f2(up, up), from2 = f2(from, from);
#pragma unroll
    for (int i = 0; i < 32; i += 2) {
      const float2 z = un2(fma2(f2u(v[i], v[i + 1]), c2, fma2(f2((float)i, (float)(i + 1)), up2, from2)));
      v[i] = __float_as_uint(z.x); v[i + 1] = __float_as_uint(z.y);
    }
  } else if (slopes) {
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __float_as_uint(fmaf(-slope, fabsf(back - (float)i), __uint_as_float(v[i]) * c));
  } else if (mod.cap_in == 0.f) {
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) * c);
  }
}

// ------------------------------------------------------------------ masks
// Bits of 32 places that lie in [lo, hi).
__device__ __forceinline__ uint32_t span_bits(int lo, int hi) {
  lo = min(max(lo, 0), 32);
  hi = min(max(hi, 0), 32);
  return lo < hi ? (0xffffffffu >> (32 - hi)) & (0xffffffffu << lo) : 0u;
}
// 32 x 32 bits over a warp: bit i of lane j becomes bit j of lane i.
__device__ __forceinline__ uint32_t transpose_bits(uint32_t x, int lane) {
  uint32_t m = 0x0000ffffu;
#pragma unroll
  for (int j = 16; j > 0; j >>= 1, m ^= m << j) {
    const uint32_t y = __shfl_xor_sync(0xffffffffu, x, j);
    x = (lane & j) ? (x & ~m) | ((y & ~m) >> j) : (x & m) | ((y & m) << j);
  }
  return x;
}

// ------------------------------------------------------------------ forward
// One CTA works on two 128-row query tiles that share their keys and values: two heads of a group on the same rows, or,
// with ungrouped heads, two row tiles of one head.  Eight softmax warps per tile: a thread has one row and half of the
// tile's 64 columns, so row sums need no shuffles and the maxima of the two halves meet (through shared memory) only
// when one outgrows the running maximum by 2^8; until then probabilities simply exceed 1, and the accumulator is not
// rescaled.  The final division uses the same maximum, so this costs no accuracy.  Warp 16 issues the copies, warp 17
// the MMAs.  While one tile's softmax runs, the tensor core works for the other.  TMEM: two 128-column score tiles (the
// bf16 probabilities over them) and two output accumulators of up to 128 columns.
// A 128 x 128 tile needs 1024 clocks of the tensor core for its two products and as many of the special-function unit for
// its exponentials (16 a clock).  It takes about 1960: with two tiles in flight neither unit is busy more than half of
// the time, and what a tile waits for is its own chain: product, scores out of TMEM, maximum, exponentials, weights back into
// TMEM, product.  64 heads over 8 kv heads, 4096 tokens, causal: 266 us (1030 TFLOP/s of the seen half); with capped scores
// 413 us (666); tensor pipe 32 %, special functions 33 %, issue slots 50 %.  A CTA of few tiles costs its start and end,
// 6 to 7 us, as much as three or four tiles: 1024 tokens of 32 heads take 22 us (390 TFLOP/s).
constexpr int kSoftmaxWarps = 16, kThreadsTc = 32 * (kSoftmaxWarps + 2);
template <int DP> struct FwdCfg {
  static constexpr int kTileB = kRows * DP * 2;
  static constexpr int kStages = DP == 128 ? 4 : 8;
  static constexpr int kSmem = 2 * kTileB + kStages * kTileB + 1024 + 512 + 2048;
};

struct FwdParams {
  CUtensorMap tq, tk, tv, to;
  AttnShape s;
  AttnTensors x;
  DeviceStatus *status;
  ScoreMod mod;
  float c;              // scores to units of log2 when nothing modifies them (MOD == 0)
  int row_units;        // row tiles (heads paired) or pairs of them (rows paired)
  int pairing;          // kPairHeads, kPairRows or kPairMirrored
  int tiles;            // row tiles
  int units;            // heads or pairs of heads
  int parts;            // CTAs that share a CTA's keys
  float *part_o;        // [parts][H][Tq][D] sums not yet divided, when parts > 1
  float2 *part_ml;      // [parts][H][Tq] maximum (log2) and sum
};
enum { kPairHeads, kPairRows, kPairMirrored };

// barrier of the 256 softmax threads of a tile; true when `vote` holds on any of them
__device__ __forceinline__ bool tile_any(int w, bool vote) {
  uint32_t r;
  asm volatile("{\n.reg .pred p, q;\nsetp.ne.u32 p, %1, 0;\nbarrier.cta.red.or.pred q, %2, 256, p;\nselp.u32 %0, 1, 0, q;\n}"
               : "=r"(r) : "r"((uint32_t)vote), "r"(w + 1) : "memory");
  return r != 0;
}
__device__ __forceinline__ void tile_sync(int w) { asm volatile("barrier.cta.sync %0, 256;" ::"r"(w + 1) : "memory"); }

// 32 accumulator columns, scaled, to the staging tile (128-byte swizzle); returns whether one is not finite
__device__ __forceinline__ bool stage_columns(uint32_t t_acc, bool any, float scale, uint32_t tile, int r, int d) {
  uint32_t o[32];
  bool bad = false;
  if (any) {
    tmem_ld32(t_acc + d, o);
    tmem_ld_wait();
  } else {
#pragma unroll
    for (int i = 0; i < 32; ++i) o[i] = 0;
  }
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    const float v = __uint_as_float(o[i]) * scale;
    bad |= !(fabsf(v) < INFINITY);
    o[i] = __float_as_uint(v);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int chunk = ((d & 63) >> 3) + i;
    st_shared_v4(tile + r * 128 + (d >> 6) * kBox + ((chunk ^ (r & 7)) << 4), pack_bf16x2(o[8 * i], o[8 * i + 1]),
                 pack_bf16x2(o[8 * i + 2], o[8 * i + 3]), pack_bf16x2(o[8 * i + 4], o[8 * i + 5]),
                 pack_bf16x2(o[8 * i + 6], o[8 * i + 7]));
  }
  return bad;
}

__device__ __forceinline__ void tmem_alloc_all(volatile uint32_t *slot) {
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32((const void *)slot)),
               "r"(512u) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free_all(uint32_t tmem) {
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
}
// MMAs already issued must finish before TMEM is released
__device__ __forceinline__ void drain_mmas(uint32_t bar) {
  tc_commit(bar);
  const unsigned long long t0 = globaltimer_ns();
  while (!mbar_try(bar, 0) && globaltimer_ns() - t0 < kWaitLimitNs) {}
}

// PARTS: several CTAs share the keys of a CTA's rows (a kernel of its own: the code for it costs the other one 2 %)
template <int DP, int MOD, bool PARTS>
__global__ void __launch_bounds__(kThreadsTc, 1) attn_fwd_tc_kernel(const __grid_constant__ FwdParams P) {
  using Cfg = FwdCfg<DP>;
  constexpr int kS = Cfg::kStages, kTileB = Cfg::kTileB;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem0 = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t *smem = smem_raw + (smem0 - smem_u32(smem_raw));
  const uint32_t ring = smem0 + 2 * kTileB, bar0 = ring + kS * kTileB;
  auto full = [&](int i) { return bar0 + 8u * i; };
  auto empty = [&](int i) { return bar0 + 8u * (kS + i); };
  auto s_full = [&](int w) { return bar0 + 8u * (2 * kS + w); };
  auto p_ready = [&](int w, int part) { return bar0 + 8u * (2 * kS + 2 + 2 * w + part); };
  auto o_full = [&](int w) { return bar0 + 8u * (2 * kS + 6 + w); };
  const uint32_t q_full = bar0 + 8u * (2 * kS + 8), drain = bar0 + 8u * (2 * kS + 9);
  uint8_t *tail = smem + 2 * kTileB + kS * kTileB + 256;
  volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(tail);
  volatile int *abort_flag = reinterpret_cast<volatile int *>(tail + 4);
  volatile int *tile_abort = reinterpret_cast<volatile int *>(tail + 8);     // [tile][iteration parity]
  int *range = reinterpret_cast<int *>(tail + 32);   // per tile: smallest start, largest end
  unsigned *bad_rows = reinterpret_cast<unsigned *>(tail + 64);              // [tile][4]
  float *exchange = reinterpret_cast<float *>(tail + 256);                   // [tile][half][128]

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const AttnShape &s = P.s;
  // the longest row tiles of a causal call come first
  const int unit = blockIdx.x % P.units, ru = P.row_units - 1 - blockIdx.x / P.units;
  auto head_of = [&](int w) { return P.pairing == kPairHeads ? 2 * unit + w : unit; };
  auto row_of = [&](int w) {
    if (P.pairing == kPairHeads) return ru * kRows;
    if (P.pairing == kPairRows) return (2 * ru + w) * kRows;
    const int other = P.tiles - 1 - ru;       // mirrored: a long row tile with a short one; the middle one is alone
    return (w == 0 ? other : ru == other ? P.tiles : ru) * kRows;
  };
  const int hk = head_of(0) / s.group;

  // the copying thread starts with what needs no other thread
  if (threadIdx.x == 32 * kSoftmaxWarps) {
    for (int i = 0; i < kS; ++i) { mbar_init(full(i), 1); mbar_init(empty(i), 1); }
    for (int w = 0; w < 2; ++w) { mbar_init(s_full(w), 1); mbar_init(p_ready(w, 0), 8); mbar_init(p_ready(w, 1), 8); mbar_init(o_full(w), 1); }
    mbar_init(q_full, 1);
    mbar_init(drain, 1);
    *abort_flag = 0;
    for (int i = 0; i < 4; ++i) tile_abort[i] = 0;
    for (int i = 0; i < 8; ++i) bad_rows[i] = 0;
    for (int w = 0; w < 2; ++w) { range[2 * w] = s.Tk; range[2 * w + 1] = 0; }
    fence_barrier_init();
    pdl_join();
    int n_q = 0;
    for (int w = 0; w < 2; ++w) n_q += row_of(w) < s.Tq;
    mbar_arrive_expect_tx(q_full, (uint32_t)(n_q * kTileB));
    for (int w = 0; w < 2; ++w)
      if (row_of(w) < s.Tq)
        for (int c = 0; c < DP / 64; ++c) tma_load_3d(smem0 + w * kTileB + c * kBox, &P.tq, q_full, c * 64, head_of(w), row_of(w));
  }
  if (warp == kSoftmaxWarps + 1) tmem_alloc_all(tmem_slot);
  if (warp == kSoftmaxWarps && lane < 4) prefetch_map(lane == 0 ? &P.tq : lane == 1 ? &P.tk : lane == 2 ? &P.tv : &P.to);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  pdl_prologue();

  const int w_mine = warp >> 3, half = (warp >> 2) & 1, r_tile = (warp & 3) * 32 + lane;
  int2 mine = make_int2(0, 0);
  const int row = warp < kSoftmaxWarps ? row_of(w_mine) + r_tile : s.Tq;
  if (row < s.Tq) mine = attn_interval(s, row);
  int lo[2], hi[2], first[2], end[2];
  if (s.n_docs > 0) {
    if (warp < kSoftmaxWarps && half == 0) {
      const bool some = mine.x < mine.y;
      const int a = __reduce_min_sync(0xffffffffu, some ? mine.x : s.Tk), b = __reduce_max_sync(0xffffffffu, some ? mine.y : 0);
      if (lane == 0) {
        atomicMin(range + 2 * w_mine, a);
        atomicMax(range + 2 * w_mine + 1, b);
      }
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      lo[w] = range[2 * w]; hi[w] = range[2 * w + 1];
    }
  } else {
    // within one document both ends of the interval grow with the row: the first and the last row tell
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      lo[w] = s.Tk; hi[w] = 0;
      if (row_of(w) >= s.Tq) continue;
      const int2 a = attn_interval(s, row_of(w)), b = attn_interval(s, min(row_of(w) + kRows, s.Tq) - 1);
      lo[w] = min(a.x, s.Tk); hi[w] = min(b.y, s.Tk);
    }
  }
  // the CTA's keys start at key0 and come in n_it tiles; tile w takes part in iterations [first[w], end[w])
  int key0 = min(lo[0], lo[1]);
  const int key1 = max(hi[0], hi[1]);
  int n_it = key1 > key0 ? (key1 - key0 + kRows - 1) / kRows : 0;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    first[w] = lo[w] < hi[w] ? (lo[w] - key0) / kRows : 0;
    end[w] = lo[w] < hi[w] ? (hi[w] - key0 + kRows - 1) / kRows : 0;
  }
  if constexpr (PARTS) {      // this CTA's stretch of them
    const int from = (int)((long long)n_it * blockIdx.y / P.parts), to = (int)((long long)n_it * (blockIdx.y + 1) / P.parts);
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      first[w] = min(max(first[w], from), to) - from;
      end[w] = min(max(end[w], from), to) - from;
    }
    key0 += from * kRows;
    n_it = to - from;
  }

  if (warp == kSoftmaxWarps) {
    // ===================== copies: K and V tiles in turn through one ring =====================
    if (lane == 0 && n_it > 0) {
      int r = 0;
      bool ok = true;
      for (; r < 2 * n_it; ++r) {
        const int st = r % kS;
        if (!wait_inline(empty(st), ((r / kS) & 1) ^ 1u, abort_flag, P.status, 400)) { ok = false; break; }
        mbar_arrive_expect_tx(full(st), kTileB);
        for (int c = 0; c < DP / 64; ++c)
          tma_load_3d(ring + st * kTileB + c * kBox, (r & 1) ? &P.tv : &P.tk, full(st), c * 64, hk, key0 + (r >> 1) * kRows);
      }
      if (!ok) {
        drain_copies(q_full, 0);
        for (int k = max(0, r - kS); k < r; ++k) drain_copies(full(k % kS), (k / kS) & 1);
      }
    }
  } else if (warp == kSoftmaxWarps + 1) {
    // ===================== MMA issuer =====================
    if (lane == 0 && n_it > 0) {
      const uint32_t idesc_s = instr_desc(kRows, 0, 0), idesc_o = instr_desc(DP, 0, 1);
      const uint64_t t_k = smem_desc(0, 16, 1024), t_mn = smem_desc(0, kBox, 1024);
      auto wait_tile = [&](int r) {
        return wait_inline(full(r % kS), (r / kS) & 1, abort_flag, P.status, 410);
      };
      auto scores = [&](int w, int it) {
        const uint32_t a = smem0 + w * kTileB, b = ring + ((2 * it) % kS) * kTileB;
#pragma unroll
        for (int k = 0; k < DP / 16; ++k)
          tc_mma_bf16(tmem + w * 128, desc_k(t_k, a, k), desc_k(t_k, b, k), idesc_s, k != 0);
        tc_commit(s_full(w));
      };
      bool ok = wait_inline(q_full, 0, abort_flag, P.status, 411) && wait_tile(0);
      if (ok) {
        tc_fence_after();
        for (int w = 0; w < 2; ++w)
          if (first[w] <= 0 && 0 < end[w]) scores(w, 0);
        tc_commit(empty(0));
      }
      for (int it = 0; it < n_it && ok; ++it) {
        const int rv = 2 * it + 1;
        ok = wait_tile(rv) && (it + 1 >= n_it || wait_tile(rv + 1));
        if (!ok) break;
        const uint32_t vt = ring + (rv % kS) * kTileB;
        for (int w = 0; w < 2; ++w) {
          if (first[w] <= it && it < end[w]) {
            // the weights come in two parts, each 32 keys of either half (over the first half of their own scores)
#pragma unroll
            for (int part = 0; part < 2; ++part) {
              ok = ok && wait_inline(p_ready(w, part), (it - first[w]) & 1, abort_flag, P.status, 412);
              if (!ok) break;
              tc_fence_after();
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const int k = 2 * part + (i & 1) + 4 * (i >> 1);
                tc_mma_bf16_ts(tmem + 256 + w * 128, tmem + w * 128 + (k >> 2) * 64 + (k & 3) * 8, desc_mn(t_mn, vt, k), idesc_o,
                               (it > first[w] || part != 0 || i != 0) ? 1u : 0u);
              }
            }
            if (!ok) break;
            if (it == end[w] - 1) tc_commit(o_full(w));
          }
          if (it + 1 < n_it && first[w] <= it + 1 && it + 1 < end[w]) {
            tc_fence_after();
            scores(w, it + 1);
          }
        }
        if (!ok) break;
        tc_commit(empty(rv % kS));
        if (it + 1 < n_it) tc_commit(empty((rv + 1) % kS));
      }
      if (!ok) drain_mmas(drain);
    }
  } else {
    // ===================== softmax and epilogue: half a row per thread =====================
    const int w = w_mine, h = head_of(w);
    const uint32_t t_lane = tmem + ((uint32_t)((warp & 3) * 32) << 16) + w * 128, t_s = t_lane + 64 * half, t_o = t_lane + 256;
    float *ex_mine = exchange + (w * 2 + half) * kRows + r_tile, *ex_other = exchange + (w * 2 + 1 - half) * kRows + r_tile;
    const float c = MOD ? 1.f : P.c;
    const float slope = (MOD && s.slopes) ? s.slopes[h] * kLog2e : 0.f;
    const int in_lo = __reduce_max_sync(0xffffffffu, mine.x), in_hi = __reduce_min_sync(0xffffffffu, mine.y);
    const int p = s.q_start + row;
    float m = -INFINITY, l = 0.f;
    bool ok = true;
    for (int it = first[w]; it < end[w]; ++it) {
      ok = wait_inline(s_full(w), (it - first[w]) & 1, abort_flag, P.status, 420);
      const int n0 = key0 + it * kRows + 64 * half;
      uint32_t v[2][32];
      float mx = -INFINITY;
      const bool warp_ok = __all_sync(0xffffffffu, ok);
      if (warp_ok) {
        tc_fence_after();
        tmem_ld32(t_s, v[0]);
        tmem_ld32(t_s + 32, v[1]);
        tmem_ld_wait();
        if (MOD) {
          modify_scores<false>(P.mod, s.slopes != nullptr, slope, (float)(p - n0), v[0], nullptr);
          modify_scores<false>(P.mod, s.slopes != nullptr, slope, (float)(p - n0 - 32), v[1], nullptr);
        }
#pragma unroll
        for (int b = 0; b < 2; ++b)
          if (n0 + 32 * b < in_lo || n0 + 32 * b + 32 > in_hi) {   // some row of the warp does not see all of these keys
            const uint32_t seen = span_bits(mine.x - n0 - 32 * b, mine.y - n0 - 32 * b);
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (!(seen >> i & 1)) v[b][i] = 0xff800000u;
          }
        float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int i = 0; i < 64; i += 2)
          top[(i >> 1) & 3] = fmaxf(fmaxf(top[(i >> 1) & 3], __uint_as_float(v[i >> 5][i & 31])), __uint_as_float(v[i >> 5][(i & 31) + 1]));
        mx = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
      }
      // one barrier per tile; a second only when a row's maximum has to move (or a wait has run out)
      if (tile_any(w, !warp_ok || it == first[w] || (mx - m) * c > 8.f)) {
        *ex_mine = mx;
        if (!warp_ok) tile_abort[2 * w + (it & 1)] = 1;
        tile_sync(w);
        if (tile_abort[2 * w + (it & 1)]) { ok = false; break; }
        mx = fmaxf(mx, *ex_other);
        if (it == first[w]) {
          m = mx;
        } else {
          const bool need = (mx - m) * c > 8.f;
          if (__any_sync(0xffffffffu, need)) {
            const float alpha = need ? ex2((m - mx) * c) : 1.f;
            if (need) m = mx;
            l *= alpha;
            // the scores' barrier also covers the product before them: the accumulator is at rest
#pragma unroll 1
            for (int d = half * (DP / 2); d < (half + 1) * (DP / 2); d += 16) {
              uint32_t o[32];
              tmem_ld16(t_o + d, o);
              tmem_ld_wait();
#pragma unroll
              for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
              tmem_st16(t_o + d, o);
            }
          }
        }
      }
      const float base = m == -INFINITY ? 0.f : -m * c;
      const uint64_t c2 = f2(c, c), base2 = f2(base, base);
      uint64_t sum0 = 0, sum1 = 0;
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        uint32_t e[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const uint64_t z = f2u(v[b][2 * i], v[b][2 * i + 1]);
          const float2 x = un2(MOD ? add2(z, base2) : fma2(z, c2, base2));
          const float x0 = ex2(x.x), x1 = ex2(x.y);
          if (i & 1) sum1 = add2(sum1, f2(x0, x1)); else sum0 = add2(sum0, f2(x0, x1));
          e[i] = pack2(x0, x1);   // the second product's operand: bf16, 2^-8 of each weight
        }
        tmem_st16(t_s + 16 * b, e);
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_ready(w, b));    // this part's product may start
      }
      const float2 sum = un2(add2(sum0, sum1));
      l += sum.x + sum.y;
    }
    // ---- epilogue
    // a tile without keys writes its zeros where its queries come in
    if (ok && row_of(w) < s.Tq) ok = wait_inline(first[w] < end[w] ? o_full(w) : q_full, 0, abort_flag, P.status, 421);
    ok = __all_sync(0xffffffffu, ok) && row_of(w) < s.Tq;
    tile_sync(w);               // the last exchange has been read
    *ex_mine = l;
    tile_sync(w);
    l += *ex_other;
    const bool in = row < s.Tq;
    if constexpr (PARTS) {
      const long long at = ((long long)blockIdx.y * s.H + h) * s.Tq + row;
      if (ok && in && half == 0) P.part_ml[at] = make_float2(m * c, l);
      if (ok && first[w] < end[w]) {
        tc_fence_after();
#pragma unroll 1
        for (int d = half * (DP / 2); d < (half + 1) * (DP / 2); d += 32) {
          uint32_t o[32];
          tmem_ld32(t_o + d, o);
          tmem_ld_wait();
#pragma unroll
          for (int i = 0; i < 32; i += 4)       // head_dim is a multiple of 8
            if (in && d + i < s.D) *reinterpret_cast<uint4 *>(P.part_o + at * s.D + d + i) = make_uint4(o[i], o[i + 1], o[i + 2], o[i + 3]);
        }
      }
      ok = false;                     // nothing to stage; sums of no key are never read
    }
    if (ok) {
      tc_fence_after();
      // a row without keys gets 0 even where a masked value made its accumulator NaN
      const bool any = first[w] < end[w] && __any_sync(0xffffffffu, l != 0.f);
      const float inv = l > 0.f ? 1.f / l : l;
      bool bad = !(l < INFINITY);
#pragma unroll 1
      for (int d = half * (DP / 2); d < (half + 1) * (DP / 2); d += 32) bad |= stage_columns(t_o, any, inv, smem0 + w * kTileB, r_tile, d);
      if (half == 0 && in) P.x.lse[(long long)h * s.Tq + row] = l == 0.f ? -INFINITY : (m * c + __log2f(l)) * kLn2;
      const unsigned votes = __ballot_sync(0xffffffffu, bad && in);
      if (lane == 0 && votes) atomicOr(bad_rows + 4 * w + (warp & 3), votes);
      fence_proxy_async_smem();
    }
    tile_sync(w);
    if (ok && lane == 0 && in && (DP == 128 ? 64 * half < s.D : half == 0)) {
      const int d = DP == 128 ? 64 * half : 0;
      tma_store_3d(&P.to, smem0 + w * kTileB + (d >> 6) * kBox + (warp & 3) * 32 * 128, d, h, row);
      finish_stores(bad_rows[4 * w + (warp & 3)] != 0);
    }
    tile_sync(w);               // both halves' stores are done before a row is written again
    if (ok) attn_each_bad_row(bad_rows + 4 * w, warp & 7, 8, [&](int r) { attn_exact_fwd_row<__nv_bfloat16>(s, P.x, h, row - r_tile + r); });
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kSoftmaxWarps + 1) {
    tc_fence_after();
    tmem_free_all(tmem);
  }
}

// ------------------------------------------------------------------ backward
// P = exp2(z - lse2) and ds = P (dP - delta) (1 - tanh^2) are formed again from S = Q K^T and dP = dO V^T, once with the
// keys as rows (dk, dv: sums over queries, and over the heads of a group, stay in TMEM) and once with the queries as
// rows (dq).  Two products more than a backward that adds dq up in memory as the key tiles finish, but every sum is
// formed by one CTA in one order: the same call gives the same bits, and nothing is zeroed or converted afterwards.
// Warps 0-15 are the softmax group (four threads per row, 32 columns each), warp 16 issues copies, warp 17 MMAs.
// Five products a tile pair against the forward's two; 64 heads over 8 kv heads, 4096 tokens, causal: 860 us (800 TFLOP/s of the
// seen half, seven products done for the five that count), 1024 tokens of 32 heads: 56 us (383).  Bound as the forward is, by a
// tile's chain: about 3900 clocks in the dk, dv kernel, whose four products take 2080, and 2740 in the dq kernel, whose three take
// 1560; leaving the exponentials out changes nothing.
// P and ds are rounded to bf16 once, 2^-8 of each at most: results are 1.5 times as far from the exact ones as their own rounding
// to bf16 alone would leave them (0.0025 against 0.0017, relative).  ds in two bf16 terms: 0.0023, but 861 -> 1046 us.
constexpr int kMaskedTiles = 4096;     // query tiles whose reach a bit is kept for (half a million rows); the rest are all visited
template <int DP> struct BwdCfg {
  static constexpr int kTileB = kRows * DP * 2;
  // dk, dv: Q tiles live until dK's product, dO tiles (with their rows' statistics) only until dV's
  static constexpr int kSlotsQ = DP == 128 ? 3 : 4, kSlotsO = DP == 128 ? 2 : 4, kSlotO = kTileB + 1024;
  static constexpr int kSmemKv = 2 * kTileB + kSlotsQ * kTileB + kSlotsO * kSlotO + 288 + kMaskedTiles / 8;
  // dq: K tiles live until dQ's product, V tiles only until dP's
  static constexpr int kSlotsK = DP == 128 ? 3 : 4, kSlotsV = DP == 128 ? 2 : 4;
  static constexpr int kSmemQ = 2 * kTileB + (kSlotsK + kSlotsV) * kTileB + 288;
};
static_assert(BwdCfg<128>::kSmemKv <= 232448 && BwdCfg<128>::kSmemQ <= 232448, "shared memory of a CTA");

struct BwdParams {
  CUtensorMap tq, tk, tv, tdo, tdq, tdk, tdv;
  AttnShape s;
  AttnTensors x;
  AttnBwdScratch w;
  DeviceStatus *status;
  int order;         // key tiles to be taken by their work; 0: as they come
  ScoreMod mod;
  float c;
};

__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ void softmax_group_sync() { asm volatile("barrier.cta.sync 1, 512;" ::: "memory"); }
// TMEM column of contraction step k of a weight tile: the four 32-column quarters keep their place over the scores
__device__ __forceinline__ uint32_t weight_col(int k) { return (uint32_t)((k >> 1) * 32 + (k & 1) * 8); }

// These kernels use the whole shared memory and cannot spend up to 1 KB on aligning it: dynamic shared memory begins
// 1024-byte aligned when a kernel has no static shared memory.  Should that ever not hold, the call reports it.
__device__ __forceinline__ bool misaligned(uint32_t smem0, DeviceStatus *status) {
  if ((smem0 & 1023u) == 0) return false;
  if (threadIdx.x == 0 && atomicCAS(&status->code, 0, (int)TEMPLORA_ERR_CUDA) == 0) status->where = 599;
  return true;
}

// ---- dk and dv: one CTA per 128 keys of a kv head, over the query tiles that reach them, for each head of the group.
// TMEM: S^T, dP^T (their weights over them), dV, dK.  The next tile's S^T is issued behind dV's product, its dP^T behind
// dK's, so the tensor core has work while the weights are formed.
template <int DP, int MOD>
__global__ void __launch_bounds__(kThreadsTc, 1) attn_dkdv_tc_kernel(const __grid_constant__ BwdParams P) {
  using Cfg = BwdCfg<DP>;
  constexpr int kTileB = Cfg::kTileB, kQ = Cfg::kSlotsQ, kO = Cfg::kSlotsO, kSlotO = Cfg::kSlotO;
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t smem0 = smem_u32(smem);
  if (misaligned(smem0, P.status)) return;
  const uint32_t ring_q = smem0 + 2 * kTileB, ring_o = ring_q + kQ * kTileB, bar0 = ring_o + kO * kSlotO;
  auto q_full = [&](int i) { return bar0 + 8u * i; };
  auto q_empty = [&](int i) { return bar0 + 8u * (kQ + i); };
  auto o_full = [&](int i) { return bar0 + 8u * (2 * kQ + i); };
  auto o_empty = [&](int i) { return bar0 + 8u * (2 * kQ + kO + i); };
  const uint32_t kv_full = bar0 + 8u * (2 * (kQ + kO)), s_full = kv_full + 8, dp_full = kv_full + 16, p_ready = kv_full + 24,
                 ds_ready = kv_full + 32, acc_full = kv_full + 40, drain = kv_full + 48;
  uint8_t *tail = smem + 2 * kTileB + kQ * kTileB + kO * kSlotO + 256;
  volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(tail);
  volatile int *abort_flag = reinterpret_cast<volatile int *>(tail + 4);
  unsigned *bad_rows = reinterpret_cast<unsigned *>(tail + 16);    // 4 words
  unsigned *active = reinterpret_cast<unsigned *>(tail + 32);      // kMaskedTiles bits

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const AttnShape &s = P.s;
  const int hk = blockIdx.x % s.Hkv, n_qt = P.w.Tq_pad / kRows;
  int k0 = (blockIdx.x / s.Hkv) * kRows;   // a causal call's longest tiles come first
  if (threadIdx.x == 0) {
    for (int i = 0; i < kQ; ++i) { mbar_init(q_full(i), 1); mbar_init(q_empty(i), 1); }
    for (int i = 0; i < kO; ++i) { mbar_init(o_full(i), 1); mbar_init(o_empty(i), 1); }
    mbar_init(kv_full, 1); mbar_init(s_full, 1); mbar_init(dp_full, 1); mbar_init(p_ready, kSoftmaxWarps);
    mbar_init(ds_ready, kSoftmaxWarps); mbar_init(acc_full, 1); mbar_init(drain, 1);
    *abort_flag = 0;
    for (int i = 0; i < 4; ++i) bad_rows[i] = 0;
    fence_barrier_init();
  }
  if (warp == kSoftmaxWarps + 1) tmem_alloc_all(tmem_slot);
  if (warp == kSoftmaxWarps && lane < 6)
    prefetch_map(lane == 0 ? &P.tk : lane == 1 ? &P.tv : lane == 2 ? &P.tq : lane == 3 ? &P.tdo : lane == 4 ? &P.tdk : &P.tdv);
  pdl_prologue();
  if (P.order > 0) {
    // Documents leave some keys many more queries than others: the key tiles are taken by the number of query tiles that reach
    // them, most first, so that a long one is not the last to start.  (5 documents in 4099 tokens, 32 / 8 heads, capped: the whole
    // backward 341 us as they come, 300 by work)
    int *count = reinterpret_cast<int *>(smem);
    for (int t = threadIdx.x; t < P.order; t += kThreadsTc) {
      int n = 0;
      for (int qt = 0; qt < n_qt; ++qt) {
        const int2 r = P.w.tiles[qt];
        n += r.x < (t + 1) * kRows && r.y > t * kRows;
      }
      count[t] = n;
    }
    __syncthreads();
    for (int t = threadIdx.x; t < P.order; t += kThreadsTc) {
      int rank = 0;
      for (int o = 0; o < P.order; ++o) rank += count[o] > count[t] || (count[o] == count[t] && o < t);
      if (rank == k0 / kRows) count[P.order] = t;
    }
    __syncthreads();
    k0 = count[P.order] * kRows;
    fence_proxy_async_smem();        // copies will write here
  }
  const int n_bits = min(n_qt, kMaskedTiles);
  for (int t0 = warp * 32; t0 < n_bits; t0 += kThreadsTc) {
    bool on = false;
    if (t0 + lane < n_bits) {
      const int2 r = P.w.tiles[t0 + lane];
      on = r.x < k0 + kRows && r.y > k0;
    }
    const unsigned word = __ballot_sync(0xffffffffu, on);
    if (lane == 0) active[t0 >> 5] = word;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  // first query tile at or behind t that reaches these keys (n_qt: none)
  auto next_tile = [&](int t) {
    while (t < n_bits) {
      const unsigned word = active[t >> 5] >> (t & 31);
      if (word) return t + __ffs(word) - 1;
      t = (t | 31) + 1;
    }
    return min(max(t, n_bits), n_qt);
  };
  // this CTA's heads of the group and query tiles, when they are dealt to several
  const int h0 = hk * s.group + (int)(blockIdx.y % P.w.head_parts), h_step = P.w.head_parts, h_end = (hk + 1) * s.group;
  const int stretch = blockIdx.y / P.w.head_parts;
  const int qt_end = (int)((long long)n_qt * (stretch + 1) / P.w.row_parts);
  const int qt_first = next_tile((int)((long long)n_qt * stretch / P.w.row_parts));
  const bool some = qt_first < qt_end;

  if (warp == kSoftmaxWarps) {
    if (lane == 0 && some) {
      mbar_arrive_expect_tx(kv_full, 2 * kTileB);
      for (int c = 0; c < DP / 64; ++c) {
        tma_load_3d(smem0 + c * kBox, &P.tk, kv_full, c * 64, hk, k0);
        tma_load_3d(smem0 + kTileB + c * kBox, &P.tv, kv_full, c * 64, hk, k0);
      }
      int rq = 0, ro = 0;
      bool ok = true;
      for (int h = h0; h < h_end && ok; h += h_step)
        for (int qt = qt_first; qt < qt_end; qt = next_tile(qt + 1)) {
          const int sq = rq % kQ, so = ro % kO;
          if (!mbar_wait_fast(q_empty(sq), ((rq / kQ) & 1) ^ 1u, abort_flag, P.status, 500)) { ok = false; break; }
          mbar_arrive_expect_tx(q_full(sq), kTileB);
          for (int c = 0; c < DP / 64; ++c) tma_load_3d(ring_q + sq * kTileB + c * kBox, &P.tq, q_full(sq), c * 64, h, qt * kRows);
          ++rq;
          if (!mbar_wait_fast(o_empty(so), ((ro / kO) & 1) ^ 1u, abort_flag, P.status, 501)) { ok = false; break; }
          mbar_arrive_expect_tx(o_full(so), kSlotO);
          for (int c = 0; c < DP / 64; ++c) tma_load_3d(ring_o + so * kSlotO + c * kBox, &P.tdo, o_full(so), c * 64, h, qt * kRows);
          bulk_load(ring_o + so * kSlotO + kTileB, P.w.stat + 2 * ((long long)h * P.w.Tq_pad + qt * kRows), 1024, o_full(so));
          ++ro;
        }
      if (!ok) {
        drain_copies(kv_full, 0);
        for (int k = max(0, rq - kQ); k < rq; ++k) drain_copies(q_full(k % kQ), (k / kQ) & 1);
        for (int k = max(0, ro - kO); k < ro; ++k) drain_copies(o_full(k % kO), (k / kO) & 1);
      }
    }
  } else if (warp == kSoftmaxWarps + 1) {
    if (lane == 0 && some) {
      const uint32_t idesc_s = instr_desc(kRows, 0, 0), idesc_o = instr_desc(DP, 0, 1);
      const uint64_t t_k = smem_desc(0, 16, 1024), t_mn = smem_desc(0, kBox, 1024);
      // rows of `a` (keys) against rows of `b` (queries), contracted over head_dim
      auto outer = [&](uint32_t d, uint32_t a, uint32_t b, uint32_t bar) {
#pragma unroll
        for (int k = 0; k < DP / 16; ++k) tc_mma_bf16(d, desc_k(t_k, a, k), desc_k(t_k, b, k), idesc_s, k != 0);
        tc_commit(bar);
      };
      auto accumulate = [&](uint32_t d, uint32_t weights, uint32_t b, bool more) {
#pragma unroll
        for (int k = 0; k < kRows / 16; ++k)
          tc_mma_bf16_ts(d, weights + weight_col(k), desc_mn(t_mn, b, k), idesc_o, (more || k != 0) ? 1u : 0u);
      };
      auto wait_q = [&](int r) { return mbar_wait_fast(q_full(r % kQ), (r / kQ) & 1, abort_flag, P.status, 510); };
      auto wait_o = [&](int r) { return mbar_wait_fast(o_full(r % kO), (r / kO) & 1, abort_flag, P.status, 511); };
      int n = 0;
      for (int qt = qt_first; qt < qt_end; qt = next_tile(qt + 1)) ++n;
      n *= (h_end - h0 + h_step - 1) / h_step;
      bool ok = mbar_wait_fast(kv_full, 0, abort_flag, P.status, 512) && wait_q(0) && wait_o(0);
      if (ok) {
        tc_fence_after();
        outer(tmem, smem0, ring_q, s_full);
        outer(tmem + 128, smem0 + kTileB, ring_o, dp_full);
      }
      for (int r = 0; r < n && ok; ++r) {
        const bool more = r + 1 < n;
        if (!(ok = mbar_wait_fast(p_ready, r & 1, abort_flag, P.status, 513))) break;
        tc_fence_after();
        accumulate(tmem + 256, tmem, ring_o + (r % kO) * kSlotO, r > 0);
        if (more) {
          if (!(ok = wait_q(r + 1))) break;
          tc_fence_after();
          outer(tmem, smem0, ring_q + ((r + 1) % kQ) * kTileB, s_full);
        }
        if (!(ok = mbar_wait_fast(ds_ready, r & 1, abort_flag, P.status, 514))) break;
        tc_fence_after();
        tc_commit(o_empty(r % kO));      // dV's product, and the statistics have been used
        accumulate(tmem + 384, tmem + 128, ring_q + (r % kQ) * kTileB, r > 0);
        tc_commit(q_empty(r % kQ));
        if (more) {
          if (!(ok = wait_o(r + 1))) break;
          tc_fence_after();
          outer(tmem + 128, smem0 + kTileB, ring_o + ((r + 1) % kO) * kSlotO, dp_full);
        }
      }
      if (ok) tc_commit(acc_full); else drain_mmas(drain);
    }
  } else {
    const int quarter = warp >> 2, row = (warp & 3) * 32 + lane, j = k0 + row;
    const uint32_t t_lane = tmem + ((uint32_t)((warp & 3) * 32) << 16), t_s = t_lane + 32 * quarter, t_dp = t_s + 128;
    const uint64_t c2 = f2(P.c, P.c);
    bool ok = true;
    int r = 0;
    for (int h = h0; h < h_end && ok; h += h_step) {
      const float slope = (MOD && s.slopes) ? s.slopes[h] * kLog2e : 0.f;
      for (int qt = qt_first; qt < qt_end; qt = next_tile(qt + 1), ++r) {
        const int2 inner = P.w.inner[4 * qt + quarter];
        const int kb = k0 + (warp & 3) * 32;        // the warp's first key
        const bool masked = kb < inner.x || kb + 32 > inner.y;
        // -lse2 of this quarter's rows, and 128 words on -delta
        const float4 *stat = reinterpret_cast<const float4 *>(smem + 2 * kTileB + kQ * kTileB + (r % kO) * kSlotO + kTileB) + 8 * quarter;
        ok = mbar_wait_fast(o_full(r % kO), (r / kO) & 1, abort_flag, P.status, 520) &&        // the statistics
             mbar_wait_fast(s_full, r & 1, abort_flag, P.status, 521);
        if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
        tc_fence_after();
        uint32_t v[32];
        float g[32];
        tmem_ld32(t_s, v);
        tmem_ld_wait();
        if (MOD) {
          // |p - j| with p = q_start + query: the columns are queries here
          modify_scores<true>(P.mod, s.slopes != nullptr, slope, (float)(j - s.q_start - qt * kRows - 32 * quarter), v, g);
        }
#pragma unroll
        for (int i = 0; i < 32; i += 4) {
          const float4 l4 = stat[i >> 2];
          const uint64_t z0 = f2u(v[i], v[i + 1]), z1 = f2u(v[i + 2], v[i + 3]);
          const float2 a = un2(MOD ? add2(z0, f2(l4.x, l4.y)) : fma2(z0, c2, f2(l4.x, l4.y)));
          const float2 b = un2(MOD ? add2(z1, f2(l4.z, l4.w)) : fma2(z1, c2, f2(l4.z, l4.w)));
          const float e[4] = {ex2(a.x), ex2(a.y), ex2(b.x), ex2(b.y)};
#pragma unroll
          for (int n = 0; n < 4; ++n) {
            v[i + n] = __float_as_uint(e[n]);
            g[i + n] = MOD ? fmaf(-g[i + n] * g[i + n], e[n], e[n]) : e[n];      // weight times the cap's slope
          }
        }
        if (masked) {
          const int2 rw = P.w.rows[qt * kRows + 32 * quarter + lane];      // a lane's row against the warp's keys, then the other way
          const uint32_t seen = transpose_bits(span_bits(rw.x - kb, rw.y - kb), lane);
#pragma unroll
          for (int i = 0; i < 32; ++i)
            if (!(seen >> i & 1)) { v[i] = 0; g[i] = 0.f; }
        }
        uint32_t e[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) e[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
        tmem_st16(t_s, e);
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_ready);
        ok = mbar_wait_fast(dp_full, r & 1, abort_flag, P.status, 522);
        if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
        tc_fence_after();
        tmem_ld32(t_dp, v);
        tmem_ld_wait();
#pragma unroll
        for (int i = 0; i < 32; i += 4) {
          const float4 d4 = stat[32 + (i >> 2)];
          const float2 a = un2(mul2(f2(g[i], g[i + 1]), add2(f2u(v[i], v[i + 1]), f2(d4.x, d4.y))));
          const float2 b = un2(mul2(f2(g[i + 2], g[i + 3]), add2(f2u(v[i + 2], v[i + 3]), f2(d4.z, d4.w))));
          e[i >> 1] = pack2(a.x, a.y);
          e[(i >> 1) + 1] = pack2(b.x, b.y);
        }
        tmem_st16(t_dp, e);
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(ds_ready);
      }
    }
    // ---- epilogue: two quarters store dv, two dk, through the resident tiles' room (every product is done)
    if (ok && some) ok = mbar_wait_fast(acc_full, 0, abort_flag, P.status, 523);
    ok = __all_sync(0xffffffffu, ok);
    const int what = quarter >> 1, col_half = quarter & 1;
    if (gridDim.y > 1) {
      if (ok) {
        tc_fence_after();
        float *to = (what ? P.w.part_dk : P.w.part_dv) + (((long long)blockIdx.y * s.Hkv + hk) * s.Tk + j) * s.D;
#pragma unroll 1
        for (int d = col_half * (DP / 2); d < (col_half + 1) * (DP / 2); d += 32) {
          uint32_t o[32];
          if (some) {
            tmem_ld32(t_lane + 256 + 128 * what + d, o);
            tmem_ld_wait();
          }
          const float scale = what ? s.scale : 1.f;
#pragma unroll
          for (int i = 0; i < 32; i += 4)       // head_dim and the rows' addresses are multiples of 8 elements
            if (j < s.Tk && d + i < s.D)
              *reinterpret_cast<float4 *>(to + d + i) =
                  some ? make_float4(__uint_as_float(o[i]) * scale, __uint_as_float(o[i + 1]) * scale, __uint_as_float(o[i + 2]) * scale,
                                     __uint_as_float(o[i + 3]) * scale)
                       : make_float4(0.f, 0.f, 0.f, 0.f);
        }
      }
      ok = false;                      // nothing to stage
    }
    const uint32_t tile = smem0 + what * kTileB;
    if (ok) {
      tc_fence_after();
      bool bad = false;
#pragma unroll 1
      for (int d = col_half * (DP / 2); d < (col_half + 1) * (DP / 2); d += 32)
        bad |= stage_columns(t_lane + 256 + 128 * what, some, what ? s.scale : 1.f, tile, row, d);
      const unsigned votes = __ballot_sync(0xffffffffu, bad && j < s.Tk);
      if (lane == 0 && votes) atomicOr(bad_rows + (warp & 3), votes);
      fence_proxy_async_smem();
    }
    softmax_group_sync();
    if (ok && lane == 0 && j < s.Tk && (DP == 128 ? 64 * col_half < s.D : col_half == 0)) {
      const int d = DP == 128 ? 64 * col_half : 0;
      tma_store_3d(what ? &P.tdk : &P.tdv, tile + (d >> 6) * kBox + (warp & 3) * 32 * 128, d, hk, j);
      finish_stores(bad_rows[warp & 3] != 0);
    }
    softmax_group_sync();    // all stores are done before a row is written again
    if (ok) attn_each_bad_row(bad_rows, warp, kSoftmaxWarps, [&](int r) { attn_exact_dkdv_row<__nv_bfloat16>(s, P.x, P.w, hk, k0 + r); });
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kSoftmaxWarps + 1) {
    tc_fence_after();
    tmem_free_all(tmem);
  }
}

// ---- dq: one CTA per 128 queries of a head.  TMEM: S, dP twice (its weights over it), dQ.  The next tile's S is issued as
// soon as the softmax group has this one's in registers, its dP into the other buffer.
template <int DP, int MOD>
__global__ void __launch_bounds__(kThreadsTc, 1) attn_dq_tc_kernel(const __grid_constant__ BwdParams P) {
  using Cfg = BwdCfg<DP>;
  constexpr int kTileB = Cfg::kTileB, kK = Cfg::kSlotsK, kV = Cfg::kSlotsV;
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t smem0 = smem_u32(smem);
  if (misaligned(smem0, P.status)) return;
  const uint32_t ring_k = smem0 + 2 * kTileB, ring_v = ring_k + kK * kTileB, bar0 = ring_v + kV * kTileB;
  auto k_full = [&](int i) { return bar0 + 8u * i; };
  auto k_empty = [&](int i) { return bar0 + 8u * (kK + i); };
  auto v_full = [&](int i) { return bar0 + 8u * (2 * kK + i); };
  auto v_empty = [&](int i) { return bar0 + 8u * (2 * kK + kV + i); };
  const uint32_t q_full = bar0 + 8u * (2 * (kK + kV)), s_full = q_full + 8, s_free = q_full + 16, acc_full = q_full + 24,
                 drain = q_full + 32;
  auto dp_full = [&](int b) { return q_full + 40 + 8u * b; };
  // two, taken in turn: S and dP of the next tile are there before this one's weights are, so that a warp's second arrival
  // can come while the issuing thread still waits for the first phase
  auto ds_ready = [&](int b) { return q_full + 56 + 8u * b; };
  uint8_t *tail = smem + (2 + kK + kV) * kTileB + 256;
  volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(tail);
  volatile int *abort_flag = reinterpret_cast<volatile int *>(tail + 4);
  unsigned *bad_rows = reinterpret_cast<unsigned *>(tail + 16);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const AttnShape &s = P.s;
  const int h = blockIdx.x % s.H, rt = P.w.Tq_pad / kRows - 1 - blockIdx.x / s.H, hk = h / s.group;
  // the copying thread starts with what needs no other thread
  if (threadIdx.x == 32 * kSoftmaxWarps) {
    for (int i = 0; i < kK; ++i) { mbar_init(k_full(i), 1); mbar_init(k_empty(i), 1); }
    for (int i = 0; i < kV; ++i) { mbar_init(v_full(i), 1); mbar_init(v_empty(i), 1); }
    mbar_init(q_full, 1); mbar_init(s_full, 1); mbar_init(s_free, kSoftmaxWarps);
    mbar_init(ds_ready(0), kSoftmaxWarps); mbar_init(ds_ready(1), kSoftmaxWarps);
    mbar_init(acc_full, 1); mbar_init(drain, 1); mbar_init(dp_full(0), 1); mbar_init(dp_full(1), 1);
    *abort_flag = 0;
    for (int i = 0; i < 4; ++i) bad_rows[i] = 0;
    fence_barrier_init();
    mbar_arrive_expect_tx(q_full, 2 * kTileB);
    for (int c = 0; c < DP / 64; ++c) {
      tma_load_3d(smem0 + c * kBox, &P.tq, q_full, c * 64, h, rt * kRows);
      tma_load_3d(smem0 + kTileB + c * kBox, &P.tdo, q_full, c * 64, h, rt * kRows);
    }
  }
  if (warp == kSoftmaxWarps + 1) tmem_alloc_all(tmem_slot);
  if (warp == kSoftmaxWarps && lane < 5)
    prefetch_map(lane == 0 ? &P.tq : lane == 1 ? &P.tdo : lane == 2 ? &P.tk : lane == 3 ? &P.tv : &P.tdq);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  pdl_beside();        // it takes the SMs that the dk, dv kernel's last CTAs leave idle
  const int2 reach = __ldcg(P.w.tiles + rt);
  const int key0 = reach.x, n_it = reach.y > reach.x ? (reach.y - reach.x + kRows - 1) / kRows : 0;

  if (warp == kSoftmaxWarps) {
    if (lane == 0 && n_it > 0) {
      bool ok = true;
      int rk = 0, rv = 0;
      for (int it = 0; it < n_it; ++it) {
        const int sk = it % kK, sv = it % kV;
        if (!mbar_wait_fast(k_empty(sk), ((it / kK) & 1) ^ 1u, abort_flag, P.status, 600)) { ok = false; break; }
        mbar_arrive_expect_tx(k_full(sk), kTileB);
        for (int c = 0; c < DP / 64; ++c) tma_load_3d(ring_k + sk * kTileB + c * kBox, &P.tk, k_full(sk), c * 64, hk, key0 + it * kRows);
        ++rk;
        if (!mbar_wait_fast(v_empty(sv), ((it / kV) & 1) ^ 1u, abort_flag, P.status, 601)) { ok = false; break; }
        mbar_arrive_expect_tx(v_full(sv), kTileB);
        for (int c = 0; c < DP / 64; ++c) tma_load_3d(ring_v + sv * kTileB + c * kBox, &P.tv, v_full(sv), c * 64, hk, key0 + it * kRows);
        ++rv;
      }
      if (!ok) {
        drain_copies(q_full, 0);
        for (int k = max(0, rk - kK); k < rk; ++k) drain_copies(k_full(k % kK), (k / kK) & 1);
        for (int k = max(0, rv - kV); k < rv; ++k) drain_copies(v_full(k % kV), (k / kV) & 1);
      }
    }
  } else if (warp == kSoftmaxWarps + 1) {
    if (lane == 0 && n_it > 0) {
      const uint32_t idesc_s = instr_desc(kRows, 0, 0), idesc_o = instr_desc(DP, 0, 1);
      const uint64_t t_k = smem_desc(0, 16, 1024), t_mn = smem_desc(0, kBox, 1024);
      auto outer = [&](uint32_t d, uint32_t a, uint32_t b, uint32_t bar) {
#pragma unroll
        for (int k = 0; k < DP / 16; ++k) tc_mma_bf16(d, desc_k(t_k, a, k), desc_k(t_k, b, k), idesc_s, k != 0);
        tc_commit(bar);
      };
      auto pair = [&](int it) {      // S and dP of a key tile
        if (!mbar_wait_fast(k_full(it % kK), (it / kK) & 1, abort_flag, P.status, 610)) return false;
        tc_fence_after();
        outer(tmem, smem0, ring_k + (it % kK) * kTileB, s_full);
        if (!mbar_wait_fast(v_full(it % kV), (it / kV) & 1, abort_flag, P.status, 611)) return false;
        tc_fence_after();
        outer(tmem + 128 + 128 * (it & 1), smem0 + kTileB, ring_v + (it % kV) * kTileB, dp_full(it & 1));
        tc_commit(v_empty(it % kV));
        return true;
      };
      bool ok = mbar_wait_fast(q_full, 0, abort_flag, P.status, 612) && pair(0);
      for (int it = 0; it < n_it && ok; ++it) {
        if (it + 1 < n_it) {
          ok = mbar_wait_fast(s_free, it & 1, abort_flag, P.status, 613);
          if (ok) {
            tc_fence_after();
            ok = pair(it + 1);
          }
          if (!ok) break;
        }
        if (!(ok = mbar_wait_fast(ds_ready(it & 1), (it >> 1) & 1, abort_flag, P.status, 614))) break;
        tc_fence_after();
#pragma unroll
        for (int k = 0; k < kRows / 16; ++k)
          tc_mma_bf16_ts(tmem + 384, tmem + 128 + 128 * (it & 1) + weight_col(k), desc_mn(t_mn, ring_k + (it % kK) * kTileB, k),
                         idesc_o, (it > 0 || k != 0) ? 1u : 0u);
        tc_commit(k_empty(it % kK));
      }
      if (ok) tc_commit(acc_full); else drain_mmas(drain);
    }
  } else {
    const int quarter = warp >> 2, r = (warp & 3) * 32 + lane, row = rt * kRows + r;
    const uint32_t t_lane = tmem + ((uint32_t)((warp & 3) * 32) << 16), t_s = t_lane + 32 * quarter;
    const float *stat = P.w.stat + 2 * ((long long)h * P.w.Tq_pad + rt * kRows);
    const float nlse = __ldcg(stat + r), ndelta = __ldcg(stat + kRows + r);
    const int2 mine = __ldcg(P.w.rows + row), inner = __ldcg(P.w.inner + 4 * rt + (warp & 3));
    const float slope = (MOD && s.slopes) ? __ldcg(s.slopes + h) * kLog2e : 0.f;
    const uint64_t c2 = f2(P.c, P.c), nlse2 = f2(nlse, nlse), ndelta2 = f2(ndelta, ndelta);
    bool ok = true;
    for (int it = 0; it < n_it; ++it) {
      const int n0 = key0 + it * kRows + 32 * quarter;
      const bool masked = n0 < inner.x || n0 + 32 > inner.y;
      ok = mbar_wait_fast(s_full, it & 1, abort_flag, P.status, 620);
      if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
      tc_fence_after();
      uint32_t v[32];
      float g[32];
      tmem_ld32(t_s, v);
      tmem_ld_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(s_free);
      if (MOD) modify_scores<true>(P.mod, s.slopes != nullptr, slope, (float)(s.q_start + row - n0), v, g);
#pragma unroll
      for (int i = 0; i < 32; i += 2) {
        const uint64_t z = f2u(v[i], v[i + 1]);
        const float2 a = un2(MOD ? add2(z, nlse2) : fma2(z, c2, nlse2));
        const float p0 = ex2(a.x), p1 = ex2(a.y);
        g[i] = MOD ? fmaf(-g[i] * g[i], p0, p0) : p0;
        g[i + 1] = MOD ? fmaf(-g[i + 1] * g[i + 1], p1, p1) : p1;
      }
      if (masked) {
        const uint32_t seen = span_bits(mine.x - n0, mine.y - n0);
#pragma unroll
        for (int i = 0; i < 32; ++i)
          if (!(seen >> i & 1)) g[i] = 0.f;
      }
      ok = mbar_wait_fast(dp_full(it & 1), (it >> 1) & 1, abort_flag, P.status, 621);
      if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
      tc_fence_after();
      const uint32_t t_dp = t_s + 128 + 128 * (it & 1);
      tmem_ld32(t_dp, v);
      tmem_ld_wait();
      uint32_t e[16];
#pragma unroll
      for (int i = 0; i < 32; i += 2) {
        const float2 a = un2(mul2(f2(g[i], g[i + 1]), add2(f2u(v[i], v[i + 1]), ndelta2)));
        e[i >> 1] = pack2(a.x, a.y);
      }
      tmem_st16(t_dp, e);
      tmem_st_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(ds_ready(it & 1));
    }
    // a tile without keys writes its zeros where its queries come in
    if (ok) ok = mbar_wait_fast(n_it > 0 ? acc_full : q_full, 0, abort_flag, P.status, 622);
    ok = __all_sync(0xffffffffu, ok);
    const bool stores = 32 * quarter < DP;
    if (ok && stores) {
      tc_fence_after();
      const bool bad = stage_columns(t_lane + 384, n_it > 0, s.scale, smem0, r, 32 * quarter);
      const unsigned votes = __ballot_sync(0xffffffffu, bad && row < s.Tq);
      if (lane == 0 && votes) atomicOr(bad_rows + (warp & 3), votes);
      fence_proxy_async_smem();
    }
    softmax_group_sync();
    if (ok && quarter == 0 && lane == 0 && row < s.Tq) {
      for (int d = 0; d < s.D; d += 64) tma_store_3d(&P.tdq, smem0 + (d >> 6) * kBox + warp * 32 * 128, d, h, row);
      finish_stores(bad_rows[warp] != 0);
    }
    __syncwarp();
    pdl_join();
    if (bad_rows[0] | bad_rows[1] | bad_rows[2] | bad_rows[3]) {
      softmax_group_sync();              // all stores are done before a row is written again
      if (ok) attn_each_bad_row(bad_rows, warp, kSoftmaxWarps, [&](int r) { attn_exact_dq_row<__nv_bfloat16>(s, P.x, h, rt * kRows + r); });
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kSoftmaxWarps + 1) {
    tc_fence_after();
    tmem_free_all(tmem);
  }
}

template <int DP, int MOD>
templora_status_t launch_bwd(const BwdParams &p, cudaStream_t st) {
  TL_TRY((allow_smem<attn_dkdv_tc_kernel<DP, MOD>>(BwdCfg<DP>::kSmemKv)));
  TL_TRY((allow_smem<attn_dq_tc_kernel<DP, MOD>>(BwdCfg<DP>::kSmemQ)));
  {
    LaunchScope scope(kKindAttention, st);
    TL_CUDA_CHECK(launch_pdl(attn_dkdv_tc_kernel<DP, MOD>, dim3((p.s.Tk + kRows - 1) / kRows * p.s.Hkv, p.w.head_parts * p.w.row_parts), dim3(kThreadsTc),
                             BwdCfg<DP>::kSmemKv, st, p));
  }
  {
    LaunchScope scope(kKindAttention, st);
    TL_CUDA_CHECK(launch_pdl(attn_dq_tc_kernel<DP, MOD>, dim3(p.w.Tq_pad / kRows * p.s.H), dim3(kThreadsTc), BwdCfg<DP>::kSmemQ, st, p));
  }
  return p.w.head_parts * p.w.row_parts == 1 ? TEMPLORA_OK : attn_add_parts(p.s, p.x, p.w, TEMPLORA_BF16, st);
}

template <int DP, int MOD, bool PARTS>
templora_status_t launch_fwd(const FwdParams &p, cudaStream_t st) {
  TL_TRY((allow_smem<attn_fwd_tc_kernel<DP, MOD, PARTS>>(FwdCfg<DP>::kSmem)));
  LaunchScope scope(kKindAttention, st);
  TL_CUDA_CHECK(launch_pdl(attn_fwd_tc_kernel<DP, MOD, PARTS>, dim3(p.row_units * p.units, p.parts), dim3(kThreadsTc),
                           FwdCfg<DP>::kSmem, st, p));
  return TEMPLORA_OK;
}
template <int DP, int MOD>
templora_status_t launch_fwd(const FwdParams &p, cudaStream_t st) {
  return p.parts > 1 ? launch_fwd<DP, MOD, true>(p, st) : launch_fwd<DP, MOD, false>(p, st);
}

// finite for every finite scale, so that scores of 0 stay 0
float log2_scale(const AttnShape &s) { return fminf(fmaxf(s.scale * kLog2e, -FLT_MAX), FLT_MAX); }
ScoreMod score_mod(const AttnShape &s) {
  // cap_in = 0 says that nothing is capped: a zero scale's scores are 0 either way
  const float in = s.softcap > 0.f && s.softcap < kNoCap ? fminf(fmaxf(s.scale / s.softcap, -1e38f), 1e38f) : 0.f;      // finite times 2 log2(e) too
  if (fabsf(in) >= FLT_MIN) return ScoreMod{in, s.softcap * kLog2e};
  return ScoreMod{0.f, log2_scale(s)};
}
bool modified(const AttnShape &s) { return s.softcap > 0.f || s.slopes || !(s.scale > 0.f); }

}  // namespace

bool attn_tc_available() { return tc_available(); }

templora_status_t attn_tc_fwd(const AttnShape &s, const AttnTensors &x, const AttnFwdParts &parts, DeviceStatus *status, cudaStream_t st) {
  FwdParams p;
  p.s = s; p.x = x; p.status = status;
  p.mod = score_mod(s);
  p.c = log2_scale(s);
  int sms = 0;
  TL_TRY(stream_sms(st, &sms));
  p.tiles = (s.Tq + kRows - 1) / kRows;
  p.units = s.group % 2 == 0 ? s.H / 2 : s.H;
  p.row_units = s.group % 2 == 0 ? p.tiles : (p.tiles + 1) / 2;
  if ((long long)p.row_units * p.units > 0x7fffffff) return TEMPLORA_ERR_UNSUPPORTED;
  // Two heads on the same rows always suit each other.  Rows of one head: neighbours, whose keys are nearly the same, keep
  // the tensor core busy with one tile while the other's softmax runs; but when all CTAs run at once, the call lasts as
  // long as the last rows' CTA, and a long tile with a short one halves that.
  p.pairing = s.group % 2 == 0 ? kPairHeads : (s.causal && p.row_units * p.units <= sms) ? kPairMirrored : kPairRows;
  if (!make_map_heads(&p.tq, x.q, s.D, s.H, s.Tq, x.ldq, kRows) || !make_map_heads(&p.tk, x.k, s.D, s.Hkv, s.Tk, x.ldk, kRows) ||
      !make_map_heads(&p.tv, x.v, s.D, s.Hkv, s.Tk, x.ldv, kRows) || !make_map_heads(&p.to, x.o, s.D, s.H, s.Tq, x.ldo, 32))
    return TEMPLORA_ERR_CUDA;
  p.parts = parts.n; p.part_o = parts.o; p.part_ml = parts.ml;
  TL_TRY(s.D <= 64 ? (modified(s) ? launch_fwd<64, 1>(p, st) : launch_fwd<64, 0>(p, st))
                   : (modified(s) ? launch_fwd<128, 1>(p, st) : launch_fwd<128, 0>(p, st)));
  return parts.n == 1 ? TEMPLORA_OK : attn_join_parts(s, x, parts, st);
}

templora_status_t attn_tc_bwd(const AttnShape &s, const AttnTensors &x, const AttnBwdScratch &w, DeviceStatus *status,
                              cudaStream_t st) {
  BwdParams p;
  p.s = s; p.x = x; p.w = w; p.status = status;
  p.mod = score_mod(s);
  p.c = log2_scale(s);
  if ((long long)(w.Tq_pad / kRows) * s.H > 0x7fffffff || ((long long)s.Tk + kRows - 1) / kRows * s.Hkv > 0x7fffffff)
    return TEMPLORA_ERR_UNSUPPORTED;
  const bool ok = make_map_heads(&p.tq, x.q, s.D, s.H, s.Tq, x.ldq, kRows) && make_map_heads(&p.tk, x.k, s.D, s.Hkv, s.Tk, x.ldk, kRows) &&
                  make_map_heads(&p.tv, x.v, s.D, s.Hkv, s.Tk, x.ldv, kRows) && make_map_heads(&p.tdo, x.dO, s.D, s.H, s.Tq, x.lddo, kRows) &&
                  make_map_heads(&p.tdq, x.dq, s.D, s.H, s.Tq, x.lddq, 32) && make_map_heads(&p.tdk, x.dk, s.D, s.Hkv, s.Tk, x.lddk, 32) &&
                  make_map_heads(&p.tdv, x.dv, s.D, s.Hkv, s.Tk, x.lddv, 32);
  if (!ok) return TEMPLORA_ERR_CUDA;
  int sms = 0;
  TL_TRY(stream_sms(st, &sms));
  const int key_tiles = (s.Tk + kRows - 1) / kRows;
  // dk and dv in parts where one CTA to a key tile would leave half the SMs idle, and has tiles enough to make up for the
  // kernel that adds the parts.  Whole against parts, causal: 1024 tokens, 8 / 1 heads of 128: 130 -> 41 us; 300 tokens, 4 / 1: 38 ->
  // 33; 128 tokens, 4 / 1: 24 -> 28; 342 tokens, 16 / 8: 28 -> 37.  As many parts as run at once (2048 tokens, 8 / 2 heads: two
  // rounds of CTAs 92 us, one 68), the heads dealt evenly.
  if ((long long)key_tiles * s.Hkv * 2 > sms || (long long)s.group * (w.Tq_pad / kRows) < 10) p.w.head_parts = p.w.row_parts = 1;
  else {
    const int fit = (int)(sms / ((long long)key_tiles * s.Hkv)), each = (s.group + fit - 1) / fit;
    p.w.head_parts = std::min(p.w.head_parts, (s.group + each - 1) / each);
    p.w.row_parts = p.w.head_parts == s.group ? std::min(p.w.row_parts, std::max(1, fit / s.group)) : 1;
  }
  p.order = s.n_docs > 0 && key_tiles <= 256 && w.Tq_pad / kRows <= 256 && (long long)key_tiles * s.Hkv > sms ? key_tiles : 0;
  if (s.D <= 64) return modified(s) ? launch_bwd<64, 1>(p, st) : launch_bwd<64, 0>(p, st);
  return modified(s) ? launch_bwd<128, 1>(p, st) : launch_bwd<128, 0>(p, st);
}

}  // namespace templora
