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

namespace templora {
namespace {

constexpr int kRows = 128;               // rows of a tile
constexpr int kBox = kRows * 64 * 2;     // bytes of one 64-column box

// ------------------------------------------------------------------ instruction wrappers beyond tc_device.cuh
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap *map, uint32_t bar, int c0, int c1, int c2) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
      ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2) : "memory");
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
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&v)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,"
      "%29,%30,%31};"
      ::"r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
        "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]), "r"(v[17]), "r"(v[18]),
        "r"(v[19]), "r"(v[20]), "r"(v[21]), "r"(v[22]), "r"(v[23]), "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]),
        "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31]), "r"(taddr)
      : "memory");
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

// K-contiguous operand tile: descriptor of contraction steps [16 k, 16 k + 16); boxes of 64 columns follow one another
__device__ __forceinline__ uint64_t desc_k(uint64_t tmpl, uint32_t tile, int k) {
  return tmpl | (uint64_t)(((tile + (k >> 2) * kBox + (k & 3) * 32) & 0x3FFFFu) >> 4);
}
// the same tile contracted over its rows: steps are 16 rows, boxes are the chunks along N
__device__ __forceinline__ uint64_t desc_mn(uint64_t tmpl, uint32_t tile, int k) {
  return tmpl | (uint64_t)(((tile + k * 2048) & 0x3FFFFu) >> 4);
}

// Score modifications in units of log2: z = tanh(s * cap_in) * cap_out - slope * |p - j| (or s * cap_out without a cap).
struct ScoreMod {
  float cap_in, cap_out;   // scale / softcap and softcap * log2(e); without a cap 0 and scale * log2(e)
};

// tanh(x) = 1 - 2 / (1 + exp(2 x)): absolute error about 1e-7, two special-function instructions
__device__ __forceinline__ float tanh_of_scaled(float x2log2e) { return fmaf(-2.f, rcp(1.f + ex2(x2log2e)), 1.f); }

// ------------------------------------------------------------------ forward
// One CTA works on two 128-row query tiles that share their keys and values: two heads of a group on the same rows, or,
// with ungrouped heads, two neighbouring row tiles.  Warps 0-3 and 4-7 are the tiles' softmax groups (one thread per
// row: no shuffles), warp 8 issues the copies, warp 9 the MMAs.  While one tile's softmax runs, the tensor core works
// for the other.  TMEM: two 128-column score tiles and two output accumulators of up to 128 columns.  The running
// maximum only moves when a row's scores outgrow it by 2^8, so that the accumulator is rarely rescaled; the final
// division uses the same maximum, so this costs no accuracy.
// Bound by the special-function unit: 128 x 128 exponentials at 16 per clock take as long (1024 clocks) as the two
// products of a tile.
constexpr int kFwdThreads = 320;
template <int DP> struct FwdCfg {
  static constexpr int kTileB = kRows * DP * 2;
  static constexpr int kStages = DP == 128 ? 5 : 8;
  static constexpr int kSmem = 2 * kTileB + kStages * kTileB + 1024 + 1024;
};

struct FwdParams {
  CUtensorMap tq, tk, tv, to;
  AttnShape s;
  AttnTensors x;
  DeviceStatus *status;
  ScoreMod mod;
  float c;              // scores to units of log2 when nothing modifies them (MOD == 0)
  int row_tiles;        // 128-row tiles (heads paired) or pairs of them (rows paired)
  int pair_heads;       // 1: two heads on the same rows
  int units;            // heads or pairs of heads
};

template <int DP, int MOD>
__global__ void __launch_bounds__(kFwdThreads, 1) attn_fwd_tc_kernel(const __grid_constant__ FwdParams P) {
  using Cfg = FwdCfg<DP>;
  constexpr int kS = Cfg::kStages, kTileB = Cfg::kTileB;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem0 = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t *smem = smem_raw + (smem0 - smem_u32(smem_raw));
  const uint32_t ring = smem0 + 2 * kTileB, bar0 = ring + kS * kTileB;
  auto full = [&](int i) { return bar0 + 8u * i; };
  auto empty = [&](int i) { return bar0 + 8u * (kS + i); };
  auto s_full = [&](int w) { return bar0 + 8u * (2 * kS + w); };
  auto p_ready = [&](int w) { return bar0 + 8u * (2 * kS + 2 + w); };
  auto o_full = [&](int w) { return bar0 + 8u * (2 * kS + 4 + w); };
  const uint32_t q_full = bar0 + 8u * (2 * kS + 6), drain = bar0 + 8u * (2 * kS + 7);
  uint8_t *tail = smem + 2 * kTileB + kS * kTileB + 256;
  volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(tail);
  volatile int *abort_flag = reinterpret_cast<volatile int *>(tail + 4);
  int *range = reinterpret_cast<int *>(tail + 16);   // per tile: smallest start, largest end, largest start, smallest end

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const AttnShape &s = P.s;
  // the longest row tiles of a causal call come first
  const int unit = blockIdx.x % P.units, rt = P.row_tiles - 1 - blockIdx.x / P.units;
  auto head_of = [&](int w) { return P.pair_heads ? 2 * unit + w : unit; };
  auto row_of = [&](int w) { return P.pair_heads ? rt * kRows : (2 * rt + w) * kRows; };
  const int hk = head_of(0) / s.group;

  if (threadIdx.x == 0) {
    for (int i = 0; i < kS; ++i) { mbar_init(full(i), 1); mbar_init(empty(i), 1); }
    for (int w = 0; w < 2; ++w) { mbar_init(s_full(w), 1); mbar_init(p_ready(w), 4); mbar_init(o_full(w), 1); }
    mbar_init(q_full, 1);
    mbar_init(drain, 1);
    *abort_flag = 0;
    for (int w = 0; w < 2; ++w) { range[4 * w] = s.Tk; range[4 * w + 1] = 0; range[4 * w + 2] = 0; range[4 * w + 3] = s.Tk; }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 9) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32((const void *)tmem_slot)),
                 "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  pdl_prologue();

  int2 mine = make_int2(0, 0);
  const int row = warp < 8 ? row_of(warp >> 2) + (warp & 3) * 32 + lane : s.Tq;
  if (warp < 8) {
    const int w = warp >> 2;
    if (row < s.Tq) mine = attn_interval(s, row);
    const bool some = mine.x < mine.y, in = row < s.Tq;
    const int a = __reduce_min_sync(0xffffffffu, some ? mine.x : s.Tk), b = __reduce_max_sync(0xffffffffu, some ? mine.y : 0);
    const int c = __reduce_max_sync(0xffffffffu, in ? mine.x : 0), d = __reduce_min_sync(0xffffffffu, in ? mine.y : s.Tk);
    if (lane == 0) {
      atomicMin(range + 4 * w, a);
      atomicMax(range + 4 * w + 1, b);
      atomicMax(range + 4 * w + 2, c);
      atomicMin(range + 4 * w + 3, d);
    }
  }
  __syncthreads();
  // the CTA's keys start at key0 and come in n_it tiles; tile w takes part in iterations [first[w], end[w])
  int lo[2], hi[2], first[2], end[2];
#pragma unroll
  for (int w = 0; w < 2; ++w) { lo[w] = range[4 * w]; hi[w] = range[4 * w + 1]; }
  const int key0 = min(lo[0], lo[1]), key1 = max(hi[0], hi[1]);
  const int n_it = key1 > key0 ? (key1 - key0 + kRows - 1) / kRows : 0;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    first[w] = lo[w] < hi[w] ? (lo[w] - key0) / kRows : 0;
    end[w] = lo[w] < hi[w] ? (hi[w] - key0 + kRows - 1) / kRows : 0;
  }

  if (warp == 8) {
    // ===================== copies: Q, then K and V tiles in turn through one ring =====================
    if (lane == 0 && n_it > 0) {
      int n_q = 0;
      for (int w = 0; w < 2; ++w) n_q += first[w] < end[w];
      mbar_arrive_expect_tx(q_full, (uint32_t)(n_q * kTileB));
      for (int w = 0; w < 2; ++w)
        if (first[w] < end[w])
          for (int c = 0; c < DP / 64; ++c)
            tma_load_3d(smem0 + w * kTileB + c * kBox, &P.tq, q_full, c * 64, head_of(w), row_of(w));
      int r = 0;
      bool ok = true;
      for (; r < 2 * n_it && ok; ++r) {
        const int st = r % kS;
        if (!mbar_wait_fast(empty(st), ((r / kS) & 1) ^ 1u, abort_flag, P.status, 400)) { ok = false; break; }
        mbar_arrive_expect_tx(full(st), kTileB);
        for (int c = 0; c < DP / 64; ++c)
          tma_load_3d(ring + st * kTileB + c * kBox, (r & 1) ? &P.tv : &P.tk, full(st), c * 64, hk, key0 + (r >> 1) * kRows);
      }
      if (!ok) {   // copies in flight must land before the CTA may exit
        const unsigned long long t0 = globaltimer_ns();
        while (!mbar_try(q_full, 0) && globaltimer_ns() - t0 < kWaitLimitNs) {}
        for (int k = max(0, r - kS); k < r; ++k)
          while (!mbar_try(full(k % kS), (k / kS) & 1) && globaltimer_ns() - t0 < kWaitLimitNs) {}
      }
    }
  } else if (warp == 9) {
    // ===================== MMA issuer =====================
    if (lane == 0 && n_it > 0) {
      const uint32_t idesc_s = instr_desc(kRows, 0, 0), idesc_o = instr_desc(DP, 0, 1);
      const uint64_t t_k = smem_desc(0, 16, 1024), t_mn = smem_desc(0, kBox, 1024);
      auto wait_tile = [&](int r) {
        return mbar_wait_fast(full(r % kS), (r / kS) & 1, abort_flag, P.status, 410);
      };
      auto scores = [&](int w, int it) {
        const uint32_t a = smem0 + w * kTileB, b = ring + ((2 * it) % kS) * kTileB;
#pragma unroll
        for (int k = 0; k < DP / 16; ++k)
          tc_mma_bf16(tmem + w * 128, desc_k(t_k, a, k), desc_k(t_k, b, k), idesc_s, k != 0);
        tc_commit(s_full(w));
      };
      bool ok = mbar_wait_fast(q_full, 0, abort_flag, P.status, 411) && wait_tile(0);
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
            if (!mbar_wait_fast(p_ready(w), (it - first[w]) & 1, abort_flag, P.status, 412)) { ok = false; break; }
            tc_fence_after();
#pragma unroll
            for (int k = 0; k < kRows / 16; ++k)
              tc_mma_bf16_ts(tmem + 256 + w * 128, tmem + w * 128 + k * 8, desc_mn(t_mn, vt, k), idesc_o,
                             (it > first[w] || k != 0) ? 1u : 0u);
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
      if (!ok) {   // MMAs already issued must finish before TMEM is released
        tc_commit(drain);
        const unsigned long long t0 = globaltimer_ns();
        while (!mbar_try(drain, 0) && globaltimer_ns() - t0 < kWaitLimitNs) {}
      }
    }
  } else {
    // ===================== softmax and epilogue: one thread per row =====================
    const int w = warp >> 2, h = head_of(w);
    const uint32_t t_s = tmem + ((uint32_t)((warp & 3) * 32) << 16) + w * 128, t_o = t_s + 256;
    const float c = MOD ? 1.f : P.c;
    const float slope = (MOD && s.slopes) ? s.slopes[h] * kLog2e : 0.f;
    const int inner_lo = range[4 * w + 2], inner_hi = range[4 * w + 3];
    const int p = s.q_start + row;
    float m = -INFINITY, l = 0.f;
    bool ok = true;
    for (int it = first[w]; it < end[w]; ++it) {
      ok = mbar_wait_fast(s_full(w), (it - first[w]) & 1, abort_flag, P.status, 420);
      if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
      tc_fence_after();
      const int n0 = key0 + it * kRows;
      uint32_t v[4][32];
#pragma unroll
      for (int b = 0; b < 4; ++b) tmem_ld32(t_s + 32 * b, v[b]);
      tmem_ld_wait();
      if (MOD) {
        if (P.mod.cap_in != 0.f) {
          const float in = P.mod.cap_in * (2.f * kLog2e), out = P.mod.cap_out;
#pragma unroll
          for (int b = 0; b < 4; ++b)
#pragma unroll
            for (int i = 0; i < 32; ++i) v[b][i] = __float_as_uint(tanh_of_scaled(__uint_as_float(v[b][i]) * in) * out);
        } else {
#pragma unroll
          for (int b = 0; b < 4; ++b)
#pragma unroll
            for (int i = 0; i < 32; ++i) v[b][i] = __float_as_uint(__uint_as_float(v[b][i]) * P.mod.cap_out);
        }
        if (s.slopes) {
          const float back = (float)(p - n0);
#pragma unroll
          for (int b = 0; b < 4; ++b)
#pragma unroll
            for (int i = 0; i < 32; ++i)
              v[b][i] = __float_as_uint(fmaf(-slope, fabsf(back - (float)(32 * b + i)), __uint_as_float(v[b][i])));
        }
      }
      if (n0 < inner_lo || n0 + kRows > inner_hi) {   // some row of the tile does not see all of these keys
        const int a = mine.x - n0;
        const unsigned n = (unsigned)(mine.y - mine.x);
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
          for (int i = 0; i < 32; ++i)
            if ((unsigned)(32 * b + i - a) >= n) v[b][i] = 0xff800000u;
      }
      float mx = -INFINITY;
#pragma unroll
      for (int b = 0; b < 4; ++b)
#pragma unroll
        for (int i = 0; i < 32; ++i) mx = fmaxf(mx, __uint_as_float(v[b][i]));
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
          for (int d = 0; d < DP; d += 32) {
            uint32_t o[32];
            tmem_ld32(t_o + d, o);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
            tmem_st32(t_o + d, o);
          }
        }
      }
      const float base = m == -INFINITY ? 0.f : -m * c;
      float sum[2] = {0.f, 0.f};
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        uint32_t e[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float x = ex2(fmaf(__uint_as_float(v[b][2 * i]), c, base)), y = ex2(fmaf(__uint_as_float(v[b][2 * i + 1]), c, base));
          sum[0] += x;
          sum[1] += y;
          e[i] = pack2(x, y);   // the second product's operand: bf16, 2^-8 of each weight
        }
        tmem_st16(t_s + 16 * b, e);
      }
      l += sum[0] + sum[1];
      tmem_st_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(p_ready(w));
    }
    // ---- epilogue
    if (ok && first[w] < end[w]) ok = mbar_wait_fast(o_full(w), 0, abort_flag, P.status, 421);
    if (__all_sync(0xffffffffu, ok) && row_of(w) < s.Tq) {
      tc_fence_after();
      const bool any = first[w] < end[w];
      const float inv = l > 0.f ? 1.f / l : l;         // 0 for a row without keys, NaN stays
      bool bad = !(l < INFINITY);
      const int r = (warp & 3) * 32 + lane;
      const uint32_t stage = smem0 + w * kTileB + r * 128;
#pragma unroll
      for (int d = 0; d < DP; d += 32) {
        uint32_t o[32];
        if (any) {
          tmem_ld32(t_o + d, o);
          tmem_ld_wait();
        } else {
#pragma unroll
          for (int i = 0; i < 32; ++i) o[i] = 0;
        }
#pragma unroll
        for (int i = 0; i < 32; ++i) {
          const float x = l == 0.f ? 0.f : __uint_as_float(o[i]) * inv;
          bad |= !(fabsf(x) < INFINITY);
          o[i] = __float_as_uint(x);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int chunk = ((d & 63) >> 3) + i;
          st_shared_v4(stage + (d >> 6) * kBox + ((chunk ^ (r & 7)) << 4), pack_bf16x2(o[8 * i], o[8 * i + 1]),
                       pack_bf16x2(o[8 * i + 2], o[8 * i + 3]), pack_bf16x2(o[8 * i + 4], o[8 * i + 5]),
                       pack_bf16x2(o[8 * i + 6], o[8 * i + 7]));
        }
      }
      const bool in = row < s.Tq;
      if (in) P.x.lse[(long long)h * s.Tq + row] = l == 0.f ? -INFINITY : (m * c + __log2f(l)) * kLn2;
      // a row whose keys are all masked gets 0 even where a masked value made its accumulator NaN
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0 && row < s.Tq) {
        for (int d = 0; d < s.D; d += 64)
          tma_store_3d(&P.to, smem0 + w * kTileB + (d >> 6) * kBox + (warp & 3) * 32 * 128, d, h, row);
        bulk_commit_group();
        bulk_wait_group_all();
      }
      __syncwarp();
      unsigned redo = __ballot_sync(0xffffffffu, bad && in);
      while (redo) {
        attn_exact_fwd_row<__nv_bfloat16>(s, P.x, h, row - lane + __ffs(redo) - 1);
        redo &= redo - 1;
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 9) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
  }
}

// ------------------------------------------------------------------ backward
// P = exp2(z - lse2) and ds = P (dP - delta) (1 - tanh^2) are formed again from S = Q K^T and dP = dO V^T, once with the
// keys as rows (dk, dv: sums over queries, and over the heads of a group, stay in TMEM) and once with the queries as
// rows (dq).  Two products more than a backward that adds dq up in memory as the key tiles finish, but every sum is
// formed by one CTA in one order: the same call gives the same bits, and nothing is zeroed or converted afterwards.
// Warps 0-7 are the softmax group (two threads per row, 64 columns each), warp 8 issues copies, warp 9 MMAs.
constexpr int kBwdThreads = 320;
constexpr int kMaskedTiles = 8192;     // query tiles whose reach a bit is kept for (a million rows); the rest are all visited
template <int DP> struct BwdCfg {
  static constexpr int kTileB = kRows * DP * 2;
  static constexpr int kStages = DP == 128 ? 2 : 4;
  static constexpr int kStageB = 2 * kTileB + 2048;    // two tiles, row statistics, row intervals
  static constexpr int kSmem = 2 * kTileB + kStages * kStageB + 1024 + 3072;
};

struct BwdParams {
  CUtensorMap tq, tk, tv, tdo, tdq, tdk, tdv;
  AttnShape s;
  AttnTensors x;
  AttnBwdScratch w;
  DeviceStatus *status;
  ScoreMod mod;
  float c;
};

__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ void softmax_group_sync() { asm volatile("bar.sync 1, 256;" ::: "memory"); }
// TMEM column of contraction step k of a weight tile: the two 64-column halves keep their place over the scores
__device__ __forceinline__ uint32_t weight_col(int k) { return (uint32_t)((k >> 2) * 64 + (k & 3) * 8); }

// One score: weight p (for the product) and g = p (1 - tanh^2) (for ds).
template <int MOD>
__device__ __forceinline__ float bwd_weight(const BwdParams &P, float sc, float lse2, float slope, float dist, float &g) {
  if (!MOD) {
    const float p = ex2(fmaf(sc, P.c, -lse2));
    g = p;
    return p;
  }
  float z, t = 0.f;
  if (P.mod.cap_in != 0.f) {
    t = tanh_of_scaled(sc * (P.mod.cap_in * (2.f * kLog2e)));
    z = t * P.mod.cap_out;
  } else {
    z = sc * P.mod.cap_out;
  }
  const float p = ex2(fmaf(-slope, fabsf(dist), z) - lse2);
  g = fmaf(-t * t, p, p);
  return p;
}

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

// ---- dk and dv: one CTA per 128 keys of a kv head, over the query tiles that reach them, for each head of the group.
// TMEM: S^T, dP^T (their weights over them), dV, dK.  The next tile's S^T is issued behind dV's product, its dP^T behind
// dK's, so the tensor core has work while the weights are formed.
template <int DP, int MOD>
__global__ void __launch_bounds__(kBwdThreads, 1) attn_dkdv_tc_kernel(const __grid_constant__ BwdParams P) {
  using Cfg = BwdCfg<DP>;
  constexpr int kS = Cfg::kStages, kTileB = Cfg::kTileB, kStageB = Cfg::kStageB;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem0 = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t *smem = smem_raw + (smem0 - smem_u32(smem_raw));
  const uint32_t ring = smem0 + 2 * kTileB, bar0 = ring + kS * kStageB;
  auto full = [&](int i) { return bar0 + 8u * i; };
  auto empty = [&](int i) { return bar0 + 8u * (kS + i); };
  const uint32_t kv_full = bar0 + 8u * (2 * kS), s_full = kv_full + 8, dp_full = kv_full + 16, p_ready = kv_full + 24,
                 ds_ready = kv_full + 32, acc_full = kv_full + 40, drain = kv_full + 48;
  uint8_t *tail = smem + 2 * kTileB + kS * kStageB + 256;
  volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(tail);
  volatile int *abort_flag = reinterpret_cast<volatile int *>(tail + 4);
  unsigned *bad_rows = reinterpret_cast<unsigned *>(tail + 16);    // 4 words
  unsigned *active = reinterpret_cast<unsigned *>(tail + 32);      // kMaskedTiles bits

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const AttnShape &s = P.s;
  const int hk = blockIdx.x % s.Hkv, k0 = (blockIdx.x / s.Hkv) * kRows;   // a causal call's longest tiles come first
  const int n_qt = P.w.Tq_pad / kRows;
  if (threadIdx.x == 0) {
    for (int i = 0; i < kS; ++i) { mbar_init(full(i), 1); mbar_init(empty(i), 1); }
    mbar_init(kv_full, 1); mbar_init(s_full, 1); mbar_init(dp_full, 1); mbar_init(p_ready, 8); mbar_init(ds_ready, 8);
    mbar_init(acc_full, 1); mbar_init(drain, 1);
    *abort_flag = 0;
    for (int i = 0; i < 4; ++i) bad_rows[i] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 9) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32((const void *)tmem_slot)),
                 "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  pdl_prologue();
  const int n_bits = min(n_qt, kMaskedTiles);
  for (int t0 = warp * 32; t0 < n_bits; t0 += kBwdThreads) {
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
  const int qt_first = next_tile(0);
  const int steps_exist = qt_first < n_qt;

  if (warp == 8) {
    if (lane == 0 && steps_exist) {
      mbar_arrive_expect_tx(kv_full, 2 * kTileB);
      for (int c = 0; c < DP / 64; ++c) {
        tma_load_3d(smem0 + c * kBox, &P.tk, kv_full, c * 64, hk, k0);
        tma_load_3d(smem0 + kTileB + c * kBox, &P.tv, kv_full, c * 64, hk, k0);
      }
      int r = 0;
      bool ok = true;
      for (int h = hk * s.group; h < (hk + 1) * s.group && ok; ++h)
        for (int qt = qt_first; qt < n_qt; qt = next_tile(qt + 1), ++r) {
          const int st = r % kS;
          if (!mbar_wait_fast(empty(st), ((r / kS) & 1) ^ 1u, abort_flag, P.status, 500)) { ok = false; break; }
          mbar_arrive_expect_tx(full(st), kStageB);
          const uint32_t dst = ring + st * kStageB;
          for (int c = 0; c < DP / 64; ++c) {
            tma_load_3d(dst + c * kBox, &P.tq, full(st), c * 64, h, qt * kRows);
            tma_load_3d(dst + kTileB + c * kBox, &P.tdo, full(st), c * 64, h, qt * kRows);
          }
          bulk_load(dst + 2 * kTileB, P.w.stat + (long long)h * P.w.Tq_pad + qt * kRows, 1024, full(st));
          bulk_load(dst + 2 * kTileB + 1024, P.w.rows + qt * kRows, 1024, full(st));
        }
      if (!ok) {
        const unsigned long long t0 = globaltimer_ns();
        while (!mbar_try(kv_full, 0) && globaltimer_ns() - t0 < kWaitLimitNs) {}
        for (int k = max(0, r - kS); k < r; ++k)
          while (!mbar_try(full(k % kS), (k / kS) & 1) && globaltimer_ns() - t0 < kWaitLimitNs) {}
      }
    }
  } else if (warp == 9) {
    if (lane == 0 && steps_exist) {
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
      int n = 0;
      for (int qt = qt_first; qt < n_qt; qt = next_tile(qt + 1)) ++n;
      n *= s.group;
      bool ok = mbar_wait_fast(kv_full, 0, abort_flag, P.status, 510) && mbar_wait_fast(full(0), 0, abort_flag, P.status, 511);
      if (ok) {
        tc_fence_after();
        outer(tmem, smem0, ring, s_full);
        outer(tmem + 128, smem0 + kTileB, ring + kTileB, dp_full);
      }
      for (int r = 0; r < n && ok; ++r) {
        const uint32_t cur = ring + (r % kS) * kStageB, nxt = ring + ((r + 1) % kS) * kStageB;
        if (!(ok = mbar_wait_fast(p_ready, r & 1, abort_flag, P.status, 512))) break;
        tc_fence_after();
        accumulate(tmem + 256, tmem, cur + kTileB, r > 0);
        if (r + 1 < n) {
          if (!(ok = mbar_wait_fast(full((r + 1) % kS), ((r + 1) / kS) & 1, abort_flag, P.status, 513))) break;
          tc_fence_after();
          outer(tmem, smem0, nxt, s_full);
        }
        if (!(ok = mbar_wait_fast(ds_ready, r & 1, abort_flag, P.status, 514))) break;
        tc_fence_after();
        accumulate(tmem + 384, tmem + 128, cur, r > 0);
        tc_commit(empty(r % kS));
        if (r + 1 < n) outer(tmem + 128, smem0 + kTileB, nxt + kTileB, dp_full);
      }
      if (ok) {
        tc_commit(acc_full);
      } else {
        tc_commit(drain);
        const unsigned long long t0 = globaltimer_ns();
        while (!mbar_try(drain, 0) && globaltimer_ns() - t0 < kWaitLimitNs) {}
      }
    }
  } else {
    const int half = warp >> 2, row = (warp & 3) * 32 + lane, j = k0 + row;
    const uint32_t t_lane = tmem + ((uint32_t)((warp & 3) * 32) << 16), t_s = t_lane + 64 * half, t_dp = t_s + 128;
    bool ok = true;
    int r = 0;
    for (int h = hk * s.group; h < (hk + 1) * s.group && ok; ++h) {
      const float slope = (MOD && s.slopes) ? s.slopes[h] * kLog2e : 0.f;
      for (int qt = qt_first; qt < n_qt; qt = next_tile(qt + 1), ++r) {
        const int2 inner = P.w.inner[qt];
        const bool masked = k0 < inner.x || k0 + kRows > inner.y;
        const uint8_t *stage = smem + 2 * kTileB + (r % kS) * kStageB + 2 * kTileB;
        const float4 *stat = reinterpret_cast<const float4 *>(stage) + 32 * half;            // two rows each
        const int4 *rows = reinterpret_cast<const int4 *>(stage + 1024) + 32 * half;
        ok = mbar_wait_fast(full(r % kS), (r / kS) & 1, abort_flag, P.status, 520) &&        // the statistics
             mbar_wait_fast(s_full, r & 1, abort_flag, P.status, 521);
        if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
        tc_fence_after();
        float g[64];
        uint32_t v[32];
        const float dist0 = (float)(s.q_start + qt * kRows + 64 * half - j);
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          tmem_ld32(t_s + 32 * b, v);
          tmem_ld_wait();
          uint32_t e[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float4 st = stat[16 * b + i];
            const int a = 32 * b + 2 * i;
            float p0 = bwd_weight<MOD>(P, __uint_as_float(v[2 * i]), st.x, slope, dist0 + (float)a, g[a]);
            float p1 = bwd_weight<MOD>(P, __uint_as_float(v[2 * i + 1]), st.z, slope, dist0 + (float)(a + 1), g[a + 1]);
            if (masked) {
              const int4 rw = rows[16 * b + i];
              if (j < rw.x || j >= rw.y) p0 = g[a] = 0.f;
              if (j < rw.z || j >= rw.w) p1 = g[a + 1] = 0.f;
            }
            e[i] = pack2(p0, p1);
          }
          tmem_st16(t_s + 16 * b, e);
        }
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_ready);
        ok = mbar_wait_fast(dp_full, r & 1, abort_flag, P.status, 522);
        if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
        tc_fence_after();
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          tmem_ld32(t_dp + 32 * b, v);
          tmem_ld_wait();
          uint32_t e[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float4 st = stat[16 * b + i];
            const int a = 32 * b + 2 * i;
            e[i] = pack2(g[a] * (__uint_as_float(v[2 * i]) - st.y), g[a + 1] * (__uint_as_float(v[2 * i + 1]) - st.w));
          }
          tmem_st16(t_dp + 16 * b, e);
        }
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(ds_ready);
      }
    }
    // ---- epilogue: the first half stores dv, the second dk, through the stages (all their copies have been consumed)
    if (ok && steps_exist) ok = mbar_wait_fast(acc_full, 0, abort_flag, P.status, 523);
    ok = __all_sync(0xffffffffu, ok);
    if (ok) {
      tc_fence_after();
      const uint32_t tile = ring + half * kTileB;
      bool bad = false;
#pragma unroll 1
      for (int d = 0; d < DP; d += 32)
        bad |= stage_columns(t_lane + 256 + 128 * half, steps_exist, half ? s.scale : 1.f, tile, row, d);
      const unsigned votes = __ballot_sync(0xffffffffu, bad && j < s.Tk);
      if (lane == 0 && votes) atomicOr(bad_rows + (warp & 3), votes);
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0 && j < s.Tk) {
        for (int d = 0; d < s.D; d += 64)
          tma_store_3d(half ? &P.tdk : &P.tdv, tile + (d >> 6) * kBox + (warp & 3) * 32 * 128, d, hk, j);
        bulk_commit_group();
        bulk_wait_group_all();
      }
    }
    softmax_group_sync();    // both halves' stores are done before a row is written again
    if (ok && half == 0)
      for (unsigned redo = bad_rows[warp]; redo; redo &= redo - 1)
        attn_exact_dkdv_row<__nv_bfloat16>(s, P.x, hk, k0 + warp * 32 + __ffs(redo) - 1);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 9) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
  }
}

// ---- dq: one CTA per 128 queries of a head.  TMEM: S, dP twice (its weights over it), dQ.  The next tile's S is issued as
// soon as the softmax group has this one's in registers, its dP into the other buffer.
template <int DP, int MOD>
__global__ void __launch_bounds__(kBwdThreads, 1) attn_dq_tc_kernel(const __grid_constant__ BwdParams P) {
  using Cfg = BwdCfg<DP>;
  constexpr int kS = Cfg::kStages, kTileB = Cfg::kTileB, kStageB = 2 * Cfg::kTileB;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem0 = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t *smem = smem_raw + (smem0 - smem_u32(smem_raw));
  const uint32_t ring = smem0 + 2 * kTileB, bar0 = ring + kS * kStageB;
  auto full = [&](int i) { return bar0 + 8u * i; };
  auto empty = [&](int i) { return bar0 + 8u * (kS + i); };
  const uint32_t q_full = bar0 + 8u * (2 * kS), s_full = q_full + 8, s_free = q_full + 16, ds_ready = q_full + 24,
                 acc_full = q_full + 32, drain = q_full + 40;
  auto dp_full = [&](int b) { return q_full + 48 + 8u * b; };
  uint8_t *tail = smem + 2 * kTileB + kS * kStageB + 256;
  volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(tail);
  volatile int *abort_flag = reinterpret_cast<volatile int *>(tail + 4);
  unsigned *bad_rows = reinterpret_cast<unsigned *>(tail + 16);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const AttnShape &s = P.s;
  const int h = blockIdx.x % s.H, rt = P.w.Tq_pad / kRows - 1 - blockIdx.x / s.H, hk = h / s.group;
  if (threadIdx.x == 0) {
    for (int i = 0; i < kS; ++i) { mbar_init(full(i), 1); mbar_init(empty(i), 1); }
    mbar_init(q_full, 1); mbar_init(s_full, 1); mbar_init(s_free, 8); mbar_init(ds_ready, 8); mbar_init(acc_full, 1);
    mbar_init(drain, 1); mbar_init(dp_full(0), 1); mbar_init(dp_full(1), 1);
    *abort_flag = 0;
    for (int i = 0; i < 4; ++i) bad_rows[i] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 9) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32((const void *)tmem_slot)),
                 "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  pdl_prologue();
  const int2 reach = P.w.tiles[rt], inner = P.w.inner[rt];
  const int key0 = reach.x, n_it = reach.y > reach.x ? (reach.y - reach.x + kRows - 1) / kRows : 0;

  if (warp == 8) {
    if (lane == 0 && n_it > 0) {
      mbar_arrive_expect_tx(q_full, 2 * kTileB);
      for (int c = 0; c < DP / 64; ++c) {
        tma_load_3d(smem0 + c * kBox, &P.tq, q_full, c * 64, h, rt * kRows);
        tma_load_3d(smem0 + kTileB + c * kBox, &P.tdo, q_full, c * 64, h, rt * kRows);
      }
      bool ok = true;
      int it = 0;
      for (; it < n_it; ++it) {
        const int st = it % kS;
        if (!mbar_wait_fast(empty(st), ((it / kS) & 1) ^ 1u, abort_flag, P.status, 600)) { ok = false; break; }
        mbar_arrive_expect_tx(full(st), kStageB);
        for (int c = 0; c < DP / 64; ++c) {
          tma_load_3d(ring + st * kStageB + c * kBox, &P.tk, full(st), c * 64, hk, key0 + it * kRows);
          tma_load_3d(ring + st * kStageB + kTileB + c * kBox, &P.tv, full(st), c * 64, hk, key0 + it * kRows);
        }
      }
      if (!ok) {
        const unsigned long long t0 = globaltimer_ns();
        while (!mbar_try(q_full, 0) && globaltimer_ns() - t0 < kWaitLimitNs) {}
        for (int k = max(0, it - kS); k < it; ++k)
          while (!mbar_try(full(k % kS), (k / kS) & 1) && globaltimer_ns() - t0 < kWaitLimitNs) {}
      }
    }
  } else if (warp == 9) {
    if (lane == 0 && n_it > 0) {
      const uint32_t idesc_s = instr_desc(kRows, 0, 0), idesc_o = instr_desc(DP, 0, 1);
      const uint64_t t_k = smem_desc(0, 16, 1024), t_mn = smem_desc(0, kBox, 1024);
      auto outer = [&](uint32_t d, uint32_t a, uint32_t b, uint32_t bar) {
#pragma unroll
        for (int k = 0; k < DP / 16; ++k) tc_mma_bf16(d, desc_k(t_k, a, k), desc_k(t_k, b, k), idesc_s, k != 0);
        tc_commit(bar);
      };
      bool ok = mbar_wait_fast(q_full, 0, abort_flag, P.status, 610) && mbar_wait_fast(full(0), 0, abort_flag, P.status, 611);
      if (ok) {
        tc_fence_after();
        outer(tmem, smem0, ring, s_full);
        outer(tmem + 128, smem0 + kTileB, ring + kTileB, dp_full(0));
      }
      for (int it = 0; it < n_it && ok; ++it) {
        const uint32_t cur = ring + (it % kS) * kStageB, nxt = ring + ((it + 1) % kS) * kStageB;
        if (it + 1 < n_it) {
          ok = mbar_wait_fast(full((it + 1) % kS), ((it + 1) / kS) & 1, abort_flag, P.status, 612) &&
               mbar_wait_fast(s_free, it & 1, abort_flag, P.status, 613);
          if (!ok) break;
          tc_fence_after();
          outer(tmem, smem0, nxt, s_full);
          outer(tmem + 128 + 128 * ((it + 1) & 1), smem0 + kTileB, nxt + kTileB, dp_full((it + 1) & 1));
        }
        if (!(ok = mbar_wait_fast(ds_ready, it & 1, abort_flag, P.status, 614))) break;
        tc_fence_after();
#pragma unroll
        for (int k = 0; k < kRows / 16; ++k)
          tc_mma_bf16_ts(tmem + 384, tmem + 128 + 128 * (it & 1) + weight_col(k), desc_mn(t_mn, cur, k), idesc_o,
                         (it > 0 || k != 0) ? 1u : 0u);
        tc_commit(empty(it % kS));
      }
      if (ok) {
        tc_commit(acc_full);
      } else {
        tc_commit(drain);
        const unsigned long long t0 = globaltimer_ns();
        while (!mbar_try(drain, 0) && globaltimer_ns() - t0 < kWaitLimitNs) {}
      }
    }
  } else {
    const int half = warp >> 2, r = (warp & 3) * 32 + lane, row = rt * kRows + r;
    const uint32_t t_lane = tmem + ((uint32_t)((warp & 3) * 32) << 16), t_s = t_lane + 64 * half;
    const float2 stat = P.w.stat[(long long)h * P.w.Tq_pad + row];
    const int2 mine = P.w.rows[row];
    const float slope = (MOD && s.slopes) ? s.slopes[h] * kLog2e : 0.f;
    bool ok = true;
    for (int it = 0; it < n_it; ++it) {
      const int n0 = key0 + it * kRows + 64 * half;
      const bool masked = key0 + it * kRows < inner.x || key0 + it * kRows + kRows > inner.y;
      ok = mbar_wait_fast(s_full, it & 1, abort_flag, P.status, 620);
      if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
      tc_fence_after();
      uint32_t v[2][32];
      tmem_ld32(t_s, v[0]);
      tmem_ld32(t_s + 32, v[1]);
      tmem_ld_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(s_free);
      float g[64];
      const float dist0 = (float)(s.q_start + row - n0);
      const int a = mine.x - n0;
      const unsigned n = (unsigned)(mine.y - mine.x);
#pragma unroll
      for (int i = 0; i < 64; ++i) {
        bwd_weight<MOD>(P, __uint_as_float(v[i >> 5][i & 31]), stat.x, slope, dist0 - (float)i, g[i]);
        if (masked && (unsigned)(i - a) >= n) g[i] = 0.f;
      }
      ok = mbar_wait_fast(dp_full(it & 1), (it >> 1) & 1, abort_flag, P.status, 621);
      if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
      tc_fence_after();
      const uint32_t t_dp = t_s + 128 + 128 * (it & 1);
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        tmem_ld32(t_dp + 32 * b, v[b]);
        tmem_ld_wait();
        uint32_t e[16];
#pragma unroll
        for (int i = 0; i < 16; ++i)
          e[i] = pack2(g[32 * b + 2 * i] * (__uint_as_float(v[b][2 * i]) - stat.y),
                       g[32 * b + 2 * i + 1] * (__uint_as_float(v[b][2 * i + 1]) - stat.y));
        tmem_st16(t_dp + 16 * b, e);
      }
      tmem_st_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(ds_ready);
    }
    if (ok && n_it > 0) ok = mbar_wait_fast(acc_full, 0, abort_flag, P.status, 622);
    ok = __all_sync(0xffffffffu, ok);
    if (ok) {
      tc_fence_after();
      bool bad = false;
#pragma unroll 1
      for (int d = half * (DP / 2); d < (half + 1) * (DP / 2); d += 32)
        bad |= stage_columns(t_lane + 384, n_it > 0, s.scale, smem0, r, d);
      const unsigned votes = __ballot_sync(0xffffffffu, bad && row < s.Tq);
      if (lane == 0 && votes) atomicOr(bad_rows + (warp & 3), votes);
      fence_proxy_async_smem();
    }
    softmax_group_sync();
    if (ok && half == 0 && lane == 0 && row < s.Tq) {
      for (int d = 0; d < s.D; d += 64) tma_store_3d(&P.tdq, smem0 + (d >> 6) * kBox + warp * 32 * 128, d, h, row);
      bulk_commit_group();
      bulk_wait_group_all();
    }
    __syncwarp();
    if (ok && half == 0)
      for (unsigned redo = bad_rows[warp]; redo; redo &= redo - 1)
        attn_exact_dq_row<__nv_bfloat16>(s, P.x, h, rt * kRows + warp * 32 + __ffs(redo) - 1);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 9) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
  }
}

template <int DP, int MOD>
templora_status_t launch_bwd(const BwdParams &p, cudaStream_t st) {
  TL_TRY((allow_smem<attn_dkdv_tc_kernel<DP, MOD>>(BwdCfg<DP>::kSmem)));
  TL_TRY((allow_smem<attn_dq_tc_kernel<DP, MOD>>(BwdCfg<DP>::kSmem)));
  {
    LaunchScope scope(kKindAttention, st);
    TL_CUDA_CHECK(launch_pdl(attn_dkdv_tc_kernel<DP, MOD>, dim3((p.s.Tk + kRows - 1) / kRows * p.s.Hkv), dim3(kBwdThreads),
                             BwdCfg<DP>::kSmem, st, p));
  }
  LaunchScope scope(kKindAttention, st);
  TL_CUDA_CHECK(launch_pdl(attn_dq_tc_kernel<DP, MOD>, dim3(p.w.Tq_pad / kRows * p.s.H), dim3(kBwdThreads),
                           BwdCfg<DP>::kSmem, st, p));
  return TEMPLORA_OK;
}

template <int DP, int MOD>
templora_status_t launch_fwd(const FwdParams &p, cudaStream_t st) {
  TL_TRY((allow_smem<attn_fwd_tc_kernel<DP, MOD>>(FwdCfg<DP>::kSmem)));
  LaunchScope scope(kKindAttention, st);
  TL_CUDA_CHECK(launch_pdl(attn_fwd_tc_kernel<DP, MOD>, dim3(p.row_tiles * p.units), dim3(kFwdThreads), FwdCfg<DP>::kSmem, st, p));
  return TEMPLORA_OK;
}

ScoreMod score_mod(const AttnShape &s) {
  if (s.softcap > 0.f) return ScoreMod{s.scale / s.softcap, s.softcap * kLog2e};
  return ScoreMod{0.f, s.scale * kLog2e};
}
bool modified(const AttnShape &s) { return s.softcap > 0.f || s.slopes || !(s.scale > 0.f); }

}  // namespace

bool attn_tc_available() { return tc_available(); }

templora_status_t attn_tc_fwd(const AttnShape &s, const AttnTensors &x, DeviceStatus *status, cudaStream_t st) {
  FwdParams p;
  p.s = s; p.x = x; p.status = status;
  p.mod = score_mod(s);
  p.c = s.scale * kLog2e;
  p.pair_heads = s.group % 2 == 0;
  p.units = p.pair_heads ? s.H / 2 : s.H;
  const int tiles = (s.Tq + kRows - 1) / kRows;
  p.row_tiles = p.pair_heads ? tiles : (tiles + 1) / 2;
  if ((long long)p.row_tiles * p.units > 0x7fffffff) return TEMPLORA_ERR_UNSUPPORTED;
  if (!make_map_heads(&p.tq, x.q, s.D, s.H, s.Tq, x.ldq, kRows) || !make_map_heads(&p.tk, x.k, s.D, s.Hkv, s.Tk, x.ldk, kRows) ||
      !make_map_heads(&p.tv, x.v, s.D, s.Hkv, s.Tk, x.ldv, kRows) || !make_map_heads(&p.to, x.o, s.D, s.H, s.Tq, x.ldo, 32))
    return TEMPLORA_ERR_CUDA;
  if (s.D <= 64) return modified(s) ? launch_fwd<64, 1>(p, st) : launch_fwd<64, 0>(p, st);
  return modified(s) ? launch_fwd<128, 1>(p, st) : launch_fwd<128, 0>(p, st);
}

templora_status_t attn_tc_bwd(const AttnShape &s, const AttnTensors &x, const AttnBwdScratch &w, DeviceStatus *status,
                              cudaStream_t st) {
  BwdParams p;
  p.s = s; p.x = x; p.w = w; p.status = status;
  p.mod = score_mod(s);
  p.c = s.scale * kLog2e;
  if ((long long)(w.Tq_pad / kRows) * s.H > 0x7fffffff || ((long long)s.Tk + kRows - 1) / kRows * s.Hkv > 0x7fffffff)
    return TEMPLORA_ERR_UNSUPPORTED;
  const bool ok = make_map_heads(&p.tq, x.q, s.D, s.H, s.Tq, x.ldq, kRows) && make_map_heads(&p.tk, x.k, s.D, s.Hkv, s.Tk, x.ldk, kRows) &&
                  make_map_heads(&p.tv, x.v, s.D, s.Hkv, s.Tk, x.ldv, kRows) && make_map_heads(&p.tdo, x.dO, s.D, s.H, s.Tq, x.lddo, kRows) &&
                  make_map_heads(&p.tdq, x.dq, s.D, s.H, s.Tq, x.lddq, 32) && make_map_heads(&p.tdk, x.dk, s.D, s.Hkv, s.Tk, x.lddk, 32) &&
                  make_map_heads(&p.tdv, x.dv, s.D, s.Hkv, s.Tk, x.lddv, 32);
  if (!ok) return TEMPLORA_ERR_CUDA;
  if (s.D <= 64) return modified(s) ? launch_bwd<64, 1>(p, st) : launch_bwd<64, 0>(p, st);
  return modified(s) ? launch_bwd<128, 1>(p, st) : launch_bwd<128, 0>(p, st);
}

}  // namespace templora
