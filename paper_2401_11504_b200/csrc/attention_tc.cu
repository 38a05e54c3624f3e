// Attention of a chunk on the 5th-generation tensor cores: forward, and the two kernels of the backward.
//
// Every product is a chain of 128 x N x 16 tcgen05 MMAs into TMEM.  The softmax weights go from registers straight back
// into TMEM (over the scores they came from) and are the next product's first operand from there, so no score ever
// touches shared or global memory.  Tiles come in by TMA as 64-column, 128-byte-swizzled boxes of 128 rows of one head;
// the same box serves as a K-contiguous operand (contraction over head_dim) and as an M/N-contiguous one (contraction
// over its rows).  Head dims up to 64 and up to 128 have a kernel each; the columns behind head_dim read as zero.
#include <unordered_map>

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

}  // namespace templora
