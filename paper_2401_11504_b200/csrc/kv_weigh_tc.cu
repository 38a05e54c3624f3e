// What attention the cached tokens receive from the many rows of a chunk, on the 5th-generation tensor cores.
#include "kv_weigh.cuh"
#include "tc_device.cuh"
#include "tc_host.h"

#include <algorithm>
#include <type_traits>

namespace templora {
namespace {

// An item is 128 places of one kv head.  Their codes become bf16 numbers in shared memory (exactly: e4m3 has 4 significant bits), the
// first operand of 128 x 128 x head_dim products S^T = K Q^T whose second operand, 128 (row, head) pairs, comes in by TMA.  Scores
// alternate between two halves of the CTA's TMEM; a thread reads those of one place and 64 pairs, 32 at a time, so that a place's sum
// stays in a register and the pairs' lse, which all threads need at once, is a broadcast from shared memory.
// Warps 0-7 form the weights (warp w: places 32 (w % 4) .., pairs 64 (w / 4) ..), warp 8 copies and issues the products, warp 9 brings
// in the pairs' lse and positions (as each of the eight did for itself, that was half of all instructions).
// Bound by the exponentials, one per pair and place on a unit of 16 a cycle and SM: 1024 rows of 4096 tokens, 32 heads of 128, take
// 53.5 us (54.5 in calls over changing inputs), the exponentials alone 26.  A tile's weights take two CTAs of an SM 2400 cycles where the unit alone takes 2048; an item's
// keys and first pairs, with nothing to weigh meanwhile, are a quarter of the time.  Next item's codes asked for ahead (57 -> 61:
// registers), an eighth of the exponentials by a polynomial on the FMA pipe (57 -> 55), scores in quarters (57 -> 59) were not kept.
// Items are drawn from the counter in the workspace head, those of the first places, which most rows see, first.
// fp32 queries are three bf16 numbers each, exactly: a kernel before this one takes them apart, and a tile's products are added up over
// the three, the smallest first.  That is bound by the tensor cores (1536 cycles a tile and SM, the exponentials 1024).
constexpr int kTcWarps = 8, kTcThreads = 32 * (kTcWarps + 2);
constexpr int kPlaces = 128, kPairs = 128;
constexpr int kPanel = 128 * 128;        // bytes of 128 rows by 64 columns of bf16
enum { kWhereQueries = 710, kWhereScores = 711, kWhereRoom = 712, kWhereSlot = 713, kWherePairs = 714 };

struct Pairs {                           // of a tile
  float nlse[kPairs], nslope[kPairs];    // -lse, -slope
  float from_tile[kPairs];               // position less the item's first
  int pos[kPairs];                       // -1: none, or a row that counts for nothing
  int any[2], plain[2];                  // of each 64: are there any; does every place of the item see all, with finite lse
};

struct WeighTcParams {
  WeighParams p;
  CUtensorMap tq;                        // queries as [row][head][dim], boxes of rows_per_tile rows of a kv head's heads by 64 dims
  int rows_per_tile;
  void *terms;                           // fp32 queries as bf16 numbers
};

// 16 codes as bf16 numbers, two 16-byte chunks of a swizzled row
__device__ __forceinline__ void widen16(const uint4 &v, uint32_t row_at, int row, int chunk) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  uint32_t out[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float2 t = values_of_codes((w[i >> 1] >> (16 * (i & 1))) & 0xffffu);
    out[i] = pack_bf16x2(__float_as_uint(t.x), __float_as_uint(t.y));
  }
  st_shared_v4(row_at + ((chunk ^ (row & 7)) << 4), out[0], out[1], out[2], out[3]);
  st_shared_v4(row_at + (((chunk + 1) ^ (row & 7)) << 4), out[4], out[5], out[6], out[7]);
}

// fp32 rows as three planes of bf16 rows, contiguous: each the leading 8 bits of what the ones before leave.
constexpr int kTerms3 = 3;
__global__ void __launch_bounds__(256) weigh_terms_kernel(const float *q, long long ldq, int width, long long plane, uint2 *out) {
  pdl_prologue();
  const float *row = q + blockIdx.x * ldq;
  const bool vectors = (ldq & 3) == 0;
  for (int v = threadIdx.x; v < width / 4; v += 256) {
    float x[4];
    if (vectors) {
      const float4 y = __ldcs(reinterpret_cast<const float4 *>(row) + v);
      x[0] = y.x; x[1] = y.y; x[2] = y.z; x[3] = y.w;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = row[4 * v + i];
    }
#pragma unroll
    for (int t = 0; t < kTerms3; ++t) {
      uint32_t top[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t bits = __float_as_uint(x[i]);
        top[i] = bits & 0xffff0000u;
        if (fabsf(x[i]) < INFINITY) x[i] -= __uint_as_float(top[i]);      // exact
        else {
          if (x[i] != x[i]) top[i] = 0x7fc00000u;
          x[i] = 0.f;
        }
      }
      out[t * plane + blockIdx.x * (long long)(width / 4) + v] = make_uint2(top[0] >> 16 | top[1], top[2] >> 16 | top[3]);
    }
  }
}

// SPLIT: in clusters whose CTAs share an item's tiles of pairs.  TERMS: bf16 numbers that make up a query's
template <int DM, bool SPLIT, int TERMS>
__global__ void __launch_bounds__(kTcThreads, 2) weigh_tc_kernel(const __grid_constant__ WeighTcParams T) {
  pdl_prologue();
  constexpr int kTile = kPanel * (DM / 64);
  const WeighParams &P = T.p;
  const CacheView &c = P.c;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem0 = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t *tail = smem_raw + (smem0 - smem_u32(smem_raw)) + 3 * kTile;
  const uint32_t ring = smem0 + kTile, bar0 = smem_u32(tail);
  const auto q_full = [&](int i) { return bar0 + 8u * i; };
  const auto q_empty = [&](int i) { return bar0 + 16 + 8u * i; };
  const auto s_full = [&](int i) { return bar0 + 32 + 8u * i; };
  const auto s_empty = [&](int i) { return bar0 + 48 + 8u * i; };
  const auto p_full = [&](int i) { return bar0 + 64 + 8u * i; };
  const auto p_empty = [&](int i) { return bar0 + 80 + 8u * i; };
  const uint32_t drain = bar0 + 96;
  volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(tail + 104);
  volatile int *abort_flag = reinterpret_cast<volatile int *>(tail + 108);
  long long *next_item = reinterpret_cast<long long *>(tail + 112);
  float *half_sum = reinterpret_cast<float *>(tail + 128);                    // of pairs 64 .. 127
  Pairs *pairs_of = reinterpret_cast<Pairs *>(half_sum + kPlaces);            // of every other tile
  long long *before = reinterpret_cast<long long *>(pairs_of + 2);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  if (tid == 32 * kTcWarps) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(q_full(i), 1);
      mbar_init(q_empty(i), 1);
      mbar_init(s_full(i), 1);
      mbar_init(s_empty(i), kTcWarps);
      mbar_init(p_full(i), 1);
      mbar_init(p_empty(i), kTcWarps);
    }
    mbar_init(drain, 1);
    fence_barrier_init();
    *abort_flag = 0;
  }
  if (warp == 0) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32((const void *)tmem_slot)), "r"(256u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  count_tiles(P, kPlaces, before, kTcThreads);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  const long long total = before[c.n_seqs];
  const int rpt = T.rows_per_tile, pairs = rpt * P.group, S = SPLIT ? (int)cluster_size() : 1, rank = SPLIT ? (int)cluster_ctarank() : 0;
  const int place_of = 32 * (warp & 3) + lane, first_pair = 64 * ((warp >> 2) & 1);      // a thread's place, its warp's pairs
  const bool modified = P.softcap > 0.f || P.slopes;
  unsigned done_tiles = 0;               // of earlier items: a stage or half is used every other tile
  unsigned landed = 0, asked = 0;        // copying thread: tiles (of a term) waited for and requested

  for (long long item = blockIdx.x / S; item < total;) {
    const int seq = find_seq(before, c.n_seqs, item);
    const SeqRows r = seq_rows(P, seq);
    const long long local = item - before[seq];
    const int hk = (int)(local % c.Hkv), tile0 = r.base + (int)(local / c.Hkv) * kPlaces;
    const int new_from = r.len - r.rows, row0 = max(tile0 - new_from, 0);
    int row1 = r.rows;
    if (P.window > 0) row1 = (int)min((long long)row1, (long long)tile0 + kPlaces - 1 + P.window - new_from);
    const int all_tiles = (row1 - row0 + rpt - 1) / rpt, tiles = (all_tiles - rank + S - 1) / S;      // this CTA's: every S-th
    const auto first_row_of = [&](int i) { return row0 + (rank + i * S) * rpt; };
    const auto request = [&](int u) {      // copying thread: the last term of a tile, which is the smallest, first
      const unsigned t = done_tiles * TERMS + u, stage = t & 1;
      const int row = (TERMS - 1 - u % TERMS) * P.n_rows + r.first_row + first_row_of(u / TERMS);
      if (!mbar_wait_fast(q_empty(stage), ((t >> 1) & 1) ^ 1, abort_flag, c.status, kWhereRoom)) return false;
      mbar_arrive_expect_tx(q_full(stage), (uint32_t)pairs * 128u * (DM / 64));
#pragma unroll
      for (int b = 0; b < DM / 64; ++b)
        tma_load_3d(ring + stage * kTile + b * kPanel, &T.tq, q_full(stage), 64 * b, hk * P.group, row);
      ++asked;
      return true;
    };
    const int j = tile0 + place_of;
    float sum = 0.f, f = 0.f;
    long long place = -1;
    if (warp < kTcWarps) {
      const int id = j < r.len ? cache_block(c, seq, j >> c.bt_log2) : -1;
      // keys: two threads a place
      const int row = tid >> 1, jr = tile0 + row, half = tid & 1;
      const int idr = jr < r.len ? cache_block(c, seq, jr >> c.bt_log2) : -1;
      const uint8_t *codes = c.k + (((long long)max(idr, 0) * c.Hkv + hk) * c.bt + (jr & (c.bt - 1))) * c.D;
      const float unit = c.k_scale[(long long)max(id, 0) * c.Hkv + hk];
      constexpr int kEach = DM / 2;      // dims of a thread
      uint4 x[kEach / 16];
#pragma unroll
      for (int i = 0; i < kEach / 16; ++i) {
        const int d = half * kEach + 16 * i;
        x[i] = idr >= 0 && d < c.D ? __ldcs(reinterpret_cast<const uint4 *>(codes + d)) : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < kEach / 16; ++i) {
        const int d = half * kEach + 16 * i;
        widen16(x[i], smem0 + (d >> 6) * kPanel + row * 128, row, (d & 63) >> 3);
      }
      if (id >= 0) {
        place = ((long long)id * c.Hkv + hk) * c.bt + (j & (c.bt - 1));
        f = finite_unit(P.scale, unit);
      }
      fence_proxy_async_smem();
    } else if (warp == kTcWarps && lane == 0) {
      if (tiles > 0) request(0);
      *next_item = S == 1 && total < (1ll << 30) ? (long long)gridDim.x + atomicAdd(&c.status->sched_next, 1) : item + gridDim.x / S;
    }
    tc_fence_before();
    __syncthreads();                     // keys are in shared memory
    if (warp == kTcWarps) {
      if (lane == 0) {
        const uint32_t idesc = instr_desc(kPairs, 0, 0);
        const uint64_t tmpl = smem_desc_template(0);
        for (int i = 0; i < tiles; ++i) {
          const unsigned t = done_tiles + i, half = t & 1;
          bool fine = true;
          for (int term = 0; term < TERMS && fine; ++term) {
            const unsigned u = t * TERMS + term, stage = u & 1;
            if (!mbar_wait_fast(q_full(stage), (u >> 1) & 1, abort_flag, c.status, kWhereQueries)) { fine = false; break; }
            ++landed;
            if (term == 0 && !mbar_wait_fast(s_empty(half), ((t >> 1) & 1) ^ 1, abort_flag, c.status, kWhereSlot)) { fine = false; break; }
            tc_fence_after();
            const int steps = (c.D + 15) / 16;
            for (int k = 0; k < steps; ++k) {
              const uint32_t at = (k >> 2) * kPanel + (k & 3) * 32;
              tc_mma_bf16(tmem + 128 * half, tmpl | (uint64_t)(((smem0 + at) & 0x3FFFFu) >> 4),
                          tmpl | (uint64_t)(((ring + stage * kTile + at) & 0x3FFFFu) >> 4), idesc, term + k > 0);
            }
            tc_commit(q_empty(stage));
            if (term == TERMS - 1) tc_commit(s_full(half));
            if (TERMS * i + term + 1 < TERMS * tiles) fine = request(TERMS * i + term + 1);
          }
          if (!fine) break;
        }
      }
      __syncwarp();
    } else if (warp == kTcWarps + 1) {
      // lse of four pairs a lane, asked for a tile ahead
      int of_row[4], of_head[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int pair = lane + 32 * k;
        of_row[k] = pair < pairs ? pair / P.group : 1 << 30;
        of_head[k] = hk * P.group + (pair < pairs ? pair % P.group : 0);
      }
      float next_lse[4];
      const auto ask = [&](int i) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int row = first_row_of(i) + of_row[k];
          next_lse[k] = load_lse(P, r.first_row + row, of_head[k], row < row1);
        }
      };
      ask(0);
      for (int i = 0; i < tiles; ++i) {
        const unsigned t = done_tiles + i;
        Pairs &out = pairs_of[t & 1];
        if (!__all_sync(0xffffffffu, mbar_wait_fast(p_empty(t & 1), ((t >> 1) & 1) ^ 1, abort_flag, c.status, kWherePairs))) break;
        bool any[4], plain[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int row = first_row_of(i) + of_row[k], p = row < row1 && next_lse[k] != INFINITY ? new_from + row : -1;
          out.nlse[lane + 32 * k] = -next_lse[k];
          out.pos[lane + 32 * k] = p;
          if (P.slopes) {
            out.nslope[lane + 32 * k] = row < row1 ? -P.slopes[of_head[k]] : 0.f;
            out.from_tile[lane + 32 * k] = (float)(p - tile0);
          }
          any[k] = __any_sync(0xffffffffu, row < row1);
          plain[k] = __all_sync(0xffffffffu, p >= tile0 + kPlaces - 1 && (P.window == 0 || p - tile0 < P.window));
        }
        if (lane < 2) {
          out.any[lane] = lane ? any[2] || any[3] : any[0] || any[1];
          out.plain[lane] = !modified && (lane ? plain[2] && plain[3] : plain[0] && plain[1]);
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(p_full(t & 1));
        if (i + 1 < tiles) ask(i + 1);
      }
    } else {
      const uint64_t f2 = pack_f2(f, f), l2 = pack_f2(kLog2e, kLog2e);
      const uint64_t in2 = pack_f2(P.cap_in, P.cap_in), cap2 = pack_f2(P.softcap, P.softcap), down2 = pack_f2(-(float)place_of, -(float)place_of);
      const unsigned reach = P.window > 0 ? (unsigned)P.window : 0x80000000u;      // how far behind a row a place may be
      uint64_t sums[2] = {0, 0};
      const uint32_t t_lane = tmem + ((uint32_t)(32 * (warp & 3)) << 16) + first_pair;
      for (int i = 0; i < tiles; ++i) {
        const unsigned t = done_tiles + i, buf = t & 1;
        if (!mbar_wait_fast(p_full(buf), (t >> 1) & 1, abort_flag, c.status, kWherePairs)) break;
        const Pairs &in = pairs_of[buf];
        const bool any = in.any[first_pair >> 6], plain = in.plain[first_pair >> 6];
        const float *nlse = in.nlse + first_pair;
        if (!mbar_wait_fast(s_full(buf), (t >> 1) & 1, abort_flag, c.status, kWhereScores)) break;
        tc_fence_after();
#pragma unroll
        for (int h = 0; h < 2; ++h) {      // 32 pairs at a time: more registers than these would spill
          uint32_t v[32];
          if (any) {
            tmem_ld32(t_lane + 128 * buf + 32 * h, v);
            tmem_ld_wait();
          }
          if (h == 1) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(s_empty(buf));
          }
          if (!any) continue;
          if (plain) {
#pragma unroll
            for (int e = 0; e < 32; e += 4) {
              const float4 n = *reinterpret_cast<const float4 *>(nlse + 32 * h + e);
              const uint64_t a = mul_f2(fma_f2(pack_f2(__uint_as_float(v[e]), __uint_as_float(v[e + 1])), f2, pack_f2(n.x, n.y)), l2);
              const uint64_t b = mul_f2(fma_f2(pack_f2(__uint_as_float(v[e + 2]), __uint_as_float(v[e + 3])), f2, pack_f2(n.z, n.w)), l2);
              const float2 x = unpack_f2(a), y = unpack_f2(b);
              sums[0] = add_f2(sums[0], pack_f2(ex2(x.x), ex2(x.y)));
              sums[1] = add_f2(sums[1], pack_f2(ex2(y.x), ex2(y.y)));
            }
          } else {
            // capped scores, slopes, and pairs that do not see the place: as weights_of does, two at a time
#pragma unroll
            for (int e = 0; e < 32; e += 4) {
              const float4 n = *reinterpret_cast<const float4 *>(nlse + 32 * h + e);
              uint64_t t[2] = {pack_f2(__uint_as_float(v[e]), __uint_as_float(v[e + 1])), pack_f2(__uint_as_float(v[e + 2]), __uint_as_float(v[e + 3]))};
              const uint64_t n2[2] = {pack_f2(n.x, n.y), pack_f2(n.z, n.w)};
              if (P.softcap > 0.f) {
#pragma unroll
                for (int k = 0; k < 2; ++k) t[k] = fma_f2(tanh_f2(mul_f2(mul_f2(t[k], f2), in2)), cap2, n2[k]);
              } else {
#pragma unroll
                for (int k = 0; k < 2; ++k) t[k] = fma_f2(t[k], f2, n2[k]);
              }
              if (P.slopes) {
                const float4 b = *reinterpret_cast<const float4 *>(in.from_tile + first_pair + 32 * h + e);
                const float4 m = *reinterpret_cast<const float4 *>(in.nslope + first_pair + 32 * h + e);
                t[0] = fma_f2(pack_f2(m.x, m.y), add_f2(pack_f2(b.x, b.y), down2), t[0]);
                t[1] = fma_f2(pack_f2(m.z, m.w), add_f2(pack_f2(b.z, b.w), down2), t[1]);
              }
              const int4 p = *reinterpret_cast<const int4 *>(in.pos + first_pair + 32 * h + e);
              const float2 x = unpack_f2(mul_f2(t[0], l2)), y = unpack_f2(mul_f2(t[1], l2));
              const auto seen = [&](int at, float w) { return (unsigned)at - (unsigned)j < reach ? w : 0.f; };
              sums[0] = add_f2(sums[0], pack_f2(seen(p.x, ex2(x.x)), seen(p.y, ex2(x.y))));
              sums[1] = add_f2(sums[1], pack_f2(seen(p.z, ex2(y.x)), seen(p.w, ex2(y.y))));
            }
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(p_empty(buf));
      }
      const float2 a = unpack_f2(sums[0]), b = unpack_f2(sums[1]);
      sum += (a.x + a.y) + (b.x + b.y);
      if (warp >= 4) half_sum[place_of] = sum;
    }
    done_tiles += tiles;
    __syncthreads();                     // products of this item have been read, its sums are there
    item = *next_item;
    if (warp < 4) sum += half_sum[place_of];
    if (SPLIT) {                         // the cluster's first CTA adds up what all have
      if (warp < 4) half_sum[place_of] = sum;
      cluster_barrier();
      if (rank == 0 && warp < 4)
        for (int k = 1; k < S; ++k) sum += __uint_as_float(peer_u32(&half_sum[place_of], k));
      if (warp == 8 && lane < S && peer_u32((const void *)abort_flag, lane)) *abort_flag = 1;      // all leave together
      cluster_barrier();
    }
    if (*abort_flag) break;
    if (rank == 0 && warp < 4 && place >= 0 && j < r.len) {
      float *at = P.weights + place;
      *at = j < new_from ? *at + sum : sum;
    }
    __syncthreads();                     // before the next item is drawn into its place
  }
  if (tid == 32 * kTcWarps) {
    for (; landed < asked; ++landed) drain_copies(q_full(landed & 1), (landed >> 1) & 1);
    tc_commit(drain);
    const unsigned long long t0 = globaltimer_ns();
    while (!mbar_try(drain, 0) && globaltimer_ns() - t0 < kWaitLimitNs) {}
    const int done = atomicAdd(&c.status->sched_done, 1);
    if (done == (int)gridDim.x - 1) {
      c.status->sched_next = 0;
      c.status->sched_done = 0;
      __threadfence();
    }
  }
  __syncthreads();
  if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(256u) : "memory");
}

template <int DM, bool SPLIT, int TERMS> templora_status_t launch(WeighTcParams &t, int S, int sms, cudaStream_t st) {
  const WeighParams &p = t.p;
  constexpr size_t fixed = 1024 + 3 * (size_t)kPanel * (DM / 64) + 128 + kPlaces * 4 + 2 * sizeof(Pairs);
  TL_TRY((allow_smem<weigh_tc_kernel<DM, SPLIT, TERMS>>(fixed + (kMaxSeqs + 1) * sizeof(long long))));
  const int heads = p.c.Hkv * p.group;
  if (!make_map_head_rows(&t.tq, TERMS > 1 ? t.terms : p.q, p.c.D, heads, (long long)TERMS * p.n_rows, TERMS > 1 ? (long long)heads * p.c.D : p.ldq, p.group,
                          t.rows_per_tile))
    return TEMPLORA_ERR_CUDA;
  if (TERMS > 1) {
    const int width = heads * p.c.D;
    LaunchScope scope(kKindKvCache, st);
    TL_CUDA_CHECK(launch_pdl(weigh_terms_kernel, dim3((unsigned)p.n_rows), dim3(256), 0, st, (const float *)p.q, p.ldq, width,
                             (long long)p.n_rows * (width / 4), reinterpret_cast<uint2 *>(t.terms)));
  }
  const long long most = (long long)p.c.n_seqs * p.c.Hkv * (((long long)p.c.max_blocks * p.c.bt + kPlaces - 1) / kPlaces + 1);
  LaunchScope scope(kKindKvCache, st);
  TL_CUDA_CHECK(launch_cluster_pdl(weigh_tc_kernel<DM, SPLIT, TERMS>, dim3((int)std::min<long long>(most, 2ll * sms / S) * S), dim3(kTcThreads), S,
                                   fixed + (size_t)(p.c.n_seqs + 1) * sizeof(long long), st, t));
  return TEMPLORA_OK;
}

}  // namespace

// bf16 rows on 16-byte boundaries, or fp32, and enough of them that products of 128 columns are not mostly empty: 32 pairs a sequence and
// kv head, in fp32, where taking the rows apart is a launch of its own, 96 (41 sequences of 160 tokens, 64 / 32 heads: 42 rows, 84 pairs, 63 us
// here and 55 by the kernel without tensor memory; one of 1171, 64 / 8 heads, 1576 pairs: 38 and 107).
bool weigh_tc_available(const WeighParams &p, int dtype) {
  return p.offsets && (dtype == TEMPLORA_BF16 ? p.ldq % 8 == 0 && p.group <= kPairs && (long long)p.n_rows * p.group >= 32ll * p.c.n_seqs
                                              : weigh_tc_terms(p.c.Hkv * p.group, p.c.D, p.n_rows, p.c.n_seqs, p.group) > 0) &&
         kernel_path() != 1 && tc_available();
}
size_t weigh_tc_terms(int heads, int dim, int n_rows, int n_seqs, int group) {
  if (group > kPairs || (long long)n_rows * group < 96ll * n_seqs || n_rows > (1 << 28)) return 0;
  return align_up((size_t)n_rows * heads * dim * 2 * kTerms3, kWsAlign);
}
templora_status_t weigh_tc(const WeighParams &p, int dtype, void *terms, cudaStream_t st) {
  WeighTcParams t{};
  t.p = p;
  t.rows_per_tile = kPairs / p.group;
  t.terms = terms;
  int sms = 0;
  TL_TRY(stream_sms(st, &sms));
  const int S = weigh_cluster(p, kPlaces, (p.n_rows / p.c.n_seqs + t.rows_per_tile - 1) / t.rows_per_tile, sms);
  const auto go = [&](auto dm) {
    constexpr int DM = decltype(dm)::value;
    if (dtype == TEMPLORA_BF16) return S > 1 ? launch<DM, true, 1>(t, S, sms, st) : launch<DM, false, 1>(t, S, sms, st);
    return S > 1 ? launch<DM, true, kTerms3>(t, S, sms, st) : launch<DM, false, kTerms3>(t, S, sms, st);
  };
  return p.c.D <= 64 ? go(std::integral_constant<int, 64>{}) : go(std::integral_constant<int, 128>{});
}

}  // namespace templora
