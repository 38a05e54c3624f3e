// What attention the cached tokens receive from new query rows: the softmax weights of the rows over the 8-bit cache, added up
// per token and kv head.
#include "kv_weigh.cuh"
#include "tc_device.cuh"
#include "tc_host.h"

#include <algorithm>
#include <type_traits>

namespace templora {
namespace {

constexpr int kWeighThreads = 256, kWeighWarps = kWeighThreads / 32;

// ------------------------------------------------------------------ queries as matrix columns
// A warp-level product has 16 tokens as rows and 8 (row, head) pairs as columns.  Lane (g = lane / 4, c = lane % 4) holds of column
// g the dims [64 b + 16 c, +16) of every 64, as it holds of the keys: the order of the dims within a product is of no matter.
// A column is scaled by a power of two that brings its largest value into [2^14, 2^15).  fp16 then holds every bit of its bf16
// values down to 2^-28 of the largest, and three terms of 11 bits every bit of its fp32 values down to 2^-29.
template <bool F32> constexpr int kTerms = F32 ? 3 : 1;
template <int DM, bool F32> struct Column {
  uint32_t f[kTerms<F32>][DM / 16][2];
  float unit;                         // what the products are in units of, times the softmax scale
};
template <bool F32> using QueryType = typename std::conditional<F32, float, __nv_bfloat16>::type;
template <int DM, bool F32> struct RawColumn { Raw16<QueryType<F32>> x[DM / 64]; };      // as it is stored
template <int DM, bool F32>
__device__ __forceinline__ void ask_column(const WeighParams &P, int row, int head, bool there, int lane, RawColumn<DM, F32> &r) {
  using T = QueryType<F32>;
  const int c = lane & 3;
  const T *q = (const T *)P.q + (long long)row * P.ldq + (long long)head * P.c.D;
  const bool vec = (P.ldq * sizeof(T)) % 16 == 0;
#pragma unroll
  for (int b = 0; b < DM / 64; ++b) {
    const int d = 64 * b + 16 * c;
#pragma unroll
    for (int i = 0; i < (int)sizeof(T); ++i) r.x[b].w[i] = make_uint4(0, 0, 0, 0);
    if (there && d < P.c.D) load16<T>(q + d, vec, r.x[b]);
  }
}
// the largest finite magnitude of 16 values
__device__ __forceinline__ float largest16(const Raw16<float> &r) {
  float v[16], amax = 0.f;
  values16(r, v);
#pragma unroll
  for (int i = 0; i < 16; ++i) if (fabsf(v[i]) < INFINITY) amax = fmaxf(amax, fabsf(v[i]));
  return amax;
}
__device__ __forceinline__ float largest16(const Raw16<__nv_bfloat16> &r) {
  const auto size = [](const uint32_t &w) { return __habs2(*reinterpret_cast<const __nv_bfloat162 *>(&w)); };
  __nv_bfloat162 m[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) m[i] = __hmax2(__hmax2(size(r.w[i].x), size(r.w[i].y)), __hmax2(size(r.w[i].z), size(r.w[i].w)));
  const float2 f = __bfloat1622float2(__hmax2(m[0], m[1]));
  float amax = fmaxf(f.x, f.y);        // NaN has been left out
  if (!(amax < INFINITY)) {
    float v[16];
    values16(r, v);
    amax = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) if (fabsf(v[i]) < INFINITY) amax = fmaxf(amax, fabsf(v[i]));
  }
  return amax;
}
template <int DM, bool F32>
__device__ __forceinline__ void form_column(const WeighParams &P, const RawColumn<DM, F32> &raw, Column<DM, F32> &r) {
  float amax = 0.f;
#pragma unroll
  for (int b = 0; b < DM / 64; ++b) amax = fmaxf(amax, largest16(raw.x[b]));
  amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
  amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
  int e = (int)(__float_as_uint(amax) >> 23) - 127 - 14;      // amax 2^-e in [2^14, 2^15)
  if (__float_as_uint(amax) < 0x00800000u) e = -126 - 14;     // zero or subnormal
  e = max(e, -120);                                           // 2^-e stays finite; such rows are below any use
  const float up = pow2f(-e);
#pragma unroll
  for (int b = 0; b < DM / 64; ++b) {
    float v[16];
    values16(raw.x[b], v);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float x0 = v[2 * i] * up, x1 = v[2 * i + 1] * up;
#pragma unroll
      for (int t = 0; t < kTerms<F32>; ++t) {
        const uint32_t h = pack_half2(x0, x1);
        r.f[t][4 * b + (i >> 1)][i & 1] = h;
        if (t + 1 < kTerms<F32>) {      // what is left; nothing of what is not finite
          const float2 y = __half22float2(*reinterpret_cast<const __half2 *>(&h));
          x0 = fabsf(x0) < INFINITY ? x0 - y.x : 0.f;
          x1 = fabsf(x1) < INFINITY ? x1 - y.y : 0.f;
        }
      }
    }
  }
  r.unit = P.scale * pow2f(e);
}

// Codes of 16 tokens: lane (g, c) holds tokens g and g + 8, bytes [16 c, 16 c + 16) of every 64.
template <int DM> struct KeyCodes { uint4 w[2][DM / 64]; };
template <int DM>
__device__ __forceinline__ void load_keys(const uint8_t *rows, int D, int lane, KeyCodes<DM> &r) {
  const int g = lane >> 2, c = lane & 3;
#pragma unroll
  for (int a = 0; a < 2; ++a)
#pragma unroll
    for (int b = 0; b < DM / 64; ++b) {
      const int d = 64 * b + 16 * c;
      r.w[a][b] = d < D ? __ldcs(reinterpret_cast<const uint4 *>(rows + (g + 8 * a) * D + d)) : make_uint4(0, 0, 0, 0);
    }
}
__device__ __forceinline__ uint32_t word_of(const uint4 &v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// ------------------------------------------------------------------ one row per sequence
// The tiles of 16 tokens of all (sequence, kv head) pairs form one list that is dealt evenly to all warps.  A warp walks its share;
// the codes of the tiles ahead are on their way into a ring in shared memory, where each lane reads back what it has copied itself, so
// that nothing waits but for its own copies.  The query of a pair stays in registers.
// Bound by the codes and weights that it streams: head_dim + 8 bytes per token and kv head.  (With the next tile's codes in registers
// instead of a ring, 100003 tokens of 32 heads of 128 took 82 us.)  They take 78 us, 5.6 TB/s, replayed from a graph, as all times in these
// files are, and 87 us, 5.0 TB/s, in calls over changing inputs; 16 sequences of up to 4096 tokens, 64 / 8 heads, capped, 14 and 16 us, of
// which the chain of length, table and first codes is 4, and then the issue of 250 instructions per 16 tokens counts.
constexpr int kRing = 4;
__device__ __forceinline__ void copy16(uint32_t to, const void *from, bool there) {      // zeros if not
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t to, const void *from, bool there) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to), "l"(from), "r"(there ? 4 : 0) : "memory");
}
__device__ __forceinline__ void copies_asked() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_landed() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
template <int DM> constexpr int kSlotBytes = 32 * (DM / 64 * 2 * 16 + 4);

// NC: how many times 8 heads a kv head may have
template <int DM, bool F32, int NC>
__global__ void __launch_bounds__(kWeighThreads, F32 || NC > 1 ? 2 : 3) weigh_step_kernel(const WeighParams P) {
  pdl_prologue();
  extern __shared__ __align__(16) uint8_t smem_raw[];
  const CacheView &c = P.c;
  const int lane = threadIdx.x & 31, g = lane >> 2, cc = lane & 3;
  constexpr int kVecs = DM / 64 * 2;
  uint8_t *ring = smem_raw + (threadIdx.x >> 5) * kRing * kSlotBytes<DM>;
  long long *before = reinterpret_cast<long long *>(smem_raw + kWeighWarps * kRing * kSlotBytes<DM>);
  if (c.n_seqs <= 32) {
    before += (threadIdx.x >> 5) * 33;
    count_tiles_of_few(P, 16, before);
  } else {
    count_tiles(P, 16, before, kWeighThreads);
  }
  const long long total = before[c.n_seqs], W = (long long)gridDim.x * kWeighWarps;
  const long long me = (long long)(threadIdx.x >> 5) * gridDim.x + blockIdx.x;
  long long t = total * me / W;
  const long long t1 = total * (me + 1) / W;
  if (t >= t1) return;
  int seq = find_seq(before, c.n_seqs, t);
  while (t < t1) {
    while (before[seq + 1] <= t) ++seq;
    const SeqRows r = seq_rows(P, seq);
    const int tiles = (r.len - r.base + 15) / 16;
    const int local = (int)((t - before[seq]) % tiles), hk = (int)((t - before[seq]) / tiles);
    const int n = (int)min((long long)(tiles - local), t1 - t);
    const int first = P.window > 0 ? max(r.len - P.window, 0) : 0, j_base = r.base + 16 * local;
    // the pair's query and its lse: asked for before anything is waited for
    RawColumn<DM, F32> raw[NC];
    float lse[NC][2], slope[NC][2];
#pragma unroll
    for (int q = 0; q < NC; ++q) {
      ask_column<DM, F32>(P, seq, hk * P.group + 8 * q + g, 8 * q + g < P.group, lane, raw[q]);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int h = 8 * q + 2 * cc + k;
        lse[q][k] = load_lse(P, seq, hk * P.group + h, h < P.group);
        slope[q][k] = P.slopes && h < P.group ? P.slopes[hk * P.group + h] : 0.f;
      }
    }
    // Lanes look up the blocks of 32 tiles at a time, half of that ahead, and their scales as soon as the blocks are known.
    const auto look_up = [&](int i) { return i < n ? cache_block(c, seq, (j_base + 16 * i) >> c.bt_log2) : -1; };
    int ids = look_up(lane), next_ids = -1;
    float scales = ids >= 0 ? c.k_scale[(long long)ids * c.Hkv + hk] : 0.f;
    const auto place_of = [&](int id, int i) { return ((long long)id * c.Hkv + hk) * c.bt + ((j_base + 16 * i) & (c.bt - 1)); };
    const auto fetch = [&](int i) {
      if (i < n) {
        if ((i & 31) == 0 && i > 0) {
          ids = next_ids;
          scales = ids >= 0 ? c.k_scale[(long long)ids * c.Hkv + hk] : 0.f;
        }
        const int id = __shfl_sync(0xffffffffu, ids, i & 31);
        if (id >= 0) {
          const long long place = place_of(id, i);
          const uint32_t slot = smem_u32(ring + (i % kRing) * kSlotBytes<DM>);
#pragma unroll
          for (int v = 0; v < kVecs; ++v) {      // token g, then g + 8; bytes [16 c, 16 c + 16) of every 64
            const int d = 64 * (v % (DM / 64)) + 16 * cc, tok = g + 8 * (v / (DM / 64));
            copy16(slot + 16 * (32 * v + lane), c.k + (place + tok) * c.D + (d < c.D ? d : 0), d < c.D);
          }
          // lanes c = 0 and 1 write their tokens g and g + 8; what the newest one's place holds does not count
          if (cc < 2) copy4(slot + 16 * 32 * kVecs + 4 * lane, P.weights + place + g + 8 * cc, j_base + 16 * i + g + 8 * cc < r.len - 1);
        }
        if ((i & 31) == 16) next_ids = look_up(i + 16 + lane);
      }
      copies_asked();
    };
#pragma unroll
    for (int i = 0; i < kRing - 1; ++i) fetch(i);
    Column<DM, F32> col[NC];
    float unit[NC][2];
#pragma unroll
    for (int q = 0; q < NC; ++q) {
      form_column<DM, F32>(P, raw[q], col[q]);
#pragma unroll
      for (int k = 0; k < 2; ++k) unit[q][k] = __shfl_sync(0xffffffffu, col[q].unit, 4 * (2 * cc + k));
    }
    int now_ids = ids;                  // of the tiles being worked on
    float now_scales = scales;
    for (int i = 0; i < n; ++i) {
      if ((i & 31) == 0) { now_ids = ids; now_scales = scales; }
      const int id = __shfl_sync(0xffffffffu, now_ids, i & 31);
      const float ks = __shfl_sync(0xffffffffu, now_scales, i & 31);
      copies_landed<kRing - 2>();
      const uint8_t *slot = ring + (i % kRing) * kSlotBytes<DM>;
      float part[NC][DM / 64][4];
#pragma unroll
      for (int b = 0; b < DM / 64; ++b) {
#pragma unroll
        for (int q = 0; q < NC; ++q) part[q][b][0] = part[q][b][1] = part[q][b][2] = part[q][b][3] = 0.f;
        const uint4 k0 = reinterpret_cast<const uint4 *>(slot)[32 * b + lane], k1 = reinterpret_cast<const uint4 *>(slot)[32 * (b + DM / 64) + lane];
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          uint32_t a0, a1, a2, a3;
          half2s_of_codes(word_of(k0, w), a0, a2);
          half2s_of_codes(word_of(k1, w), a1, a3);
#pragma unroll
          for (int q = 0; q < NC; ++q)
#pragma unroll
            for (int s = kTerms<F32> - 1; s >= 0; --s) mma_16816(part[q][b], a0, a1, a2, a3, col[q].f[s][4 * b + w][0], col[q].f[s][4 * b + w][1]);
        }
      }
      const float old = reinterpret_cast<const float *>(slot + 16 * 32 * kVecs)[lane];
      fetch(i + kRing - 1);             // into the slot of the tile before
      const int j = j_base + 16 * i + g;
      float sum[2] = {0.f, 0.f};
#pragma unroll
      for (int q = 0; q < NC; ++q)
#pragma unroll
        for (int k2 = 0; k2 < 2; ++k2) {
          const float f = finite_unit(unit[q][k2], ks);
#pragma unroll
          for (int a = 0; a < 2; ++a) {
            const float s = DM == 64 ? part[q][0][2 * a + k2] : part[q][0][2 * a + k2] + part[q][DM / 64 - 1][2 * a + k2];
            sum[a] += weight_of(P, s, f, lse[q][k2], slope[q][k2], r.len - 1 - j - 8 * a);
          }
        }
#pragma unroll
      for (int a = 0; a < 2; ++a) {
        sum[a] += __shfl_xor_sync(0xffffffffu, sum[a], 1);
        sum[a] += __shfl_xor_sync(0xffffffffu, sum[a], 2);
      }
      const int mine = j + 8 * cc;
      if (cc < 2 && id >= 0 && mine >= first && mine < r.len) P.weights[place_of(id, i) + g + 8 * cc] = old + (cc == 0 ? sum[0] : sum[1]);
    }
    t += n;
  }
}

// ------------------------------------------------------------------ many rows per sequence
// A CTA takes 8 x 16 MT tokens of one kv head, 16 MT a warp, whose keys stay in registers as fp16, and walks the (row, head) pairs
// that see any of them, 64 at a time through shared memory: each warp brings 8 of them in.  The CTAs of a cluster (MT 1) share out the pairs.
// For few rows, and for rows that TMA cannot bring in.  Bound by an item's chain (table, codes, rows, products) where pairs are few (43 sequences of up
// to 3402 tokens, 3 rows, 16 / 8 heads of 96: 46 us, floor 9), by the issue of products and weights where they are many.
constexpr int kStageColumns = 8 * kWeighWarps;
template <int DM, bool F32, int MT>
__global__ void __launch_bounds__(kWeighThreads, 2) weigh_rows_kernel(const WeighParams P) {
  pdl_prologue();
  extern __shared__ __align__(16) uint8_t smem_raw[];
  constexpr int kTile = 16 * MT * kWeighWarps, kSteps = DM / 16, kFrag = kTerms<F32> * kSteps * 32;
  uint2 *frag = reinterpret_cast<uint2 *>(smem_raw);                               // [8 columns][term][step][lane]
  float4 *info = reinterpret_cast<float4 *>(frag + kWeighWarps * kFrag);           // unit, lse, slope, position of a column
  float *joined = reinterpret_cast<float *>(info + kStageColumns);                 // this CTA's sums, for the cluster's first
  long long *before = reinterpret_cast<long long *>(joined + kTile);
  const CacheView &c = P.c;
  const int S = MT == 1 ? (int)cluster_size() : 1, rank = MT == 1 ? (int)cluster_ctarank() : 0;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, cc = lane & 3;
  count_tiles(P, kTile, before, kWeighThreads);
  const long long total = before[c.n_seqs];
  for (long long item = blockIdx.x / S; item < total; item += gridDim.x / S) {
    const int seq = find_seq(before, c.n_seqs, item);
    const SeqRows r = seq_rows(P, seq);
    const int tiles = (r.len - r.base + kTile - 1) / kTile;
    const int hk = (int)((item - before[seq]) / tiles), tile0 = r.base + (int)((item - before[seq]) % tiles) * kTile;
    const int j0 = tile0 + warp * 16 * MT, new_from = r.len - r.rows;
    uint32_t a[MT][kSteps][4];
    float ks[MT], sum[MT][2];
    long long place[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      const int j = j0 + 16 * m;
      const int id = j < r.len ? cache_block(c, seq, j >> c.bt_log2) : -1;
      place[m] = id >= 0 ? ((long long)id * c.Hkv + hk) * c.bt + (j & (c.bt - 1)) : -1;
      ks[m] = id >= 0 ? c.k_scale[(long long)id * c.Hkv + hk] : 0.f;
      KeyCodes<DM> k;
#pragma unroll
      for (int b = 0; b < DM / 64; ++b) k.w[0][b] = k.w[1][b] = make_uint4(0, 0, 0, 0);
      if (id >= 0) load_keys<DM>(c.k + place[m] * c.D, c.D, lane, k);
#pragma unroll
      for (int b = 0; b < DM / 64; ++b)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          half2s_of_codes(word_of(k.w[0][b], w), a[m][4 * b + w][0], a[m][4 * b + w][2]);
          half2s_of_codes(word_of(k.w[1][b], w), a[m][4 * b + w][1], a[m][4 * b + w][3]);
        }
      sum[m][0] = sum[m][1] = 0.f;
    }
    // rows that see any of the tile's tokens
    const int row0 = max(tile0 - new_from, 0);
    int row1 = r.rows;
    if (P.window > 0) row1 = (int)min((long long)row1, (long long)tile0 + kTile - 1 + P.window - new_from);
    const long long col1 = (long long)row1 * P.group;
    const unsigned reach = P.window > 0 ? (unsigned)P.window : 0x80000000u;      // how far behind a row a place may be
    for (long long col0 = (long long)row0 * P.group + rank * kStageColumns; col0 < col1; col0 += S * kStageColumns) {
      __syncthreads();                // the columns before have been used
      {
        const long long col = col0 + 8 * warp + g;
        const bool there = col < col1;
        const int row = there ? (int)(col / P.group) : 0, head = hk * P.group + (there ? (int)(col % P.group) : 0);
        Column<DM, F32> x;
        RawColumn<DM, F32> raw;
        ask_column<DM, F32>(P, r.first_row + row, head, there, lane, raw);
        form_column<DM, F32>(P, raw, x);
#pragma unroll
        for (int t = 0; t < kTerms<F32>; ++t)
#pragma unroll
          for (int s = 0; s < kSteps; ++s) frag[warp * kFrag + (t * kSteps + s) * 32 + lane] = make_uint2(x.f[t][s][0], x.f[t][s][1]);
        if (cc == 0)      // a column that is none stands before all places
          info[8 * warp + g] = make_float4(x.unit, load_lse(P, r.first_row + row, head, there),
                                           P.slopes && there ? P.slopes[head] : 0.f, __int_as_float(there ? new_from + row : -1));
      }
      __syncthreads();
      const int chunks = (int)min((long long)kWeighWarps, (col1 - col0 + 7) / 8);
      for (int ch = 0; ch < chunks; ++ch) {
        // positions grow with the columns: does any of these see any of the warp's tokens?
        const int p_first = __float_as_int(info[8 * ch].w), p_last = __float_as_int(info[min(8 * ch + 7, (int)min((long long)kStageColumns, col1 - col0) - 1)].w);
        if (j0 >= r.len || p_last < j0 || (P.window > 0 && (long long)p_first - (j0 + 16 * MT - 1) >= P.window)) continue;
        float acc[MT][4];
#pragma unroll
        for (int m = 0; m < MT; ++m) acc[m][0] = acc[m][1] = acc[m][2] = acc[m][3] = 0.f;
#pragma unroll
        for (int t = kTerms<F32> - 1; t >= 0; --t)
#pragma unroll
          for (int s = 0; s < kSteps; ++s) {
            const uint2 b = frag[ch * kFrag + (t * kSteps + s) * 32 + lane];
#pragma unroll
            for (int m = 0; m < MT; ++m) mma_16816(acc[m], a[m][s][0], a[m][s][1], a[m][s][2], a[m][s][3], b.x, b.y);
          }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const float4 x = info[8 * ch + 2 * cc + k];
          const int p = __float_as_int(x.w);
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            const float f = finite_unit(x.x, ks[m]);
            const int back = p - (j0 + 16 * m + g);
            const float2 w = unpack_f2(weights_of(P, acc[m][k], acc[m][2 + k], f, x.y, x.z, back));
            if ((unsigned)back < reach) sum[m][0] += w.x;
            if ((unsigned)(back - 8) < reach) sum[m][1] += w.y;
          }
        }
      }
    }
#pragma unroll
    for (int m = 0; m < MT; ++m) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        sum[m][h] += __shfl_xor_sync(0xffffffffu, sum[m][h], 1);
        sum[m][h] += __shfl_xor_sync(0xffffffffu, sum[m][h], 2);
      }
      if (S > 1 && cc < 2) joined[(warp * MT + m) * 16 + g + 8 * cc] = cc == 0 ? sum[m][0] : sum[m][1];
    }
    if (S > 1) cluster_barrier();
    if (rank == 0) {
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        const int j = j0 + 16 * m + g + 8 * cc;
        if (cc < 2 && place[m] >= 0 && j < r.len) {
          float *at = P.weights + place[m] + g + 8 * cc, add = cc == 0 ? sum[m][0] : sum[m][1];
          for (int k = 1; k < S; ++k) add += __uint_as_float(peer_u32(&joined[(warp * MT + m) * 16 + g + 8 * cc], k));
          *at = j < new_from ? *at + add : add;
        }
      }
    }
    if (S > 1) cluster_barrier();      // sums have been read
  }
}

// ------------------------------------------------------------------ host side
templora_status_t check_weigh(const templora_attn_t *a, const templora_kv_cache_t *c, int n_rows, bool pointers) {
  TL_TRY(attn_check_desc(a));
  TL_TRY(check_cache(c, pointers));
  if (n_rows <= 0 || a->n_kv_heads != c->n_kv_heads || a->head_dim != c->head_dim) return TEMPLORA_ERR_INVALID_ARG;
  if (a->n_docs != 0 || a->prefix_lens || n_rows > (1 << 30)) return TEMPLORA_ERR_UNSUPPORTED;
  return TEMPLORA_OK;
}

template <int DM, bool F32, int MT>
templora_status_t launch_rows(const WeighParams &p, int sms, cudaStream_t st) {
  constexpr size_t stage = (size_t)kWeighWarps * kTerms<F32> * (DM / 16) * 32 * sizeof(uint2) + kStageColumns * sizeof(float4) +
                           16 * MT * kWeighWarps * sizeof(float);
  constexpr int tile = 16 * MT * kWeighWarps;
  TL_TRY((allow_smem<weigh_rows_kernel<DM, F32, MT>>(stage + (kMaxSeqs + 1) * sizeof(long long))));
  const long long most = (long long)p.c.n_seqs * p.c.Hkv * (((long long)p.c.max_blocks * p.c.bt + tile - 1) / tile + 1);
  const int S = MT > 1 ? 1 : weigh_cluster(p, tile, ((long long)p.n_rows * p.group / p.c.n_seqs + kStageColumns - 1) / kStageColumns, sms);
  LaunchScope scope(kKindKvCache, st);
  TL_CUDA_CHECK(launch_cluster_pdl(weigh_rows_kernel<DM, F32, MT>, dim3((int)std::min<long long>(most, 2ll * sms / S) * S), dim3(kWeighThreads), S,
                                   stage + (size_t)(p.c.n_seqs + 1) * sizeof(long long), st, p));
  return TEMPLORA_OK;
}
template <int DM, bool F32, int NC>
templora_status_t launch_step(const WeighParams &p, int sms, cudaStream_t st) {
  constexpr size_t rings = (size_t)kWeighWarps * kRing * kSlotBytes<DM>;
  const size_t counts = std::max<size_t>((size_t)(p.c.n_seqs + 1), kWeighWarps * 33) * sizeof(long long);
  TL_TRY((allow_smem<weigh_step_kernel<DM, F32, NC>>(rings + (kMaxSeqs + 1) * sizeof(long long))));
  const long long tiles = (long long)p.c.n_seqs * p.c.Hkv * (((long long)p.c.max_blocks * p.c.bt + 15) / 16);
  const int ctas = (int)std::min<long long>((tiles + kWeighWarps - 1) / kWeighWarps, (F32 || NC > 1 ? 2ll : 3ll) * sms);
  LaunchScope scope(kKindKvCache, st);
  TL_CUDA_CHECK(launch_pdl(weigh_step_kernel<DM, F32, NC>, dim3(ctas), dim3(kWeighThreads), rings + counts, st, p));
  return TEMPLORA_OK;
}
template <int DM, bool F32>
templora_status_t launch_weigh(const WeighParams &p, cudaStream_t st) {
  int sms = 0;
  TL_TRY(stream_sms(st, &sms));
  // the columns of one row of up to 8 heads, in bf16 16, stay in registers
  if (!p.offsets && p.group <= 8) return launch_step<DM, F32, 1>(p, sms, st);
  if constexpr (!F32) {
    if (!p.offsets && p.group <= 16) return launch_step<DM, F32, 2>(p, sms, st);
  }
  const long long places = (long long)p.c.max_blocks * p.c.bt, pairs = (long long)p.c.n_seqs * p.c.Hkv;
  // 256 places a CTA, or 128 where that many would leave SMs idle (61 rows of three sequences of 1501 tokens, 16 / 4 heads, fp32, by this
  // kernel: 17.4 and 13.3 us)
  if (pairs * (places / 256 + 1) < sms) return launch_rows<DM, F32, 1>(p, sms, st);
  return launch_rows<DM, F32, 2>(p, sms, st);
}

}  // namespace
}  // namespace templora

using namespace templora;

extern "C" {

size_t templora_kv_cache_weigh_workspace_bytes(const templora_attn_t *attn, const templora_kv_cache_t *cache, int32_t n_rows) {
  if (check_weigh(attn, cache, n_rows, false) != TEMPLORA_OK) return 0;
  return kStatusBytes + (attn->dtype == TEMPLORA_F32 ? weigh_tc_terms(attn->n_heads, attn->head_dim, n_rows, cache->n_seqs, attn->n_heads / attn->n_kv_heads) : 0);
}

templora_status_t templora_kv_cache_weigh(const templora_attn_t *attn, const templora_kv_cache_t *cache, const int32_t *seq_lens,
                                          const int32_t *row_offsets, int32_t n_rows, const void *q, int64_t ld_q,
                                          const float *lse, int64_t lse_row, int64_t lse_head, float *weights, void *ws,
                                          size_t ws_bytes, void *stream) {
  TL_TRY(check_weigh(attn, cache, n_rows, true));
  if (!seq_lens || !q || !lse || !weights || !aligned16(q) || lse_row < 0 || lse_head < 0) return TEMPLORA_ERR_INVALID_ARG;
  if (!word_aligned(seq_lens) || !word_aligned(row_offsets) || !word_aligned(lse) || !word_aligned(weights)) return TEMPLORA_ERR_INVALID_ARG;
  if (!row_offsets && n_rows != cache->n_seqs) return TEMPLORA_ERR_INVALID_ARG;
  const long long lq = row_stride(ld_q, (long long)attn->n_heads * attn->head_dim);
  if (lq < 0) return TEMPLORA_ERR_INVALID_ARG;
  TL_TRY(check_workspace(ws, ws_bytes, kStatusBytes));
  const bool f32 = attn->dtype == TEMPLORA_F32;
  WeighParams p{};
  p.c = view(cache, seq_lens, ws);
  p.q = q; p.lse = lse; p.slopes = attn->slopes; p.weights = weights; p.offsets = row_offsets;
  p.ldq = lq; p.lse_row = lse_row; p.lse_head = lse_head;
  p.n_rows = n_rows; p.group = attn->n_heads / attn->n_kv_heads; p.window = attn->window;
  p.scale = attn->scale;
  p.softcap = attn->softcap >= kNoCap ? 0.f : attn->softcap;
  p.cap_in = p.softcap > 0.f ? fminf(1.f / p.softcap, 3e38f) : 0.f;      // finite for the smallest caps too
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  if (weigh_tc_available(p, attn->dtype)) {
    if (f32) TL_TRY(check_workspace(ws, ws_bytes, kStatusBytes + weigh_tc_terms(attn->n_heads, attn->head_dim, n_rows, cache->n_seqs, p.group)));
    return weigh_tc(p, attn->dtype, reinterpret_cast<uint8_t *>(ws) + kStatusBytes, st);
  }
  if (f32) return attn->head_dim <= 64 ? launch_weigh<64, true>(p, st) : launch_weigh<128, true>(p, st);
  return attn->head_dim <= 64 ? launch_weigh<64, false>(p, st) : launch_weigh<128, false>(p, st);
}

}  // extern "C"
