// Cutting sequences of the 8-bit key/value cache down to a number of tokens: the choice of the tokens by their weights, and their
// way into other blocks.
#include "cluster.cuh"
#include "kv_cache.cuh"
#include "tc_host.h"

#include <algorithm>

namespace templora {
namespace {

using u64 = unsigned long long;

struct EvictParams {
  CacheView from, to;                 // to.seq_lens is not used
  const float *weights;
  float *to_weights;
  int *new_lens;
  int keep, first, recent;
  int *list, *counts;                 // [pair][keep] places of the kept tokens, [pair] how many; pair = sequence * Hkv + head
  int cap;                            // places whose keys fit a CTA's shared memory
};

// ------------------------------------------------------------------ the choice
// One cluster per (sequence, kv head) finds the weight of the last token that is kept by counting the tokens' order keys by
// digits of 11, 11 and 10 bits, the highest first, then writes down the kept places in order: of those of that very weight, the first.
// The CTAs share the places evenly and keep their keys in shared memory where they fit.  The cluster's counts are looked through by one
// warp, first those of groups of 32 bins: when every CTA read all of the others' counts, that took 37000 cycles a digit on eight CTAs.
// A bin that is kept whole ends the search.  Few places are compared one with another instead.
// Bound by the latency of its steps (length, table, weights, three counts, a scan), not by the 4 bytes per place.
constexpr int kSelThreads = 512, kSelWarps = kSelThreads / 32, kBins = 2048, kGroups = kBins / 32;
constexpr int kFewPlaces = 256;       // compared one with another

// A sequence that cannot be moved whole is not moved at all.  A barrier.
template <int TH> __device__ __forceinline__ bool cannot_move(const EvictParams &P, int n, const int *table, const int *to_table) {
  const CacheView &c = P.from;
  bool bad = n < 0 || n > (long long)c.max_blocks * c.bt;
  if (bad) {
    if (threadIdx.x == 0) report(c.status, kWhereLength);
  } else {
    const int from = (n + c.bt - 1) >> c.bt_log2, to = (min(n, P.keep) + c.bt - 1) >> c.bt_log2;
#pragma unroll 4
    for (int b = threadIdx.x; b < from; b += TH) bad |= (unsigned)table[b] >= (unsigned)c.n_blocks;
    for (int b = threadIdx.x; b < to; b += TH) bad |= (unsigned)to_table[b] >= (unsigned)P.to.n_blocks;
    if (bad) report(c.status, kWhereTable);
  }
  return __syncthreads_or(bad);
}
// Of up to kFewPlaces keys, a thread one, the m largest, of equal ones the first: how many kept ones stand before the thread's, or
// -1 if its own is not kept.  all: kFewPlaces words; part: one per 32 of them.
__device__ __forceinline__ int choose_few(uint32_t *all, uint32_t *part, uint32_t k, int places, int m) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid < kFewPlaces) all[tid] = k;
  __syncthreads();
  int before = 0;                     // keys that come before this one
  if (tid < places)
    for (int i = 0; i < places; i += 4) {
      const uint4 x = *reinterpret_cast<const uint4 *>(all + i);      // behind the last: 0
      const auto ahead = [&](uint32_t other, int at) { before += other >= (at < tid ? k : k + 1); };
      ahead(x.x, i);
      ahead(x.y, i + 1);
      ahead(x.z, i + 2);
      ahead(x.w, i + 3);
    }
  const unsigned kept = __ballot_sync(0xffffffffu, tid < places && before < m);
  if (lane == 0 && warp < kFewPlaces / 32) part[warp] = __popc(kept);
  __syncthreads();
  int at = __popc(kept & ((1u << lane) - 1));
  for (int w = 0; w < warp && w < kFewPlaces / 32; ++w) at += part[w];
  return (kept >> lane) & 1 ? at : -1;
}

__global__ void __launch_bounds__(kSelThreads, 2) evict_select_kernel(const EvictParams P) {
  pdl_prologue();
  extern __shared__ __align__(16) uint32_t keys[];
  __shared__ __align__(16) uint32_t hist[2][kBins];
  __shared__ __align__(8) uint32_t group[2][kGroups];
  __shared__ uint32_t part[kSelWarps], more[kSelWarps], found[4];
  __shared__ __align__(8) uint32_t mine[2];
  const CacheView &c = P.from;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int C = (int)cluster_size(), rank = (int)cluster_ctarank();
  const auto barrier = [&] { if (C == 1) __syncthreads(); else cluster_barrier(); };
  const auto peer = [&](const uint32_t *p, int r) { return C == 1 ? *p : peer_u32(p, r); };
  const auto peer2 = [&](const uint32_t *p, int r) { return C == 1 ? *reinterpret_cast<const u64 *>(p) : peer_u64(p, r); };
  const int pair = blockIdx.x / C, seq = pair / c.Hkv, hk = pair - seq * c.Hkv;
  const int n = c.seq_lens[seq];
  const int *table = c.table + (long long)seq * c.max_blocks, *to_table = P.to.table + (long long)seq * P.to.max_blocks;
  for (int b = tid; b < 2 * kBins; b += kSelThreads) (&hist[0][0])[b] = 0;

  const bool bad = cannot_move<kSelThreads>(P, n, table, to_table);
  const int count = bad ? 0 : min(n, P.keep);
  int *list = P.list + (long long)pair * P.keep;
  if (rank == 0 && tid == 0) P.counts[pair] = count;
  if (bad || n <= P.keep) {
    for (int i = rank * kSelThreads + tid; i < count; i += C * kSelThreads) list[i] = i;
    return;
  }
  const int m = P.keep - P.first - P.recent, places = n - P.first - P.recent;      // m < places
  const int slice = (places + C - 1) / C, lo = min(rank * slice, places), own = min(lo + slice, places) - lo;
  const bool held = slice <= P.cap && m > 0;
  const auto load = [&](int i) {
    const int j = P.first + lo + i;
    return P.weights[((long long)table[j >> c.bt_log2] * c.Hkv + hk) * c.bt + (j & (c.bt - 1))];
  };
  const bool few = C == 1 && places <= kFewPlaces;
  if (held && !few) {
    constexpr int U = 8;              // on their way at once
    for (int i0 = tid; i0 < own; i0 += U * kSelThreads) {
      float w[U];
#pragma unroll
      for (int e = 0; e < U; ++e) w[e] = i0 + e * kSelThreads < own ? load(i0 + e * kSelThreads) : 0.f;
#pragma unroll
      for (int e = 0; e < U; ++e) {
        if (i0 + e * kSelThreads >= own) break;
        const uint32_t k = order_key(w[e]);
        keys[i0 + e * kSelThreads] = k;
        atomicAdd(&hist[0][k >> 21], 1u);
      }
    }
  }
  for (int i = rank * kSelThreads + tid; i < P.first; i += C * kSelThreads) list[i] = i;
  for (int i = rank * kSelThreads + tid; i < P.recent; i += C * kSelThreads) list[P.keep - P.recent + i] = n - P.recent + i;
  if (m == 0) return;

  if (few) {
    const int at = choose_few(hist[0], part, tid < places ? order_key(load(tid)) : 0, places, m);
    if (at >= 0) list[P.first + at] = P.first + tid;
    return;
  }

  // visit(i, key) for i = from, from + by, ... < to, four keys on their way at once
  const auto over = [&](int from, int to, int by, auto visit) {
    if (held) {
#pragma unroll 4
      for (int i = from; i < to; i += by) visit(i, keys[i]);
    } else {
#pragma unroll 4
      for (int i = from; i < to; i += by) visit(i, order_key(load(i)));
    }
  };
  uint32_t prefix = 0, left = m;      // `left` tokens are still to be found among the keys that begin with `prefix`
#pragma unroll
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
    uint32_t *h = hist[pass & 1], *sums = group[pass & 1];
    if (pass > 0 || !held)
      over(tid, own, kSelThreads, [&](int, uint32_t k) {
        if (pass == 0 || k >> (shift + bits) == prefix) atomicAdd(&h[(k >> shift) & ((1u << bits) - 1)], 1u);
      });
    __syncthreads();
    for (int b = tid; b < kBins; b += kSelThreads) {
      const uint32_t v = __reduce_add_sync(0xffffffffu, h[b]);
      if (lane == 0) sums[b >> 5] = v;
    }
    barrier();
    if (pass == 1)                    // everyone has read the first counts
      for (int b = tid; b < kBins; b += kSelThreads) hist[0][b] = 0;
    if (warp == 0) {                  // from the highest key down
      uint32_t v0 = 0, v1 = 0;
#pragma unroll
      for (int r = 0; r < kMaxCluster; ++r) {
        const u64 two = r < C ? peer2(&sums[kGroups - 2 - 2 * lane], r) : 0;
        v0 += (uint32_t)(two >> 32);
        v1 += (uint32_t)two;
      }
      uint32_t upto = v0 + v1;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t u = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += u;
      }
      const int l = __ffs(__ballot_sync(0xffffffffu, upto >= left)) - 1;
      const uint32_t first_of = __shfl_sync(0xffffffffu, v0, l);
      uint32_t above = __shfl_sync(0xffffffffu, upto - v0 - v1, l);
      int grp = kGroups - 1 - 2 * l;
      if (above + first_of < left) { above += first_of; --grp; }
      uint32_t v = 0;
#pragma unroll
      for (int r = 0; r < kMaxCluster; ++r) v += r < C ? peer(&h[grp * 32 + 31 - lane], r) : 0;
      upto = v;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t u = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += u;
      }
      const int at = __ffs(__ballot_sync(0xffffffffu, above + upto >= left)) - 1;
      if (lane == at) {
        found[0] = grp * 32 + 31 - lane;
        found[1] = above + upto - v;
        found[2] = v;
      }
    }
    __syncthreads();
    prefix = prefix << bits | found[0];
    left -= found[1];
    if (pass < 2 && found[2] == left) {      // the bin is kept whole; it is not the last, since not all places are kept
      prefix = (prefix << shift) - 1;
      left = 0;
      break;
    }
  }

  // kept: every key above `prefix`, and the first `left` equal to it.  Each warp takes a stretch of the slice.
  const int stretch = ((own + kSelWarps - 1) / kSelWarps + 31) & ~31;
  const int i0 = min(warp * stretch, own), i1 = min(i0 + stretch, own);
  uint32_t gt = 0, eq = 0;
  over(i0 + lane, i1, 32, [&](int, uint32_t k) {
    gt += k > prefix;
    eq += k == prefix;
  });
  gt = __reduce_add_sync(0xffffffffu, gt);
  eq = __reduce_add_sync(0xffffffffu, eq);
  if (lane == 0) { part[warp] = gt; more[warp] = eq; }
  __syncthreads();
  if (warp == 0) {
    const uint32_t x = __reduce_add_sync(0xffffffffu, lane < kSelWarps ? part[lane] : 0), y = __reduce_add_sync(0xffffffffu, lane < kSelWarps ? more[lane] : 0);
    if (lane == 0) { mine[0] = x; mine[1] = y; }
  }
  if (C > 1) {
    cluster_barrier();
    if (warp == 0) {                  // of the CTAs before this one
      const u64 x = lane < rank ? peer_u64(mine, lane) : 0;
      const uint32_t g = __reduce_add_sync(0xffffffffu, (uint32_t)x), e = __reduce_add_sync(0xffffffffu, (uint32_t)(x >> 32));
      if (lane == 0) { found[2] = g; found[3] = e; }
    }
    __syncthreads();
  }
  gt = C > 1 ? found[2] : 0;
  eq = C > 1 ? found[3] : 0;
  for (int w = 0; w < warp; ++w) { gt += part[w]; eq += more[w]; }
  // keys 32 at a time; the last places of a stretch are visited alone
  const auto write = [&](int i, uint32_t k, bool in) {
    const unsigned above = __ballot_sync(0xffffffffu, in && k > prefix), same = __ballot_sync(0xffffffffu, in && k == prefix);
    const unsigned before = (1u << lane) - 1;
    const uint32_t rank_eq = eq + __popc(same & before);
    if (((above >> lane) & 1) || (((same >> lane) & 1) && rank_eq < left))
      list[P.first + gt + __popc(above & before) + min(rank_eq, left)] = P.first + lo + i;
    gt += __popc(above);
    eq += __popc(same);
  };
  const int whole = i0 + ((i1 - i0) & ~31);
  over(i0 + lane, whole, 32, [&](int i, uint32_t k) { write(i, k, true); });
  if (whole < i1) {
    const bool in = whole + lane < i1;
    write(whole + lane, !in ? 0 : held ? keys[whole + lane] : order_key(load(whole + lane)), in);
  }
  if (C > 1) cluster_barrier();       // the others may still read this CTA's counts
}

// ------------------------------------------------------------------ the way
// A CTA moves up to 128 tokens of one kv head: it looks up where they all stand, a thread a token, then block by block, as many at once
// as four vectors of 16 codes per thread hold, reads their codes into registers, finds the scales that the blocks need, and writes
// them; codes whose scale stays are copied as they are.
// Bound by HBM: head_dim bytes of keys and of values read and written per token, by one chain of dependent reads (count, place, table,
// codes) for 128 tokens instead of one for each block.  16 sequences of 2112 tokens cut to 2048, 8 heads of 128: 37 us with the choice, which
// takes 7 of them, replayed from a graph; 134 MB then move at 4.5 TB/s.  In calls over changing inputs 40 us.  (256 tokens a CTA: 3 us more.)
constexpr int kMoveThreads = 256, kMoveVecs = 4, kMoveTokens = 128;

// The largest magnitude among 16 codes, as the bits of an fp16 number, in which every code is exact; NaN does not count, unless
// all are.
__device__ __forceinline__ uint32_t largest_code(const uint4 &v) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  __half2 top;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t a, b;
    half2s_of_codes(w[i], a, b);
    const __half2 m = __hmax2(__habs2(*reinterpret_cast<const __half2 *>(&a)), __habs2(*reinterpret_cast<const __half2 *>(&b)));
    top = i == 0 ? m : __hmax2(top, m);
  }
  return __half_as_ushort(__hmax(__low2half(top), __high2half(top)));
}
__device__ __forceinline__ bool power_of_two(uint32_t bits) { return (bits & 0x807fffffu) == 0 && bits - 1 < 0x7f7fffffu; }   // a positive normal number's
// exponent of the scale that a code (as fp16 bits, NaN for none) times the number with the bits `scale` needs
__device__ __forceinline__ int exponent_needed(uint32_t code, uint32_t scale) {
  if (code == 0 || code > 0x7c00u) return -126;
  if (power_of_two(scale)) return (int)(code >> 10) - 15 + (int)(scale >> 23) - 127 - 8 + ((code & 0x3ffu) > 0x300u);
  if (!(fabsf(__uint_as_float(scale)) < INFINITY)) return -126;      // its values are NaN
  // in fp64, where the product is exact and, of a huge scale, finite
  const double v = fabs((double)__half2float(__ushort_as_half((unsigned short)code)) * (double)__uint_as_float(scale));
  const long long bits = __double_as_longlong(v);
  return (int)(bits >> 52) - 1023 - 8 + ((bits & 0xfffffffffffffll) > 0xc000000000000ll);
}
// Codes of a scale with the bits `from` as codes of 2^e.  A power of two times a code is exact in fp16 wherever it is not below half
// of e4m3's smallest value.
__device__ __forceinline__ uint4 recode(const uint4 &v, uint32_t from, int e) {
  if (from == (uint32_t)(e + 127) << 23) return v;
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  uint32_t out[4];
  if (power_of_two(from)) {
    // only zeros and NaN could be raised further than 2^18, which two factors hold
    const int by = min((int)(from >> 23) - 127 - e, 30), high = max(by - 15, 0), low = by - high;
    const __half up = __ushort_as_half((unsigned short)(low < -24 ? 0 : low < -14 ? 1 << (low + 24) : (low + 15) << 10));
    const __half2 f = __halves2half2(up, up), f2 = __float2half2_rn((float)(1 << high));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t a, b;
      half2s_of_codes(w[i], a, b);
      __half2 x = __hmul2(*reinterpret_cast<const __half2 *>(&a), f), y = __hmul2(*reinterpret_cast<const __half2 *>(&b), f);
      if (high > 0) { x = __hmul2(x, f2); y = __hmul2(y, f2); }
      asm("{\n.reg .b16 l, h;\ncvt.rn.satfinite.e4m3x2.f16x2 l, %1;\ncvt.rn.satfinite.e4m3x2.f16x2 h, %2;\nmov.b32 %0, {l, h};\n}"
          : "=r"(out[i]) : "r"(*reinterpret_cast<const uint32_t *>(&x)), "r"(*reinterpret_cast<const uint32_t *>(&y)));
    }
    return make_uint4(out[0], out[1], out[2], out[3]);
  }
  // Any other scale, as of a cache that another program has filled: the product has up to 28 bits and is rounded once, since it is cut off
  // and its last bit set where something was cut off, which the codes' 4 bits then round as they would the whole.
  const float scale = __uint_as_float(from);
  float by = scale / pow2f(e);        // exact, or of less than half of e4m3's smallest value
  if (!(fabsf(scale) < INFINITY)) by = __uint_as_float(0x7fffffffu);
  else if (fabsf(by) > 1048576.f) by = copysignf(1048576.f, by);      // as above: zeros stay zeros
  float f[16];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float2 t = values_of_codes((w[i >> 1] >> (16 * (i & 1))) & 0xffffu);
    const auto product = [&](float x) {
      const float y = __fmul_rz(x, by);
      return fmaf(x, by, -y) != 0.f ? __uint_as_float(__float_as_uint(y) | 1u) : y;
    };
    f[2 * i] = product(t.x); f[2 * i + 1] = product(t.y);
  }
  return encode16(f, 1.f);
}

struct MoveShared {
  long long row_of[kMoveTokens];
  uint32_t scale_of[2][kMoveTokens];
  long long plane_of[kMoveTokens / 16];
  int top[2][kMoveTokens / 16];       // exponents of the blocks' scales
};
// Tokens t0 .. t0 + live of those that are kept; list: where these stand.
__device__ __forceinline__ void move_tokens(const EvictParams &P, MoveShared &sh, int seq, int hk, int t0, int live, const int *list) {
  auto &row_of = sh.row_of;
  auto &scale_of = sh.scale_of;
  auto &plane_of = sh.plane_of;
  auto &top = sh.top;
  const CacheView &c = P.from;
  const int tid = threadIdx.x;
  if (tid < live) {
    const int j = list[tid];
    const long long to = (long long)P.to.table[(long long)seq * P.to.max_blocks + ((t0 + tid) >> c.bt_log2)] * c.Hkv + hk;
    const long long from = (long long)c.table[(long long)seq * c.max_blocks + (j >> c.bt_log2)] * c.Hkv + hk;
    const long long row = from * c.bt + (j & (c.bt - 1));
    row_of[tid] = row;
    scale_of[0][tid] = __float_as_uint(c.k_scale[from]);
    scale_of[1][tid] = __float_as_uint(c.v_scale[from]);
    if ((tid & (c.bt - 1)) == 0) plane_of[tid >> c.bt_log2] = to;
    P.to_weights[to * c.bt + (tid & (c.bt - 1))] = P.weights[row];
  }
  if (tid < 2 * (kMoveTokens / 16)) (&top[0][0])[tid] = -126;
  __syncthreads();
  const int vpr = c.D / 16;
  const unsigned per_row = (65535u + vpr) / vpr;      // v / vpr = v * per_row >> 16 for v < 1024
  const int vecs = live * vpr;        // at most kMoveThreads * kMoveVecs
  {
    uint4 x[2][kMoveVecs];
    int token[kMoveVecs], rest[kMoveVecs];
#pragma unroll
    for (int n = 0; n < kMoveVecs; ++n) {
      const int v = tid + n * kMoveThreads, t = (int)(v * per_row >> 16);
      token[n] = v < vecs ? t : -1;
      rest[n] = v - t * vpr;
      if (token[n] < 0) continue;
      const long long at = row_of[token[n]] * vpr + rest[n];
      x[0][n] = __ldcs(reinterpret_cast<const uint4 *>(c.k) + at);
      x[1][n] = __ldcs(reinterpret_cast<const uint4 *>(c.v) + at);
    }
#pragma unroll
    for (int n = 0; n < kMoveVecs; ++n) {
      const int blk = token[n] >= 0 ? token[n] >> c.bt_log2 : -1;
      const unsigned same = __match_any_sync(0xffffffffu, blk);      // a warp's vectors belong to one block, or two
#pragma unroll
      for (int kv = 0; kv < 2; ++kv) {
        const int e = __reduce_max_sync(same, blk >= 0 ? exponent_needed(largest_code(x[kv][n]), scale_of[kv][token[n]]) : -126);
        if ((tid & 31) == __ffs(same) - 1 && e > -126) atomicMax(&top[kv][blk], min(e, 127));
      }
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < kMoveVecs; ++n) {
      if (token[n] < 0) continue;
      const int t = token[n], blk = t >> c.bt_log2;
      const long long at = (plane_of[blk] * c.bt + (t & (c.bt - 1))) * vpr + rest[n];
#pragma unroll
      for (int kv = 0; kv < 2; ++kv) {
        const int e = top[kv][blk];
        reinterpret_cast<uint4 *>(kv ? P.to.v : P.to.k)[at] = recode(x[kv][n], scale_of[kv][t], e);
        if (rest[n] == 0 && (t & (c.bt - 1)) == 0) (kv ? P.to.v_scale : P.to.k_scale)[plane_of[blk]] = pow2f(e);
      }
    }
  }
}

__global__ void __launch_bounds__(kMoveThreads, 4) evict_move_kernel(const EvictParams P) {
  pdl_prologue();
  __shared__ MoveShared sh;
  const int hk = blockIdx.y, seq = blockIdx.z, pair = seq * P.from.Hkv + hk, t0 = blockIdx.x * kMoveTokens;
  const int count = P.counts[pair];
  if (blockIdx.x == 0 && hk == 0 && threadIdx.x == 0) P.new_lens[seq] = count;
  const int live = min(kMoveTokens, count - t0);
  if (live > 0) move_tokens(P, sh, seq, hk, t0, live, P.list + (long long)pair * P.keep + t0);
}

// Choice and way of one (sequence, kv head) by one CTA, where a sequence has few places and few are kept: one launch.
__global__ void __launch_bounds__(kMoveThreads, 3) evict_few_kernel(const EvictParams P) {
  static_assert(kMoveThreads >= kFewPlaces, "a thread a place");
  pdl_prologue();
  __shared__ MoveShared sh;
  __shared__ __align__(16) uint32_t all[kFewPlaces];
  __shared__ uint32_t part[kFewPlaces / 32];
  __shared__ int list[kFewPlaces];
  const CacheView &c = P.from;
  const int tid = threadIdx.x, pair = blockIdx.x, seq = pair / c.Hkv, hk = pair - seq * c.Hkv;
  const int n = c.seq_lens[seq];
  const int *table = c.table + (long long)seq * c.max_blocks;
  const bool bad = cannot_move<kMoveThreads>(P, n, table, P.to.table + (long long)seq * P.to.max_blocks);
  const int count = bad ? 0 : min(n, P.keep);
  if (hk == 0 && tid == 0) P.new_lens[seq] = count;
  if (bad || n <= P.keep) {
    if (tid < count) list[tid] = tid;
  } else {
    const int m = P.keep - P.first - P.recent, places = n - P.first - P.recent, j = P.first + tid;
    const uint32_t k = tid < places ? order_key(P.weights[((long long)table[j >> c.bt_log2] * c.Hkv + hk) * c.bt + (j & (c.bt - 1))]) : 0;
    const int at = choose_few(all, part, k, places, m);
    if (at >= 0) list[P.first + at] = j;
    if (tid < P.first) list[tid] = tid;
    if (tid < P.recent) list[P.keep - P.recent + tid] = n - P.recent + tid;
  }
  __syncthreads();
  if (tid < count) P.list[(long long)pair * P.keep + tid] = list[tid];
  for (int t0 = 0; t0 < count; t0 += kMoveTokens) {
    if (t0 > 0) __syncthreads();      // the tokens before have been moved
    move_tokens(P, sh, seq, hk, t0, min(kMoveTokens, count - t0), list + t0);
  }
}

// ------------------------------------------------------------------ host side
constexpr int kMostCap = 24576;      // keys: 96 KB, two CTAs per SM

struct Scratch { size_t counts, list, bytes; };
Scratch scratch(const templora_kv_cache_t *c, int keep) {
  const size_t pairs = (size_t)c->n_seqs * c->n_kv_heads;
  Scratch s;
  s.counts = kStatusBytes;
  s.list = s.counts + align_up(pairs * sizeof(int), 256);
  s.bytes = s.list + align_up(pairs * (size_t)keep * sizeof(int), kWsAlign);
  return s;
}

}  // namespace
}  // namespace templora

using namespace templora;

extern "C" {

size_t templora_kv_cache_evict_workspace_bytes(const templora_kv_cache_t *cache, int32_t n_keep) {
  return check_cache(cache, false) == TEMPLORA_OK && n_keep > 0 ? scratch(cache, n_keep).bytes : 0;
}

templora_status_t templora_kv_cache_evict(const templora_kv_cache_t *cache, const float *weights, const int32_t *seq_lens,
                                          const templora_kv_cache_t *to, float *to_weights, int32_t *new_lens, int32_t n_keep,
                                          int32_t n_first, int32_t n_recent, int32_t *kept, void *ws, size_t ws_bytes, void *stream) {
  TL_TRY(check_cache(cache, true));
  TL_TRY(check_cache(to, true));
  if (!weights || !seq_lens || !to_weights || !new_lens) return TEMPLORA_ERR_INVALID_ARG;
  if (!word_aligned(weights) || !word_aligned(seq_lens) || !word_aligned(to_weights) || !word_aligned(new_lens) || !word_aligned(kept))
    return TEMPLORA_ERR_INVALID_ARG;
  if (to->n_kv_heads != cache->n_kv_heads || to->head_dim != cache->head_dim || to->block_tokens != cache->block_tokens ||
      to->n_seqs != cache->n_seqs)
    return TEMPLORA_ERR_INVALID_ARG;
  if (n_keep < 1 || n_first < 0 || n_recent < 0 || (long long)n_first + n_recent > n_keep ||
      n_keep > (long long)to->max_blocks * to->block_tokens)
    return TEMPLORA_ERR_INVALID_ARG;
  if (to->k == cache->k && to->block_table == cache->block_table) return TEMPLORA_ERR_INVALID_ARG;      // what is read would be written
  const Scratch s = scratch(cache, n_keep);
  TL_TRY(check_workspace(ws, ws_bytes, s.bytes));
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  int sms = 0;
  TL_TRY(stream_sms(st, &sms));
  EvictParams p{};
  p.from = view(cache, seq_lens, ws);
  p.to = view(to, nullptr, ws);
  p.weights = weights; p.to_weights = to_weights; p.new_lens = new_lens;
  p.keep = n_keep; p.first = n_first; p.recent = n_recent;
  p.counts = reinterpret_cast<int *>(reinterpret_cast<uint8_t *>(ws) + s.counts);
  p.list = kept ? kept : reinterpret_cast<int *>(reinterpret_cast<uint8_t *>(ws) + s.list);
  // few places and few kept: one launch (2 heads, 90 tokens cut to 48: 4.7 us, 7.0 by two), unless the new lengths take the place of the
  // old, which its other CTAs may not have read yet
  const uintptr_t old_at = reinterpret_cast<uintptr_t>(seq_lens), new_at = reinterpret_cast<uintptr_t>(new_lens), size = (uintptr_t)cache->n_seqs * sizeof(int);
  const bool lens_apart = new_at + size <= old_at || old_at + size <= new_at;
  if (lens_apart && (long long)cache->max_blocks * cache->block_tokens - n_first - n_recent <= kFewPlaces && n_keep <= kFewPlaces) {
    LaunchScope scope(kKindKvCache, st);
    TL_CUDA_CHECK(launch_pdl(evict_few_kernel, dim3((unsigned)((long long)cache->n_seqs * cache->n_kv_heads)), dim3(kMoveThreads), 0, st, p));
    return TEMPLORA_OK;
  }
  // as few CTAs to a pair as keep its places; more while a wave holds them all and each has some thousand places (3 sequences of 13249
  // tokens, 2 heads: 20.2 us with 8192 a CTA, 18.1 with 4096, 16.2 with 2048, 15.7 with 1024; 2312 tokens, 2 heads: 11.6 with 2048, 12.9 with less)
  const long long pairs = (long long)cache->n_seqs * cache->n_kv_heads, places = (long long)cache->max_blocks * cache->block_tokens;
  int C = 1;
  while (C < kMaxCluster && (places > (long long)C * kMostCap || (pairs * C * 2 <= 9ll * sms / 5 && places / (2 * C) >= 2048))) C *= 2;
  p.cap = (int)std::min<long long>((places + C - 1) / C, kMostCap);
  TL_TRY((allow_smem<evict_select_kernel>((size_t)kMostCap * sizeof(uint32_t))));
  {
    LaunchScope scope(kKindKvCache, st);
    TL_CUDA_CHECK(launch_cluster_pdl(evict_select_kernel, dim3((unsigned)(pairs * C)), dim3(kSelThreads), C,
                                     (size_t)p.cap * sizeof(uint32_t), st, p));
  }
  LaunchScope scope(kKindKvCache, st);
  TL_CUDA_CHECK(launch_pdl(evict_move_kernel, dim3((n_keep + kMoveTokens - 1) / kMoveTokens, cache->n_kv_heads, cache->n_seqs), dim3(kMoveThreads),
                           0, st, p));
  return TEMPLORA_OK;
}

}  // extern "C"
