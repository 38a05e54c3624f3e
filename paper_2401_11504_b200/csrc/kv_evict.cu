// Cutting sequences of the 8-bit key/value cache down to a number of tokens: the choice of the tokens by their weights, and their
// way into other blocks.
#include "cluster.cuh"
#include "kv_cache.cuh"
#include "tc_host.h"

#include <algorithm>

namespace templora {
namespace {

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
// The CTAs share the places evenly, keep their keys in shared memory where they fit, and add up each other's counts.
// Bound by the latency of its steps (lengths, table, weights, three counts, a scan), not by the 4 bytes per place.
constexpr int kSelThreads = 512, kSelWarps = kSelThreads / 32, kBins = 2048;

__global__ void __launch_bounds__(kSelThreads) evict_select_kernel(const EvictParams P) {
  pdl_prologue();
  extern __shared__ __align__(16) uint32_t keys[];
  __shared__ uint32_t hist[2][kBins];
  __shared__ uint32_t part[kSelWarps], more[kSelWarps], found[2], mine[2];
  const CacheView &c = P.from;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int C = (int)cluster_size(), rank = (int)cluster_ctarank();
  const int pair = blockIdx.x / C, seq = pair / c.Hkv, hk = pair - seq * c.Hkv;
  const int n = c.seq_lens[seq];
  const int *table = c.table + (long long)seq * c.max_blocks, *to_table = P.to.table + (long long)seq * P.to.max_blocks;

  // a sequence that cannot be moved whole is not moved at all
  bool bad = n < 0 || n > (long long)c.max_blocks * c.bt;
  if (bad) {
    if (tid == 0) report(c.status, kWhereLength);
  } else {
    for (int b = tid; b < (n + c.bt - 1) >> c.bt_log2; b += kSelThreads) bad |= (unsigned)table[b] >= (unsigned)c.n_blocks;
    for (int b = tid; b < (min(n, P.keep) + c.bt - 1) >> c.bt_log2; b += kSelThreads) bad |= (unsigned)to_table[b] >= (unsigned)P.to.n_blocks;
    if (bad) report(c.status, kWhereTable);
  }
  bad = __syncthreads_or(bad);
  const int count = bad ? 0 : min(n, P.keep);
  int *list = P.list + (long long)pair * P.keep;
  if (rank == 0 && tid == 0) P.counts[pair] = count;
  if (bad || n <= P.keep) {
    for (int i = rank * kSelThreads + tid; i < count; i += C * kSelThreads) list[i] = i;
    return;
  }
  for (int i = rank * kSelThreads + tid; i < P.first; i += C * kSelThreads) list[i] = i;
  for (int i = rank * kSelThreads + tid; i < P.recent; i += C * kSelThreads) list[P.keep - P.recent + i] = n - P.recent + i;
  const int m = P.keep - P.first - P.recent, places = n - P.first - P.recent;      // m < places
  if (m == 0) return;

  const int slice = (places + C - 1) / C, lo = min(rank * slice, places), own = min(lo + slice, places) - lo;
  const bool held = slice <= P.cap;
  auto load = [&](int i) {
    const int j = P.first + lo + i;
    const long long at = ((long long)table[j >> c.bt_log2] * c.Hkv + hk) * c.bt + (j & (c.bt - 1));
    return order_key(P.weights[at]);
  };
  for (int b = tid; b < 2 * kBins; b += kSelThreads) (&hist[0][0])[b] = 0;
  if (held)
    for (int i = tid; i < own; i += kSelThreads) keys[i] = load(i);
  __syncthreads();

  uint32_t prefix = 0, left = m;      // `left` tokens are still to be found among the keys that begin with `prefix`
#pragma unroll
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
    uint32_t *h = hist[pass & 1];
    for (int i = tid; i < own; i += kSelThreads) {
      const uint32_t k = held ? keys[i] : load(i);
      if (pass == 0 || k >> (shift + bits) == prefix) atomicAdd(&h[(k >> shift) & ((1u << bits) - 1)], 1u);
    }
    cluster_barrier();
    if (pass == 1)                    // everyone has read the first counts
      for (int b = tid; b < kBins; b += kSelThreads) hist[0][b] = 0;
    // bins from the highest key down, four to a thread
    uint32_t bin[4] = {0, 0, 0, 0}, sum = 0;
    for (int r = 0; r < C; ++r)
#pragma unroll
      for (int e = 0; e < 4; ++e) bin[e] += peer_u32(&h[kBins - 1 - 4 * tid - e], r);
#pragma unroll
    for (int e = 0; e < 4; ++e) sum += bin[e];
    uint32_t upto = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t u = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += u;
    }
    if (lane == 31) part[warp] = upto;
    __syncthreads();
    uint32_t above = upto - sum;
    for (int w = 0; w < warp; ++w) above += part[w];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (above < left && left <= above + bin[e]) {
        found[0] = kBins - 1 - 4 * tid - e;
        found[1] = above;
      }
      above += bin[e];
    }
    __syncthreads();
    prefix = prefix << bits | found[0];
    left -= found[1];
    __syncthreads();                  // read before the next pass writes; cleared counts are visible
  }

  // kept: every key above `prefix`, and the first `left` equal to it.  Each warp takes a stretch of the slice.
  const int stretch = ((own + kSelWarps - 1) / kSelWarps + 31) & ~31;
  const int i0 = min(warp * stretch, own), i1 = min(i0 + stretch, own);
  uint32_t gt = 0, eq = 0;
  for (int i = i0 + lane; i < i1; i += 32) {
    const uint32_t k = held ? keys[i] : load(i);
    gt += k > prefix;
    eq += k == prefix;
  }
  gt = __reduce_add_sync(0xffffffffu, gt);
  eq = __reduce_add_sync(0xffffffffu, eq);
  if (lane == 0) { part[warp] = gt; more[warp] = eq; }
  __syncthreads();
  if (tid == 0) {
    mine[0] = mine[1] = 0;
    for (int w = 0; w < kSelWarps; ++w) { mine[0] += part[w]; mine[1] += more[w]; }
  }
  cluster_barrier();
  gt = eq = 0;
  for (int r = 0; r < rank; ++r) { gt += peer_u32(&mine[0], r); eq += peer_u32(&mine[1], r); }
  for (int w = 0; w < warp; ++w) { gt += part[w]; eq += more[w]; }
  for (int i = i0; i < i1; i += 32) {
    const bool in = i + lane < i1;
    const uint32_t k = !in ? 0 : held ? keys[i + lane] : load(i + lane);
    const unsigned above = __ballot_sync(0xffffffffu, in && k > prefix), same = __ballot_sync(0xffffffffu, in && k == prefix);
    const unsigned before = (1u << lane) - 1;
    const uint32_t rank_eq = eq + __popc(same & before);
    if (((above >> lane) & 1) || (((same >> lane) & 1) && rank_eq < left))
      list[P.first + gt + __popc(above & before) + min(rank_eq, left)] = P.first + lo + i + lane;
    gt += __popc(above);
    eq += __popc(same);
  }
  cluster_barrier();                 // the others may still read this CTA's counts
}

// ------------------------------------------------------------------ the way
// A CTA fills one block of one kv head: it looks up where its tokens stand, reads their codes into registers, finds the scales that
// they need, and writes them; codes whose scale stays are copied as they are.
// Bound by HBM: head_dim bytes of keys and of values read and written per token.
constexpr int kMoveThreads = 256;

// the largest magnitude among 16 codes, as a code; NaN does not count
__device__ __forceinline__ uint32_t largest_code(const uint4 &v) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t m = w[i] & 0x7f7f7f7fu;
    top = __vmaxu4(top, m & ~__vcmpeq4(m, 0x7f7f7f7fu));
  }
  top = __vmaxu4(top, top >> 16);
  return max(top & 0xffu, (top >> 8) & 0xffu);
}
// exponent of the scale that a code times `scale` needs: in fp64, where the product of a huge scale is finite
__device__ __forceinline__ int exponent_needed(uint32_t code, float scale) {
  const double v = fabs((double)values_of_codes(code).x * (double)scale);
  const long long bits = __double_as_longlong(v);
  const int e = (int)(bits >> 52) - 1023 - 8 + ((bits & 0xfffffffffffffll) > 0xc000000000000ll);
  return min(max(e, -126), 127);
}
__device__ __forceinline__ uint4 recode(const uint4 &v, float ratio) {
  if (ratio == 1.f) return v;
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  float f[16];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float2 t = values_of_codes((w[i >> 1] >> (16 * (i & 1))) & 0xffffu);
    f[2 * i] = t.x; f[2 * i + 1] = t.y;
  }
  return encode16(f, ratio);
}

template <int NV>
__global__ void __launch_bounds__(kMoveThreads) evict_move_kernel(const EvictParams P) {
  pdl_prologue();
  __shared__ long long row_of[128];
  __shared__ float scale_of[2][128];
  __shared__ int top[2][kMoveThreads / 32];
  const CacheView &c = P.from;
  const int tid = threadIdx.x, hk = blockIdx.y, seq = blockIdx.z, pair = seq * c.Hkv + hk, b0 = blockIdx.x * c.bt;
  const int count = P.counts[pair];
  if (blockIdx.x == 0 && hk == 0 && tid == 0) P.new_lens[seq] = count;
  if (b0 >= count) return;
  const int live = min(c.bt, count - b0);
  const long long plane = (long long)P.to.table[(long long)seq * P.to.max_blocks + blockIdx.x] * c.Hkv + hk;
  if (tid < live) {
    const int j = P.list[(long long)pair * P.keep + b0 + tid];
    const long long from = (long long)c.table[(long long)seq * c.max_blocks + (j >> c.bt_log2)] * c.Hkv + hk;
    const long long row = from * c.bt + (j & (c.bt - 1));
    row_of[tid] = row;
    scale_of[0][tid] = c.k_scale[from];
    scale_of[1][tid] = c.v_scale[from];
    P.to_weights[plane * c.bt + tid] = P.weights[row];
  }
  __syncthreads();
  const int vpr = c.D / 16, vecs = live * vpr;
  uint4 x[2][NV];
  int e[2] = {-126, -126};
#pragma unroll
  for (int n = 0; n < NV; ++n) {
    const int v = tid + n * kMoveThreads;
    if (v >= vecs) continue;
    const long long at = row_of[v / vpr] * vpr + v % vpr;
    x[0][n] = __ldcs(reinterpret_cast<const uint4 *>(c.k) + at);
    x[1][n] = __ldcs(reinterpret_cast<const uint4 *>(c.v) + at);
  }
#pragma unroll
  for (int n = 0; n < NV; ++n) {
    const int v = tid + n * kMoveThreads;
    if (v >= vecs) continue;
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      const uint32_t code = largest_code(x[kv][n]);
      if (code) e[kv] = max(e[kv], exponent_needed(code, scale_of[kv][v / vpr]));
    }
  }
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) {
    e[kv] = __reduce_max_sync(0xffffffffu, e[kv]);
    if ((tid & 31) == 0) top[kv][tid >> 5] = e[kv];
  }
  __syncthreads();
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) {
#pragma unroll
    for (int w = 0; w < kMoveThreads / 32; ++w) e[kv] = max(e[kv], top[kv][w]);
    const float unit = pow2f(e[kv]);
    uint8_t *codes = (kv ? P.to.v : P.to.k) + plane * c.bt * c.D;
    if (tid == 0) (kv ? P.to.v_scale : P.to.k_scale)[plane] = unit;
#pragma unroll
    for (int n = 0; n < NV; ++n) {
      const int v = tid + n * kMoveThreads;
      if (v >= vecs) continue;
      // only zeros and NaN could be raised further than 2^18; the bound keeps zeros zero
      const float ratio = fminf(scale_of[kv][v / vpr] / unit, 1048576.f);
      reinterpret_cast<uint4 *>(codes)[v] = recode(x[kv][n], ratio);
    }
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

template <int NV>
templora_status_t launch_move(const EvictParams &p, dim3 grid, cudaStream_t st) {
  LaunchScope scope(kKindKvCache, st);
  TL_CUDA_CHECK(launch_pdl(evict_move_kernel<NV>, grid, dim3(kMoveThreads), 0, st, p));
  return TEMPLORA_OK;
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
  // more CTAs to a pair while SMs are idle and each still has some thousand places
  const long long pairs = (long long)cache->n_seqs * cache->n_kv_heads, places = (long long)cache->max_blocks * cache->block_tokens;
  int C = 1;
  while (C < kMaxCluster && pairs * C * 2 <= 2ll * sms && places / C > 2048) C *= 2;
  p.cap = (int)std::min<long long>((places + C - 1) / C, kMostCap);
  TL_TRY((allow_smem<evict_select_kernel>((size_t)kMostCap * sizeof(uint32_t))));
  {
    LaunchScope scope(kKindKvCache, st);
    TL_CUDA_CHECK(launch_cluster_pdl(evict_select_kernel, dim3((unsigned)(pairs * C)), dim3(kSelThreads), C,
                                     (size_t)p.cap * sizeof(uint32_t), st, p));
  }
  const dim3 grid((n_keep + cache->block_tokens - 1) / cache->block_tokens, cache->n_kv_heads, cache->n_seqs);
  const int vecs = (cache->block_tokens * cache->head_dim / 16 + kMoveThreads - 1) / kMoveThreads;     // 1 to 4
  if (vecs == 1) return launch_move<1>(p, grid, st);
  if (vecs == 2) return launch_move<2>(p, grid, st);
  return launch_move<4>(p, grid, st);
}

}  // extern "C"
