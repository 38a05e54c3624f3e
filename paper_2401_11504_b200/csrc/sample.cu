// The choice of the next token: temperature, top-k, top-p, min-p, and the inverse of the running sum at a given random number.
#include "attention.cuh"
#include "cluster.cuh"
#include "tc_host.h"

#include <algorithm>

namespace templora {
namespace {

struct SampleParams {
  const void *logits;
  long long ld;
  int rows, vocab, slice;             // slice: tokens of a CTA
  const float *temperature, *top_p, *min_p, *u;
  const int *top_k;
  int *tokens;
  float *logprobs;
};

// A cluster of CTAs takes a row: each CTA keeps the order keys of a stretch of the vocabulary in shared memory.  Kept tokens are those
// whose key is above `cut`, and the first `ties` of those whose key is `cut`.  Neither filter sorts: the tokens are counted (top-k), or
// their weights added up (top-p), in bins of descending logits, then within the bin where the border falls, until that bin holds few
// tokens, which are compared one with another, or one value only.  All sums are integers, in units of 2^-44 of the largest weight.
constexpr int kSampleThreads = 512, kSampleWarps = kSampleThreads / 32;
constexpr int kSampleBins = 1024, kFew = 128;
constexpr int kMaxVocab = 1 << 18;    // sums stay below 2^62
constexpr int kMostSlice = 24576;
using u64 = unsigned long long;

struct Exchange { u64 a, b; };        // what CTAs tell each other
struct Shared {
  uint32_t count[kSampleBins], low[kSampleBins], high[kSampleBins];   // of a bin: tokens, and the sum of their weights
  Exchange ex[2];
  u64 part[2][kSampleWarps];
  uint32_t few[kFew], all[kFew], few_count;
  u64 all_w[kFew];
  u64 found[3];                       // bin or key, what is above it, tokens in it
  uint32_t bin_count;
};

struct Row {
  float top, lowest;                  // largest and smallest of the logits that count
  double top_d, inv_t;                // 1 / temperature
};
// w_i in units of 2^-44, rounded to the nearest
__device__ __forceinline__ u64 weight(const Row &r, uint32_t key) {
  const double d = ((double)key_value(key) - r.top_d) * r.inv_t;
  return d < -31.2 ? 0 : __double2ull_rn(exp(d) * 17592186044416.0);
}

__device__ __forceinline__ u64 warp_sum(u64 v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ u64 warp_upto(u64 v) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const u64 t = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += t;
  }
  return v;
}

template <typename T> __device__ __forceinline__ float logit(const T *p);
template <> __device__ __forceinline__ float logit<float>(const float *p) { return __ldcs(p); }
template <> __device__ __forceinline__ float logit<__nv_bfloat16>(const __nv_bfloat16 *p) {
  return __uint_as_float((uint32_t)__ldcs(reinterpret_cast<const unsigned short *>(p)) << 16);
}
// the keys of n logits, 16 bytes at a time where they lie on such a boundary
template <typename T> __device__ __forceinline__ void load_keys(const T *x, int n, uint32_t *keys) {
  constexpr int N = 16 / sizeof(T);
  const int head = min(n, (int)((16 - (reinterpret_cast<uintptr_t>(x) & 15)) & 15) / (int)sizeof(T));
  const int vecs = (n - head) / N, tail = head + vecs * N;
  for (int i = threadIdx.x; i < head; i += kSampleThreads) keys[i] = order_key(logit(x + i));
#pragma unroll 4
  for (int v = threadIdx.x; v < vecs; v += kSampleThreads) {
    const uint4 w = __ldcs(reinterpret_cast<const uint4 *>(x + head) + v);
    const uint32_t in[4] = {w.x, w.y, w.z, w.w};
    uint32_t *k = keys + head + v * N;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (sizeof(T) == 4) {
        k[e] = order_key(__uint_as_float(in[e]));
      } else {
        k[2 * e] = order_key(__uint_as_float(in[e] << 16));
        k[2 * e + 1] = order_key(__uint_as_float(in[e] & 0xffff0000u));
      }
    }
  }
  for (int i = tail + threadIdx.x; i < n; i += kSampleThreads) keys[i] = order_key(logit(x + i));
}

struct Group {                        // the cluster, and this CTA in it
  int C, rank, own;
  const uint32_t *keys;
  Shared *sh;
  int turn;                           // which of the exchange's two halves is next
};
// every CTA's (a, b): sums over all, and over the ranks before
__device__ __forceinline__ void exchange_sums(Group &g, u64 a, u64 b, u64 &sum_a, u64 &sum_b, u64 &before_a, u64 &before_b) {
  if (threadIdx.x == 0) g.sh->ex[g.turn] = Exchange{a, b};
  cluster_barrier();
  sum_a = sum_b = before_a = before_b = 0;
  for (int r = 0; r < g.C; ++r) {
    const u64 x = peer_u64(&g.sh->ex[g.turn].a, r), y = peer_u64(&g.sh->ex[g.turn].b, r);
    sum_a += x; sum_b += y;
    if (r < g.rank) { before_a += x; before_b += y; }
  }
  g.turn ^= 1;
}
// largest a and b over the cluster, from every thread's
__device__ __forceinline__ void exchange_max(Group &g, u64 &a, u64 &b) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    a = max(a, __shfl_xor_sync(0xffffffffu, a, o));
    b = max(b, __shfl_xor_sync(0xffffffffu, b, o));
  }
  if (lane == 0) { g.sh->part[0][warp] = a; g.sh->part[1][warp] = b; }
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < kSampleWarps; ++w) { a = max(a, g.sh->part[0][w]); b = max(b, g.sh->part[1][w]); }
    g.sh->ex[g.turn] = Exchange{a, b};
  }
  cluster_barrier();
  a = b = 0;
  for (int r = 0; r < g.C; ++r) {
    a = max(a, peer_u64(&g.sh->ex[g.turn].a, r));
    b = max(b, peer_u64(&g.sh->ex[g.turn].b, r));
  }
  g.turn ^= 1;
}

struct Border { uint32_t cut, ties; u64 tied; };      // kept: keys above cut, and the first `ties` of the `tied` that equal it

// Finds the last token of the shortest run of tokens, largest logits first and starting behind nothing, whose number reaches want
// (WEIGHTS false) or whose weights reach the share p of all their sum (WEIGHTS true).  Only keys above floor.cut, and floor.ties of
// those that equal it, are there; what is wanted is among them.
template <bool WEIGHTS>
__device__ Border find_border(Group &g, const Row &row, u64 want, double p, const Border &floor) {
  Shared &sh = *g.sh;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  // first bins: equal steps of the logit.  Each step of the arithmetic is monotone, so that bins are runs of keys.
  const float span = WEIGHTS ? fminf(row.top - row.lowest, 40.f / (float)row.inv_t) : row.top - row.lowest;
  const float per = fminf((kSampleBins - 1) / span, 1e30f);
  uint32_t k_high = 0xffffffffu, k_low = floor.cut;    // keys that the border is among
  int shift = -1;
  u64 gone = 0;                                         // what is above k_high
  for (int level = 0;; ++level) {
    for (int b = tid; b < kSampleBins; b += kSampleThreads) {
      sh.count[b] = 0;
      if (WEIGHTS) sh.low[b] = sh.high[b] = 0;
    }
    __syncthreads();
    auto bin_of = [&](uint32_t key) {
      return shift < 0 ? (int)fminf((row.top - key_value(key)) * per, (float)(kSampleBins - 1)) : (int)((k_high - key) >> shift);
    };
    for (int i = tid; i < g.own; i += kSampleThreads) {
      const uint32_t key = g.keys[i];
      if (key == 0 || key < k_low || key > k_high) continue;
      const int b = bin_of(key);
      atomicAdd(&sh.count[b], 1u);
      if (WEIGHTS) {
        const u64 w = weight(row, key);
        const uint32_t lo = (uint32_t)w, old = atomicAdd(&sh.low[b], lo);
        const uint32_t hi = (uint32_t)(w >> 32) + (old + lo < old);
        if (hi) atomicAdd(&sh.high[b], hi);
      }
    }
    cluster_barrier();
    constexpr int kEach = kSampleBins / kSampleThreads;
    u64 in[kEach], sum = 0;
    uint32_t cnt[kEach];
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int b = tid * kEach + e;
      in[e] = cnt[e] = 0;
      for (int r = 0; r < g.C; ++r) {
        const uint32_t n = peer_u32(&sh.count[b], r);
        cnt[e] += n;
        if (WEIGHTS) { if (n) in[e] += peer_u32(&sh.low[b], r) + ((u64)peer_u32(&sh.high[b], r) << 32); }
        else in[e] += n;
      }
      sum += in[e];
    }
    u64 upto = warp_upto(sum);
    if (lane == 31) sh.part[0][warp] = upto;
    __syncthreads();
    u64 before = gone + upto - sum, all = 0;
    for (int w = 0; w < kSampleWarps; ++w) {
      if (w < warp) before += sh.part[0][w];
      all += sh.part[0][w];
    }
    if (WEIGHTS && level == 0) {
      // of those that equal the floor, only some are there
      if (floor.tied > floor.ties) all -= (floor.tied - floor.ties) * weight(row, floor.cut);
      want = min(max((u64)ceil(p * (double)all), 1ull), all);
    }
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      if (before < want && want <= before + in[e]) {
        sh.found[0] = tid * kEach + e;
        sh.found[1] = before;
        sh.bin_count = cnt[e];
      }
      before += in[e];
    }
    if (tid == 0) sh.few_count = 0;
    __syncthreads();
    const int bin = (int)sh.found[0];
    gone = sh.found[1];
    const uint32_t tokens = sh.bin_count;
    // the bin's smallest and largest key, and its keys if they are few
    u64 hi = 0, lo = 0;
    for (int i = tid; i < g.own; i += kSampleThreads) {
      const uint32_t key = g.keys[i];
      if (key == 0 || key < k_low || key > k_high || bin_of(key) != bin) continue;
      hi = max(hi, (u64)key);
      lo = max(lo, (u64)~key);
      if (tokens <= kFew) sh.few[atomicAdd(&sh.few_count, 1u)] = key;
    }
    exchange_max(g, hi, lo);          // its barrier makes the lists visible too
    k_high = (uint32_t)hi;
    k_low = ~(uint32_t)lo;
    if (k_low == k_high) {
      const u64 w = WEIGHTS ? weight(row, k_low) : 1;
      const u64 ties = w ? (want - gone + w - 1) / w : 1;
      cluster_barrier();              // counts of this level have been read
      return Border{k_low, (uint32_t)min(ties, (u64)tokens), tokens};
    }
    if (tokens <= kFew) {
      int at = 0;
      for (int r = 0; r < g.C; ++r) {
        const int n = (int)peer_u32(&sh.few_count, r);
        for (int i = tid; i < n; i += kSampleThreads) sh.all[at + i] = peer_u32(&sh.few[i], r);
        at += n;
      }
      __syncthreads();
      uint32_t key = 0;
      if (tid < (int)tokens) {
        key = sh.all[tid];
        sh.all_w[tid] = WEIGHTS ? weight(row, key) : 1;
      }
      __syncthreads();
      if (tid < (int)tokens) {
        u64 above = gone, equal = 0;
        for (int i = 0; i < (int)tokens; ++i) {
          const uint32_t other = sh.all[i];
          if (other > key) above += sh.all_w[i];
          equal += other == key;
        }
        const u64 w = sh.all_w[tid];
        if (above < want && want <= above + equal * w) {     // equal keys write the same
          sh.found[0] = key;
          sh.found[1] = w ? (want - above + w - 1) / w : 1;
          sh.found[2] = equal;
        }
      }
      cluster_barrier();              // lists and counts have been read
      return Border{(uint32_t)sh.found[0], (uint32_t)sh.found[1], sh.found[2]};
    }
    const uint32_t range = k_high - k_low;
    shift = max(0, 32 - __clz(range) - 10);
    cluster_barrier();                // counts of this level have been read
  }
}

template <typename T>
__global__ void __launch_bounds__(kSampleThreads) sample_kernel(const SampleParams P) {
  pdl_prologue();
  extern __shared__ __align__(16) uint32_t keys[];
  __shared__ Shared sh;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  Group g;
  g.C = (int)cluster_size();
  g.rank = (int)cluster_ctarank();
  g.keys = keys;
  g.sh = &sh;
  g.turn = 0;
  const int r = blockIdx.x / g.C, lo = min(g.rank * P.slice, P.vocab);
  g.own = min(lo + P.slice, P.vocab) - lo;
  load_keys((const T *)P.logits + (long long)r * P.ld + lo, g.own, keys);
  const float temperature = P.temperature ? P.temperature[r] : 1.f;
  const int k = P.top_k ? P.top_k[r] : 0;
  const float top_p = P.top_p ? P.top_p[r] : 1.f;
  float min_p = P.min_p ? P.min_p[r] : 0.f, u = P.u[r];
  min_p = min_p > 0.f ? fminf(min_p, 1.f) : 0.f;
  u = u > 0.f ? u : 0.f;
  __syncthreads();

  // largest logit, the first of equal ones, and the smallest
  u64 best = 0, least = 0;
  for (int i = tid; i < g.own; i += kSampleThreads) {
    const uint32_t key = keys[i];
    if (key == 0) continue;
    best = max(best, (u64)key << 32 | (uint32_t)~(lo + i));
    least = max(least, (u64)~key);
  }
  exchange_max(g, best, least);
  const bool greedy = !(temperature > 0.f) || k == 1;
  if (best == 0 || greedy) {
    if (g.rank == 0 && tid == 0) {
      P.tokens[r] = best == 0 ? -1 : (int)~(uint32_t)best;
      if (P.logprobs) P.logprobs[r] = best == 0 ? -INFINITY : 0.f;
    }
    cluster_barrier();                // the others may still read this CTA's exchange
    return;
  }
  Row row;
  uint32_t top_key = (uint32_t)(best >> 32);
  row.lowest = key_value(~(uint32_t)least);
  if (key_value(top_key) == INFINITY) {      // infinite logits have all the weight, in equal shares
    for (int i = tid; i < g.own; i += kSampleThreads) keys[i] = keys[i] == top_key ? 0x80000000u : 0;
    top_key = 0x80000000u;
    row.lowest = 0.f;
    __syncthreads();
  }
  row.top = key_value(top_key);
  row.top_d = row.top;
  row.inv_t = 1.0 / (double)temperature;

  Border cut{0, 0, 0};
  if (k > 1 && k < P.vocab) {
    u64 there = 0, n = 0, x, y;
    for (int i = tid; i < g.own; i += kSampleThreads) there += keys[i] != 0;
    there = warp_sum(there);
    if (lane == 0) sh.part[0][warp] = there;
    __syncthreads();
    for (int w = 0; w < kSampleWarps; ++w) n += sh.part[0][w];
    exchange_sums(g, n, 0, there, n, x, y);
    if (there > (u64)k) cut = find_border<false>(g, row, k, 0.0, cut);
  }
  if (top_p < 1.f) cut = find_border<true>(g, row, 0, fmax((double)top_p, 0.0), cut);

  // Each warp takes a stretch of the slice; ties are numbered in the order of the vocabulary.
  const int stretch = ((g.own + kSampleWarps - 1) / kSampleWarps + 31) & ~31;
  const int i0 = min(warp * stretch, g.own), i1 = min(i0 + stretch, g.own);
  u64 ties_before = 0;
  const bool some_ties = cut.tied > cut.ties;
  if (some_ties) {
    u64 n = 0, s, x, y;
    for (int i = i0 + lane; i < i1; i += 32) n += keys[i] == cut.cut;
    n = warp_sum(n);
    __syncthreads();
    if (lane == 0) sh.part[0][warp] = n;
    __syncthreads();
    n = 0;
    for (int w = 0; w < kSampleWarps; ++w) {
      n += sh.part[0][w];
      if (w < warp) ties_before += sh.part[0][w];
    }
    exchange_sums(g, n, 0, s, n, x, y);
    ties_before += x;
  }
  auto kept_weight = [&](int i, uint32_t &ties) -> u64 {      // of token i = the lane's; ties: those before the warp's 32
    const uint32_t key = i < i1 ? keys[i] : 0;
    bool in = key > cut.cut;
    if (key != 0 && key == cut.cut) in = true;
    if (some_ties) {
      const unsigned same = __ballot_sync(0xffffffffu, key != 0 && key == cut.cut);
      if (key == cut.cut) in = key != 0 && ties + __popc(same & ((1u << lane) - 1)) < cut.ties;
      ties += __popc(same);
    }
    if (!in) return 0;
    const double d = ((double)key_value(key) - row.top_d) * row.inv_t;
    if (d < -31.2) return 0;
    const double w = exp(d);
    return w < (double)min_p ? 0 : __double2ull_rn(w * 17592186044416.0);
  };
  u64 sum = 0;
  uint32_t ties = (uint32_t)ties_before;
  for (int i = i0; i < i1; i += 32) sum += kept_weight(i + lane, ties);
  sum = warp_sum(sum);
  __syncthreads();
  if (lane == 0) sh.part[1][warp] = sum;
  __syncthreads();
  u64 mine = 0, before = 0, total, x, y, z;
  for (int w = 0; w < kSampleWarps; ++w) {
    mine += sh.part[1][w];
    if (w < warp) before += sh.part[1][w];
  }
  exchange_sums(g, mine, 0, total, x, y, z);
  before += y;
  // the first token at which the running sum is above u times the total
  const u64 target = min((u64)floor(fmin((double)u, 1.0) * (double)total), total - 1);
  if (before <= target && target < before + sum) {
    ties = (uint32_t)ties_before;
    for (int i = i0; i < i1; i += 32) {
      const u64 w = kept_weight(i + lane, ties), upto = before + warp_upto(w);
      const unsigned past = __ballot_sync(0xffffffffu, upto > target);
      if (past) {
        if (lane == __ffs(past) - 1) {
          P.tokens[r] = lo + i + lane;
          if (P.logprobs)
            P.logprobs[r] = (float)(((double)key_value(keys[i + lane]) - row.top_d) * row.inv_t - log((double)total * (1.0 / 17592186044416.0)));
        }
        break;
      }
      before = __shfl_sync(0xffffffffu, upto, 31);
    }
  }
  cluster_barrier();                  // the others may still read this CTA's exchange
}

template <typename T>
templora_status_t launch_sample(SampleParams &p, cudaStream_t st) {
  int sms = 0;
  TL_TRY(stream_sms(st, &sms));
  // as few CTAs to a row as hold its keys with two CTAs per SM; more while SMs are idle and a CTA keeps some thousand tokens
  int C = 1;
  while (C < kMaxCluster && p.vocab > C * kMostSlice) C *= 2;
  while (C < kMaxCluster && (long long)p.rows * C * 2 <= sms && p.vocab / C > 2048) C *= 2;
  p.slice = (p.vocab + C - 1) / C;
  TL_TRY((allow_smem<sample_kernel<T>>((size_t)kMaxVocab / kMaxCluster * sizeof(uint32_t))));
  LaunchScope scope(kKindSample, st);
  TL_CUDA_CHECK(launch_cluster_pdl(sample_kernel<T>, dim3((unsigned)(p.rows * C)), dim3(kSampleThreads), C,
                                   (size_t)p.slice * sizeof(uint32_t), st, p));
  return TEMPLORA_OK;
}

}  // namespace
}  // namespace templora

using namespace templora;

extern "C" templora_status_t templora_sample(const templora_sample_t *s, int32_t rows, void *stream) {
  if (!s || rows <= 0 || s->vocab <= 0 || !s->logits || !s->u || !s->tokens || (reinterpret_cast<uintptr_t>(s->logits) & 15) != 0)
    return TEMPLORA_ERR_INVALID_ARG;
  if (!word_aligned(s->temperature) || !word_aligned(s->top_k) || !word_aligned(s->top_p) || !word_aligned(s->min_p) || !word_aligned(s->u) ||
      !word_aligned(s->tokens) || !word_aligned(s->logprobs))
    return TEMPLORA_ERR_INVALID_ARG;
  if (s->dtype != TEMPLORA_F32 && s->dtype != TEMPLORA_BF16) return TEMPLORA_ERR_UNSUPPORTED;
  if (s->vocab > kMaxVocab || rows > (1 << 24)) return TEMPLORA_ERR_UNSUPPORTED;
  const long long ld = s->ld == 0 ? s->vocab : s->ld;
  if (ld < s->vocab || ld > (1ll << 31)) return TEMPLORA_ERR_INVALID_ARG;
  SampleParams p{s->logits, ld, rows, s->vocab, 0, s->temperature, s->top_p, s->min_p, s->u, s->top_k, s->tokens, s->logprobs};
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  return s->dtype == TEMPLORA_F32 ? launch_sample<float>(p, st) : launch_sample<__nv_bfloat16>(p, st);
}
