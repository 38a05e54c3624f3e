// The choice of the next token: temperature, top-k, top-p, min-p, and the inverse of the running sum at a given random number.
#include "attention.cuh"
#include "cluster.cuh"
#include "tc_host.h"

#include <algorithm>
#include <cfloat>

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

// A cluster of CTAs takes a row: each CTA keeps the logits of a stretch of the vocabulary in shared memory, and what they find
// they tell each other through it.  No filter sorts the row; each first finds few tokens that hold all that may be kept, if there are
// such, and then one CTA sorts these and finishes the row:
//   top-k, up to 256: the k-th largest of the threads' largest logits is a bound that the k largest tokens do not fall below.
//   top-p: the weights are added up in bins of descending logits; the border falls into one of them.
// Where the tokens are many, the border is searched for within its bin, and another pass adds up the weights of the tokens above it.
// All sums are integers, in units of 2^-44 of the largest weight, so that neither the order of atomics nor the number of CTAs changes a
// result.
// Bound by latency: a row's few passes over shared memory, and the steps between its CTAs.  One row of 32000, top-k and top-p, 8.2 us; 64 rows of
// 32000 under all filters, 27; 24 rows of 128251, top-p, 47, of which weights in bins are 10; 192 rows of 64000, min-p, 33: replayed from a
// graph, over logits that are in L2 by then, as all times here.  In calls over changing logits 8.5, 27.5, 48 and 37.
constexpr int kSampleBins = 1024, kGroups = 32;      // bins, and groups of bins that are looked through first
constexpr int kFew = 64;              // tokens that are compared one with another to find a border
constexpr int kList = 256;            // tokens that one CTA sorts
constexpr int kGather = 1024;         // tokens that are put into finer bins without another pass
constexpr int kMaxVocab = 1 << 18;    // sums stay below 2^62
constexpr int kMostBytes = 69632;     // logits of a CTA: two CTAs per SM
constexpr uint32_t kLeastKey = 0x00800000u;          // order_key of the least finite number
using u64 = unsigned long long;

struct Exchange { u64 a, b; };        // what CTAs tell each other
struct Shared {
  uint32_t field[3][kSampleBins];     // of a bin: the weights of its tokens, in fields of 17 bits that are added up by themselves
  u64 sum[kSampleBins], group[kGroups];
  u64 list[kGather], above[kList];    // this CTA's tokens in the border's bin, and above it: key << 32 | ~index, in order of the filters
  u64 all[kGather], list_w[kList];
  Exchange ex[2], got;
  int counts[2][kMaxCluster];         // of the CTAs' lists
  u64 part[2][32];
  u64 found[3];
  uint32_t found_count;
  alignas(8) uint32_t listed;
  uint32_t listed_above;              // read as one with the one before
  double power[64];                   // 2^(i / 64)
};

struct Row {
  float top, t;                       // largest logit that counts; temperature
  double top_d, inv_t, per64, min_p;  // per64: 64 log2(e) / temperature
  float floor;                        // below it a logit has no weight
  const double *power;
};
// w_i for logits not below the floor: 2^(n / 64) from a table times the first six terms of the series of 2^(x / 64), |x| <= 1/2, whose
// rest is below 2^-54.  (The library's exp spends twice the instructions; it serves every argument.)
__device__ __forceinline__ double weight_value(const Row &r, float logit) {
  constexpr double kRound = 6755399441055744.0, l = 0.010830424696249145;     // 1.5 * 2^52; log(2) / 64
  const double d = ((double)logit - r.top_d) * r.per64, m = d + kRound, x = d - (m - kRound);
  const int n = __double2loint(m);
  double p = fma(x, l * l * l * l * l / 120, l * l * l * l / 24);
  p = fma(x, p, l * l * l / 6);
  p = fma(x, p, l * l / 2);
  p = fma(x, p, l);
  p = fma(x, p, 1.0) * r.power[n & 63];
  return __hiloint2double(__double2hiint(p) + ((n >> 6) << 20), __double2loint(p));
}
// in units of 2^-44, rounded to the nearest: the low bits of a number just above 2^52
__device__ __forceinline__ u64 fixed_weight(double w) {
  return (u64)__double_as_longlong(fma(w, 17592186044416.0, 4503599627370496.0)) & 0xfffffffffffffull;
}
__device__ __forceinline__ u64 weight(const Row &r, float logit) { return logit >= r.floor ? fixed_weight(weight_value(r, logit)) : 0; }
__device__ __forceinline__ u64 weight_of_key(const Row &r, uint32_t key) { return weight(r, key_value(key)); }

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

// ------------------------------------------------------------------ a stretch of the vocabulary
// Logits stay as they are stored, 16 bytes at a time; places in front of the first and behind the last token hold -infinity.
// Comparisons leave out NaN by themselves, and bounds above -infinity that.
template <typename T> struct Vec;
template <> struct Vec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ float at(const uint4 &w, int e) { return __uint_as_float(e == 0 ? w.x : e == 1 ? w.y : e == 2 ? w.z : w.w); }
  static __device__ __forceinline__ void put(uint4 &w, int e, float v) { (e == 0 ? w.x : e == 1 ? w.y : e == 2 ? w.z : w.w) = __float_as_uint(v); }
  static __device__ __forceinline__ float most(const uint4 &w) { return fmaxf(fmaxf(at(w, 0), at(w, 1)), fmaxf(at(w, 2), at(w, 3))); }
};
template <> struct Vec<__nv_bfloat16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ float at(const uint4 &w, int e) {
    const uint32_t v = (e >> 1) == 0 ? w.x : (e >> 1) == 1 ? w.y : (e >> 1) == 2 ? w.z : w.w;
    return __uint_as_float(e & 1 ? v & 0xffff0000u : v << 16);
  }
  static __device__ __forceinline__ void put(uint4 &w, int e, float x) {      // x: a bf16 number
    uint32_t &v = (e >> 1) == 0 ? w.x : (e >> 1) == 1 ? w.y : (e >> 1) == 2 ? w.z : w.w;
    v = e & 1 ? (v & 0xffffu) | (__float_as_uint(x) & 0xffff0000u) : (v & 0xffff0000u) | __float_as_uint(x) >> 16;
  }
  static __device__ __forceinline__ float most(const uint4 &w) {
    const auto pair = [](const uint32_t &v) { return *reinterpret_cast<const __nv_bfloat162 *>(&v); };
    const float2 m = __bfloat1622float2(__hmax2(__hmax2(pair(w.x), pair(w.y)), __hmax2(pair(w.z), pair(w.w))));
    return fmaxf(m.x, m.y);
  }
};

struct Group {                        // the cluster, and this CTA in it
  int C, rank;
  uint4 *x;                           // logits
  int vecs, pad, lo;                  // vectors of logits; token of place i: lo + i - pad
  Shared *sh;
  int turn;                           // which of the exchange's two halves is next
  __device__ __forceinline__ void barrier() const {
    if (C == 1) __syncthreads();
    else cluster_barrier();
  }
  __device__ __forceinline__ u64 peer(const u64 *p, int r) const { return C == 1 ? *p : peer_u64(p, r); }
  template <typename T> __device__ __forceinline__ u64 token(float logit, int v, int e) const {
    return (u64)order_key(logit) << 32 | (uint32_t)~(lo + v * Vec<T>::N + e - pad);
  }
};
// Reads a stretch of n logits; returns the largest that the thread has read.
template <typename T, int TH> __device__ __forceinline__ float load_logits(Group &g, const T *x, int n) {
  using V = Vec<T>;
  constexpr int N = V::N;
  const int head = min(n, (int)((16 - (reinterpret_cast<uintptr_t>(x) & 15)) & 15) / (int)sizeof(T));
  g.pad = (N - head) & (N - 1);
  g.vecs = (g.pad + n + N - 1) / N;
  const int first = (g.pad + head) / N, full = (n - head) / N;      // whole vectors: `full` from vector `first`
  float most = -INFINITY;
  const uint4 *in = reinterpret_cast<const uint4 *>(x + head);
#pragma unroll 4
  for (int v = threadIdx.x; v < full; v += TH) {
    const uint4 w = __ldcs(in + v);
    most = fmaxf(most, V::most(w));
    g.x[first + v] = w;
  }
  // at most one vector in front of these and one behind
  const int v = threadIdx.x == 0 && first > 0 ? 0 : threadIdx.x == 1 && first + full < g.vecs ? first + full : -1;
  if (v >= 0) {
    uint4 w = make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const int i = v * N + e - g.pad;
      V::put(w, e, i >= 0 && i < n ? attn_ld(x + i) : -INFINITY);
    }
    most = fmaxf(most, V::most(w));
    g.x[v] = w;
  }
  return most;
}

// ------------------------------------------------------------------ between the CTAs of a cluster
// One warp reads what the others have to say, a lane a CTA: were all warps to, their loads would queue up (2000 cycles instead of 300).
// every CTA's a: the sum over all, and over the ranks before
__device__ __forceinline__ void exchange_sum(Group &g, u64 a, u64 &sum, u64 &before) {
  Shared &sh = *g.sh;
  if (threadIdx.x == 0) sh.ex[g.turn].a = a;
  g.barrier();
  if (threadIdx.x < 32) {
    const int lane = threadIdx.x;
    const u64 x = lane < g.C ? g.peer(&sh.ex[g.turn].a, lane) : 0, upto = warp_upto(x);
    if (lane == 31) sh.got.a = upto;
    if (lane == g.rank) sh.got.b = upto - x;
  }
  __syncthreads();
  sum = sh.got.a;
  before = sh.got.b;
  g.turn ^= 1;
}
// largest a and b in the block, from every thread's
template <int TH> __device__ __forceinline__ void block_max(Shared &sh, uint32_t &a, uint32_t &b) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  a = __reduce_max_sync(0xffffffffu, a);
  b = __reduce_max_sync(0xffffffffu, b);
  if (lane == 0) sh.part[0][warp] = (u64)a << 32 | b;
  __syncthreads();
  const u64 v = lane < TH / 32 ? sh.part[0][lane] : 0;
  a = __reduce_max_sync(0xffffffffu, (uint32_t)(v >> 32));
  b = __reduce_max_sync(0xffffffffu, (uint32_t)v);
  __syncthreads();
}
// largest a, b, c over the cluster, from values that all threads of a CTA have
__device__ __forceinline__ void exchange_max(Group &g, uint32_t &a, uint32_t &b, uint32_t &c) {
  if (g.C == 1) return;
  Shared &sh = *g.sh;
  if (threadIdx.x == 0) sh.ex[g.turn] = Exchange{(u64)a << 32 | b, c};
  g.barrier();
  if (threadIdx.x < 32) {
    const int lane = threadIdx.x;
    u64 x = 0, y = 0;
    if (lane < g.C) {
      x = g.peer(&sh.ex[g.turn].a, lane);
      y = g.peer(&sh.ex[g.turn].b, lane);
    }
    a = __reduce_max_sync(0xffffffffu, (uint32_t)(x >> 32));
    b = __reduce_max_sync(0xffffffffu, (uint32_t)x);
    c = __reduce_max_sync(0xffffffffu, (uint32_t)y);
    if (lane == 0) sh.got = Exchange{(u64)a << 32 | b, c};
  }
  __syncthreads();
  a = (uint32_t)(sh.got.a >> 32);
  b = (uint32_t)sh.got.a;
  c = (uint32_t)sh.got.b;
  g.turn ^= 1;
}
// tokens in the lists of all CTAs: above a bin, and in it.  A barrier, behind which the lists may be read.
__device__ __forceinline__ void exchange_counts(Group &g, uint32_t &above, uint32_t &in) {
  Shared &sh = *g.sh;
  g.barrier();
  if (threadIdx.x < 32) {
    const int lane = threadIdx.x;
    uint32_t x = 0, y = 0;
    if (lane < g.C) {
      const u64 both = g.peer(reinterpret_cast<const u64 *>(&sh.listed), lane);
      sh.counts[0][lane] = x = (uint32_t)both;
      sh.counts[1][lane] = y = (uint32_t)(both >> 32);
    }
    x = __reduce_add_sync(0xffffffffu, x);
    y = __reduce_add_sync(0xffffffffu, y);
    if (lane == 0) sh.got.a = (u64)y << 32 | x;
  }
  __syncthreads();
  above = (uint32_t)(sh.got.a >> 32);
  in = (uint32_t)sh.got.a;
}
// Copies the lists of all CTAs, counted before, into sh.all.
template <int TH> __device__ __forceinline__ void copy_lists(Group &g, bool with_above) {
  Shared &sh = *g.sh;
  int total = 0;
  for (int r = 0; r < g.C; ++r) total += sh.counts[0][r] + (with_above ? sh.counts[1][r] : 0);
  for (int i = threadIdx.x; i < total; i += TH) {
    int at = i, r = 0;
    for (;; ++r) {
      const int n = sh.counts[0][r] + (with_above ? sh.counts[1][r] : 0);
      if (at < n) break;
      at -= n;
    }
    const int n = sh.counts[0][r];
    sh.all[i] = g.peer(at < n ? &sh.list[at] : &sh.above[at - n], r);
  }
}

// ------------------------------------------------------------------ where a filter ends
struct Border {
  uint32_t cut, ties;                 // kept: keys above cut, and the first `ties` of the `tied` that equal it
  u64 tied;
  u64 want;                           // what the sum had to reach
  bool listed;                        // instead: every token down to the border, and some below, are in the CTAs' lists
};
// bins of descending logits in equal steps, or, with shift >= 0, of descending keys
struct Bins {
  float top, per;
  uint32_t high;
  int shift;
  __device__ __forceinline__ uint32_t of(float logit) const {
    // each step of the arithmetic is monotone, so that bins are runs of logits
    return shift < 0 ? (uint32_t)fminf((top - logit) * per, (float)(kSampleBins - 1)) : (high - order_key(logit)) >> shift;
  }
  __device__ __forceinline__ uint32_t of_key(uint32_t key) const { return (high - key) >> shift; }
  // no key of bin b or a bin above it is below this
  __device__ __forceinline__ uint32_t least_key(uint32_t b) const {
    if (b == kSampleBins - 1) return kLeastKey;
    if (shift < 0) return max(order_key(top - ((float)(b + 1) / per * 1.000001f + fabsf(top) * 1e-6f)), kLeastKey);
    const uint32_t down = ((b + 1) << shift) - 1;
    return down >= high ? kLeastKey : high - down;
  }
};
__device__ __forceinline__ void clear_bins(Shared &sh, int threads, bool weights) {
  for (int b = threadIdx.x; b < (weights ? 3 : 1) * kSampleBins; b += threads) (&sh.field[0][0])[b] = 0;
}
// A bin's tokens are at most 2^15, its fields' sums stay below 2^32.
__device__ __forceinline__ void add_weight(Shared &sh, uint32_t bin, u64 w) {
  atomicAdd(&sh.field[0][bin], (uint32_t)w & 0x1ffffu);
  atomicAdd(&sh.field[1][bin], (uint32_t)(w >> 17) & 0x1ffffu);
  if (w >> 34) atomicAdd(&sh.field[2][bin], (uint32_t)(w >> 34));
}
// Between two barriers of the block: the bins' sums from their fields, and the groups'.  more: what the last bin has besides.
template <int TH, bool WEIGHTS> __device__ __forceinline__ void sum_bins(Shared &sh, u64 more) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int b = threadIdx.x; b < kSampleBins; b += TH) {
    u64 v = sh.field[0][b];
    if (WEIGHTS) v += ((u64)sh.field[1][b] << 17) + ((u64)sh.field[2][b] << 34);
    if (b == kSampleBins - 1) v += more;
    sh.sum[b] = v;
    v = warp_sum(v);
    if (lane == 0) sh.group[b >> 5] = v;
  }
}
// The bin where the running sum over all CTAs, beginning at `gone`, reaches want; one warp.  want 0: the share p of all, less `absent`.
// Leaves the bin, what is above it, and want in sh.found; ~0 as the bin where all do not reach it.
__device__ __forceinline__ void find_bin(Group &g, u64 gone, u64 want, double p, u64 absent) {
  Shared &sh = *g.sh;
  const int lane = threadIdx.x & 31;
  u64 v = 0;
#pragma unroll
  for (int r = 0; r < kMaxCluster; ++r) v += r < g.C ? g.peer(&sh.group[lane], r) : 0;
  u64 upto = warp_upto(v);
  const u64 all = __shfl_sync(0xffffffffu, upto, 31) - absent;
  if (want == 0) want = min(max((u64)ceil(p * (double)all), 1ull), all);
  unsigned past = __ballot_sync(0xffffffffu, gone + upto >= want);
  if (!past) {
    if (lane == 0) sh.found[0] = ~0ull;
    return;
  }
  const int grp = __ffs(past) - 1;
  gone += __shfl_sync(0xffffffffu, upto - v, grp);
  v = 0;
#pragma unroll
  for (int r = 0; r < kMaxCluster; ++r) v += r < g.C ? g.peer(&sh.sum[grp * 32 + lane], r) : 0;
  upto = warp_upto(v);
  past = __ballot_sync(0xffffffffu, gone + upto >= want);
  if (lane == __ffs(past) - 1) {
    sh.found[0] = grp * 32 + lane;
    sh.found[1] = gone + upto - v;
    sh.found[2] = want;
  }
}
__device__ __forceinline__ uint32_t key_of(u64 token) { return (uint32_t)(token >> 32); }

// The border among the n tokens of sh.all; `gone` is above them.  Finer and finer bins, until few tokens are left to be compared
// one with another.  Each CTA by itself.
template <int TH, bool WEIGHTS>
__device__ Border border_of_list(Shared &sh, const Row &row, int n, u64 want, u64 gone) {
  const int tid = threadIdx.x, warp = tid >> 5;
  uint32_t most = 0, least = 0;
  __syncthreads();
  for (int i = tid; i < n; i += TH) {
    most = max(most, key_of(sh.all[i]));
    least = max(least, ~key_of(sh.all[i]));
  }
  block_max<TH>(sh, most, least);
  uint32_t k_high = most, k_low = ~least;
  int in_bin = n;
  while (in_bin > kFew && k_low != k_high) {
    const Bins bins{0.f, 0.f, k_high, max(0, 32 - __clz(k_high - k_low) - 10)};
    clear_bins(sh, TH, WEIGHTS);
    __syncthreads();
    for (int i = tid; i < n; i += TH) {
      const uint32_t key = key_of(sh.all[i]);
      if (key < k_low || key > k_high) continue;
      if (WEIGHTS) add_weight(sh, bins.of_key(key), weight_of_key(row, key));
      else atomicAdd(&sh.field[0][bins.of_key(key)], 1u);
    }
    if (tid == 0) sh.found_count = 0;
    __syncthreads();
    sum_bins<TH, WEIGHTS>(sh, 0);
    __syncthreads();
    if (warp == 0) {                  // as find_bin does, within the CTA
      const int lane = tid;
      u64 v = sh.group[lane], upto = warp_upto(v);
      const int grp = __ffs(__ballot_sync(0xffffffffu, gone + upto >= want)) - 1;
      const u64 before = gone + __shfl_sync(0xffffffffu, upto - v, grp);
      v = sh.sum[grp * 32 + lane];
      upto = warp_upto(v);
      if (lane == __ffs(__ballot_sync(0xffffffffu, before + upto >= want)) - 1) {
        sh.found[0] = grp * 32 + lane;
        sh.found[1] = before + upto - v;
      }
    }
    __syncthreads();
    const uint32_t bin = (uint32_t)sh.found[0];
    gone = sh.found[1];
    k_low = max(k_low, bins.least_key(bin));
    k_high -= bin << bins.shift;
    // how many it holds
    int c = 0;
    for (int i = tid; i < n; i += TH) c += key_of(sh.all[i]) >= k_low && key_of(sh.all[i]) <= k_high;
    c = __reduce_add_sync(0xffffffffu, c);
    if ((tid & 31) == 0 && c) atomicAdd(&sh.found_count, (uint32_t)c);
    __syncthreads();
    in_bin = (int)sh.found_count;
    __syncthreads();
  }
  if (k_low == k_high) {
    const u64 w = WEIGHTS ? weight_of_key(row, k_low) : 1;
    return Border{k_low, (uint32_t)min(w ? (want - gone + w - 1) / w : 1, (u64)in_bin), (u64)in_bin, want, false};
  }
  if (tid == 0) sh.listed = 0;
  __syncthreads();
  for (int i = tid; i < n; i += TH) {
    const uint32_t key = key_of(sh.all[i]);
    if (key < k_low || key > k_high) continue;
    const uint32_t at = atomicAdd(&sh.listed, 1u);
    sh.list[at] = key;
    sh.list_w[at] = WEIGHTS ? weight_of_key(row, key) : 1;
  }
  __syncthreads();
  if (tid < in_bin) {
    const u64 key = sh.list[tid], w = sh.list_w[tid];
    u64 over = gone, equal = 0;
    for (int j = 0; j < in_bin; ++j) {
      const u64 other = sh.list[j];
      if (other > key) over += sh.list_w[j];
      equal += other == key;
    }
    if (over < want && want <= over + equal * w) {           // equal keys write the same
      sh.found[0] = key;
      sh.found[1] = w ? (want - over + w - 1) / w : 1;
      sh.found[2] = equal;
    }
  }
  __syncthreads();
  const Border found{(uint32_t)sh.found[0], (uint32_t)sh.found[1], sh.found[2], want, false};
  __syncthreads();
  return found;
}

// Finds the last token of the shortest run of tokens, largest logits first, whose number reaches `want` (WEIGHTS false; all, where there
// are no more than that) or whose weights reach the share p of all their sum (WEIGHTS true).  Only keys above floor.cut, and
// floor.ties of those that equal it, are there; what is wanted is among them.  may_list: the tokens down to the border may be listed
// instead if they are few.
template <typename T, int TH, bool WEIGHTS>
__device__ Border find_border(Group &g, const Row &row, u64 want, double p, const Border &floor, bool may_list) {
  using V = Vec<T>;
  Shared &sh = *g.sh;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  // Of the tokens with less than (1 - p) / vocab of the largest weight, all together have less than 1 - p of the sum: the border of
  // top-p is above them, and they share the last bin.
  float span = row.t * (__logf((float)kMaxVocab / (float)(1.0 - p)) + 0.1f);
  if (!WEIGHTS) {
    uint32_t least = 0, none = 0, no = 0;
    for (int v = tid; v < g.vecs; v += TH) {
      const uint4 x = g.x[v];
#pragma unroll
      for (int e = 0; e < V::N; ++e)
        if (V::at(x, e) > -INFINITY) least = max(least, ~order_key(V::at(x, e)));
    }
    block_max<TH>(sh, least, none);
    exchange_max(g, least, none, no);
    span = row.top - key_value(~least);
  }
  Bins bins{row.top, fminf((kSampleBins - 1) / span, 1e30f), 0, -1};
  uint32_t k_high = 0xff7fffffu, k_low = max(floor.cut, kLeastKey);      // keys that the border is among: at first all but infinities'
  u64 gone = 0;                                         // what is above k_high
  if (WEIGHTS) want = 0;
  // of those that equal the floor, only some are there
  const u64 absent = WEIGHTS && floor.tied > floor.ties ? (floor.tied - floor.ties) * weight_of_key(row, floor.cut) : 0;
  for (int level = 0;; ++level) {
    clear_bins(sh, TH, WEIGHTS);
    __syncthreads();
    u64 last = 0;                     // of the last bin, which may hold nearly all tokens
    const float x_low = WEIGHTS ? fmaxf(key_value(k_low), row.floor) : key_value(k_low), x_high = key_value(k_high);
    for (int v = tid; v < g.vecs; v += TH) {
      const uint4 x = g.x[v];
      if (!(V::most(x) >= x_low)) continue;
#pragma unroll
      for (int half = 0; half < V::N; half += 4) {
        uint32_t bin[4];
        u64 w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float l = V::at(x, half + e);
          const bool in = l >= x_low && l <= x_high;
          bin[e] = in ? bins.of(l) : kSampleBins;
          w[e] = !in ? 0 : WEIGHTS ? fixed_weight(weight_value(row, l)) : 1;
          if (bin[e] == kSampleBins - 1) last += w[e];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (bin[e] < kSampleBins - 1) {
            if (WEIGHTS) add_weight(sh, bin[e], w[e]);
            else atomicAdd(&sh.field[0][bin[e]], 1u);
          }
      }
    }
    last = warp_sum(last);
    if (lane == 0) sh.part[0][warp] = last;
    if (tid == 0) sh.listed = sh.listed_above = 0;
    __syncthreads();
    last = 0;
    for (int i = 0; i < TH / 32; ++i) last += sh.part[0][i];
    sum_bins<TH, WEIGHTS>(sh, last);
    g.barrier();
    if (warp == 0) find_bin(g, gone, want, p, absent);
    __syncthreads();
    if (!WEIGHTS && sh.found[0] == ~0ull) {
      g.barrier();              // sums have been read
      return Border{0, 0, 0, 0, false};
    }
    const uint32_t bin = (uint32_t)sh.found[0], from = max(k_low, bins.least_key(bin));
    gone = sh.found[1];
    want = sh.found[2];
    // the bin's tokens if they are not too many, its smallest and largest key, and the tokens above it
    uint32_t hi = 0, lo = 0, none = 0;
    const bool list_above = may_list && level == 0;
    const float x_from = key_value(from);
    for (int v = tid; v < g.vecs; v += TH) {
      const uint4 x = g.x[v];
      if (!(V::most(x) >= x_from)) continue;
#pragma unroll
      for (int e = 0; e < V::N; ++e) {
        const float l = V::at(x, e);
        if (!(l >= x_from && l <= x_high)) continue;
        const uint32_t b = bins.of(l);
        if (b == bin) {
          const uint32_t key = order_key(l), at = atomicAdd(&sh.listed, 1u);
          hi = max(hi, key);
          lo = max(lo, ~key);
          if (at < kGather) sh.list[at] = g.token<T>(l, v, e);
        } else if (b < bin && list_above) {
          const uint32_t at = atomicAdd(&sh.listed_above, 1u);
          if (at < kList) sh.above[at] = g.token<T>(l, v, e);
        }
      }
    }
    uint32_t above, tokens;
    exchange_counts(g, above, tokens);
    if (list_above && above + tokens <= kList) return Border{0, 0, 0, want, true};
    if (tokens <= kGather) {
      copy_lists<TH>(g, false);
      g.barrier();              // lists and sums have been read: each CTA goes on by itself
      return border_of_list<TH, WEIGHTS>(sh, row, (int)tokens, want, gone);
    }
    block_max<TH>(sh, hi, lo);
    exchange_max(g, hi, lo, none);    // its barrier: lists and sums have been read
    k_high = hi;
    k_low = ~lo;
    if (k_low == k_high) {
      const u64 w = WEIGHTS ? weight_of_key(row, k_low) : 1;
      return Border{k_low, (uint32_t)min(w ? (want - gone + w - 1) / w : 1, (u64)tokens), tokens, want, false};
    }
    bins = Bins{0.f, 0.f, k_high, max(0, 32 - __clz(k_high - k_low) - 10)};
  }
}

// what the row's draw is told by
__device__ __forceinline__ u64 draw_at(float u, u64 total) {
  return min((u64)floor(fmin((double)u, 1.0) * (double)total), total - 1);
}
__device__ __forceinline__ void store_token(const SampleParams &P, int r, const Row &row, int token, float logit, u64 total) {
  P.tokens[r] = token;
  if (P.logprobs)
    P.logprobs[r] = (float)(((double)logit - row.top_d) * row.inv_t - log((double)total * (1.0 / 17592186044416.0)));
}

// The row's end where the CTAs' lists hold every token that may be kept, n in all, up to kGather with top-k, else kList: the first
// CTA sorts them, two threads to a token.  most: how many top-k leaves; want: the weight that top-p has to reach, or, with p < 1, its
// share of what top-k leaves.  A barrier has made the lists complete.
template <int TH> __device__ void finish_listed(Group &g, const SampleParams &P, int r, const Row &row, int n, uint32_t most, u64 want, double p, float u) {
  Shared &sh = *g.sh;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (g.rank == 0) copy_lists<TH>(g, true);
  g.barrier();                  // lists have been read
  if (g.rank != 0) return;
  if (n > kList) {
    // exactly `most` are left, of equal ones the first in the vocabulary
    const Border cut = border_of_list<TH, false>(sh, row, n, most, 0);
    if (tid == 0) sh.listed = 0;
    __syncthreads();
    for (int i = tid; i < n; i += TH) {
      const u64 x = sh.all[i];
      if (key_of(x) < cut.cut) continue;
      uint32_t rank = 0;
      if (key_of(x) == cut.cut && cut.tied > cut.ties)
        for (int j = 0; j < n; ++j) rank += key_of(sh.all[j]) == cut.cut && sh.all[j] > x;
      if (key_of(x) > cut.cut || rank < cut.ties) sh.list[atomicAdd(&sh.listed, 1u)] = x;
    }
    __syncthreads();
    n = (int)sh.listed;
    if (tid < n) sh.all[tid] = sh.list[tid];
    __syncthreads();
  }
  static_assert(TH >= 2 * kList, "two threads to a token");
  const int at = tid >> 1;
  u64 mine = at < n ? sh.all[at] : 0;
  int ahead = 0;
  if (at < n)
    for (int i = tid & 1; i < n; i += 2) ahead += sh.all[i] > mine;
  ahead += __shfl_xor_sync(0xffffffffu, ahead, 1);
  if (at < n && !(tid & 1)) sh.list[ahead] = mine;
  __syncthreads();
  // The tokens from the largest down, one to a pair of threads.
  if (tid >= 2 * kList) return;
  const auto meet = [] { asm volatile("bar.sync 1, %0;" ::"n"(2 * kList) : "memory"); };
  const int left = min(n, (int)most), half = tid & 1;
  mine = at < left ? sh.list[at] : 0;
  const float logit = key_value(key_of(mine));
  const double w = at < left && logit >= row.floor ? weight_value(row, logit) : 0.0;
  u64 fixed = half ? 0 : fixed_weight(w);
  u64 upto = warp_upto(fixed), total = 0;
  if (lane == 31) sh.part[0][warp] = upto;
  meet();
  for (int x = 0; x < kList / 16; ++x) {
    if (x < warp) upto += sh.part[0][x];
    total += sh.part[0][x];
  }
  if (p < 1.0) want = max((u64)ceil(p * (double)total), 1ull);
  if (upto - fixed >= want || w < row.min_p) fixed = 0;
  total = warp_sum(fixed);
  if (lane == 0) sh.part[1][warp] = total;
  if (!half) sh.list_w[at] = fixed;
  meet();
  total = 0;
  for (int x = 0; x < kList / 16; ++x) total += sh.part[1][x];
  const u64 target = draw_at(u, total);
  // in the order of the vocabulary: the weight of the tokens before
  const uint32_t index = ~(uint32_t)mine;
  fixed = __shfl_sync(0xffffffffu, fixed, lane & 30);
  u64 before = 0;
  if (fixed)
    for (int i = half; i < left; i += 2)
      if (~(uint32_t)sh.list[i] < index) before += sh.list_w[i];
  before += __shfl_xor_sync(0xffffffffu, before, 1);
  if (!half && before <= target && target < before + fixed) store_token(P, r, row, (int)index, logit, total);
}
// Lists the tokens whose logits are not below `from`.
template <typename T, int TH> __device__ __forceinline__ void list_from(Group &g, float from) {
  using V = Vec<T>;
  Shared &sh = *g.sh;
  for (int v = threadIdx.x; v < g.vecs; v += TH) {
    const uint4 x = g.x[v];
    if (!(V::most(x) >= from)) continue;
#pragma unroll
    for (int e = 0; e < V::N; ++e) {
      const float l = V::at(x, e);
      if (!(l >= from)) continue;
      const uint32_t at = atomicAdd(&sh.listed, 1u);
      if (at < kGather) sh.list[at] = g.token<T>(l, v, e);
    }
  }
}
// A key that at least k of the CTA's tokens reach, from the threads' largest logits, or the least if fewer threads have any; and one
// that `share` of them reach.  They are counted in equal steps down from the CTA's largest, as far as the smallest of them.
template <int TH>
__device__ __forceinline__ void bounds_of_largest(Shared &sh, float own, uint32_t top_key, uint32_t least, uint32_t k, uint32_t share,
                                                  uint32_t &of_k, uint32_t &of_share) {
  const int lane = threadIdx.x & 31;
  const float top = key_value(top_key);
  const Bins bins{top, fminf((kSampleBins - 1) / (top - key_value(~least)), 1e30f), 0, -1};
  clear_bins(sh, TH, false);
  __syncthreads();
  if (own > -INFINITY) atomicAdd(&sh.field[0][bins.of(own)], 1u);
  __syncthreads();
  sum_bins<TH, false>(sh, 0);
  __syncthreads();
  // every warp for itself
  const u64 groups = sh.group[lane], upto = warp_upto(groups);
  const auto reached_by = [&](uint32_t n) -> uint32_t {
    unsigned past = __ballot_sync(0xffffffffu, upto >= n);
    if (!past) return kLeastKey;
    const int grp = __ffs(past) - 1;
    const u64 before = __shfl_sync(0xffffffffu, upto - groups, grp);
    past = __ballot_sync(0xffffffffu, before + warp_upto(sh.sum[grp * 32 + lane]) >= n);
    return bins.least_key(grp * 32 + __ffs(past) - 1);
  };
  of_k = reached_by(k);
  of_share = share == k ? of_k : reached_by(share);
}

template <typename T, int TH>
__global__ void __launch_bounds__(TH, 1024 / TH) sample_kernel(const SampleParams P) {
  using V = Vec<T>;
  pdl_prologue();
  extern __shared__ uint4 stretch_of_row[];
  __shared__ Shared sh;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  Group g;
  g.C = (int)cluster_size();
  g.rank = (int)cluster_ctarank();
  g.x = stretch_of_row;
  g.sh = &sh;
  g.turn = 0;
  const int r = blockIdx.x / g.C;
  g.lo = min(g.rank * P.slice, P.vocab);
  const float temperature = P.temperature ? P.temperature[r] : 1.f;
  const int k = P.top_k ? P.top_k[r] : 0;
  const float top_p = P.top_p ? P.top_p[r] : 1.f;
  float min_p = P.min_p ? P.min_p[r] : 0.f, u = P.u[r];
  if (tid < 64) sh.power[tid] = exp2(tid * (1.0 / 64));
  min_p = min_p > 0.f ? fminf(min_p, 1.f) : 0.f;
  u = u > 0.f ? u : 0.f;
  Row row;
  row.t = temperature;
  row.inv_t = 1.0 / (double)temperature;
  row.per64 = row.inv_t * 92.332482616893656;
  row.min_p = min_p;
  row.power = sh.power;
  const float own = load_logits<T, TH>(g, (const T *)P.logits + (long long)r * P.ld + g.lo, min(g.lo + P.slice, P.vocab) - g.lo);
  if (tid == 0) sh.listed = sh.listed_above = 0;
  const bool greedy = !(temperature > 0.f) || k == 1, few = k > 1 && k <= kList && k < P.vocab;
  uint32_t top_key = order_key(own), least = top_key ? ~top_key : 0, bound = 0, of_share = kLeastKey;      // least: of the threads' largest
  block_max<TH>(sh, top_key, least);
  if (few && !greedy && top_key) bounds_of_largest<TH>(sh, own, top_key, least, k, (k + g.C - 1) / g.C, bound, of_share);
  // Tokens down to one CTA's k-th are enough, and so are those down to the least of all CTAs' shares of k: the higher of the two lists fewer.
  uint32_t share_down = ~of_share;
  exchange_max(g, top_key, share_down, bound);
  bound = max(bound, ~share_down);
  if (top_key == 0 || greedy) {
    // the first token of the largest logit
    const float top = key_value(top_key);
    uint32_t first = 0, none = 0;
    for (int v = tid; v < g.vecs && top_key; v += TH) {
      const uint4 x = g.x[v];
      if (V::most(x) < top) continue;
#pragma unroll
      for (int e = 0; e < V::N; ++e)
        if (V::at(x, e) == top) first = max(first, (uint32_t)g.token<T>(top, v, e));
    }
    block_max<TH>(sh, first, none);
    exchange_max(g, first, none, bound);
    if (g.rank == 0 && tid == 0) {
      P.tokens[r] = top_key ? (int)~first : -1;
      if (P.logprobs) P.logprobs[r] = top_key ? 0.f : -INFINITY;
    }
    g.barrier();                // the others may still read this CTA's exchange
    return;
  }
  const bool infinite = key_value(top_key) == INFINITY;
  if (infinite) {                     // infinite logits have all the weight, in equal shares
    for (int v = tid; v < g.vecs; v += TH) {
      const uint4 x = g.x[v];
      uint4 y = make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int e = 0; e < V::N; ++e) V::put(y, e, V::at(x, e) == INFINITY ? 0.f : -INFINITY);
      g.x[v] = y;
    }
    top_key = 0x80000000u;
    __syncthreads();
  }
  row.top = key_value(top_key);
  row.top_d = row.top;
  // exp(-31.2) is below half of 2^-44.  The bound is rounded down, to a number that may be far below if the next one up is above.
  row.floor = fmaxf(__fsub_rd(row.top, __fmul_ru(31.25f, temperature)), -FLT_MAX);
  while (((double)row.floor - row.top_d) * row.inv_t < -45.0) row.floor = nextafterf(row.floor, INFINITY);
  // logits below this one fall short of min-p for certain
  float least_min = -FLT_MAX;
  if (min_p > 0.f) least_min = fmaxf(row.top + temperature * (__logf(min_p) * 1.000001f - 1e-4f) - fabsf(row.top) * 2e-7f, -FLT_MAX);

  Border cut{0, 0, 0, 0, false};
  uint32_t above, tokens;
  if (few && !infinite) {
    list_from<T, TH>(g, key_value(max(bound, kLeastKey)));
    exchange_counts(g, above, tokens);
    if (tokens <= kGather) {
      finish_listed<TH>(g, P, r, row, (int)tokens, k, ~0ull, top_p < 1.f ? fmax((double)top_p, 0.0) : 1.0, u);
      return;
    }
    g.barrier();                // counts have been read
  }
  if (k > 1 && k < P.vocab) cut = find_border<T, TH, false>(g, row, k, 0.0, cut, false);
  if (top_p < 1.f) {
    cut = find_border<T, TH, true>(g, row, 0, fmax((double)top_p, 0.0), cut, cut.cut == 0);
    if (cut.listed) {
      exchange_counts(g, above, tokens);
      finish_listed<TH>(g, P, r, row, (int)(above + tokens), kList, cut.want, 1.0, u);
      return;
    }
  }

  // Each warp takes a stretch of the slice, a lane a vector at a time; ties are numbered in the order of the vocabulary.
  const int stretch = ((g.vecs + (TH / 32) - 1) / (TH / 32) + 31) & ~31;
  const int v0 = min(warp * stretch, g.vecs), v1 = min(v0 + stretch, g.vecs);
  u64 ties_before = 0;
  const bool some_ties = cut.tied > cut.ties;
  const float x_cut = cut.cut ? key_value(cut.cut) : -FLT_MAX;
  if (some_ties) {
    u64 n = 0, s, before;
    for (int v = v0 + lane; v < v1; v += 32) {
      const uint4 x = g.x[v];
#pragma unroll
      for (int e = 0; e < V::N; ++e) n += V::at(x, e) == x_cut;
    }
    n = warp_sum(n);
    __syncthreads();
    if (lane == 0) sh.part[0][warp] = n;
    __syncthreads();
    n = 0;
    for (int w = 0; w < TH / 32; ++w) {
      n += sh.part[0][w];
      if (w < warp) ties_before += sh.part[0][w];
    }
    exchange_sum(g, n, s, before);
    ties_before += before;
  }
  const float from = fmaxf(fmaxf(x_cut, row.floor), least_min);      // logits below it are not kept, or without weight
  uint32_t ties = (uint32_t)ties_before;      // those before the warp's 32 vectors
  // weights of the lane's vector v, 0 of tokens that are not kept; their sum
  auto weights = [&](int v, u64 (&w)[V::N]) {
    uint4 x = make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u);      // -infinity, or NaN
    if (v < v1) x = g.x[v];
    u64 s = 0;
    uint32_t rank = 0;
    if (some_ties) {
      uint32_t n = 0;
#pragma unroll
      for (int e = 0; e < V::N; ++e) n += V::at(x, e) == x_cut;
      const uint32_t upto = (uint32_t)warp_upto(n);
      rank = ties + upto - n;
      ties += __shfl_sync(0xffffffffu, upto, 31);
    }
#pragma unroll
    for (int e = 0; e < V::N; ++e) w[e] = 0;
    if (V::most(x) >= from) {
#pragma unroll
      for (int e = 0; e < V::N; ++e) {
        const float l = V::at(x, e);
        if (!(l >= from) || (some_ties && l == x_cut && rank++ >= cut.ties)) continue;
        const double value = weight_value(row, l);
        w[e] = value < row.min_p ? 0 : fixed_weight(value);
        s += w[e];
      }
    }
    return s;
  };
  // sums of the warp's 32 vectors at a time stay in shared memory, so that none but those of the drawn token are formed again
  static_assert(kMaxVocab / kMaxCluster / 4 <= kSampleBins * 32, "room for them");
  constexpr int kRounds = kSampleBins / (TH / 32);
  u64 sum = 0, w[V::N];
  for (int v = v0, i = 0; v < v1; v += 32, ++i) {
    const u64 s = warp_sum(weights(v + lane, w));
    if (lane == 0) sh.sum[warp * kRounds + i] = s;
    sum += s;
  }
  __syncthreads();
  if (lane == 0) sh.part[1][warp] = sum;
  __syncthreads();
  u64 ours = 0, before = 0, total, x;
  for (int i = 0; i < TH / 32; ++i) {
    ours += sh.part[1][i];
    if (i < warp) before += sh.part[1][i];
  }
  exchange_sum(g, ours, total, x);
  before += x;
  // the first token at which the running sum is above u times the total
  const u64 target = draw_at(u, total);
  if (before <= target && target < before + sum) {
    int v = v0;
    for (int i = 0; before + sh.sum[warp * kRounds + i] <= target; ++i) {
      before += sh.sum[warp * kRounds + i];
      v += 32;
    }
    ties = (uint32_t)ties_before;
    if (some_ties)
      for (int o = v0; o < v; o += 32) weights(o + lane, w);       // numbers the ties
    const u64 s = weights(v + lane, w), upto = before + warp_upto(s);
    u64 at = upto - s;
    if (at <= target && target < upto) {
#pragma unroll
      for (int e = 0; e < V::N; ++e) {
        if (at <= target && target < at + w[e]) store_token(P, r, row, g.lo + (v + lane) * V::N + e - g.pad, V::at(g.x[v + lane], e), total);
        at += w[e];
      }
    }
  }
  g.barrier();                  // the others may still read this CTA's exchange
}

template <typename T>
templora_status_t launch_sample(SampleParams &p, cudaStream_t st) {
  int sms = 0;
  TL_TRY(stream_sms(st, &sms));
  // Two CTAs per SM keep their logits in shared memory, as far as a row's cluster goes.  More CTAs take a row where a wave still holds
  // all of them (nine tenths of two CTAs per SM: clusters of eight do not fill every group of SMs) and each has some thousand
  // tokens, since a step between CTAs costs as much as passes over that many: 11 rows of 15026, top-k and top-p, 31 us on one CTA a row,
  // 22 on eight; one row of 1000, 4.6 on one, 6.2 on two.  Beyond a wave two CTAs of a row that fill each other's waits do for it
  // (214 rows of 16273: 37 us on one, 34 on two, 41 on four).
  int C = 1;
  while (C < kMaxCluster && p.vocab > C * std::min(kMostBytes / (int)sizeof(T), kMaxVocab / kMaxCluster)) C *= 2;
  while (C < kMaxCluster && (long long)p.rows * C * 2 <= 9 * sms / 5 && p.vocab / (2 * C) >= 2500) C *= 2;
  if (C == 1 && p.vocab >= 16000) C = 2;
  constexpr int N = 16 / sizeof(T);
  p.slice = (p.vocab + C - 1) / C;
  const auto bytes = [](int slice) { return (size_t)((slice + 2 * N - 2) / N) * 16; };      // up to N - 1 places in front
  const dim3 grid((unsigned)(p.rows * C));
  const size_t largest = bytes(kMaxVocab / kMaxCluster);      // of the larger type
  LaunchScope scope(kKindSample, st);
  // a CTA that no other fits beside has all the warps of the SM (16 rows of 180286, fp32: 34 us with half of them, 30 with all); a stretch
  // of bf16 logits always leaves room for another
  if constexpr (kMaxVocab / kMaxCluster * sizeof(T) + 16 > kMostBytes) {
    if (bytes(p.slice) > kMostBytes) {
      TL_TRY((allow_smem<sample_kernel<T, 1024>>(largest)));
      TL_CUDA_CHECK(launch_cluster_pdl(sample_kernel<T, 1024>, grid, dim3(1024), C, bytes(p.slice), st, p));
      return TEMPLORA_OK;
    }
  }
  TL_TRY((allow_smem<sample_kernel<T, 512>>(largest)));
  TL_CUDA_CHECK(launch_cluster_pdl(sample_kernel<T, 512>, grid, dim3(512), C, bytes(p.slice), st, p));
  return TEMPLORA_OK;
}

}  // namespace
}  // namespace templora

using namespace templora;

extern "C" templora_status_t templora_sample(const templora_sample_t *s, int32_t rows, void *stream) {
  if (!s || rows <= 0 || s->vocab <= 0 || !s->logits || !s->u || !s->tokens) return TEMPLORA_ERR_INVALID_ARG;
  if (!word_aligned(s->temperature) || !word_aligned(s->top_k) || !word_aligned(s->top_p) || !word_aligned(s->min_p) || !word_aligned(s->u) ||
      !word_aligned(s->tokens) || !word_aligned(s->logprobs))
    return TEMPLORA_ERR_INVALID_ARG;
  if (s->dtype != TEMPLORA_F32 && s->dtype != TEMPLORA_BF16) return TEMPLORA_ERR_UNSUPPORTED;
  if ((reinterpret_cast<uintptr_t>(s->logits) & (s->dtype == TEMPLORA_F32 ? 3 : 1)) != 0) return TEMPLORA_ERR_INVALID_ARG;
  if (s->vocab > kMaxVocab || rows > (1 << 24)) return TEMPLORA_ERR_UNSUPPORTED;
  const long long ld = s->ld == 0 ? s->vocab : s->ld;
  if (ld < s->vocab || ld > (1ll << 31)) return TEMPLORA_ERR_INVALID_ARG;
  SampleParams p{s->logits, ld, rows, s->vocab, 0, s->temperature, s->top_p, s->min_p, s->u, s->top_k, s->tokens, s->logprobs};
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  return s->dtype == TEMPLORA_F32 ? launch_sample<float>(p, st) : launch_sample<__nv_bfloat16>(p, st);
}
