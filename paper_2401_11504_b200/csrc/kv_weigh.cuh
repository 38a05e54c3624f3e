// Shared by the kernels that add up the weights of cached tokens: a call's parameters, what each sequence asks for, and a weight.
#pragma once
#include "cluster.cuh"
#include "kv_cache.cuh"

#include <algorithm>

namespace templora {

struct WeighParams {
  CacheView c;
  const void *q;
  const float *lse, *slopes;
  float *weights;
  const int *offsets;                 // nullptr: one row per sequence
  long long ldq, lse_row, lse_head;
  int n_rows, group, window;
  float scale, softcap, cap_in;       // cap_in: 1 / softcap
};

// ------------------------------------------------------------------ what a sequence asks for
struct SeqRows { int len, first_row, rows, base; };      // base: first place looked at, a multiple of 16
__device__ __forceinline__ SeqRows seq_rows(const WeighParams &P, int s) {
  SeqRows r;
  r.len = P.c.seq_lens[s];
  r.first_row = s;
  r.rows = 1;
  if (P.offsets) {
    r.first_row = min(max(P.offsets[s], 0), P.n_rows);
    r.rows = max(min(P.offsets[s + 1], P.n_rows) - r.first_row, 0);
  }
  if (r.len < 0 || (long long)r.len > (long long)P.c.max_blocks * P.c.bt) {
    report(P.c.status, kWhereLength);
    r.len = 0;
  }
  r.base = P.window > 0 ? (int)max((long long)r.len - r.rows - P.window + 1, 0ll) & ~15 : 0;
  return r;
}
// before[s]: tiles of `tile` places, times kv heads, of the sequences before s.  Whole block; before has n_seqs + 1 entries.
__device__ __forceinline__ void count_tiles(const WeighParams &P, int tile, long long *before, int threads) {
  const int tid = threadIdx.x, n = P.c.n_seqs;
  for (int s = tid; s < n; s += threads) {
    const SeqRows r = seq_rows(P, s);
    before[s + 1] = r.rows > 0 ? (long long)((r.len - r.base + tile - 1) / tile) * P.c.Hkv : 0;
  }
  if (tid == 0) before[0] = 0;
  __syncthreads();
  if (tid < 32) {
    long long sum = 0;
    for (int s0 = 0; s0 < n; s0 += 32) {
      long long v = s0 + tid < n ? before[s0 + tid + 1] : 0;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const long long u = __shfl_up_sync(0xffffffffu, v, o);
        if (tid >= o) v += u;
      }
      if (s0 + tid < n) before[s0 + tid + 1] = sum + v;
      sum += __shfl_sync(0xffffffffu, v, 31);
    }
  }
  __syncthreads();
}
// The same by one warp for up to 32 sequences, into an array of its own: neither a barrier nor a second warp to wait for.
__device__ __forceinline__ void count_tiles_of_few(const WeighParams &P, int tile, long long *before) {
  const int lane = threadIdx.x & 31, n = P.c.n_seqs;
  long long v = 0;
  if (lane < n) {
    const SeqRows r = seq_rows(P, lane);
    if (r.rows > 0) v = (long long)((r.len - r.base + tile - 1) / tile) * P.c.Hkv;
  }
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long u = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += u;
  }
  if (lane == 0) before[0] = 0;
  if (lane < n) before[lane + 1] = v;
  __syncwarp();
}
// last sequence with before[s] <= at; a whole warp
__device__ __forceinline__ int find_seq(const long long *before, int n, long long at) {
  int a = 0, b = n;
  while (b - a > 32) {
    const int m = (a + b) >> 1;
    if (before[m] <= at) a = m; else b = m;
  }
  const int s = a + (threadIdx.x & 31);
  return a + 31 - __clz(__ballot_sync(0xffffffffu, s < b && before[s] <= at));
}

// ------------------------------------------------------------------ a weight
// log of the softmax's sum; +infinity for a row (or a column that is none) that counts for nothing
__device__ __forceinline__ float load_lse(const WeighParams &P, int row, int head, bool there) {
  const float v = there ? P.lse[row * P.lse_row + head * P.lse_head] : INFINITY;
  return v == -INFINITY ? INFINITY : v;
}
__device__ __forceinline__ uint64_t pack_f2(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 unpack_f2(uint64_t v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ uint64_t fma_f2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t mul_f2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t add_f2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// exp(z - lse).  Uncapped scores are subtracted in one fused step from the product, so that a weight's relative error is
// 2^-24 |z - lse| whatever z is.  tanh as in the decode step's attention: relative to its value, by a polynomial near 0.
__device__ __forceinline__ float weight_of(const WeighParams &P, float s, float f, float lse, float slope, int back) {
  float t;
  if (P.softcap > 0.f) {
    const float x = s * f * P.cap_in, u = x * x;
    t = x * fmaf(u, fmaf(u, fmaf(u, fmaf(u, fmaf(u, kTanh5, kTanh4), kTanh3), kTanh2), kTanh1), kTanh0);
    if (!(fabsf(x) <= kTanhPolyMax)) t = fmaf(-2.f, __fdividef(1.f, 1.f + ex2(x * (2.f * kLog2e))), 1.f);
    t = fmaf(t, P.softcap, -lse);
  } else {
    t = fmaf(s, f, -lse);
  }
  t = fmaf(-slope, (float)back, t);
  return lse == INFINITY ? 0.f : ex2(t * kLog2e);
}
// The same two numbers at a time, where there is more to compute than to load.  (In the decode step's kernel it took registers that
// it lacks: 58724 tokens, 32 heads of 64, 36.6 us with one at a time, 38.8 with two.)
__device__ __forceinline__ uint64_t tanh_f2(uint64_t x) {
  const auto both = [](float v) { return pack_f2(v, v); };
  const uint64_t u = mul_f2(x, x);
  uint64_t p = fma_f2(u, both(kTanh5), both(kTanh4));
  p = fma_f2(u, p, both(kTanh3));
  p = fma_f2(u, p, both(kTanh2));
  p = fma_f2(u, p, both(kTanh1));
  p = mul_f2(x, fma_f2(u, p, both(kTanh0)));
  const float2 v = unpack_f2(x);
  if (fmaxf(fabsf(v.x), fabsf(v.y)) > kTanhPolyMax) {
    float2 t = unpack_f2(p);
    const auto far = [](float z) { return fmaf(-2.f, __fdividef(1.f, 1.f + ex2(z * (2.f * kLog2e))), 1.f); };
    if (fabsf(v.x) > kTanhPolyMax) t.x = far(v.x);
    if (fabsf(v.y) > kTanhPolyMax) t.y = far(v.y);
    p = pack_f2(t.x, t.y);
  }
  return p;
}

// of a row for the scores of two places, `back` and back - 8 behind it
__device__ __forceinline__ uint64_t weights_of(const WeighParams &P, float s0, float s1, float f, float lse, float slope, int back) {
  const uint64_t f2 = pack_f2(f, f), nlse = pack_f2(-lse, -lse);
  uint64_t t = pack_f2(s0, s1);
  if (P.softcap > 0.f) t = fma_f2(tanh_f2(mul_f2(mul_f2(t, f2), pack_f2(P.cap_in, P.cap_in))), pack_f2(P.softcap, P.softcap), nlse);
  else t = fma_f2(t, f2, nlse);
  if (P.slopes) t = fma_f2(pack_f2(-slope, -slope), pack_f2((float)back, (float)(back - 8)), t);
  const float2 x = unpack_f2(mul_f2(t, pack_f2(kLog2e, kLog2e)));
  return lse == INFINITY ? 0 : pack_f2(ex2(x.x), ex2(x.y));
}
// a product's unit times the block's scale, finite so that a zero product stays zero
__device__ __forceinline__ float finite_unit(float unit, float ks) { return fminf(fmaxf(unit * ks, -3e38f), 3e38f); }


// Where items are few, a cluster of CTAs takes one and deals out its pairs, `stages` portions of them, and its first CTA adds up their
// sums: how many CTAs.  places: of an item.  Five sequences of 1996 tokens, 16 / 1 heads, 80 rows under a window of 67: 53 us on one CTA an
// item, 17 on eight.
inline int weigh_cluster(const WeighParams &p, int places, long long stages, int sms) {
  // places that any row may see
  const long long table = (long long)p.c.max_blocks * p.c.bt;
  const long long seen = p.window > 0 ? std::min<long long>(table, (long long)p.window + p.n_rows / p.c.n_seqs + p.c.bt) : table;
  const long long items = (long long)p.c.n_seqs * p.c.Hkv * ((seen + places - 1) / places);
  int S = 1;
  while (S < kMaxCluster && items * S * 2 <= 9 * sms / 5 && stages >= 2 * S) S *= 2;
  return S;
}

bool weigh_tc_available(const WeighParams &p, int dtype);      // the tensor-core kernel handles this call, and is worth it
size_t weigh_tc_terms(int heads, int dim, int n_rows, int n_seqs, int group);      // bytes that it takes for fp32 queries, or 0
templora_status_t weigh_tc(const WeighParams &p, int dtype, void *terms, cudaStream_t st);

}  // namespace templora
