// Shared by the attention kernels: the parameters of a call, the allowed keys of a query row, the score
// modifications, and the row-by-row forms that never let a masked place touch a result.
#pragma once
#include <atomic>

#include "common.cuh"

namespace templora {

// Masks, score modifications and head layout of one call (a checked copy of templora_attn_t).
struct AttnShape {
  int H, Hkv, group, D;
  int Tq, Tk, q_start;
  int causal, window, n_docs;
  float scale, softcap;
  const float *slopes;
  const int *doc_offsets, *prefix_lens;
};
// Tensors of one call; ld_*: elements between rows.
struct AttnTensors {
  const void *q, *k, *v, *dO;
  void *o, *dq, *dk, *dv;
  float *lse;
  long long ldq, ldk, ldv, ldo, lddo, lddq, lddk, lddv;
};

// Scratch of the backward on the tensor-core path, inside the caller's workspace (attention_tc.cu).
struct AttnBwdScratch {
  float *stat;       // [H][Tq_pad / 128][2][128]: of a tile's rows, -lse (in the kernels' units) and -delta
  int2 *rows;        // [Tq_pad]: allowed keys
  int2 *tiles;       // [Tq_pad / 128]: smallest start and largest end of the tile's rows
  int2 *inner;       // [Tq_pad / 32]: largest start and smallest end of 32 rows: keys that all of them see
  int Tq_pad;
  // dk and dv in parts (by head of a group and by stretch of queries), added up in order afterwards (attn_add_parts)
  float *part_dk, *part_dv;   // [parts][Hkv][Tk][D]
  int head_parts, row_parts;
  // generic kernel: dq in parts (by stretch of keys)
  float *part_dq;             // [key_parts][H][Tq][D]
  int key_parts;
};

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

#ifdef __CUDACC__
// Allowed keys [x, y) of query row i.  Every mask of the library (causal, prefix, window, document) leaves one interval.
// Offsets and prefix lengths come from device memory and are clamped, so no content reads outside [0, Tk).
__device__ __forceinline__ int2 attn_interval(const AttnShape &s, int i) {
  const int p = s.q_start + i;
  int lo = 0, hi = s.Tk, d = 0;
  if (s.n_docs > 0) {
    int a = 0, b = s.n_docs + 1;   // first entry greater than p
    while (a < b) {
      const int m = (a + b) >> 1;
      if (s.doc_offsets[m] <= p) a = m + 1; else b = m;
    }
    d = a - 1;
    if (d < 0 || d >= s.n_docs) return make_int2(0, 0);
    lo = min(max(s.doc_offsets[d], 0), s.Tk);
    hi = min(max(s.doc_offsets[d + 1], lo), s.Tk);
  }
  const int start = lo;
  if (s.causal) {
    int reach = p + 1;
    if (s.prefix_lens) reach = max(reach, start + min(max(s.prefix_lens[d], 0), s.Tk));
    hi = min(hi, reach);
  }
  if (s.window > 0) {
    lo = max(lo, p - s.window + 1);
    if (!s.causal) hi = min(hi, p + s.window);
  }
  return make_int2(lo, max(hi, lo));
}

// tanh(x) = x f(x^2) for |x| <= 0.75, f the least-squares polynomial on Chebyshev nodes weighted for the absolute error: 1.3e-8,
// 8e-8 with fp32 rounding, and relative to tanh as small, which a cap of any size needs.
constexpr float kTanhPolyMax = 0.75f;
constexpr float kTanh0 = 0.999999884f, kTanh1 = -0.333325704f, kTanh2 = 0.133210675f, kTanh3 = -0.0531544633f, kTanh4 = 0.0192263854f,
                kTanh5 = -0.00447591339f;
// A cap beyond this changes no fp32 score that matters, and its products with constants would overflow.
constexpr float kNoCap = 1e37f;

__device__ __forceinline__ float attn_warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

template <typename T> __device__ __forceinline__ float attn_ld(const T *p);
template <> __device__ __forceinline__ float attn_ld<float>(const float *p) { return *p; }
template <> __device__ __forceinline__ float attn_ld<__nv_bfloat16>(const __nv_bfloat16 *p) { return __bfloat162float(*p); }
__device__ __forceinline__ void attn_st(float *p, float v) { *p = v; }
__device__ __forceinline__ void attn_st(__nv_bfloat16 *p, float v) { *p = __float2bfloat16_rn(v); }

// z = score of (row at position p, key j) from the plain product; t = tanh(..) when capped, else 0.
__device__ __forceinline__ float attn_score(const AttnShape &s, float slope, float dot, int p, int j, float &t) {
  float z = dot * s.scale;
  t = 0.f;
  if (s.softcap > 0.f) {
    t = tanhf(z / s.softcap);
    z = t * s.softcap;
  }
  return z - slope * fabsf((float)(p - j));
}

// ------------------------------------------------------------------ row-by-row forms
// A matrix product multiplies masked probabilities (zeros) with whatever the masked rows hold, and 0 * Inf is NaN.  A
// kernel that has stored a non-finite value recomputes that row here, over the allowed keys alone, unless a value that the row
// sees makes those places non-finite: the columns of a result do not mix, so that the stored row is right then.  One warp per row;
// never reached while the inputs are finite.  Asking first matters once a step has gone wrong: a NaN among the first tokens' values is
// seen by every later row, while only rows at a mask's edge share a tile with hidden places.  1800 tokens, 8 / 1 heads of 128 in
// bf16: forward 45 us, backward 61; a NaN in v at token 0 81 and 96 (33 and 92 ms with all rows formed again), at token 900, hidden
// from four rows of its tile, 465 and 436; a NaN in dO of row 0, hidden from the other 127 keys of its tile, 10 ms.
constexpr int kMaxPerLane = 4;   // head_dim <= 128
__device__ __forceinline__ bool attn_finite(float v) { return fabsf(v) < INFINITY; }
// a stored result, past L1: a line there may be older than what a copy has written behind it
__device__ __forceinline__ float attn_stored(const float *p) { return __ldcg(p); }
__device__ __forceinline__ float attn_stored(const __nv_bfloat16 *p) { return __bfloat162float(__ldcg(p)); }

// -lse (times the kernels' scale) and -delta of row i, as the backward's first kernel left them
__device__ __forceinline__ float2 attn_row_stat(const AttnBwdScratch &w, int h, int i) {
  const float *p = w.stat + 2 * ((long long)h * w.Tq_pad + (i & ~127)) + (i & 127);
  return make_float2(p[0], p[128]);
}

// Is every non-finite place of row i's stored o due to what the row sees?  A bad score makes lse NaN, which no hidden place does.
// Else, one open column after another: the first key with a bad value there, 128 keys at a time.
template <typename T>
static __device__ __noinline__ bool attn_fwd_explained(const AttnShape &s, const AttnTensors &x, int h, int i, int2 r) {
  __syncwarp();
  const int lane = threadIdx.x & 31;
  if (isnan(attn_stored(x.lse + (long long)h * s.Tq + i))) return true;
  const T *o = (const T *)x.o + (long long)i * x.ldo + (long long)h * s.D;
  const T *v = (const T *)x.v + (long long)(h / s.group) * s.D;
  bool open[kMaxPerLane], some = false;
#pragma unroll
  for (int e = 0; e < kMaxPerLane; ++e) {
    open[e] = lane + 32 * e < s.D && !attn_finite(attn_stored(o + lane + 32 * e));
    some |= open[e];
  }
  if (!__any_sync(0xffffffffu, some)) return false;
  for (;;) {
    int d = -1, key = -1;
#pragma unroll
    for (int e = 0; e < kMaxPerLane; ++e) {
      const unsigned votes = __ballot_sync(0xffffffffu, open[e]);
      if (d < 0 && votes) d = 32 * e + __ffs(votes) - 1;
    }
    if (d < 0) return true;
    for (int j0 = r.x; j0 < r.y && key < 0; j0 += 128) {
      float at[4];
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        const int j = j0 + 32 * n + lane;
        at[n] = j < r.y ? attn_ld(v + (long long)j * x.ldv + d) : 0.f;
      }
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        const unsigned votes = __ballot_sync(0xffffffffu, !attn_finite(at[n]));
        if (key < 0 && votes) key = j0 + 32 * n + __ffs(votes) - 1;
      }
    }
    if (key < 0) return false;
#pragma unroll
    for (int e = 0; e < kMaxPerLane; ++e)
      if (open[e]) open[e] = attn_finite(attn_ld(v + (long long)key * x.ldv + lane + 32 * e));
  }
}

// The same for key j's stored dk and dv.  A row whose lse is NaN, or whose delta is not finite, brings a bad ds to every place of
// dk; one whose lse is NaN, or dO bad at a place, a bad term to dv there.
template <typename T>
static __device__ __noinline__ bool attn_dkdv_explained(const AttnShape &s, const AttnTensors &x, const AttnBwdScratch &w, int hk, int j) {
  __syncwarp();
  const int lane = threadIdx.x & 31;
  const long long k_at = (long long)j * x.lddk + (long long)hk * s.D, v_at = (long long)j * x.lddv + (long long)hk * s.D;
  bool open[kMaxPerLane], some = false;      // of dv; dk is explained as a whole
#pragma unroll
  for (int e = 0; e < kMaxPerLane; ++e) {
    const int c = lane + 32 * e;
    open[e] = c < s.D && !attn_finite(attn_stored((const T *)x.dv + v_at + c));
    some |= open[e] || (c < s.D && !attn_finite(attn_stored((const T *)x.dk + k_at + c)));
  }
  if (!__any_sync(0xffffffffu, some)) return false;
  for (int i0 = 0; i0 < s.Tq; i0 += 32) {
    int2 r = make_int2(0, 0);
    if (i0 + lane < s.Tq) r = attn_interval(s, i0 + lane);
    const bool sees = r.x <= j && j < r.y;
    if (!__any_sync(0xffffffffu, sees)) continue;
    auto bad_row = [&](int h) {
      const float2 st = attn_row_stat(w, h, i0 + lane);      // (the scratch holds whole tiles of rows)
      return sees && (isnan(st.x) || !attn_finite(st.y));
    };
    bool bad = false;
    for (int h = hk * s.group; h < (hk + 1) * s.group; ++h) bad |= bad_row(h);
    if (!__any_sync(0xffffffffu, bad)) continue;
    for (int h = hk * s.group; h < (hk + 1) * s.group; ++h)
      for (unsigned rows = __ballot_sync(0xffffffffu, bad_row(h)); rows; rows &= rows - 1) {
        const int i = i0 + __ffs(rows) - 1;
        const bool all = isnan(attn_row_stat(w, h, i).x);
        const T *dO = (const T *)x.dO + (long long)i * x.lddo + (long long)h * s.D;
        some = false;
#pragma unroll
        for (int e = 0; e < kMaxPerLane; ++e) {
          if (open[e]) open[e] = !all && attn_finite(attn_ld(dO + lane + 32 * e));
          some |= open[e];
        }
        if (!__any_sync(0xffffffffu, some)) return true;
      }
  }
  return false;
}

// A lane's own row against one that the whole warp reads.  vec: both can be read 16 bytes at a time.
template <typename T>
__device__ __forceinline__ float attn_lane_dot(const T *own, const T *common, int D, bool vec) {
  constexpr int N = 16 / sizeof(T);
  float even = 0.f, odd = 0.f;
  int d = 0;
  if (vec) {
#pragma unroll 4
    for (; d < D; d += N) {
      const uint4 a = *reinterpret_cast<const uint4 *>(own + d), b = *reinterpret_cast<const uint4 *>(common + d);
      const T *pa = reinterpret_cast<const T *>(&a), *pb = reinterpret_cast<const T *>(&b);
#pragma unroll
      for (int n = 0; n < N; n += 2) {
        even = fmaf(attn_ld(pa + n), attn_ld(pb + n), even);
        odd = fmaf(attn_ld(pa + n + 1), attn_ld(pb + n + 1), odd);
      }
    }
    return even + odd;
  }
#pragma unroll 8
  for (; d + 2 <= D; d += 2) {
    even = fmaf(attn_ld(own + d), attn_ld(common + d), even);
    odd = fmaf(attn_ld(own + d + 1), attn_ld(common + d + 1), odd);
  }
  if (d < D) even = fmaf(attn_ld(own + d), attn_ld(common + d), even);
  return even + odd;
}
// sum += weights of `lanes` times the rows that these lanes stand for, `row` + lane * ld; a lane adds up dims lane + 32 e.  Four
// rows in flight (more cost the kernels registers); rows of other lanes are not read.
template <typename T>
__device__ __forceinline__ void attn_lane_sum(float (&sum)[kMaxPerLane], float weight, unsigned lanes, const T *row, long long ld, int D) {
  const int lane = threadIdx.x & 31;
  constexpr int kAhead = 4;
#pragma unroll 1
  for (int n0 = 0; n0 < 32; n0 += kAhead) {
    float at[kAhead][kMaxPerLane];
#pragma unroll
    for (int n = 0; n < kAhead; ++n)
#pragma unroll
      for (int e = 0; e < kMaxPerLane; ++e)
        at[n][e] = (lanes >> (n0 + n) & 1) && lane + 32 * e < D ? attn_ld(row + (n0 + n) * ld + lane + 32 * e) : 0.f;
#pragma unroll
    for (int n = 0; n < kAhead; ++n) {
      const float w = __shfl_sync(0xffffffffu, weight, n0 + n);
      if (lanes >> (n0 + n) & 1)
#pragma unroll
        for (int e = 0; e < kMaxPerLane; ++e) sum[e] = fmaf(w, at[n][e], sum[e]);
    }
  }
}
template <typename T> __device__ __forceinline__ bool attn_vec(int D, long long ld_a, long long ld_b) {
  return ((D | ld_a | ld_b) & (16 / (int)sizeof(T) - 1)) == 0;
}
// Rows of a tile whose bits are set in four words, dealt to n_warps warps.
template <typename F> __device__ __forceinline__ void attn_each_bad_row(const unsigned *words, int warp, int n_warps, F redo) {
  int n = 0;
  for (int w = 0; w < 4; ++w)
    for (unsigned rows = words[w]; rows; rows &= rows - 1)
      if (n++ % n_warps == warp) redo(32 * w + __ffs(rows) - 1);
}
__device__ __forceinline__ unsigned attn_first_lanes(int n) { return n >= 32 ? 0xffffffffu : (1u << n) - 1u; }

// o and lse of row i of head h, 32 keys at a time, one to a lane
template <typename T>
static __device__ __noinline__ void attn_exact_fwd_row(const AttnShape &s, const AttnTensors &x, int h, int i) {
  const int lane = threadIdx.x & 31, hk = h / s.group, p = s.q_start + i;
  const int2 r = attn_interval(s, i);
  if (attn_fwd_explained<T>(s, x, h, i, r)) return;
  const float slope = s.slopes ? s.slopes[h] : 0.f;
  const T *q = (const T *)x.q + (long long)i * x.ldq + (long long)h * s.D;
  const bool vec = attn_vec<T>(s.D, x.ldq, x.ldk);
  float acc[kMaxPerLane] = {}, m = -INFINITY, l = 0.f;
  for (int j0 = r.x; j0 < r.y; j0 += 32) {
    const int j = j0 + lane;
    const T *v = (const T *)x.v + (long long)j0 * x.ldv + (long long)hk * s.D;
    float z = -INFINITY, t;
    if (j < r.y) z = attn_score(s, slope, attn_lane_dot((const T *)x.k + (long long)j * x.ldk + (long long)hk * s.D, q, s.D, vec), p, j, t);
    float mn = z;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mn = fmaxf(mn, __shfl_xor_sync(0xffffffffu, mn, o));
    mn = fmaxf(m, mn);
    const float a = (m == mn) ? 1.f : expf(m - mn), w = (z == -INFINITY) ? 0.f : expf(z - mn);
    l = l * a + attn_warp_sum(w);
#pragma unroll
    for (int e = 0; e < kMaxPerLane; ++e) acc[e] *= a;
    attn_lane_sum(acc, w, attn_first_lanes(r.y - j0), v, x.ldv, s.D);
    m = mn;
  }
  T *o = (T *)x.o + (long long)i * x.ldo + (long long)h * s.D;
#pragma unroll
  for (int e = 0; e < kMaxPerLane; ++e)
    if (lane + 32 * e < s.D) attn_st(o + lane + 32 * e, r.x < r.y ? acc[e] / l : 0.f);
  if (lane == 0) x.lse[(long long)h * s.Tq + i] = r.x < r.y ? m + logf(l) : -INFINITY;
}

// dq of row i of head h.  With lse NaN or a delta that is not finite every ds of the row is bad, and so every place of dq, as it is
// stored: the forward has brought a bad value that the row sees into one of the two.
template <typename T>
static __device__ __noinline__ void attn_exact_dq_row(const AttnShape &s, const AttnTensors &x, int h, int i) {
  __syncwarp();
  const int lane = threadIdx.x & 31, hk = h / s.group, p = s.q_start + i;
  const int2 r = attn_interval(s, i);
  const float slope = s.slopes ? s.slopes[h] : 0.f;
  const long long at = (long long)h * s.D;
  const T *q = (const T *)x.q + (long long)i * x.ldq + at, *dO = (const T *)x.dO + (long long)i * x.lddo + at;
  const bool vec = attn_vec<T>(s.D, x.ldq, x.ldk), vec_o = attn_vec<T>(s.D, x.lddo, x.ldv);
  float acc[kMaxPerLane] = {}, delta = 0.f;
#pragma unroll
  for (int e = 0; e < kMaxPerLane; ++e)
    if (lane + 32 * e < s.D) delta += attn_ld(dO + lane + 32 * e) * attn_ld((const T *)x.o + (long long)i * x.ldo + at + lane + 32 * e);
  delta = attn_warp_sum(delta);
  const float lse = x.lse[(long long)h * s.Tq + i];
  if (r.x < r.y && (isnan(lse) || !attn_finite(delta))) return;
  for (int j0 = r.x; j0 < r.y; j0 += 32) {
    const int j = j0 + lane;
    float ds = 0.f, t;
    if (j < r.y) {
      const float z = attn_score(s, slope, attn_lane_dot((const T *)x.k + (long long)j * x.ldk + (long long)hk * s.D, q, s.D, vec), p, j, t);
      const float dp = attn_lane_dot((const T *)x.v + (long long)j * x.ldv + (long long)hk * s.D, dO, s.D, vec_o);
      ds = expf(z - lse) * (dp - delta) * (1.f - t * t) * s.scale;
    }
    attn_lane_sum(acc, ds, attn_first_lanes(r.y - j0), (const T *)x.k + (long long)j0 * x.ldk + (long long)hk * s.D, x.ldk, s.D);
  }
#pragma unroll
  for (int e = 0; e < kMaxPerLane; ++e)
    if (lane + 32 * e < s.D) attn_st((T *)x.dq + (long long)i * x.lddq + at + lane + 32 * e, acc[e]);
}

// dk and dv of key j of kv head hk, 32 rows of a head at a time
template <typename T>
static __device__ __noinline__ void attn_exact_dkdv_row(const AttnShape &s, const AttnTensors &x, const AttnBwdScratch &w, int hk, int j) {
  if (attn_dkdv_explained<T>(s, x, w, hk, j)) return;
  const int lane = threadIdx.x & 31;
  const T *k = (const T *)x.k + (long long)j * x.ldk + (long long)hk * s.D, *v = (const T *)x.v + (long long)j * x.ldv + (long long)hk * s.D;
  const bool vec = attn_vec<T>(s.D, x.ldq, x.ldk), vec_o = attn_vec<T>(s.D, x.lddo, x.ldv);
  float dk[kMaxPerLane] = {}, dv[kMaxPerLane] = {};
  for (int i0 = 0; i0 < s.Tq; i0 += 32) {
    const int i = i0 + lane;
    int2 r = make_int2(0, 0);
    if (i < s.Tq) r = attn_interval(s, i);
    const bool sees = r.x <= j && j < r.y;
    const unsigned rows = __ballot_sync(0xffffffffu, sees);
    if (!rows) continue;
    for (int h = hk * s.group; h < (hk + 1) * s.group; ++h) {
      const T *q = (const T *)x.q + (long long)i0 * x.ldq + (long long)h * s.D, *dO = (const T *)x.dO + (long long)i0 * x.lddo + (long long)h * s.D;
      float pr = 0.f, ds = 0.f, t;
      if (sees) {
        const float z = attn_score(s, s.slopes ? s.slopes[h] : 0.f, attn_lane_dot(q + lane * x.ldq, k, s.D, vec), s.q_start + i, j, t);
        pr = expf(z - x.lse[(long long)h * s.Tq + i]);
        ds = pr * (attn_lane_dot(dO + lane * x.lddo, v, s.D, vec_o) + attn_row_stat(w, h, i).y) * (1.f - t * t) * s.scale;
      }
      attn_lane_sum(dk, ds, rows, q, x.ldq, s.D);
      attn_lane_sum(dv, pr, rows, dO, x.lddo, s.D);
    }
  }
#pragma unroll
  for (int e = 0; e < kMaxPerLane; ++e) {
    const int c = lane + 32 * e;
    if (c >= s.D) continue;
    attn_st((T *)x.dk + (long long)j * x.lddk + (long long)hk * s.D + c, dk[e]);
    attn_st((T *)x.dv + (long long)j * x.lddv + (long long)hk * s.D + c, dv[e]);
  }
}
#endif  // __CUDACC__

#ifdef __CUDACC__
// Lets a kernel use `bytes` of dynamic shared memory (the same number in every call); asked once per device.
template <auto Kernel> templora_status_t allow_smem(size_t bytes) {
  static std::atomic<uint64_t> done{0};
  int dev = 0;
  TL_CUDA_CHECK(cudaGetDevice(&dev));
  if (dev < 64 && ((done.load(std::memory_order_relaxed) >> dev) & 1)) return TEMPLORA_OK;
  TL_CUDA_CHECK(cudaFuncSetAttribute(Kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
  if (dev < 64) done.fetch_or(1ull << dev, std::memory_order_relaxed);
  return TEMPLORA_OK;
}
#endif
// SMs of the current device, at most the cap of the stream (templora_set_stream_sm_limit)
templora_status_t stream_sms(cudaStream_t st, int *sms);

// tensor-core kernels (attention_tc.cu): bf16, head_dim and row strides multiples of 8
bool attn_tc_available();
// Partial results of the forward where several CTAs share the keys of a few rows, inside the caller's workspace
struct AttnFwdParts {
  int n;             // 1: none
  float *o;          // [n][H][Tq][D]
  float2 *ml;        // [n][H][Tq]: maximum (in units of log2 on the tensor-core path) and sum
};
templora_status_t attn_join_parts(const AttnShape &s, const AttnTensors &x, const AttnFwdParts &parts, cudaStream_t st);   // of the tensor-core path
templora_status_t attn_tc_fwd(const AttnShape &s, const AttnTensors &x, const AttnFwdParts &parts, DeviceStatus *status, cudaStream_t st);
templora_status_t attn_tc_bwd(const AttnShape &s, const AttnTensors &x, const AttnBwdScratch &w, DeviceStatus *status,
                              cudaStream_t st);
// kernels for every type and layout (attention.cu)
templora_status_t attn_simt_fwd(const AttnShape &s, const AttnTensors &x, const AttnFwdParts &parts, int dtype, cudaStream_t st);
templora_status_t attn_add_parts(const AttnShape &s, const AttnTensors &x, const AttnBwdScratch &w, int dtype, cudaStream_t st);

// fp32 and int32 arrays that are read word by word
inline bool word_aligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3) == 0; }
// checks of a templora_attn_t that involve neither lengths nor tensors (attention.cu)
templora_status_t attn_check_desc(const templora_attn_t *a);

}  // namespace templora
