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
// kernel that finds a non-finite value in a result it is about to store recomputes that row here, over the allowed
// keys alone.  One warp per row; slow, and never reached while the inputs are finite.
constexpr int kMaxPerLane = 4;   // head_dim <= 128

template <typename T>
static __device__ __noinline__ void attn_exact_fwd_row(const AttnShape &s, const AttnTensors &x, int h, int i) {
  const int lane = threadIdx.x & 31, hk = h / s.group, p = s.q_start + i;
  const int2 r = attn_interval(s, i);
  const float slope = s.slopes ? s.slopes[h] : 0.f;
  const T *q = (const T *)x.q + (long long)i * x.ldq + (long long)h * s.D;
  float acc[kMaxPerLane] = {}, qv[kMaxPerLane], m = -INFINITY, l = 0.f;
#pragma unroll
  for (int e = 0; e < kMaxPerLane; ++e) qv[e] = lane + 32 * e < s.D ? attn_ld(q + lane + 32 * e) : 0.f;
  for (int j = r.x; j < r.y; ++j) {
    const T *k = (const T *)x.k + (long long)j * x.ldk + (long long)hk * s.D;
    const T *v = (const T *)x.v + (long long)j * x.ldv + (long long)hk * s.D;
    float dot = 0.f, t;
#pragma unroll
    for (int e = 0; e < kMaxPerLane; ++e) if (lane + 32 * e < s.D) dot = fmaf(qv[e], attn_ld(k + lane + 32 * e), dot);
    const float z = attn_score(s, slope, attn_warp_sum(dot), p, j, t);
    const float mn = fmaxf(m, z), a = (m == mn) ? 1.f : expf(m - mn), w = (z == -INFINITY) ? 0.f : expf(z - mn);
    l = l * a + w;
#pragma unroll
    for (int e = 0; e < kMaxPerLane; ++e)
      if (lane + 32 * e < s.D) acc[e] = acc[e] * a + w * attn_ld(v + lane + 32 * e);
    m = mn;
  }
  T *o = (T *)x.o + (long long)i * x.ldo + (long long)h * s.D;
#pragma unroll
  for (int e = 0; e < kMaxPerLane; ++e)
    if (lane + 32 * e < s.D) attn_st(o + lane + 32 * e, r.x < r.y ? acc[e] / l : 0.f);
  if (lane == 0) x.lse[(long long)h * s.Tq + i] = r.x < r.y ? m + logf(l) : -INFINITY;
}

// dq of row i of head h
template <typename T>
static __device__ __noinline__ void attn_exact_dq_row(const AttnShape &s, const AttnTensors &x, int h, int i) {
  const int lane = threadIdx.x & 31, hk = h / s.group, p = s.q_start + i;
  const int2 r = attn_interval(s, i);
  const float slope = s.slopes ? s.slopes[h] : 0.f;
  const long long at = (long long)h * s.D;
  float qv[kMaxPerLane], dov[kMaxPerLane], acc[kMaxPerLane] = {}, delta = 0.f;
#pragma unroll
  for (int e = 0; e < kMaxPerLane; ++e) {
    const int c = lane + 32 * e;
    qv[e] = dov[e] = 0.f;
    if (c >= s.D) continue;
    qv[e] = attn_ld((const T *)x.q + (long long)i * x.ldq + at + c);
    dov[e] = attn_ld((const T *)x.dO + (long long)i * x.lddo + at + c);
    delta += dov[e] * attn_ld((const T *)x.o + (long long)i * x.ldo + at + c);
  }
  delta = attn_warp_sum(delta);
  const float lse = x.lse[(long long)h * s.Tq + i];
  for (int j = r.x; j < r.y; ++j) {
    const T *k = (const T *)x.k + (long long)j * x.ldk + (long long)hk * s.D;
    const T *v = (const T *)x.v + (long long)j * x.ldv + (long long)hk * s.D;
    float dot = 0.f, dp = 0.f, t;
#pragma unroll
    for (int e = 0; e < kMaxPerLane; ++e)
      if (lane + 32 * e < s.D) {
        dot = fmaf(qv[e], attn_ld(k + lane + 32 * e), dot);
        dp = fmaf(dov[e], attn_ld(v + lane + 32 * e), dp);
      }
    const float z = attn_score(s, slope, attn_warp_sum(dot), p, j, t);
    const float ds = expf(z - lse) * (attn_warp_sum(dp) - delta) * (1.f - t * t) * s.scale;
#pragma unroll
    for (int e = 0; e < kMaxPerLane; ++e) if (lane + 32 * e < s.D) acc[e] = fmaf(ds, attn_ld(k + lane + 32 * e), acc[e]);
  }
#pragma unroll
  for (int e = 0; e < kMaxPerLane; ++e)
    if (lane + 32 * e < s.D) attn_st((T *)x.dq + (long long)i * x.lddq + at + lane + 32 * e, acc[e]);
}

// dk and dv of key j of kv head hk
template <typename T>
static __device__ __noinline__ void attn_exact_dkdv_row(const AttnShape &s, const AttnTensors &x, int hk, int j) {
  const int lane = threadIdx.x & 31;
  float kv[kMaxPerLane], vv[kMaxPerLane], dk[kMaxPerLane] = {}, dv[kMaxPerLane] = {};
#pragma unroll
  for (int e = 0; e < kMaxPerLane; ++e) {
    const int c = lane + 32 * e;
    kv[e] = c < s.D ? attn_ld((const T *)x.k + (long long)j * x.ldk + (long long)hk * s.D + c) : 0.f;
    vv[e] = c < s.D ? attn_ld((const T *)x.v + (long long)j * x.ldv + (long long)hk * s.D + c) : 0.f;
  }
  for (int i0 = 0; i0 < s.Tq; i0 += 32) {
    int2 r = make_int2(0, 0);
    if (i0 + lane < s.Tq) r = attn_interval(s, i0 + lane);
    unsigned rows = __ballot_sync(0xffffffffu, r.x <= j && j < r.y);
    while (rows) {
      const int i = i0 + __ffs(rows) - 1;
      rows &= rows - 1;
      for (int h = hk * s.group; h < (hk + 1) * s.group; ++h) {
        const long long at = (long long)h * s.D;
        float qv[kMaxPerLane], dov[kMaxPerLane], dot = 0.f, dp = 0.f, delta = 0.f, t;
#pragma unroll
        for (int e = 0; e < kMaxPerLane; ++e) {
          const int c = lane + 32 * e;
          qv[e] = dov[e] = 0.f;
          if (c >= s.D) continue;
          qv[e] = attn_ld((const T *)x.q + (long long)i * x.ldq + at + c);
          dov[e] = attn_ld((const T *)x.dO + (long long)i * x.lddo + at + c);
          dot = fmaf(qv[e], kv[e], dot);
          dp = fmaf(dov[e], vv[e], dp);
          delta = fmaf(dov[e], attn_ld((const T *)x.o + (long long)i * x.ldo + at + c), delta);
        }
        const float z = attn_score(s, s.slopes ? s.slopes[h] : 0.f, attn_warp_sum(dot), s.q_start + i, j, t);
        const float pr = expf(z - x.lse[(long long)h * s.Tq + i]);
        const float ds = pr * (attn_warp_sum(dp) - attn_warp_sum(delta)) * (1.f - t * t) * s.scale;
#pragma unroll
        for (int e = 0; e < kMaxPerLane; ++e) {
          dk[e] = fmaf(ds, qv[e], dk[e]);
          dv[e] = fmaf(pr, dov[e], dv[e]);
        }
      }
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
