// Attention of a chunk: entry points, argument checks, the backward's row statistics, and the kernels for every type
// and layout (fp32, and bf16 shapes the tensor-core kernels do not take).  attention_tc.cu has the tensor-core forms.
#include "attention.cuh"
#include "tc_host.h"

#include <algorithm>

namespace templora {
namespace {

// ------------------------------------------------------------------ generic kernels
// 256 threads as a 16 x 16 grid; a tile is TL rows by TL columns (64, or 32 where 64 would leave SMs without a CTA), thread
// (ty, tx) owns rows ty + 16 a and columns tx + 16 b, so that 16-byte shared-memory reads along head_dim hit different banks
// (row pitch D + 4 words: eight neighbouring lanes start four words apart).  At TL = 64 a thread reads 8 vectors per four
// values of head_dim for 64 FMAs; the kernels are bound by the fp32 pipes and shared memory, and on small calls by the
// latency of a tile, which the smaller one quarters.  fp32, 32 heads over 8 kv heads of 128, 1500 tokens, causal: forward 745 us
// (25 TFLOP/s), backward 2.5 ms (18); 17 queries behind 79 tokens, 4 heads of 64: 10 us.
constexpr int kSimtThreads = 256;
constexpr int kVisitBits = 8192;      // query tiles whose reach the dk, dv kernel keeps a bit for
template <int DM> constexpr int kPitch = DM + 4;
template <int TL> constexpr int kPitchP = TL + 4;

// Rows [row0, row0 + TL) of one head, zero outside [0, n_rows) and behind head_dim, as fp32 in shared memory: fetch() requests
// them, put() stores them.  With 32-row tiles a step's tiles are fetched a step ahead (a step is about as long as a round
// trip to memory); 64-row tiles would take too many registers for that, and their steps are long.
template <typename T, int DM, int TL> struct TileCopy {
  static constexpr int N = 16 / sizeof(T), kVecs = TL * DM / N, kPer = (kVecs + kSimtThreads - 1) / kSimtThreads;
  static constexpr bool kAhead = TL == 32;
  uint4 v[kPer];
  __device__ __forceinline__ void fetch(const T *src, long long ld, int row0, int n_rows, int D, bool vec) {
    if (!vec) return;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int e = threadIdx.x + i * kSimtThreads, r = e / (DM / N), c = (e % (DM / N)) * N;
      v[i] = (e < kVecs && row0 + r >= 0 && row0 + r < n_rows && c < D)
                 ? *reinterpret_cast<const uint4 *>(src + (long long)(row0 + r) * ld + c) : make_uint4(0, 0, 0, 0);
    }
  }
  __device__ __forceinline__ void put(float *dst, const T *src, long long ld, int row0, int n_rows, int D, bool vec) {
    if (vec) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int e = threadIdx.x + i * kSimtThreads, r = e / (DM / N), c = (e % (DM / N)) * N;
        if (e >= kVecs) break;
        const T *x = reinterpret_cast<const T *>(&v[i]);
#pragma unroll
        for (int k = 0; k < N; k += 4)
          *reinterpret_cast<float4 *>(dst + r * kPitch<DM> + c + k) =
              make_float4(attn_ld(x + k), attn_ld(x + k + 1), attn_ld(x + k + 2), attn_ld(x + k + 3));
      }
    } else {
      for (int e = threadIdx.x; e < TL * DM; e += kSimtThreads) {
        const int r = e / DM, c = e % DM;
        dst[r * kPitch<DM> + c] = (row0 + r >= 0 && row0 + r < n_rows && c < D) ? attn_ld(src + (long long)(row0 + r) * ld + c) : 0.f;
      }
    }
  }
  __device__ __forceinline__ void load(float *dst, const T *src, long long ld, int row0, int n_rows, int D, bool vec) {
    fetch(src, ld, row0, n_rows, D, vec);
    put(dst, src, ld, row0, n_rows, D, vec);
  }
};

// acc[a][b] = sum_d X[ty + 16 a][d] Y[tx + 16 b][d]
template <int DM, int TL>
__device__ __forceinline__ void dot_tile(float (&acc)[TL / 16][TL / 16], const float *X, const float *Y, int ty, int tx) {
  constexpr int NA = TL / 16;
#pragma unroll
  for (int a = 0; a < NA; ++a)
#pragma unroll
    for (int b = 0; b < NA; ++b) acc[a][b] = 0.f;
#pragma unroll 4
  for (int d = 0; d < DM; d += 4) {
    float4 xa[NA], yb[NA];
#pragma unroll
    for (int a = 0; a < NA; ++a) xa[a] = *reinterpret_cast<const float4 *>(X + (ty + 16 * a) * kPitch<DM> + d);
#pragma unroll
    for (int b = 0; b < NA; ++b) yb[b] = *reinterpret_cast<const float4 *>(Y + (tx + 16 * b) * kPitch<DM> + d);
#pragma unroll
    for (int a = 0; a < NA; ++a)
#pragma unroll
      for (int b = 0; b < NA; ++b) {
        acc[a][b] = fmaf(xa[a].x, yb[b].x, acc[a][b]);
        acc[a][b] = fmaf(xa[a].y, yb[b].y, acc[a][b]);
        acc[a][b] = fmaf(xa[a].z, yb[b].z, acc[a][b]);
        acc[a][b] = fmaf(xa[a].w, yb[b].w, acc[a][b]);
      }
  }
}

// out[a][4 c + e] += sum_j W[ty + 16 a][j] Y[j][64 c + 4 tx + e]
template <int DM, int TL>
__device__ __forceinline__ void weighted_sum(float (&out)[TL / 16][DM / 16], const float *W, const float *Y, int ty, int tx) {
  constexpr int NA = TL / 16;
#pragma unroll 2
  for (int j = 0; j < TL; j += 4) {
    float4 w[NA];
#pragma unroll
    for (int a = 0; a < NA; ++a) w[a] = *reinterpret_cast<const float4 *>(W + (ty + 16 * a) * kPitchP<TL> + j);
#pragma unroll
    for (int jj = 0; jj < 4; ++jj)
#pragma unroll
      for (int c = 0; c < DM / 64; ++c) {
        const float4 y = *reinterpret_cast<const float4 *>(Y + (j + jj) * kPitch<DM> + 64 * c + 4 * tx);
#pragma unroll
        for (int a = 0; a < NA; ++a) {
          const float f = jj == 0 ? w[a].x : jj == 1 ? w[a].y : jj == 2 ? w[a].z : w[a].w;
          out[a][4 * c] = fmaf(f, y.x, out[a][4 * c]);
          out[a][4 * c + 1] = fmaf(f, y.y, out[a][4 * c + 1]);
          out[a][4 * c + 2] = fmaf(f, y.z, out[a][4 * c + 2]);
          out[a][4 * c + 3] = fmaf(f, y.w, out[a][4 * c + 3]);
        }
      }
  }
}

// smallest start and largest end of the allowed keys of rows [row0, row0 + TL); every thread gets them
template <int TL>
__device__ __forceinline__ int2 tile_range(const AttnShape &s, int row0, int2 *rows) {
  __shared__ int range[2];
  if (threadIdx.x == 0) { range[0] = s.Tk; range[1] = 0; }
  __syncthreads();
  if (threadIdx.x < TL) {
    const int2 r = row0 + threadIdx.x < s.Tq ? attn_interval(s, row0 + threadIdx.x) : make_int2(0, 0);
    rows[threadIdx.x] = r;
    if (r.x < r.y) {
      atomicMin(&range[0], r.x);
      atomicMax(&range[1], r.y);
    }
  }
  __syncthreads();
  return make_int2(range[0], range[1]);
}

// This CTA's stretch of a tile's keys, in steps of TL.  PARTS: several CTAs share them (kernels of their own: 17 queries, 10.8 us with
// both forms in one, 10.2 without).
template <int TL, bool PARTS> __device__ __forceinline__ int2 key_stretch(int2 range) {
  if (!PARTS || range.y <= range.x) return range;
  const int steps = (range.y - range.x + TL - 1) / TL;
  const int a = (int)((long long)steps * blockIdx.z / gridDim.z), b = (int)((long long)steps * (blockIdx.z + 1) / gridDim.z);
  return make_int2(range.x + a * TL, min(range.y, range.x + b * TL));
}

template <typename T, int DM, int TL, bool PARTS>
__global__ void __launch_bounds__(kSimtThreads) attn_simt_fwd_kernel(const AttnShape s, const AttnTensors x, const AttnFwdParts parts) {
  pdl_prologue();
  constexpr int N = 16 / sizeof(T);
  const bool vec = ((s.D | x.ldq | x.ldk | x.ldv | x.lddo) & (N - 1)) == 0;      // (the forward's lddo is 0)
  extern __shared__ __align__(16) float sm[];
  float *Q = sm, *KV = Q + TL * kPitch<DM>, *P = KV + TL * kPitch<DM>;
  __shared__ int2 rows[TL];
  const int h = blockIdx.y, hk = h / s.group, q0 = (gridDim.x - 1 - blockIdx.x) * TL;      // a causal call's longest rows first
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const int2 range = key_stretch<TL, PARTS>(tile_range<TL>(s, q0, rows));
  const T *ks = (const T *)x.k + (long long)hk * s.D, *vs = (const T *)x.v + (long long)hk * s.D;
  using Copy = TileCopy<T, DM, TL>;
  Copy ck, cv;
  ck.fetch(ks, x.ldk, range.x, range.y, s.D, vec && Copy::kAhead);
  cv.fetch(vs, x.ldv, range.x, range.y, s.D, vec && Copy::kAhead);
  { Copy cq; cq.load(Q, (const T *)x.q + (long long)h * s.D, x.ldq, q0, s.Tq, s.D, vec); }
  const float slope = s.slopes ? s.slopes[h] : 0.f;
  float m[TL / 16], l[TL / 16], acc[TL / 16][DM / 16];
#pragma unroll
  for (int a = 0; a < TL / 16; ++a) {
    m[a] = -INFINITY; l[a] = 0.f;
#pragma unroll
    for (int c = 0; c < DM / 16; ++c) acc[a][c] = 0.f;
  }
  for (int k0 = range.x; k0 < range.y; k0 += TL) {
    __syncthreads();
    if (!Copy::kAhead) ck.fetch(ks, x.ldk, k0, range.y, s.D, vec);
    ck.put(KV, ks, x.ldk, k0, range.y, s.D, vec);
    __syncthreads();
    if (Copy::kAhead) ck.fetch(ks, x.ldk, k0 + TL, range.y, s.D, vec);
    float sc[TL / 16][TL / 16];
    dot_tile<DM, TL>(sc, Q, KV, ty, tx);
#pragma unroll
    for (int a = 0; a < TL / 16; ++a) {
      const int2 r = rows[ty + 16 * a];
      float mx = -INFINITY, t;
#pragma unroll
      for (int b = 0; b < TL / 16; ++b) {
        const int j = k0 + tx + 16 * b;
        sc[a][b] = (j >= r.x && j < r.y) ? attn_score(s, slope, sc[a][b], s.q_start + q0 + ty + 16 * a, j, t) : -INFINITY;
        mx = fmaxf(mx, sc[a][b]);
      }
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
      const float mn = fmaxf(m[a], mx), base = mn == -INFINITY ? 0.f : mn;
      const float alpha = expf(m[a] - base);
      float sum = 0.f;
#pragma unroll
      for (int b = 0; b < TL / 16; ++b) {
        const float w = expf(sc[a][b] - base);
        sum += w;
        P[(ty + 16 * a) * kPitchP<TL> + tx + 16 * b] = w;
      }
      l[a] = l[a] * alpha + sum;
      m[a] = mn;
#pragma unroll
      for (int c = 0; c < DM / 16; ++c) acc[a][c] *= alpha;
    }
    __syncthreads();
    if (!Copy::kAhead) cv.fetch(vs, x.ldv, k0, range.y, s.D, vec);
    cv.put(KV, vs, x.ldv, k0, range.y, s.D, vec);
    __syncthreads();
    if (Copy::kAhead) cv.fetch(vs, x.ldv, k0 + TL, range.y, s.D, vec);
    weighted_sum<DM, TL>(acc, P, KV, ty, tx);
  }
  bool redo[TL / 16];
#pragma unroll
  for (int a = 0; a < TL / 16; ++a) {
    const int i = q0 + ty + 16 * a;
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) l[a] += __shfl_xor_sync(0xffffffffu, l[a], o);
    if constexpr (PARTS) {
      const long long at = ((long long)blockIdx.z * s.H + h) * s.Tq + i;
      if (i < s.Tq && tx == 0) parts.ml[at] = make_float2(m[a], l[a]);
#pragma unroll
      for (int c = 0; c < DM / 16; ++c) {
        const int d = 64 * (c / 4) + 4 * tx + (c & 3);
        if (i < s.Tq && d < s.D) parts.o[at * s.D + d] = acc[a][c];
      }
      redo[a] = false;
      continue;
    }
    const float inv = l[a] == 0.f ? 0.f : 1.f / l[a];
    bool bad = !(l[a] < INFINITY);
    T *o = (T *)x.o + (long long)i * x.ldo + (long long)h * s.D;
#pragma unroll
    for (int c = 0; c < DM / 16; ++c) {
      const int d = 64 * (c / 4) + 4 * tx + (c & 3);
      const float v = acc[a][c] * inv;
      bad |= !(fabsf(v) < INFINITY) && d < s.D;
      if (i < s.Tq && d < s.D) attn_st(o + d, v);
    }
    if (i < s.Tq && tx == 0) x.lse[(long long)h * s.Tq + i] = l[a] == 0.f ? -INFINITY : m[a] + logf(l[a]);
    redo[a] = bad && i < s.Tq;
  }
  // non-finite rows again, over their allowed keys alone (each half of a warp holds one row)
  __syncwarp();
#pragma unroll
  for (int a = 0; a < TL / 16; ++a) {
    const unsigned votes = __ballot_sync(0xffffffffu, redo[a]);
    const int base = q0 + (ty & ~1) + 16 * a;
    if (votes & 0xffffu) attn_exact_fwd_row<T>(s, x, h, base);
    if (votes >> 16) attn_exact_fwd_row<T>(s, x, h, base + 1);
  }
}

// One step of the backward on a 64 x 64 tile of scores: from sc = q.k and dp = dO.v the weights P and ds (without scale).
__device__ __forceinline__ void bwd_weights(const AttnShape &s, float slope, float sc, float dp, int i, int j, int2 r,
                                            float2 stat, float &p, float &ds) {   // stat: -lse, -delta
  p = ds = 0.f;
  if (j < r.x || j >= r.y) return;
  float t;
  const float z = attn_score(s, slope, sc, s.q_start + i, j, t);
  p = expf(z + stat.x);
  ds = p * (dp + stat.y) * (1.f - t * t);
}

// dk, dv of a tile of keys: loops over the heads that share it and over the query tiles that reach it, or over its part of both
template <typename T, int DM, int TL>
__global__ void __launch_bounds__(kSimtThreads) attn_simt_dkdv_kernel(const AttnShape s, const AttnTensors x,
                                                                      const __grid_constant__ AttnBwdScratch w) {
  pdl_prologue();
  constexpr int N = 16 / sizeof(T);
  const bool vec = ((s.D | x.ldq | x.ldk | x.ldv | x.lddo) & (N - 1)) == 0;
  extern __shared__ __align__(16) float sm[];
  constexpr int kT = TL * kPitch<DM>;
  float *K = sm, *V = K + kT, *Q = V + kT, *DO = Q + kT, *P = DO + kT, *DS = P + TL * kPitchP<TL>;
  __shared__ int2 rows[TL];
  __shared__ float2 stat[TL];
  const int hk = blockIdx.y, k0 = blockIdx.x * TL;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  // query tiles with a row that sees one of these keys (a warp looks at one tile); those behind the last bit are all visited
  __shared__ unsigned active[kVisitBits / 32];
  const int n_qt = (s.Tq + TL - 1) / TL, n_bits = min(n_qt, kVisitBits);
  for (int i = threadIdx.x; i < kVisitBits / 32; i += kSimtThreads) active[i] = 0;
  __syncthreads();
  for (int t = threadIdx.x >> 5; t < n_bits; t += kSimtThreads / 32) {
    const int2 reach = w.tiles[t * TL / 128];
    if (reach.x >= k0 + TL || reach.y <= k0) continue;
    bool on = false;
    for (int i = threadIdx.x & 31; i < TL; i += 32) {
      const int2 r = w.rows[t * TL + i];
      on |= r.x < k0 + TL && r.y > k0 && r.x < r.y;
    }
    if (__any_sync(0xffffffffu, on) && (threadIdx.x & 31) == 0) atomicOr(&active[t >> 5], 1u << (t & 31));
  }
  using Copy = TileCopy<T, DM, TL>;
  {
    Copy c;
    c.load(K, (const T *)x.k + (long long)hk * s.D, x.ldk, k0, s.Tk, s.D, vec);
    c.load(V, (const T *)x.v + (long long)hk * s.D, x.ldv, k0, s.Tk, s.D, vec);
  }
  __syncthreads();
  // the steps: query tiles of the first head, then of the next
  const int t_begin = (int)((long long)n_qt * (blockIdx.z / w.head_parts) / w.row_parts);
  const int t_end = (int)((long long)n_qt * (blockIdx.z / w.head_parts + 1) / w.row_parts);
  auto next_step = [&](int &h, int &t) {
    for (++t;; ++t) {
      if (t >= t_end) {
        if ((h += w.head_parts) >= (hk + 1) * s.group) return false;
        t = t_begin;
        if (t >= t_end) return false;
      }
      if (t >= n_bits) return true;
      const unsigned word = active[t >> 5] >> (t & 31);
      if (word & 1) return true;
      if (word == 0) t |= 31;
    }
  };
  float dk[TL / 16][DM / 16], dv[TL / 16][DM / 16];
#pragma unroll
  for (int a = 0; a < TL / 16; ++a)
#pragma unroll
    for (int c = 0; c < DM / 16; ++c) dk[a][c] = dv[a][c] = 0.f;
  Copy cq, co;
  int h = hk * s.group + (int)(blockIdx.z % w.head_parts), t = t_begin - 1;
  bool more = next_step(h, t);
  auto fetch = [&]() {
    cq.fetch((const T *)x.q + (long long)h * s.D, x.ldq, t * TL, s.Tq, s.D, vec);
    co.fetch((const T *)x.dO + (long long)h * s.D, x.lddo, t * TL, s.Tq, s.D, vec);
  };
  if (Copy::kAhead && more) fetch();
  while (more) {
    {
      const int q0 = t * TL;
      const float slope = s.slopes ? s.slopes[h] : 0.f;
      __syncthreads();
      if (!Copy::kAhead) fetch();
      cq.put(Q, (const T *)x.q + (long long)h * s.D, x.ldq, q0, s.Tq, s.D, vec);
      co.put(DO, (const T *)x.dO + (long long)h * s.D, x.lddo, q0, s.Tq, s.D, vec);
      if (threadIdx.x < TL) {
        rows[threadIdx.x] = w.rows[q0 + threadIdx.x];
        stat[threadIdx.x] = attn_row_stat(w, h, q0 + threadIdx.x);
      }
      __syncthreads();
      more = next_step(h, t);
      if (Copy::kAhead && more) fetch();
      float sc[TL / 16][TL / 16], dp[TL / 16][TL / 16];
      dot_tile<DM, TL>(sc, K, Q, ty, tx);    // rows: keys, columns: queries
      dot_tile<DM, TL>(dp, V, DO, ty, tx);
#pragma unroll
      for (int a = 0; a < TL / 16; ++a)
#pragma unroll
        for (int b = 0; b < TL / 16; ++b) {
          const int i = tx + 16 * b;
          float p, ds;
          bwd_weights(s, slope, sc[a][b], dp[a][b], q0 + i, k0 + ty + 16 * a, rows[i], stat[i], p, ds);
          P[(ty + 16 * a) * kPitchP<TL> + i] = p;
          DS[(ty + 16 * a) * kPitchP<TL> + i] = ds;
        }
      __syncthreads();
      weighted_sum<DM, TL>(dv, P, DO, ty, tx);
      weighted_sum<DM, TL>(dk, DS, Q, ty, tx);
    }
  }
  if (gridDim.z > 1) {
    const long long at = ((long long)blockIdx.z * s.Hkv + hk) * s.Tk;
#pragma unroll
    for (int a = 0; a < TL / 16; ++a) {
      const int j = k0 + ty + 16 * a;
#pragma unroll
      for (int c = 0; c < DM / 16; ++c) {
        const int d = 64 * (c / 4) + 4 * tx + (c & 3);
        if (d >= s.D || j >= s.Tk) continue;
        w.part_dk[(at + j) * s.D + d] = dk[a][c] * s.scale;
        w.part_dv[(at + j) * s.D + d] = dv[a][c];
      }
    }
    return;
  }
  bool redo[TL / 16];
#pragma unroll
  for (int a = 0; a < TL / 16; ++a) {
    const int j = k0 + ty + 16 * a;
    bool bad = false;
#pragma unroll
    for (int c = 0; c < DM / 16; ++c) {
      const int d = 64 * (c / 4) + 4 * tx + (c & 3);
      const float gk = dk[a][c] * s.scale;
      if (d >= s.D || j >= s.Tk) continue;
      bad |= !(fabsf(gk) < INFINITY) || !(fabsf(dv[a][c]) < INFINITY);
      attn_st((T *)x.dk + (long long)j * x.lddk + (long long)hk * s.D + d, gk);
      attn_st((T *)x.dv + (long long)j * x.lddv + (long long)hk * s.D + d, dv[a][c]);
    }
    redo[a] = bad;
  }
  __syncwarp();
#pragma unroll
  for (int a = 0; a < TL / 16; ++a) {
    const unsigned votes = __ballot_sync(0xffffffffu, redo[a]);
    const int base = k0 + (ty & ~1) + 16 * a;
    if (votes & 0xffffu) attn_exact_dkdv_row<T>(s, x, w, hk, base);
    if (votes >> 16) attn_exact_dkdv_row<T>(s, x, w, hk, base + 1);
  }
}

// adds the parts up, in order: one warp per key and head
template <typename T>
__global__ void __launch_bounds__(kSimtThreads) attn_add_parts_kernel(const AttnShape s, const AttnTensors x,
                                                                           const __grid_constant__ AttnBwdScratch w) {
  pdl_prologue();
  const long long row = (long long)blockIdx.x * (kSimtThreads / 32) + (threadIdx.x >> 5);     // hk * Tk + j
  if (row >= (long long)s.Hkv * s.Tk) return;
  const int lane = threadIdx.x & 31, hk = (int)(row / s.Tk), j = (int)(row % s.Tk), parts = w.head_parts * w.row_parts;
  bool bad = false;
#pragma unroll
  for (int e = 0; e < kMaxPerLane; ++e) {
    const int d = lane + 32 * e;
    if (d >= s.D) continue;
    float gk = 0.f, gv = 0.f;
    for (int p = 0; p < parts; ++p) {
      const long long at = ((long long)p * s.Hkv * s.Tk + row) * s.D + d;
      gk += w.part_dk[at];
      gv += w.part_dv[at];
    }
    bad |= !(fabsf(gk) < INFINITY) || !(fabsf(gv) < INFINITY);
    attn_st((T *)x.dk + (long long)j * x.lddk + (long long)hk * s.D + d, gk);
    attn_st((T *)x.dv + (long long)j * x.lddv + (long long)hk * s.D + d, gv);
  }
  if (__any_sync(0xffffffffu, bad)) attn_exact_dkdv_row<T>(s, x, w, hk, j);
}

// the same for dq: one warp per row and head
template <typename T>
__global__ void __launch_bounds__(kSimtThreads) attn_add_dq_parts_kernel(const AttnShape s, const AttnTensors x, const AttnBwdScratch w) {
  pdl_prologue();
  const long long rows = (long long)s.H * s.Tq, row = (long long)blockIdx.x * (kSimtThreads / 32) + (threadIdx.x >> 5);   // h * Tq + i
  if (row >= rows) return;
  const int lane = threadIdx.x & 31, h = (int)(row / s.Tq), i = (int)(row % s.Tq);
  bool bad = false;
#pragma unroll
  for (int e = 0; e < kMaxPerLane; ++e) {
    const int d = lane + 32 * e;
    if (d >= s.D) continue;
    float g = 0.f;
    for (int p = 0; p < w.key_parts; ++p) g += w.part_dq[(p * rows + row) * s.D + d];
    bad |= !(fabsf(g) < INFINITY);
    attn_st((T *)x.dq + (long long)i * x.lddq + (long long)h * s.D + d, g);
  }
  if (__any_sync(0xffffffffu, bad)) attn_exact_dq_row<T>(s, x, h, i);
}

template <typename T, int DM, int TL, bool PARTS>
__global__ void __launch_bounds__(kSimtThreads) attn_simt_dq_kernel(const AttnShape s, const AttnTensors x,
                                                                    const AttnBwdScratch w) {
  pdl_prologue();
  constexpr int N = 16 / sizeof(T);
  const bool vec = ((s.D | x.ldq | x.ldk | x.ldv | x.lddo) & (N - 1)) == 0;
  extern __shared__ __align__(16) float sm[];
  constexpr int kT = TL * kPitch<DM>;
  float *Q = sm, *DO = Q + kT, *K = DO + kT, *V = K + kT, *DS = V + kT;
  __shared__ int2 rows[TL];
  __shared__ float2 stat[TL];
  const int h = blockIdx.y, hk = h / s.group, q0 = (gridDim.x - 1 - blockIdx.x) * TL;      // a causal call's longest rows first
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const float slope = s.slopes ? s.slopes[h] : 0.f;
  const int2 range = key_stretch<TL, PARTS>(tile_range<TL>(s, q0, rows));
  const T *ks = (const T *)x.k + (long long)hk * s.D, *vs = (const T *)x.v + (long long)hk * s.D;
  using Copy = TileCopy<T, DM, TL>;
  Copy ck, cv;
  ck.fetch(ks, x.ldk, range.x, range.y, s.D, vec && Copy::kAhead);
  cv.fetch(vs, x.ldv, range.x, range.y, s.D, vec && Copy::kAhead);
  {
    Copy c;
    c.load(Q, (const T *)x.q + (long long)h * s.D, x.ldq, q0, s.Tq, s.D, vec);
    c.load(DO, (const T *)x.dO + (long long)h * s.D, x.lddo, q0, s.Tq, s.D, vec);
  }
  if (threadIdx.x < TL) stat[threadIdx.x] = attn_row_stat(w, h, q0 + threadIdx.x);
  float dq[TL / 16][DM / 16];
#pragma unroll
  for (int a = 0; a < TL / 16; ++a)
#pragma unroll
    for (int c = 0; c < DM / 16; ++c) dq[a][c] = 0.f;
  for (int k0 = range.x; k0 < range.y; k0 += TL) {
    __syncthreads();
    if (!Copy::kAhead) {
      ck.fetch(ks, x.ldk, k0, range.y, s.D, vec);
      cv.fetch(vs, x.ldv, k0, range.y, s.D, vec);
    }
    ck.put(K, ks, x.ldk, k0, range.y, s.D, vec);
    cv.put(V, vs, x.ldv, k0, range.y, s.D, vec);
    __syncthreads();
    if (Copy::kAhead) {
      ck.fetch(ks, x.ldk, k0 + TL, range.y, s.D, vec);
      cv.fetch(vs, x.ldv, k0 + TL, range.y, s.D, vec);
    }
    float sc[TL / 16][TL / 16], dp[TL / 16][TL / 16];
    dot_tile<DM, TL>(sc, Q, K, ty, tx);
    dot_tile<DM, TL>(dp, DO, V, ty, tx);
#pragma unroll
    for (int a = 0; a < TL / 16; ++a)
#pragma unroll
      for (int b = 0; b < TL / 16; ++b) {
        const int i = ty + 16 * a;
        float p, ds;
        bwd_weights(s, slope, sc[a][b], dp[a][b], q0 + i, k0 + tx + 16 * b, rows[i], stat[i], p, ds);
        DS[i * kPitchP<TL> + tx + 16 * b] = ds;
      }
    __syncthreads();
    weighted_sum<DM, TL>(dq, DS, K, ty, tx);
  }
  bool redo[TL / 16];
#pragma unroll
  for (int a = 0; a < TL / 16; ++a) {
    const int i = q0 + ty + 16 * a;
    bool bad = false;
#pragma unroll
    for (int c = 0; c < DM / 16; ++c) {
      const int d = 64 * (c / 4) + 4 * tx + (c & 3);
      const float g = dq[a][c] * s.scale;
      if (d >= s.D || i >= s.Tq) continue;
      if constexpr (PARTS) {
        w.part_dq[(((long long)blockIdx.z * s.H + h) * s.Tq + i) * s.D + d] = g;
        continue;
      }
      bad |= !(fabsf(g) < INFINITY);
      attn_st((T *)x.dq + (long long)i * x.lddq + (long long)h * s.D + d, g);
    }
    redo[a] = bad;
  }
  __syncwarp();
#pragma unroll
  for (int a = 0; a < TL / 16; ++a) {
    const unsigned votes = __ballot_sync(0xffffffffu, redo[a]);
    const int base = q0 + (ty & ~1) + 16 * a;
    if (votes & 0xffffu) attn_exact_dq_row<T>(s, x, h, base);
    if (votes >> 16) attn_exact_dq_row<T>(s, x, h, base + 1);
  }
}

// ------------------------------------------------------------------ row statistics of the backward
// Eight lanes per row: delta = dO . o, 16 bytes per lane and load.  stat = -lse * lse_scale and -delta.  Rows behind Tq
// get lse = +infinity (their probabilities come out 0) and an empty interval.  Blocks of head 0 also write the rows'
// intervals and their tiles'.  Bound by HBM (o and dO read once) on long calls, by the latency of one read on short ones:
// every row of a tile is asked for at once.  (1024 tokens, 32 heads of 128 in bf16, with the kernels behind it: 62.5 us,
// and 66.6 with a quarter of the rows at a time.)
constexpr int kPrepRows = 128, kPrepThreads = 8 * kPrepRows;
template <typename T>
__global__ void __launch_bounds__(kPrepThreads) attn_bwd_prep_kernel(const AttnShape s, const AttnTensors x, const AttnBwdScratch w,
                                                            float lse_scale) {
  pdl_prologue();
  constexpr int N = 16 / sizeof(T);
  const int h = blockIdx.y, row0 = blockIdx.x * kPrepRows, sub = threadIdx.x & 7;
  const bool vec = ((s.D | x.lddo | x.ldo) & (N - 1)) == 0;
  float *stat = w.stat + 2 * ((long long)h * w.Tq_pad + row0);
  const int r = threadIdx.x >> 3, i = row0 + r;
  const float lse = i < s.Tq ? x.lse[(long long)h * s.Tq + i] : 0.f;
  float delta = 0.f;
  if (i < s.Tq) {
    const T *a = (const T *)x.dO + (long long)i * x.lddo + (long long)h * s.D;
    const T *b = (const T *)x.o + (long long)i * x.ldo + (long long)h * s.D;
    if (vec) {
#pragma unroll
      for (int n = 0; n < 128 / (8 * N); ++n) {
        const int c = (n * 8 + sub) * N;
        if (c < s.D) {
          const uint4 va = *reinterpret_cast<const uint4 *>(a + c), vb = *reinterpret_cast<const uint4 *>(b + c);
          const T *pa = reinterpret_cast<const T *>(&va), *pb = reinterpret_cast<const T *>(&vb);
#pragma unroll
          for (int e = 0; e < N; ++e) delta = fmaf(attn_ld(pa + e), attn_ld(pb + e), delta);
        }
      }
    } else {
      for (int c = sub; c < s.D; c += 8) delta = fmaf(attn_ld(a + c), attn_ld(b + c), delta);
    }
  }
#pragma unroll
  for (int o = 1; o < 8; o <<= 1) delta += __shfl_xor_sync(0xffffffffu, delta, o);
  if (sub == 0) {
    stat[r] = i < s.Tq ? -lse * lse_scale : -INFINITY;
    stat[kPrepRows + r] = i < s.Tq ? -delta : 0.f;
  }
  if (h != 0) return;
  __shared__ int range[2];
  if (threadIdx.x == 0) { range[0] = s.Tk; range[1] = 0; }
  __syncthreads();
  if (threadIdx.x < kPrepRows) {
    const int i = row0 + threadIdx.x;
    const bool in = i < s.Tq;           // rows behind the last have no weight anyway
    const int2 r = in ? attn_interval(s, i) : make_int2(0, 0);
    w.rows[i] = r;
    const bool some = r.x < r.y;
    const int lo = __reduce_min_sync(0xffffffffu, some ? r.x : s.Tk), hi = __reduce_max_sync(0xffffffffu, some ? r.y : 0);
    const int a = __reduce_max_sync(0xffffffffu, in ? r.x : 0), b = __reduce_min_sync(0xffffffffu, in ? r.y : s.Tk);
    if ((threadIdx.x & 31) == 0) {
      atomicMin(&range[0], lo);
      atomicMax(&range[1], hi);
      w.inner[i >> 5] = make_int2(a, b);
    }
  }
  __syncthreads();
  if (threadIdx.x == 0) w.tiles[blockIdx.x] = make_int2(range[0], range[1]);
}

// ------------------------------------------------------------------ rows whose keys several CTAs shared
// One warp per row and head: the parts' sums, weighted by their maxima, in order.  A part that saw no key of the row (sum 0) has
// written no values.  LOG2: maxima in units of log2.
template <typename T, bool LOG2>
__global__ void __launch_bounds__(kSimtThreads) attn_join_parts_kernel(const AttnShape s, const AttnTensors x, const AttnFwdParts parts) {
  pdl_prologue();
  const long long rows = (long long)s.H * s.Tq, row = (long long)blockIdx.x * (kSimtThreads / 32) + (threadIdx.x >> 5);   // h * Tq + i
  if (row >= rows) return;
  const int lane = threadIdx.x & 31, h = (int)(row / s.Tq), i = (int)(row % s.Tq);
  float top = -INFINITY;
  for (int p = 0; p < parts.n; ++p) {
    const float2 ml = parts.ml[p * rows + row];
    if (ml.y != 0.f) top = fmaxf(top, ml.x);
  }
  float sum = 0.f, acc[kMaxPerLane] = {};
  for (int p = 0; p < parts.n; ++p) {
    const float2 ml = parts.ml[p * rows + row];
    if (ml.y == 0.f) continue;
    const float a = LOG2 ? exp2f(ml.x - top) : expf(ml.x - top);
    sum = fmaf(a, ml.y, sum);
#pragma unroll
    for (int e = 0; e < kMaxPerLane; ++e)
      if (lane + 32 * e < s.D) acc[e] = fmaf(a, parts.o[(p * rows + row) * s.D + lane + 32 * e], acc[e]);
  }
  bool bad = !(sum < INFINITY);
#pragma unroll
  for (int e = 0; e < kMaxPerLane; ++e) {
    if (lane + 32 * e >= s.D) continue;
    const float v = sum == 0.f ? 0.f : acc[e] / sum;
    bad |= !(fabsf(v) < INFINITY);
    attn_st((T *)x.o + (long long)i * x.ldo + (long long)h * s.D + lane + 32 * e, v);
  }
  if (lane == 0) x.lse[row] = sum == 0.f ? -INFINITY : LOG2 ? (top + log2f(sum)) * kLn2 : top + logf(sum);
  if (__any_sync(0xffffffffu, bad)) attn_exact_fwd_row<T>(s, x, h, i);
}

template <typename T, bool LOG2>
templora_status_t join_parts(const AttnShape &s, const AttnTensors &x, const AttnFwdParts &parts, cudaStream_t st) {
  LaunchScope scope(kKindAttention, st);
  const long long rows = (long long)s.H * s.Tq, per = kSimtThreads / 32;
  TL_CUDA_CHECK(launch_pdl(attn_join_parts_kernel<T, LOG2>, dim3((unsigned)((rows + per - 1) / per)), dim3(kSimtThreads), 0, st, s, x,
                           parts));
  return TEMPLORA_OK;
}
template <typename T, int DM, int TL, bool PARTS>
templora_status_t simt_fwd(const AttnShape &s, const AttnTensors &x, const AttnFwdParts &parts, cudaStream_t st) {
  const size_t smem = (2 * TL * kPitch<DM> + TL * kPitchP<TL>) * sizeof(float);
  TL_TRY((allow_smem<attn_simt_fwd_kernel<T, DM, TL, PARTS>>(smem)));
  LaunchScope scope(kKindAttention, st);
  TL_CUDA_CHECK(launch_pdl(attn_simt_fwd_kernel<T, DM, TL, PARTS>, dim3((s.Tq + TL - 1) / TL, s.H, parts.n), dim3(kSimtThreads), smem, st,
                           s, x, parts));
  return TEMPLORA_OK;
}
template <typename T, int DM, int TL>
templora_status_t simt_fwd(const AttnShape &s, const AttnTensors &x, const AttnFwdParts &parts, cudaStream_t st) {
  if (parts.n == 1) return simt_fwd<T, DM, TL, false>(s, x, parts, st);
  TL_TRY((simt_fwd<T, DM, TL, true>(s, x, parts, st)));
  return join_parts<T, false>(s, x, parts, st);
}
template <typename T>
templora_status_t add_parts(const AttnShape &s, const AttnTensors &x, const AttnBwdScratch &w, cudaStream_t st) {
  LaunchScope scope(kKindAttention, st);
  const long long rows = (long long)s.Hkv * s.Tk, per = kSimtThreads / 32;
  TL_CUDA_CHECK(launch_pdl(attn_add_parts_kernel<T>, dim3((unsigned)((rows + per - 1) / per)), dim3(kSimtThreads), 0, st, s, x, w));
  return TEMPLORA_OK;
}
template <typename T, int DM, int TL>
templora_status_t simt_dkdv(const AttnShape &s, const AttnTensors &x, const AttnBwdScratch &w, cudaStream_t st) {
  const size_t smem = (4 * TL * kPitch<DM> + 2 * TL * kPitchP<TL>) * sizeof(float);
  TL_TRY((allow_smem<attn_simt_dkdv_kernel<T, DM, TL>>(smem)));
  const int parts = w.head_parts * w.row_parts;
  {
    LaunchScope scope(kKindAttention, st);
    TL_CUDA_CHECK(launch_pdl(attn_simt_dkdv_kernel<T, DM, TL>, dim3((s.Tk + TL - 1) / TL, s.Hkv, parts), dim3(kSimtThreads), smem, st,
                             s, x, w));
  }
  return parts == 1 ? TEMPLORA_OK : add_parts<T>(s, x, w, st);
}
template <typename T, int DM, int TL, bool PARTS>
templora_status_t simt_dq(const AttnShape &s, const AttnTensors &x, const AttnBwdScratch &w, cudaStream_t st) {
  const size_t smem = (4 * TL * kPitch<DM> + TL * kPitchP<TL>) * sizeof(float);
  TL_TRY((allow_smem<attn_simt_dq_kernel<T, DM, TL, PARTS>>(smem)));
  LaunchScope scope(kKindAttention, st);
  TL_CUDA_CHECK(launch_pdl(attn_simt_dq_kernel<T, DM, TL, PARTS>, dim3((s.Tq + TL - 1) / TL, s.H, w.key_parts), dim3(kSimtThreads), smem,
                           st, s, x, w));
  return TEMPLORA_OK;
}
template <typename T, int DM, int TL>
templora_status_t simt_dq(const AttnShape &s, const AttnTensors &x, const AttnBwdScratch &w, cudaStream_t st) {
  if (w.key_parts == 1) return simt_dq<T, DM, TL, false>(s, x, w, st);
  TL_TRY((simt_dq<T, DM, TL, true>(s, x, w, st)));
  LaunchScope scope(kKindAttention, st);
  const long long rows = (long long)s.H * s.Tq, per = kSimtThreads / 32;
  TL_CUDA_CHECK(launch_pdl(attn_add_dq_parts_kernel<T>, dim3((unsigned)((rows + per - 1) / per)), dim3(kSimtThreads), 0, st, s, x, w));
  return TEMPLORA_OK;
}
// Tiles of 32 rows, whose steps take a quarter of the time, where 64-row ones would take at most every second SM; causal in
// fp32, 64 against 32 rows: 500 tokens, 8 / 2 heads of 64: 55 -> 33 us forward; 1000 tokens, 8 heads of 128: 172 -> 217 us.
template <typename T, int DM>
templora_status_t simt_fwd(const AttnShape &s, const AttnTensors &x, const AttnFwdParts &parts, int sms, cudaStream_t st) {
  return ((s.Tq + 63) / 64) * (long long)s.H * parts.n * 2 <= sms ? simt_fwd<T, DM, 32>(s, x, parts, st) : simt_fwd<T, DM, 64>(s, x, parts, st);
}
template <typename T, int DM>
templora_status_t simt_bwd(const AttnShape &s, const AttnTensors &x, const AttnBwdScratch &w, int sms, cudaStream_t st) {
  if (((s.Tk + 63) / 64) * (long long)s.Hkv * (w.head_parts * w.row_parts) * 2 <= sms) TL_TRY((simt_dkdv<T, DM, 32>(s, x, w, st)));
  else TL_TRY((simt_dkdv<T, DM, 64>(s, x, w, st)));
  return ((s.Tq + 63) / 64) * (long long)s.H * w.key_parts * 2 <= sms ? simt_dq<T, DM, 32>(s, x, w, st) : simt_dq<T, DM, 64>(s, x, w, st);
}

template <typename T>
templora_status_t prep(const AttnShape &s, const AttnTensors &x, const AttnBwdScratch &w, float lse_scale, cudaStream_t st) {
  LaunchScope scope(kKindAttention, st);
  TL_CUDA_CHECK(launch_pdl(attn_bwd_prep_kernel<T>, dim3(w.Tq_pad / kPrepRows, s.H), dim3(kPrepThreads), 0, st, s, x, w,
                           lse_scale));
  return TEMPLORA_OK;
}

// ------------------------------------------------------------------ host side
bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

constexpr int kMaxLen = 1 << 30;   // positions and their sums stay inside 32 bits

templora_status_t check_lengths(int Tq, int Tk, int q_start) {
  if (Tq <= 0 || Tk <= 0 || q_start < 0) return TEMPLORA_ERR_INVALID_ARG;
  if (Tq > kMaxLen || Tk > kMaxLen || q_start > kMaxLen - Tq) return TEMPLORA_ERR_UNSUPPORTED;
  return TEMPLORA_OK;
}

// The backward splits dk and dv (the tensor-core kernel by a rule of its own, within these parts) where one CTA per tile of 64 keys and kv head would leave most SMs idle: by the heads
// of a group, then into stretches of at least eight query tiles, up to about four CTAs per SM of a B200.  Whole against split,
// causal in fp32: 1000 tokens, 8 / 8 heads of 128: 525 -> 467 us; 512 tokens, 16 / 4 heads: 593 -> 280 us; 2000 tokens, 2 / 1
// heads: 1510 -> 803 us; 1500 tokens, 32 / 8 heads: 3046 -> 2532 us.  Only sizes enter the rule, since the workspace is asked for
// with nothing else.
void split_dkdv(const templora_attn_t *a, int Tq, int Tk, AttnBwdScratch *w) {
  const long long base = ((long long)Tk + 63) / 64 * a->n_kv_heads, want = (4 * 148 + base - 1) / base;
  const int group = a->n_heads / a->n_kv_heads;
  w->head_parts = (int)std::min<long long>(want, group);
  const long long rows = std::min((want + group - 1) / group, ((long long)Tq + 511) / 512);
  w->row_parts = (int)std::clamp<long long>(rows, 1, 8);
}

long long keys_in_reach(const templora_attn_t *a, int Tk) {
  return a->window > 0 ? std::min<long long>(Tk, (a->causal ? 1ll : 2ll) * a->window + 256) : Tk;
}
// The tensor-core forward splits the keys where its CTAs (two 128-row tiles each) leave most SMs idle: as many parts as run at once, of
// four key tiles at least.  Whole against parts, causal: 62 queries behind 2374 tokens, 16 / 16 heads of 128: 49 -> 26 us; 43 behind
// 4000, 8 / 1: 80 -> 28; 2048 tokens, 4 / 1: 42 -> 36; in two parts 1803 tokens, 8 / 8: 41 -> 46, so two have to be long.
int fwd_parts(const templora_attn_t *a, int Tq, int Tk) {
  const bool heads = a->n_heads / a->n_kv_heads % 2 == 0;
  const long long tiles = ((long long)Tq + 127) / 128, ctas = heads ? tiles * (a->n_heads / 2) : (tiles + 1) / 2 * a->n_heads;
  const long long rounds = (keys_in_reach(a, Tk) + 511) / 512;
  const int n = (int)std::min(148 / ctas, rounds);
  return n >= 3 || (n == 2 && rounds >= 6) ? n : 1;
}
// The generic forward and dq kernel: up to about four CTAs per SM of a B200, of 512 keys at least.  Whole against parts, causal in
// fp32: 2000 tokens, 2 / 1 heads of 128: forward 265 -> 177 us, backward 799 -> 377; 4246 tokens, one head of 96: 556 -> 234, 1374 -> 682;
// 1500 tokens, 32 / 8 heads (no parts): 750, 2530.
int generic_parts(const templora_attn_t *a, int Tq, int Tk) {
  const long long ctas = ((long long)Tq + 63) / 64 * a->n_heads;
  return (int)std::clamp(std::min((4 * 148 + ctas - 1) / ctas, keys_in_reach(a, Tk) / 512), 1ll, 64ll);
}
size_t fwd_scratch_bytes(const templora_attn_t *a, int n, int Tq, AttnFwdParts *parts, uint8_t *base) {
  const size_t rows = n > 1 ? (size_t)n * a->n_heads * Tq : 0, o = align_up(rows * a->head_dim * sizeof(float), kWsAlign);
  if (parts) *parts = AttnFwdParts{n, (float *)(base + kStatusBytes), (float2 *)(base + kStatusBytes + o)};
  return kStatusBytes + o + rows * sizeof(float2);
}

size_t dkdv_part_bytes(const templora_attn_t *a, int Tk, const AttnBwdScratch &s) {
  const size_t parts = (size_t)s.head_parts * s.row_parts;
  return parts > 1 ? align_up(parts * a->n_kv_heads * (size_t)Tk * a->head_dim * sizeof(float), kWsAlign) : 0;
}
size_t dq_part_bytes(const templora_attn_t *a, int Tq, int key_parts) {
  return key_parts > 1 ? align_up((size_t)key_parts * a->n_heads * Tq * a->head_dim * sizeof(float), kWsAlign) : 0;
}
// statistics and intervals of the backward's rows
size_t row_scratch_bytes(const templora_attn_t *a, int Tq, AttnBwdScratch *w, uint8_t *base) {
  const size_t pad = align_up((size_t)Tq, 128), tiles = pad / 128;
  size_t off = kStatusBytes;
  auto take = [&](size_t bytes) { uint8_t *p = base + off; off += align_up(bytes, kWsAlign); return p; };
  uint8_t *stat = take(pad * a->n_heads * 2 * sizeof(float)), *rows = take(pad * sizeof(int2));
  uint8_t *t = take(tiles * sizeof(int2)), *in = take(tiles * 4 * sizeof(int2));
  *w = AttnBwdScratch{(float *)stat, (int2 *)rows, (int2 *)t, (int2 *)in, (int)pad};
  return off;
}
size_t scratch_bytes(const templora_attn_t *a, int Tq, int Tk, AttnBwdScratch *w, uint8_t *base) {
  size_t off = row_scratch_bytes(a, Tq, w, base);
  split_dkdv(a, Tq, Tk, w);
  if (const size_t bytes = dkdv_part_bytes(a, Tk, *w)) {
    w->part_dk = (float *)(base + off);
    w->part_dv = (float *)(base + off + bytes);
    off += 2 * bytes;
  }
  w->key_parts = generic_parts(a, Tq, Tk);
  if (const size_t bytes = dq_part_bytes(a, Tq, w->key_parts)) {
    w->part_dq = (float *)(base + off);
    off += bytes;
  }
  return off;
}

// What a call at these lengths needs, whichever direction and path it takes.
size_t call_bytes(const templora_attn_t *a, int Tq, int Tk) {
  AttnBwdScratch w;
  const int n = std::max(fwd_parts(a, Tq, Tk), generic_parts(a, Tq, Tk));
  return std::max(scratch_bytes(a, Tq, Tk, &w, nullptr), fwd_scratch_bytes(a, n, Tq, nullptr, nullptr));
}
// The most that a call at these lengths or shorter ones needs: fewer rows are split into more parts, so that 1024 tokens can need
// more than 4096.  Parts by keys do not get fewer as Tk grows, nor parts by queries as Tq does; and with as many tiles of 64 (or 128)
// rows the longest takes most.  Nothing is split from 4 * 148 tiles on.
size_t longest_bytes(const templora_attn_t *a, int Tq, int Tk) {
  AttnBwdScratch w;
  size_t dkdv = 0, dq = 0, fwd = 0;
  auto each_tile_count = [](int T, int heads, auto body) {
    const int tiles = (int)std::min(((long long)T + 63) / 64, 4 * 148ll / heads + 1);
    for (int t = 1; t <= tiles; ++t) body((int)std::min<long long>(T, 64ll * t));
  };
  each_tile_count(Tk, a->n_kv_heads, [&](int len) {
    split_dkdv(a, Tq, len, &w);
    dkdv = std::max(dkdv, dkdv_part_bytes(a, len, w));
  });
  each_tile_count(Tq, a->n_heads, [&](int len) {
    const int generic = generic_parts(a, len, Tk);
    dq = std::max(dq, dq_part_bytes(a, len, generic));
    fwd = std::max(fwd, fwd_scratch_bytes(a, std::max(fwd_parts(a, len, Tk), generic), len, nullptr, nullptr));
  });
  return std::max(row_scratch_bytes(a, Tq, &w, nullptr) + 2 * dkdv + dq, fwd);
}

templora_status_t check_call(const templora_attn_t *a, const templora_attn_io_t *io, int Tq, int Tk, int q_start,
                             bool bwd, AttnShape *s, AttnTensors *x) {
  TL_TRY(attn_check_desc(a));
  TL_TRY(check_lengths(Tq, Tk, q_start));
  if (!io || !io->q || !io->k || !io->v || !io->o || !io->lse) return TEMPLORA_ERR_INVALID_ARG;
  if (!aligned16(io->q) || !aligned16(io->k) || !aligned16(io->v) || !aligned16(io->o) || !aligned16(io->lse))
    return TEMPLORA_ERR_INVALID_ARG;
  if (bwd) {
    if (!io->dO || !io->dq || !io->dk || !io->dv) return TEMPLORA_ERR_INVALID_ARG;
    if (!aligned16(io->dO) || !aligned16(io->dq) || !aligned16(io->dk) || !aligned16(io->dv)) return TEMPLORA_ERR_INVALID_ARG;
  }
  const long long nq = (long long)a->n_heads * a->head_dim, nk = (long long)a->n_kv_heads * a->head_dim;
  bool ok = true;
  auto ld = [&](int64_t given, long long width) {
    if (given == 0) return width;
    ok = ok && given >= width && given <= (1ll << 31);
    return (long long)given;
  };
  *s = AttnShape{a->n_heads, a->n_kv_heads, a->n_heads / a->n_kv_heads, a->head_dim, Tq, Tk, q_start, a->causal,
                 a->window > kMaxLen ? kMaxLen : a->window, a->n_docs, a->scale, a->softcap, a->slopes, a->doc_offsets,
                 a->prefix_lens};
  *x = AttnTensors{};
  x->q = io->q; x->k = io->k; x->v = io->v; x->o = io->o; x->lse = io->lse;
  x->ldq = ld(io->ld_q, nq); x->ldk = ld(io->ld_k, nk); x->ldv = ld(io->ld_v, nk); x->ldo = ld(io->ld_o, nq);
  if (bwd) {
    x->dO = io->dO; x->dq = io->dq; x->dk = io->dk; x->dv = io->dv;
    x->lddo = ld(io->ld_dO, nq); x->lddq = ld(io->ld_dq, nq); x->lddk = ld(io->ld_dk, nk); x->lddv = ld(io->ld_dv, nk);
  }
  return ok ? TEMPLORA_OK : TEMPLORA_ERR_INVALID_ARG;
}

templora_status_t check_workspace(const void *ws, size_t ws_bytes, size_t need) {
  if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255) != 0 || ws_bytes < need) return TEMPLORA_ERR_WORKSPACE;
  return TEMPLORA_OK;
}

// Does the call run on the tensor cores?  16-byte rows are what their copies need.
bool use_tc(const AttnShape &s, const AttnTensors &x, int dtype) {
  if (kernel_path() == 1 || dtype != TEMPLORA_BF16) return false;
  if ((s.D | x.ldq | x.ldk | x.ldv | x.ldo | x.lddo | x.lddq | x.lddk | x.lddv) & 7) return false;
  return attn_tc_available();
}

}  // namespace

templora_status_t stream_sms(cudaStream_t st, int *sms) {
  DeviceInfo *di = device_info();
  if (!di) return TEMPLORA_ERR_CUDA;
  *sms = stream_sm_limit(st, di->sm_count);
  return TEMPLORA_OK;
}

templora_status_t attn_check_desc(const templora_attn_t *a) {
  if (!a) return TEMPLORA_ERR_INVALID_ARG;
  if (a->n_heads <= 0 || a->n_kv_heads <= 0 || a->head_dim <= 0 || a->n_heads % a->n_kv_heads != 0) return TEMPLORA_ERR_INVALID_ARG;
  if (a->dtype != TEMPLORA_F32 && a->dtype != TEMPLORA_BF16) return TEMPLORA_ERR_UNSUPPORTED;
  if (a->head_dim > 128 || a->n_heads > 65535) return TEMPLORA_ERR_UNSUPPORTED;
  if (!(a->scale - a->scale == 0.f) || !(a->softcap >= 0.f) || !(a->softcap - a->softcap == 0.f)) return TEMPLORA_ERR_INVALID_ARG;
  if ((a->causal != 0 && a->causal != 1) || a->window < 0 || a->n_docs < 0 || a->n_docs > (1 << 24)) return TEMPLORA_ERR_INVALID_ARG;
  if (a->n_docs > 0 && !a->doc_offsets) return TEMPLORA_ERR_INVALID_ARG;
  if (!word_aligned(a->slopes) || !word_aligned(a->doc_offsets) || !word_aligned(a->prefix_lens)) return TEMPLORA_ERR_INVALID_ARG;
  if (a->prefix_lens && !a->causal) return TEMPLORA_ERR_INVALID_ARG;
  if (a->prefix_lens && a->window > 0) return TEMPLORA_ERR_UNSUPPORTED;
  return TEMPLORA_OK;
}

templora_status_t attn_simt_fwd(const AttnShape &s, const AttnTensors &x, const AttnFwdParts &parts, int dtype, cudaStream_t st) {
  int sms = 0;
  TL_TRY(stream_sms(st, &sms));
  if (dtype == TEMPLORA_F32) return s.D <= 64 ? simt_fwd<float, 64>(s, x, parts, sms, st) : simt_fwd<float, 128>(s, x, parts, sms, st);
  return s.D <= 64 ? simt_fwd<__nv_bfloat16, 64>(s, x, parts, sms, st) : simt_fwd<__nv_bfloat16, 128>(s, x, parts, sms, st);
}

templora_status_t attn_join_parts(const AttnShape &s, const AttnTensors &x, const AttnFwdParts &parts, cudaStream_t st) {
  return join_parts<__nv_bfloat16, true>(s, x, parts, st);
}
templora_status_t attn_add_parts(const AttnShape &s, const AttnTensors &x, const AttnBwdScratch &w, int dtype, cudaStream_t st) {
  return dtype == TEMPLORA_F32 ? add_parts<float>(s, x, w, st) : add_parts<__nv_bfloat16>(s, x, w, st);
}

templora_status_t attn_simt_bwd(const AttnShape &s, const AttnTensors &x, const AttnBwdScratch &w, int dtype, cudaStream_t st) {
  int sms = 0;
  TL_TRY(stream_sms(st, &sms));
  if (dtype == TEMPLORA_F32) {
    TL_TRY(prep<float>(s, x, w, 1.f, st));
    return s.D <= 64 ? simt_bwd<float, 64>(s, x, w, sms, st) : simt_bwd<float, 128>(s, x, w, sms, st);
  }
  TL_TRY(prep<__nv_bfloat16>(s, x, w, 1.f, st));
  return s.D <= 64 ? simt_bwd<__nv_bfloat16, 64>(s, x, w, sms, st) : simt_bwd<__nv_bfloat16, 128>(s, x, w, sms, st);
}

}  // namespace templora

using namespace templora;

extern "C" {

size_t templora_attention_workspace_bytes(const templora_attn_t *attn, int32_t Tq, int32_t Tk) {
  if (attn_check_desc(attn) != TEMPLORA_OK || check_lengths(Tq, Tk, 0) != TEMPLORA_OK) return 0;
  return longest_bytes(attn, Tq, Tk);
}

templora_status_t templora_attention_fwd(const templora_attn_t *attn, const templora_attn_io_t *io, int32_t Tq,
                                         int32_t Tk, int32_t q_start, void *ws, size_t ws_bytes, void *stream) {
  AttnShape s;
  AttnTensors x;
  TL_TRY(check_call(attn, io, Tq, Tk, q_start, false, &s, &x));
  TL_TRY(check_workspace(ws, ws_bytes, call_bytes(attn, Tq, Tk)));
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  const bool tc = use_tc(s, x, attn->dtype);
  AttnFwdParts parts;
  fwd_scratch_bytes(attn, tc ? fwd_parts(attn, Tq, Tk) : generic_parts(attn, Tq, Tk), Tq, &parts, reinterpret_cast<uint8_t *>(ws));
  if (tc) return attn_tc_fwd(s, x, parts, reinterpret_cast<DeviceStatus *>(ws), st);
  return attn_simt_fwd(s, x, parts, attn->dtype, st);
}

templora_status_t templora_attention_bwd(const templora_attn_t *attn, const templora_attn_io_t *io, int32_t Tq,
                                         int32_t Tk, int32_t q_start, void *ws, size_t ws_bytes, void *stream) {
  AttnShape s;
  AttnTensors x;
  AttnBwdScratch w;
  TL_TRY(check_call(attn, io, Tq, Tk, q_start, true, &s, &x));
  scratch_bytes(attn, Tq, Tk, &w, reinterpret_cast<uint8_t *>(ws));
  TL_TRY(check_workspace(ws, ws_bytes, call_bytes(attn, Tq, Tk)));
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  if (use_tc(s, x, attn->dtype)) {
    TL_TRY(prep<__nv_bfloat16>(s, x, w, kLog2e, st));
    return attn_tc_bwd(s, x, w, reinterpret_cast<DeviceStatus *>(ws), st);
  }
  return attn_simt_bwd(s, x, w, attn->dtype, st);
}

}  // extern "C"
