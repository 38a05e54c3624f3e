// Attention of a chunk: entry points, argument checks, the backward's row statistics, and the kernels for every type
// and layout (fp32, and bf16 shapes the tensor-core kernels do not take).  attention_tc.cu has the tensor-core forms.
#include "attention.cuh"
#include "tc_host.h"

namespace templora {
namespace {

// ------------------------------------------------------------------ generic kernels
// 256 threads as a 16 x 16 grid; a tile is TL rows by TL columns (64, or 32 where 64 would leave SMs without a CTA), thread
// (ty, tx) owns rows ty + 16 a and columns tx + 16 b, so that 16-byte shared-memory reads along head_dim hit different banks
// (row pitch D + 4 words: eight neighbouring lanes start four words apart).  At TL = 64 a thread reads 8 vectors per four
// values of head_dim for 64 FMAs; the kernels are bound by the fp32 pipes and shared memory, and on small calls by the
// latency of a tile, which the smaller one quarters.
constexpr int kSimtThreads = 256;
template <int DM> constexpr int kPitch = DM + 4;
template <int TL> constexpr int kPitchP = TL + 4;

// rows [row0, row0 + TL) of one head, zero outside [0, n_rows) and behind head_dim, as fp32
template <typename T, int DM, int TL>
__device__ __forceinline__ void load_tile(float *dst, const T *src, long long ld, int row0, int n_rows, int D, bool vec) {
  constexpr int N = 16 / sizeof(T);
  if (vec) {      // 16 bytes per load, all of a thread's loads in flight together
    constexpr int kVecs = TL * DM / N, kPer = (kVecs + kSimtThreads - 1) / kSimtThreads;
    uint4 v[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int e = threadIdx.x + i * kSimtThreads, r = e / (DM / N), c = (e % (DM / N)) * N;
      v[i] = (e < kVecs && row0 + r >= 0 && row0 + r < n_rows && c < D)
                 ? *reinterpret_cast<const uint4 *>(src + (long long)(row0 + r) * ld + c) : make_uint4(0, 0, 0, 0);
    }
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
    return;
  }
  for (int e = threadIdx.x; e < TL * DM; e += kSimtThreads) {
    const int r = e / DM, c = e % DM;
    dst[r * kPitch<DM> + c] = (row0 + r >= 0 && row0 + r < n_rows && c < D) ? attn_ld(src + (long long)(row0 + r) * ld + c) : 0.f;
  }
}

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

template <typename T, int DM, int TL>
__global__ void __launch_bounds__(kSimtThreads) attn_simt_fwd_kernel(const AttnShape s, const AttnTensors x) {
  pdl_prologue();
  constexpr int N = 16 / sizeof(T);
  const bool vec = ((s.D | x.ldq | x.ldk | x.ldv | x.lddo) & (N - 1)) == 0;      // (the forward's lddo is 0)
  extern __shared__ __align__(16) float sm[];
  float *Q = sm, *KV = Q + TL * kPitch<DM>, *P = KV + TL * kPitch<DM>;
  __shared__ int2 rows[TL];
  const int h = blockIdx.y, hk = h / s.group, q0 = blockIdx.x * TL;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const int2 range = tile_range<TL>(s, q0, rows);
  load_tile<T, DM, TL>(Q, (const T *)x.q + (long long)h * s.D, x.ldq, q0, s.Tq, s.D, vec);
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
    load_tile<T, DM, TL>(KV, (const T *)x.k + (long long)hk * s.D, x.ldk, k0, range.y, s.D, vec);
    __syncthreads();
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
    load_tile<T, DM, TL>(KV, (const T *)x.v + (long long)hk * s.D, x.ldv, k0, range.y, s.D, vec);
    __syncthreads();
    weighted_sum<DM, TL>(acc, P, KV, ty, tx);
  }
  bool redo[TL / 16];
#pragma unroll
  for (int a = 0; a < TL / 16; ++a) {
    const int i = q0 + ty + 16 * a;
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) l[a] += __shfl_xor_sync(0xffffffffu, l[a], o);
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

// -lse and -delta of row i
__device__ __forceinline__ float2 row_stat(const AttnBwdScratch &w, int h, int i) {
  const float *p = w.stat + 2 * ((long long)h * w.Tq_pad + (i & ~127)) + (i & 127);
  return make_float2(p[0], p[128]);
}

// dk, dv of a 64-row tile of keys: loops over the heads that share it and over the query tiles that reach it
template <typename T, int DM, int TL>
__global__ void __launch_bounds__(kSimtThreads) attn_simt_dkdv_kernel(const AttnShape s, const AttnTensors x,
                                                                      const AttnBwdScratch w) {
  pdl_prologue();
  constexpr int N = 16 / sizeof(T);
  const bool vec = ((s.D | x.ldq | x.ldk | x.ldv | x.lddo) & (N - 1)) == 0;      // (the forward's lddo is 0)
  extern __shared__ __align__(16) float sm[];
  constexpr int kT = TL * kPitch<DM>;
  float *K = sm, *V = K + kT, *Q = V + kT, *DO = Q + kT, *P = DO + kT, *DS = P + TL * kPitchP<TL>;
  __shared__ int2 rows[TL];
  __shared__ float2 stat[TL];
  const int hk = blockIdx.y, k0 = blockIdx.x * TL;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  load_tile<T, DM, TL>(K, (const T *)x.k + (long long)hk * s.D, x.ldk, k0, s.Tk, s.D, vec);
  load_tile<T, DM, TL>(V, (const T *)x.v + (long long)hk * s.D, x.ldv, k0, s.Tk, s.D, vec);
  float dk[TL / 16][DM / 16], dv[TL / 16][DM / 16];
#pragma unroll
  for (int a = 0; a < TL / 16; ++a)
#pragma unroll
    for (int c = 0; c < DM / 16; ++c) dk[a][c] = dv[a][c] = 0.f;
  for (int h = hk * s.group; h < (hk + 1) * s.group; ++h) {
    const float slope = s.slopes ? s.slopes[h] : 0.f;
    for (int q0 = 0; q0 < s.Tq; q0 += TL) {
      const int2 reach = w.tiles[q0 / 128];
      if (reach.x >= k0 + TL || reach.y <= k0) continue;   // uniform over the block
      __syncthreads();
      load_tile<T, DM, TL>(Q, (const T *)x.q + (long long)h * s.D, x.ldq, q0, s.Tq, s.D, vec);
      load_tile<T, DM, TL>(DO, (const T *)x.dO + (long long)h * s.D, x.lddo, q0, s.Tq, s.D, vec);
      if (threadIdx.x < TL) {
        rows[threadIdx.x] = w.rows[q0 + threadIdx.x];
        stat[threadIdx.x] = row_stat(w, h, q0 + threadIdx.x);
      }
      __syncthreads();
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
    if (votes & 0xffffu) attn_exact_dkdv_row<T>(s, x, hk, base);
    if (votes >> 16) attn_exact_dkdv_row<T>(s, x, hk, base + 1);
  }
}

template <typename T, int DM, int TL>
__global__ void __launch_bounds__(kSimtThreads) attn_simt_dq_kernel(const AttnShape s, const AttnTensors x,
                                                                    const AttnBwdScratch w) {
  pdl_prologue();
  constexpr int N = 16 / sizeof(T);
  const bool vec = ((s.D | x.ldq | x.ldk | x.ldv | x.lddo) & (N - 1)) == 0;      // (the forward's lddo is 0)
  extern __shared__ __align__(16) float sm[];
  constexpr int kT = TL * kPitch<DM>;
  float *Q = sm, *DO = Q + kT, *K = DO + kT, *V = K + kT, *DS = V + kT;
  __shared__ int2 rows[TL];
  __shared__ float2 stat[TL];
  const int h = blockIdx.y, hk = h / s.group, q0 = blockIdx.x * TL;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const float slope = s.slopes ? s.slopes[h] : 0.f;
  load_tile<T, DM, TL>(Q, (const T *)x.q + (long long)h * s.D, x.ldq, q0, s.Tq, s.D, vec);
  load_tile<T, DM, TL>(DO, (const T *)x.dO + (long long)h * s.D, x.lddo, q0, s.Tq, s.D, vec);
  const int2 range = tile_range<TL>(s, q0, rows);
  if (threadIdx.x < TL) stat[threadIdx.x] = row_stat(w, h, q0 + threadIdx.x);
  float dq[TL / 16][DM / 16];
#pragma unroll
  for (int a = 0; a < TL / 16; ++a)
#pragma unroll
    for (int c = 0; c < DM / 16; ++c) dq[a][c] = 0.f;
  for (int k0 = range.x; k0 < range.y; k0 += TL) {
    __syncthreads();
    load_tile<T, DM, TL>(K, (const T *)x.k + (long long)hk * s.D, x.ldk, k0, range.y, s.D, vec);
    load_tile<T, DM, TL>(V, (const T *)x.v + (long long)hk * s.D, x.ldv, k0, range.y, s.D, vec);
    __syncthreads();
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
// intervals and their tiles'.  Bound by HBM (o and dO read once).
constexpr int kPrepRows = 128;
template <typename T>
__global__ void __launch_bounds__(256) attn_bwd_prep_kernel(const AttnShape s, const AttnTensors x, const AttnBwdScratch w,
                                                            float lse_scale) {
  pdl_prologue();
  constexpr int N = 16 / sizeof(T);
  const int h = blockIdx.y, row0 = blockIdx.x * kPrepRows, sub = threadIdx.x & 7;
  const bool vec = ((s.D | x.lddo | x.ldo) & (N - 1)) == 0;
  float *stat = w.stat + 2 * ((long long)h * w.Tq_pad + row0);
#pragma unroll
  for (int pass = 0; pass < kPrepRows / 32; ++pass) {
    const int r = pass * 32 + (threadIdx.x >> 3), i = row0 + r;
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
      stat[r] = i < s.Tq ? -x.lse[(long long)h * s.Tq + i] * lse_scale : -INFINITY;
      stat[kPrepRows + r] = i < s.Tq ? -delta : 0.f;
    }
  }
  if (h != 0) return;
  __shared__ int range[4];
  if (threadIdx.x == 0) { range[0] = s.Tk; range[1] = 0; range[2] = 0; range[3] = s.Tk; }
  __syncthreads();
  if (threadIdx.x < kPrepRows) {
    const int i = row0 + threadIdx.x;
    const int2 r = i < s.Tq ? attn_interval(s, i) : make_int2(0, 0);
    w.rows[i] = r;
    if (r.x < r.y) {
      atomicMin(&range[0], r.x);
      atomicMax(&range[1], r.y);
    }
    if (i < s.Tq) {
      atomicMax(&range[2], r.x);
      atomicMin(&range[3], r.y);
    }
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    w.tiles[blockIdx.x] = make_int2(range[0], range[1]);
    w.inner[blockIdx.x] = make_int2(range[2], range[3]);
  }
}

template <typename T, int DM, int TL>
templora_status_t simt_fwd(const AttnShape &s, const AttnTensors &x, cudaStream_t st) {
  const size_t smem = (2 * TL * kPitch<DM> + TL * kPitchP<TL>) * sizeof(float);
  TL_TRY((allow_smem<attn_simt_fwd_kernel<T, DM, TL>>(smem)));
  LaunchScope scope(kKindAttention, st);
  TL_CUDA_CHECK(launch_pdl(attn_simt_fwd_kernel<T, DM, TL>, dim3((s.Tq + TL - 1) / TL, s.H), dim3(kSimtThreads), smem, st, s, x));
  return TEMPLORA_OK;
}
template <typename T, int DM, int TL>
templora_status_t simt_dkdv(const AttnShape &s, const AttnTensors &x, const AttnBwdScratch &w, cudaStream_t st) {
  const size_t smem = (4 * TL * kPitch<DM> + 2 * TL * kPitchP<TL>) * sizeof(float);
  TL_TRY((allow_smem<attn_simt_dkdv_kernel<T, DM, TL>>(smem)));
  LaunchScope scope(kKindAttention, st);
  TL_CUDA_CHECK(launch_pdl(attn_simt_dkdv_kernel<T, DM, TL>, dim3((s.Tk + TL - 1) / TL, s.Hkv), dim3(kSimtThreads), smem, st, s, x, w));
  return TEMPLORA_OK;
}
template <typename T, int DM, int TL>
templora_status_t simt_dq(const AttnShape &s, const AttnTensors &x, const AttnBwdScratch &w, cudaStream_t st) {
  const size_t smem = (4 * TL * kPitch<DM> + TL * kPitchP<TL>) * sizeof(float);
  TL_TRY((allow_smem<attn_simt_dq_kernel<T, DM, TL>>(smem)));
  LaunchScope scope(kKindAttention, st);
  TL_CUDA_CHECK(launch_pdl(attn_simt_dq_kernel<T, DM, TL>, dim3((s.Tq + TL - 1) / TL, s.H), dim3(kSimtThreads), smem, st, s, x, w));
  return TEMPLORA_OK;
}
// Fewer CTAs of 64-row tiles than SMs: 32-row tiles, whose steps take a quarter of the time.
template <typename T, int DM>
templora_status_t simt_fwd(const AttnShape &s, const AttnTensors &x, int sms, cudaStream_t st) {
  return ((s.Tq + 63) / 64) * (long long)s.H < sms ? simt_fwd<T, DM, 32>(s, x, st) : simt_fwd<T, DM, 64>(s, x, st);
}
template <typename T, int DM>
templora_status_t simt_bwd(const AttnShape &s, const AttnTensors &x, const AttnBwdScratch &w, int sms, cudaStream_t st) {
  if (((s.Tk + 63) / 64) * (long long)s.Hkv < sms) TL_TRY((simt_dkdv<T, DM, 32>(s, x, w, st)));
  else TL_TRY((simt_dkdv<T, DM, 64>(s, x, w, st)));
  return ((s.Tq + 63) / 64) * (long long)s.H < sms ? simt_dq<T, DM, 32>(s, x, w, st) : simt_dq<T, DM, 64>(s, x, w, st);
}

template <typename T>
templora_status_t prep(const AttnShape &s, const AttnTensors &x, const AttnBwdScratch &w, float lse_scale, cudaStream_t st) {
  LaunchScope scope(kKindAttention, st);
  TL_CUDA_CHECK(launch_pdl(attn_bwd_prep_kernel<T>, dim3(w.Tq_pad / kPrepRows, s.H), dim3(256), 0, st, s, x, w, lse_scale));
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

size_t scratch_bytes(const templora_attn_t *a, int Tq, AttnBwdScratch *w, uint8_t *base) {
  const size_t pad = align_up((size_t)Tq, 128), tiles = pad / 128;
  size_t off = kStatusBytes;
  auto take = [&](size_t bytes) { uint8_t *p = base + off; off += align_up(bytes, kWsAlign); return p; };
  uint8_t *stat = take(pad * a->n_heads * 2 * sizeof(float)), *rows = take(pad * sizeof(int2));
  uint8_t *t = take(tiles * sizeof(int2)), *in = take(tiles * sizeof(int2));
  if (w) *w = AttnBwdScratch{(float *)stat, (int2 *)rows, (int2 *)t, (int2 *)in, (int)pad};
  return off;
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
  if (a->prefix_lens && !a->causal) return TEMPLORA_ERR_INVALID_ARG;
  if (a->prefix_lens && a->window > 0) return TEMPLORA_ERR_UNSUPPORTED;
  return TEMPLORA_OK;
}

templora_status_t attn_simt_fwd(const AttnShape &s, const AttnTensors &x, int dtype, cudaStream_t st) {
  int sms = 0;
  TL_TRY(stream_sms(st, &sms));
  if (dtype == TEMPLORA_F32) return s.D <= 64 ? simt_fwd<float, 64>(s, x, sms, st) : simt_fwd<float, 128>(s, x, sms, st);
  return s.D <= 64 ? simt_fwd<__nv_bfloat16, 64>(s, x, sms, st) : simt_fwd<__nv_bfloat16, 128>(s, x, sms, st);
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
  return scratch_bytes(attn, Tq, nullptr, nullptr);
}

templora_status_t templora_attention_fwd(const templora_attn_t *attn, const templora_attn_io_t *io, int32_t Tq,
                                         int32_t Tk, int32_t q_start, void *ws, size_t ws_bytes, void *stream) {
  AttnShape s;
  AttnTensors x;
  TL_TRY(check_call(attn, io, Tq, Tk, q_start, false, &s, &x));
  TL_TRY(check_workspace(ws, ws_bytes, scratch_bytes(attn, Tq, nullptr, nullptr)));
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  if (use_tc(s, x, attn->dtype)) return attn_tc_fwd(s, x, reinterpret_cast<DeviceStatus *>(ws), st);
  return attn_simt_fwd(s, x, attn->dtype, st);
}

templora_status_t templora_attention_bwd(const templora_attn_t *attn, const templora_attn_io_t *io, int32_t Tq,
                                         int32_t Tk, int32_t q_start, void *ws, size_t ws_bytes, void *stream) {
  AttnShape s;
  AttnTensors x;
  AttnBwdScratch w;
  TL_TRY(check_call(attn, io, Tq, Tk, q_start, true, &s, &x));
  TL_TRY(check_workspace(ws, ws_bytes, scratch_bytes(attn, Tq, &w, reinterpret_cast<uint8_t *>(ws))));
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  if (use_tc(s, x, attn->dtype)) {
    TL_TRY(prep<__nv_bfloat16>(s, x, w, kLog2e, st));
    return attn_tc_bwd(s, x, w, reinterpret_cast<DeviceStatus *>(ws), st);
  }
  return attn_simt_bwd(s, x, w, attn->dtype, st);
}

}  // extern "C"
