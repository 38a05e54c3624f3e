// Shared by the kernels of the 8-bit key/value cache: the device view of a cache, encoding and decoding of its codes, and the
// argument checks of the calls that take one.
#pragma once
#include "attention.cuh"

#include <cuda_fp16.h>
#include <cuda_fp8.h>

namespace templora {

// ------------------------------------------------------------------ device view of a cache
struct CacheView {
  uint8_t *k, *v;
  float *k_scale, *v_scale;
  const int *table;
  const int *seq_lens;
  int Hkv, D, bt, bt_log2, n_blocks, n_seqs, max_blocks;
  DeviceStatus *status;
};
enum { kWhereTable = 700, kWhereLength = 701, kWhereCodes = 702 };   // location tags of the device status record

__device__ __forceinline__ void report(DeviceStatus *st, int where) {
  if (atomicCAS(&st->code, 0, (int)TEMPLORA_ERR_INVALID_ARG) == 0) st->where = where;
}
// Block b of a sequence, or -1 (recorded) when the table names none.
__device__ __forceinline__ int cache_block(const CacheView &c, int seq, int b) {
  const int id = c.table[(long long)seq * c.max_blocks + b];
  if ((unsigned)id < (unsigned)c.n_blocks) return id;
  report(c.status, kWhereTable);
  return -1;
}

// ------------------------------------------------------------------ encoding
// Exponent e of the block scale for values up to amax: the smallest >= -126 with amax <= 448 * 2^e = 1.75 * 2^(e+8).
__device__ __forceinline__ int scale_exponent(float amax) {
  const uint32_t bits = __float_as_uint(amax);
  if (bits < 0x00800000u) return -126;
  const int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u);
  return e < -126 ? -126 : e;
}
__device__ __forceinline__ float pow2f(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }   // e in [-126, 127]

__device__ __forceinline__ uint32_t encode2(float a, float b) {
  // the conversion saturates; an infinity is not a value the cache can stand for
  if (!(fabsf(a) < INFINITY)) a = __uint_as_float(0x7fffffffu);
  if (!(fabsf(b) < INFINITY)) b = __uint_as_float(0x7fffffffu);
  return __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
}
__device__ __forceinline__ uint32_t half2_of_codes(uint32_t two) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((unsigned short)two));
  return h;
}
// both pairs of a register
__device__ __forceinline__ void half2s_of_codes(uint32_t four, uint32_t &a, uint32_t &b) {
  asm("{\n.reg .b16 l, h;\nmov.b32 {l, h}, %2;\ncvt.rn.f16x2.e4m3x2 %0, l;\ncvt.rn.f16x2.e4m3x2 %1, h;\n}" : "=r"(a), "=r"(b) : "r"(four));
}
__device__ __forceinline__ float2 values_of_codes(uint32_t two) {
  const uint32_t h = half2_of_codes(two);
  return __half22float2(*reinterpret_cast<const __half2 *>(&h));
}

// 16 values as they are stored, and as fp32
template <typename T> struct Raw16 { uint4 w[sizeof(T)]; };
// two neighbouring bf16, or one fp32, as a word
__device__ __forceinline__ uint32_t load_word(const __nv_bfloat16 *p) {
  return (uint32_t)__bfloat16_as_ushort(p[0]) | (uint32_t)__bfloat16_as_ushort(p[1]) << 16;
}
__device__ __forceinline__ uint32_t load_word(const float *p) { return __float_as_uint(*p); }
template <typename T>
__device__ __forceinline__ void load16(const T *p, bool vec, Raw16<T> &r) {
  constexpr int N = 4 / sizeof(T);      // values of a word
  if (vec) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T); ++i) r.w[i] = __ldcs(reinterpret_cast<const uint4 *>(p) + i);
  } else {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T); ++i, p += 4 * N) r.w[i] = make_uint4(load_word(p), load_word(p + N), load_word(p + 2 * N), load_word(p + 3 * N));
  }
}
__device__ __forceinline__ void values16(const Raw16<float> &r, float (&f)[16]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[4 * i] = __uint_as_float(r.w[i].x); f[4 * i + 1] = __uint_as_float(r.w[i].y);
    f[4 * i + 2] = __uint_as_float(r.w[i].z); f[4 * i + 3] = __uint_as_float(r.w[i].w);
  }
}
__device__ __forceinline__ void values16(const Raw16<__nv_bfloat16> &r, float (&f)[16]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t w[4] = {r.w[i].x, r.w[i].y, r.w[i].z, r.w[i].w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      f[8 * i + 2 * e] = __uint_as_float(w[e] << 16);
      f[8 * i + 2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
    }
  }
}
__device__ __forceinline__ uint4 encode16(const float (&f)[16], float inv) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    w[i] = encode2(f[4 * i] * inv, f[4 * i + 1] * inv) | (encode2(f[4 * i + 2] * inv, f[4 * i + 3] * inv) << 16);
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// ------------------------------------------------------------------ warp-level products
__device__ __forceinline__ void mma_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                          uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// ------------------------------------------------------------------ host side
constexpr int kMaxSeqs = 4096;
inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

inline templora_status_t check_cache(const templora_kv_cache_t *c, bool pointers) {
  if (!c || c->n_kv_heads <= 0 || c->head_dim <= 0 || c->block_tokens <= 0 || c->n_blocks <= 0 || c->n_seqs <= 0 ||
      c->max_blocks <= 0)
    return TEMPLORA_ERR_INVALID_ARG;
  if (c->head_dim > 128 || c->head_dim % 16 != 0) return TEMPLORA_ERR_UNSUPPORTED;
  if (c->block_tokens != 16 && c->block_tokens != 32 && c->block_tokens != 64 && c->block_tokens != 128)
    return TEMPLORA_ERR_UNSUPPORTED;
  // positions stay inside 31 bits, a block's head is a coordinate of the copies; kv heads are a grid dimension
  if (c->n_seqs > kMaxSeqs || c->n_kv_heads > 65535 || (long long)c->max_blocks * c->block_tokens > (1ll << 30) ||
      (long long)c->n_blocks * c->n_kv_heads > 0x7fffffffll)
    return TEMPLORA_ERR_UNSUPPORTED;
  if (!pointers) return TEMPLORA_OK;
  if (!c->k || !c->v || !c->k_scale || !c->v_scale || !c->block_table) return TEMPLORA_ERR_INVALID_ARG;
  if (!aligned16(c->k) || !aligned16(c->v) || !aligned16(c->k_scale) || !aligned16(c->v_scale) || !aligned16(c->block_table))
    return TEMPLORA_ERR_INVALID_ARG;
  return TEMPLORA_OK;
}
inline CacheView view(const templora_kv_cache_t *c, const int32_t *seq_lens, void *ws) {
  int lg = 4;
  while ((1 << lg) < c->block_tokens) ++lg;
  return CacheView{(uint8_t *)c->k, (uint8_t *)c->v, c->k_scale, c->v_scale, c->block_table, seq_lens, c->n_kv_heads,
                   c->head_dim, c->block_tokens, lg, c->n_blocks, c->n_seqs, c->max_blocks, (DeviceStatus *)ws};
}
inline templora_status_t check_workspace(const void *ws, size_t ws_bytes, size_t need) {
  if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255) != 0 || ws_bytes < need) return TEMPLORA_ERR_WORKSPACE;
  return TEMPLORA_OK;
}
// row stride in elements: 0 = contiguous; -1 = refused
inline long long row_stride(int64_t given, long long width) {
  if (given == 0) return width;
  return given >= width && given <= (1ll << 31) ? given : -1;
}

}  // namespace templora
