// The 8-bit key/value cache: encoding new tokens into it, and the attention of a decode step over it.
#include "kv_cache.cuh"
#include "tc_device.cuh"
#include "tc_host.h"

namespace templora {
namespace {

// A unit of work is one block of one sequence that gets new tokens, for one head and one of k, v: it reads the new rows
// (kept in registers as stored: NV vectors of 16 values per thread, block_tokens x head_dim in all), reduces their largest
// magnitude, and writes codes and scale.  Units are found by their first new row: a thread per row looks whether its row
// starts a sequence's new rows or a block.  Bound by HBM on long appends (2 or 4 bytes read, 1 written per value), by latency
// on single tokens; a unit is a chain of dependent reads (length, table, rows), so many CTAs per SM matter more than wide ones.
// About 2800 tokens of three sequences, 32 heads of 128 in bf16: 21 us, 3.3 TB/s; one token for each of 16 sequences: 9 us.
constexpr int kAppendThreads = 256;
template <typename T, int NV>
__global__ void __launch_bounds__(kAppendThreads) kv_append_kernel(const CacheView c, const int *new_offsets, int n_new,
                                                                   const T *k_new, const T *v_new, long long ld_k,
                                                                   long long ld_v, int rows_per_cta) {
  pdl_prologue();
  __shared__ int4 units[128];        // sequence, position, first row, rows
  __shared__ int n_units;
  __shared__ float part[kAppendThreads / 32];
  const int head = blockIdx.y, tid = threadIdx.x;
  const bool is_v = blockIdx.z != 0;
  if (tid == 0) n_units = 0;
  __syncthreads();
  const int row = blockIdx.x * rows_per_cta + tid;
  if (tid < rows_per_cta && row < n_new) {
    int seq = row, first = row, end = row + 1;
    if (new_offsets) {
      int a = 0, b = c.n_seqs + 1;   // first entry greater than row
      while (a < b) {
        const int m = (a + b) >> 1;
        if (new_offsets[m] <= row) a = m + 1; else b = m;
      }
      seq = a - 1;
      if (seq >= 0 && seq < c.n_seqs) { first = new_offsets[seq]; end = min(new_offsets[seq + 1], n_new); }
    }
    if (seq >= 0 && seq < c.n_seqs) {
      const long long pos = (long long)c.seq_lens[seq] + (row - (long long)first);
      const bool starts = row == max(first, 0) || (pos & (c.bt - 1)) == 0;
      if (c.seq_lens[seq] < 0 || pos >= (long long)c.max_blocks * c.bt) report(c.status, kWhereLength);
      else if (starts && end > row) {
        const int count = min(c.bt - (int)(pos & (c.bt - 1)), end - row);
        units[atomicAdd(&n_units, 1)] = make_int4(seq, (int)pos, row, count);   // any order: units are independent
      }
    }
  }
  __syncthreads();
  const T *src = is_v ? v_new : k_new;
  const long long ld = is_v ? ld_v : ld_k;
  const int vpr = c.D / 16;          // vectors per row
  const bool vec = (ld * sizeof(T)) % 16 == 0;
  for (int u = 0; u < n_units; ++u) {
    const int4 unit = units[u];
    const int block = cache_block(c, unit.x, unit.y >> c.bt_log2);
    if (block < 0) continue;
    const int held = unit.y & (c.bt - 1);
    Raw16<T> x[NV];
    float amax = 0.f;
#pragma unroll
    for (int n = 0; n < NV; ++n) {
      const int e = tid + n * kAppendThreads;
      if (e < unit.w * vpr) load16<T>(src + (long long)(unit.z + e / vpr) * ld + (long long)head * c.D + (e % vpr) * 16, vec, x[n]);
    }
#pragma unroll
    for (int n = 0; n < NV; ++n) {
      if (tid + n * kAppendThreads >= unit.w * vpr) break;
      float f[16];
      values16(x[n], f);
#pragma unroll
      for (int i = 0; i < 16; ++i) if (fabsf(f[i]) < INFINITY) amax = fmaxf(amax, fabsf(f[i]));
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
    if ((tid & 31) == 0) part[tid >> 5] = amax;
    const long long at = (long long)block * c.Hkv + head;
    float *scale = (is_v ? c.v_scale : c.k_scale) + at;
    uint8_t *codes = (is_v ? c.v : c.k) + at * c.bt * c.D;
    const float before = held > 0 ? *scale : 0.f;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kAppendThreads / 32; ++w) amax = fmaxf(amax, part[w]);
    const float after = fmaxf(before, pow2f(scale_exponent(amax)));
    __syncthreads();   // part and the old scale have been read
    if (tid == 0) *scale = after;
    if (held > 0 && before != after) {
      const float ratio = before / after;
      for (int e = tid; e < held * vpr; e += kAppendThreads) {
        uint4 *p = reinterpret_cast<uint4 *>(codes) + e;
        const uint4 w = *p;
        const uint32_t in[4] = {w.x, w.y, w.z, w.w};
        float f[16];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float2 t = values_of_codes((in[i >> 1] >> (16 * (i & 1))) & 0xffffu);
          f[2 * i] = t.x; f[2 * i + 1] = t.y;
        }
        *p = encode16(f, ratio);
      }
    }
    const float inv = 1.f / after;     // a power of two: exact
#pragma unroll
    for (int n = 0; n < NV; ++n) {
      const int e = tid + n * kAppendThreads;
      if (e >= unit.w * vpr) break;
      float f[16];
      values16(x[n], f);
      reinterpret_cast<uint4 *>(codes + (long long)held * c.D)[e] = encode16(f, inv);
    }
  }
}

// ------------------------------------------------------------------ decode attention
// The tokens of all (sequence, kv head, group of heads) pairs, in units of 64, form one list that is dealt to the CTAs:
// whole CTAs to each pair where pairs are few, else evenly, a share holding whole pairs and up to two partial ones.  Partial
// results (running maximum, sum, weighted values) meet in the workspace, and the CTA that finishes a pair last joins them in
// list order.
//
// Bound by the codes it streams: 1 byte per value, a token of one kv head is 2 * head_dim bytes for 2 * 2 * head_dim * heads
// flops.  Each warp has a ring of its own in shared memory that the copy engine fills, 16 tokens' keys and values (4 KB) a
// slot, requested by the warp itself as it empties one: 96 KB in flight per SM and no barrier between warps until a piece is
// done.  The copies swizzle their rows, and the rows and dims are dealt to the lanes so that 16-byte reads hit every bank.
// bf16: scores and weighted values on warp-level tensor-core instructions with the tokens as rows (S^T = K Q^T with 16 tokens
// x 8 heads, O^T = V^T P^T with 16 dims x 8 heads), codes converted in registers.  fp32: the same walk with fp32 FMAs, one
// head at a time, so that grouped heads read and convert a code once each (16 sequences of up to 4096 tokens, 64 / 8 heads: 150 us,
// where bf16 takes 26).
// 100003 tokens of 32 heads of 128: 154 us, 5.3 TB/s, as long as a plain sum over as many bytes takes; 16 sequences
// of up to 4096 tokens, 8 kv heads, capped: 32 us: about 8 until the first codes are there (lengths, table, queries), 15 of codes, 4 of joins, then the end.
// With 16-byte loads straight into registers, one step ahead: 158 and 45 us.
constexpr int kDecThreads = 192, kDecWarps = kDecThreads / 32, kDecCtasPerSm = 2;
constexpr int kUnit = 64;             // tokens of a unit
constexpr int kHeads = 8;             // heads of a pair (MMA columns)
constexpr int kMaxDecCtas = (kStatusBytes - sizeof(DeviceStatus)) / 2;   // 16-bit arrival counters in the workspace head
constexpr int kMaxPieces = 64;
constexpr int kRingBytes = 8192;      // of a warp: 2 steps of 16 tokens of 128 dims (3: 3% slower)
constexpr float kShift = 14.f;        // probabilities are held as 2^14 p in fp16: down to 2^-28 p without loss

struct DecodeParams {
  CacheView c;
  const void *q;
  void *o;
  float *lse, *part;                  // part: [CTA][2][heads_of_pair * (DM + 4)]: values, maximum, sum
  unsigned *arrived;
  const float *slopes;
  long long ldq, ldo;
  int H, group, chunks, window;       // chunks: pairs per kv head
  float scale, softcap, cap_in, cap_out;      // 1 / softcap, softcap log2(e)
  CUtensorMap tk, tv;                 // codes as [block, head][token][dim], boxes of 16 tokens
};

__device__ __forceinline__ uint32_t transpose_8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
// Rows and dims are dealt to the lanes in this order, so that lanes whose 16-byte reads go together hit different banks:
// bits (b2 b1 b0) of an index name the token, or the piece of a row, (b0 b2 b1).
__device__ __forceinline__ int dealt(int i) { return ((i & 1) << 2) | (i >> 1); }

// Codes of 16 tokens in registers.  Lane (g = lane / 4, c = lane % 4) holds, of the keys, tokens dealt(g) and dealt(g) + 8, bytes
// [16 c, 16 c + 16) of every 64; of the values, tokens c, c + 4, c + 8, c + 12 (rows 2c, 2c+1, 2c+8, 2c+9 of the product), bytes
// [dealt(g) DM/8, (dealt(g)+1) DM/8).
template <int DM> struct Codes {
  uint4 k[2][DM / 64];
  uint32_t v[4][DM / 32];
};
__device__ __forceinline__ uint4 lds128(uint32_t at) {
  uint4 w;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w.x), "=r"(w.y), "=r"(w.z), "=r"(w.w) : "r"(at));
  return w;
}
// from a slot: 16 rows of DM bytes of keys, then of values, as the copies swizzle them
template <int DM>
__device__ __forceinline__ void read_codes(uint32_t slot, Codes<DM> &r, int lane) {
  const int g = dealt(lane >> 2), c = lane & 3;
  auto piece = [](int row, int chunk) { return row * DM + ((DM == 128 ? chunk ^ (row & 7) : chunk ^ ((row >> 1) & 3)) << 4); };
#pragma unroll
  for (int a = 0; a < 2; ++a)
#pragma unroll
    for (int b = 0; b < DM / 64; ++b) r.k[a][b] = lds128(slot + piece(g + 8 * a, 4 * b + c));
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const int row = c + 4 * t;      // rows 2c, 2c+1, 2c+8, 2c+9 of the product
    if constexpr (DM == 128) {
      const uint4 w = lds128(slot + 16 * DM + piece(row, g));
      r.v[t][0] = w.x; r.v[t][1] = w.y; r.v[t][2] = w.z; r.v[t][3] = w.w;
    } else {
      const uint32_t at = slot + 16 * DM + piece(row, g >> 1) + 8 * (g & 1);
      asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(r.v[t][0]), "=r"(r.v[t][1]) : "r"(at));
    }
  }
}

// score in units of log2 from the product already scaled by `scale`.  Capped: near 0 by the polynomial, else tanh(x) = 1 - 2 / (1 +
// exp(2x)), whose absolute error of 1e-7 is then a relative one (the hardware's approximate tanh is only good to 2^-11, which a
// cap of 50 would turn into 0.02 on a score)
__device__ __forceinline__ float decode_score(const DecodeParams &P, float z, float slope, int back) {
  if (P.softcap > 0.f) {
    const float x = z * P.cap_in, u = x * x;
    float t = x * fmaf(u, fmaf(u, fmaf(u, fmaf(u, fmaf(u, kTanh5, kTanh4), kTanh3), kTanh2), kTanh1), kTanh0);
    if (!(fabsf(x) <= kTanhPolyMax)) t = fmaf(-2.f, __fdividef(1.f, 1.f + ex2(x * (2.f * kLog2e))), 1.f);
    z = t * P.cap_out;
  } else {
    z *= kLog2e;
  }
  return fmaf(-slope * kLog2e, (float)back, z);
}

constexpr uint32_t kNoUnit = 0xffffffffu, kPlain = 0x3f800001u;      // no scale yet; units of 1 for good
// of a positive normal fp32 number's bits
__device__ __forceinline__ bool power_of_two(uint32_t bits) { return (bits & 0x807fffffu) == 0 && bits - 1 < 0x7f7fffffu; }

// State of one warp over a piece: bf16 runs 8 heads as MMA columns, fp32 one head.
template <int DM, bool F32> struct WarpState;

template <int DM> struct WarpState<DM, false> {
  uint32_t qf[DM / 16][2];            // Q^T fragments: head g, dims as Codes::k deals them
  float qs[2], slope[2];              // of heads 2c, 2c + 1: scale of the normalised query, slope
  float m[2], l[2], acc[DM / 16][4];
  uint32_t unit;                      // acc is in units of this fp32 number (its bits), the scale of the values' last block
  int low, high;                      // exponents of the smallest and largest unit so far
  // a lane's query values, as they are stored: head g, dims 64 b + 16 c .. of every 64
  struct Query { uint4 w[DM / 32]; };
  static __device__ __forceinline__ void ask(const DecodeParams &P, int seq, int h0, int nh, int lane, Query &r) {
    const int g = lane >> 2, c = lane & 3;
    const __nv_bfloat16 *q = (const __nv_bfloat16 *)P.q + (long long)seq * P.ldq + (long long)(h0 + g) * P.c.D;
#pragma unroll
    for (int b = 0; b < DM / 32; ++b) {
      const int d = 64 * (b >> 1) + 16 * c + 8 * (b & 1);
      r.w[b] = make_uint4(0, 0, 0, 0);
      if (g >= nh || d >= P.c.D) continue;
      if ((P.ldq & 7) == 0) {
        r.w[b] = __ldg(reinterpret_cast<const uint4 *>(q + d));
      } else {
        r.w[b] = make_uint4(load_word(q + d), load_word(q + d + 2), load_word(q + d + 4), load_word(q + d + 6));
      }
    }
  }
  __device__ __forceinline__ void start(const DecodeParams &P, const Query &r, int h0, int nh, int lane) {
    const int c = lane & 3;
    // a query row is scaled by a power of two so that its largest value is in [2^14, 2^15): fp16 then holds every bit
    // of its bf16 values down to 2^-28 of the largest
    float amax = 0.f, f[DM / 16][4];
#pragma unroll
    for (int s = 0; s < DM / 16; ++s) {
      const uint4 w = r.w[s >> 1];
      const uint32_t lo = (s & 1) ? w.z : w.x, hi = (s & 1) ? w.w : w.y;
      f[s][0] = __uint_as_float(lo << 16); f[s][1] = __uint_as_float(lo & 0xffff0000u);
      f[s][2] = __uint_as_float(hi << 16); f[s][3] = __uint_as_float(hi & 0xffff0000u);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (fabsf(f[s][e]) < INFINITY) amax = fmaxf(amax, fabsf(f[s][e]));
    }
    amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
    amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
    int e = (int)(__float_as_uint(amax) >> 23) - 127 - 14;      // amax 2^-e in [2^14, 2^15)
    if (__float_as_uint(amax) < 0x00800000u) e = -126 - 14;     // zero or subnormal
    e = max(e, -120);                                           // 2^-e stays finite; such rows are below any use
    const float up = pow2f(-e);
#pragma unroll
    for (int s = 0; s < DM / 16; ++s) {
      qf[s][0] = pack_half2(f[s][0] * up, f[s][1] * up);
      qf[s][1] = pack_half2(f[s][2] * up, f[s][3] * up);
    }
    const float down = P.scale * pow2f(e);
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      qs[n] = __shfl_sync(0xffffffffu, down, (2 * c + n) * 4);
      slope[n] = (P.slopes && 2 * c + n < nh) ? P.slopes[h0 + 2 * c + n] : 0.f;
      m[n] = -INFINITY; l[n] = 0.f;
    }
#pragma unroll
    for (int i = 0; i < DM / 16; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) acc[i][k] = 0.f;
    unit = kNoUnit;
  }
  // 16 tokens from j0; those outside [first, len) count for nothing
  __device__ __forceinline__ void step(const DecodeParams &P, Codes<DM> &r, float ks, float vs, int j0, int first, int len, int lane) {
    const int g = lane >> 2, c = lane & 3;
    float part[DM / 64][4], s[4];       // one chain of products per 64 dims
#pragma unroll
    for (int b = 0; b < DM / 64; ++b) {
      part[b][0] = part[b][1] = part[b][2] = part[b][3] = 0.f;
      const uint32_t w0[4] = {r.k[0][b].x, r.k[0][b].y, r.k[0][b].z, r.k[0][b].w};
      const uint32_t w1[4] = {r.k[1][b].x, r.k[1][b].y, r.k[1][b].z, r.k[1][b].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t a0, a1, a2, a3;
        half2s_of_codes(w0[i], a0, a2);
        half2s_of_codes(w1[i], a1, a3);
        mma_16816(part[b], a0, a1, a2, a3, qf[4 * b + i][0], qf[4 * b + i][1]);
      }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) s[k] = DM == 64 ? part[0][k] : part[0][k] + part[DM / 64 - 1][k];
    const bool edge = j0 < first || j0 + 16 > len;
    float mx[2];
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      const float f = qs[n] * ks;
#pragma unroll
      for (int a = 0; a < 2; ++a) {
        const int j = j0 + dealt(g) + 8 * a;
        float z = decode_score(P, s[2 * a + n] * f, slope[n], len - 1 - j);
        if (edge && (j < first || j >= len)) z = -INFINITY;
        s[2 * a + n] = z;
      }
      mx[n] = fmaxf(s[n], s[2 + n]);
    }
    if (edge) {   // what lies behind the last token is not part of the sequence: 0 * NaN must not arise
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int j = j0 + c + 4 * t;
        if (j < first || j >= len)
#pragma unroll
          for (int i = 0; i < DM / 32; ++i) r.v[t][i] = 0;
      }
    }
    // The maximum follows only when a score is beyond twice its power of two (probabilities stay below 2^15, fp16 holds them), and the
    // products add up in the tensor cores while neither it nor the block scale changes: 2^-24 of a sum each time.
    float alpha[2] = {1.f, 1.f};
    bool direct = true;
    if (__any_sync(0xffffffffu, mx[0] > m[0] + 1.f || mx[1] > m[1] + 1.f)) {
#pragma unroll
      for (int n = 0; n < 2; ++n) {
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) mx[n] = fmaxf(mx[n], __shfl_xor_sync(0xffffffffu, mx[n], o));
        const float mn = fmaxf(m[n], mx[n]);
        alpha[n] = ex2(m[n] - (mn == -INFINITY ? 0.f : mn));
        m[n] = mn;
        l[n] *= alpha[n];
      }
      direct = false;
    }
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      const float base = (m[n] == -INFINITY ? 0.f : m[n]) - kShift;
      s[n] = ex2(s[n] - base);
      s[2 + n] = ex2(s[2 + n] - base);
      l[n] += s[n] + s[2 + n];
    }
    const uint32_t b0 = transpose_8x8(pack_half2(s[0], s[1])), b1 = transpose_8x8(pack_half2(s[2], s[3]));
    // A scale as the cache writes it is a power of two.  Sums stay below 2^54 in their block's unit, so that units at most 2^60 apart
    // neither overflow nor lose anything; beyond that, or for any other scale, sums are kept in units of 1.
    const uint32_t bits = __float_as_uint(vs);
    float times = 1.f;                // what becomes of the sums so far
    if (bits != unit && unit != kPlain) {
      const int e = (int)(bits >> 23) - 127;
      const bool first = unit == kNoUnit;
      low = first ? e : min(low, e);
      high = first ? e : max(high, e);
      if (power_of_two(bits) && high - low <= 60) {
        if (!first) times = pow2f((int)(unit >> 23) - 127 - e);
        unit = bits;
      } else {
        if (!first) times = __uint_as_float(unit);
        unit = kPlain;
      }
      direct = false;
    }
    if (unit != kPlain) {
      if (!direct) {
#pragma unroll
        for (int i = 0; i < DM / 16; ++i)
#pragma unroll
          for (int k = 0; k < 4; ++k) acc[i][k] *= alpha[k & 1] * times;
      }
#pragma unroll
      for (int i = 0; i < DM / 16; ++i) weigh(acc[i], r, i, b0, b1);
    } else {
#pragma unroll
      for (int i = 0; i < DM / 16; ++i) {
        float t[4] = {0.f, 0.f, 0.f, 0.f};
        weigh(t, r, i, b0, b1);
#pragma unroll
        for (int k = 0; k < 4; ++k) acc[i][k] = fmaf(acc[i][k] * times, alpha[k & 1], vs * t[k]);
      }
    }
  }
  // bytes 2i, 2i+1 of the four tokens: rows g and g + 8 of this MMA are dims dealt(g) DM/8 + 2i and + 1
  static __device__ __forceinline__ void weigh(float (&d)[4], const Codes<DM> &r, int i, uint32_t b0, uint32_t b1) {
    const uint32_t sel = (i & 1) ? 0x7362u : 0x5140u;
    const uint32_t lo = __byte_perm(r.v[0][i / 2], r.v[1][i / 2], sel), hi = __byte_perm(r.v[2][i / 2], r.v[3][i / 2], sel);
    uint32_t a0, a1, a2, a3;
    half2s_of_codes(lo, a0, a1);
    half2s_of_codes(hi, a2, a3);
    mma_16816(d, a0, a1, a2, a3, b0, b1);
  }
  // maximum, sum and weighted values of every head to shared memory: sm[head * (DM + 4) + ...]
  __device__ __forceinline__ void finish(float *sm, int lane) {
    const int g = lane >> 2, c = lane & 3;
    const float one = unit == kNoUnit || unit == kPlain ? 1.f : __uint_as_float(unit);
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      float sum = l[n];
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      float *p = sm + (2 * c + n) * (DM + 4);
      if (g == 0) { p[DM] = m[n]; p[DM + 1] = sum; }
#pragma unroll
      for (int i = 0; i < DM / 16; ++i) {
        p[dealt(g) * (DM / 8) + 2 * i] = acc[i][n] * one;
        p[dealt(g) * (DM / 8) + 2 * i + 1] = acc[i][2 + n] * one;
      }
    }
  }
};

template <int DM> struct WarpState<DM, true> {
  float q[DM / 4], slope;             // this lane's dims of the query, scaled
  float m, l, acc[DM / 8];            // acc: dims [g DM/8, ..) summed over this lane's tokens
  struct Query { float q[DM / 4]; };
  static __device__ __forceinline__ void ask(const DecodeParams &P, int seq, int h0, int, int lane, Query &r) {
    const int c = lane & 3;
    const float *p = (const float *)P.q + (long long)seq * P.ldq + (long long)h0 * P.c.D;
#pragma unroll
    for (int e = 0; e < DM / 4; ++e) {
      const int d = 64 * (e / 16) + 16 * c + (e & 15);
      r.q[e] = d < P.c.D ? p[d] : 0.f;
    }
  }
  __device__ __forceinline__ void start(const DecodeParams &P, const Query &r, int h0, int, int) {
#pragma unroll
    for (int e = 0; e < DM / 4; ++e) q[e] = r.q[e];
    slope = P.slopes ? P.slopes[h0] : 0.f;
    m = -INFINITY; l = 0.f;
#pragma unroll
    for (int i = 0; i < DM / 8; ++i) acc[i] = 0.f;
  }
  __device__ __forceinline__ void step(const DecodeParams &P, Codes<DM> &r, float ks, float vs, int j0, int first, int len, int lane) {
    const int g = lane >> 2, c = lane & 3;
    float s[2];
#pragma unroll
    for (int a = 0; a < 2; ++a) {
      float dot = 0.f;
#pragma unroll
      for (int b = 0; b < DM / 64; ++b) {
        const uint32_t w[4] = {r.k[a][b].x, r.k[a][b].y, r.k[a][b].z, r.k[a][b].w};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float2 f = values_of_codes((w[i >> 1] >> (16 * (i & 1))) & 0xffffu);
          dot = fmaf(q[16 * b + 2 * i], f.x, dot);
          dot = fmaf(q[16 * b + 2 * i + 1], f.y, dot);
        }
      }
      dot += __shfl_xor_sync(0xffffffffu, dot, 1);
      dot += __shfl_xor_sync(0xffffffffu, dot, 2);
      const int j = j0 + dealt(g) + 8 * a;
      float z = dot * ks * P.scale;
      if (P.softcap > 0.f) z = P.softcap * tanhf(z / P.softcap);
      z = (z - slope * (float)(len - 1 - j)) * kLog2e;
      s[a] = (j < first || j >= len) ? -INFINITY : z;
    }
    float mx = fmaxf(s[0], s[1]);
#pragma unroll
    for (int o = 4; o < 32; o <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
    const float mn = fmaxf(m, mx), base = mn == -INFINITY ? 0.f : mn, alpha = exp2f(m - base);
    m = mn;
    s[0] = exp2f(s[0] - base);
    s[1] = exp2f(s[1] - base);
    l = l * alpha + (s[0] + s[1]);    // the four lanes of a token hold the same value
#pragma unroll
    for (int i = 0; i < DM / 8; ++i) acc[i] *= alpha;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int tok = 2 * c + (t & 1);                        // row g' of the keys' layout
      const float p = __shfl_sync(0xffffffffu, s[t >> 1], tok * 4) * vs;
      const int j = j0 + c + 4 * t;
      const bool in = j >= first && j < len;
#pragma unroll
      for (int i = 0; i < DM / 16; ++i) {
        const float2 f = values_of_codes((r.v[t][i >> 1] >> (16 * (i & 1))) & 0xffffu);
        acc[2 * i] = in ? fmaf(p, f.x, acc[2 * i]) : acc[2 * i];
        acc[2 * i + 1] = in ? fmaf(p, f.y, acc[2 * i + 1]) : acc[2 * i + 1];
      }
    }
  }
  __device__ __forceinline__ void finish(float *sm, int lane) {
    const int g = lane >> 2, c = lane & 3;
#pragma unroll
    for (int o = 4; o < 32; o <<= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
#pragma unroll
    for (int i = 0; i < DM / 8; ++i) {
      acc[i] += __shfl_xor_sync(0xffffffffu, acc[i], 1);
      acc[i] += __shfl_xor_sync(0xffffffffu, acc[i], 2);
      if (c == 0) sm[dealt(g) * (DM / 8) + i] = acc[i];
    }
    if (lane == 0) { sm[DM] = m; sm[DM + 1] = l; }
  }
};

// four dims of a finished row, or of what is left of one
template <int DM, bool F32>
__device__ __forceinline__ void decode_store(const DecodeParams &P, int seq, int h, int d, float4 v, float m, float l) {
  const float r[4] = {v.x, v.y, v.z, v.w};
  if (d < P.c.D)                      // dims come in fours, and their number is a multiple of 16
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float o = l == 0.f ? 0.f : r[k] / l;
      const long long at = (long long)seq * P.ldo + (long long)h * P.c.D + d + k;
      if constexpr (F32) ((float *)P.o)[at] = o;
      else ((__nv_bfloat16 *)P.o)[at] = __float2bfloat16_rn(o);
    }
  if (d == 0 && P.lse) P.lse[(long long)seq * P.H + h] = l == 0.f ? -INFINITY : (m + log2f(l) - (F32 ? 0.f : kShift)) * kLn2;
}

// Joins the partial results of nh heads: part i of head h has DM values, a maximum and a sum at slot i of the
// CTAs from c_first on.  All parts' weights first (w: nh * (n + 2) floats of
// shared memory), then the values, eight loads in flight, the first of them requested ahead of the weights: one after the other,
// 300 parts took 240 us.  Sums run in the parts' order.
template <int DM, bool F32>
__device__ __forceinline__ void join_parts(const DecodeParams &P, int c_first, int n, int seq, int h0, int nh, float *w) {
  constexpr int kRow = DM + 4, kPart = (F32 ? 1 : kHeads) * kRow;
  // through L2: a line of this CTA's L1 may hold a neighbouring slot's older contents
  auto part = [&](int i, int h) { return P.part + ((long long)(c_first + i) * 2 + (i == 0 ? 1 : 0)) * kPart + h * kRow; };
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, items = nh * (DM / 4);
  float *top = w + nh * n, *total = top + nh;
  constexpr int kAhead = 4;
  float4 x[2][kAhead];
  auto load = [&](int e, int i) {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const int at = e + b * kDecThreads;
      if (at < items)
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
          if (i + k < n) x[b][k] = __ldcg(reinterpret_cast<const float4 *>(part(i + k, at / (DM / 4)) + 4 * (at % (DM / 4))));
    }
  };
  load(threadIdx.x, 0);
  for (int h = warp; h < nh; h += kDecWarps) {
    float m = -INFINITY, l = 0.f;
    float2 t = make_float2(-INFINITY, 0.f);
    for (int i = lane; i < n; i += 32) {
      t = __ldcg(reinterpret_cast<const float2 *>(part(i, h) + DM));
      w[h * n + i] = t.x;
      m = fmaxf(m, t.x);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    const float base = m == -INFINITY ? 0.f : m;
    for (int i = lane; i < n; i += 32) {
      const float a = exp2f(w[h * n + i] - base);      // a part without tokens has maximum -infinity and weight 0
      w[h * n + i] = a;
      l = fmaf(a, n <= 32 ? t.y : __ldcg(part(i, h) + DM + 1), l);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
    if (lane == 0) { top[h] = m; total[h] = l; }
  }
  __syncthreads();
  for (int e = threadIdx.x; e < items; e += 2 * kDecThreads) {
    float4 v[2] = {make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f)};
    for (int i = 0; i < n; i += kAhead) {
      if (i > 0 || e != (int)threadIdx.x) load(e, i);
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int at = e + b * kDecThreads;
        if (at < items) {
          const float *a = w + at / (DM / 4) * n + i;
#pragma unroll
          for (int k = 0; k < kAhead; ++k)
            if (i + k < n) {
              v[b].x = fmaf(a[k], x[b][k].x, v[b].x); v[b].y = fmaf(a[k], x[b][k].y, v[b].y);
              v[b].z = fmaf(a[k], x[b][k].z, v[b].z); v[b].w = fmaf(a[k], x[b][k].w, v[b].w);
            }
        }
      }
    }
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const int at = e + b * kDecThreads, h = at / (DM / 4);
      if (at < items) decode_store<DM, F32>(P, seq, h0 + h, 4 * (at % (DM / 4)), v[b], top[h], total[h]);
    }
  }
}

template <int DM, bool F32>
__global__ void __launch_bounds__(kDecThreads, kDecCtasPerSm) decode_attention_kernel(const __grid_constant__ DecodeParams P) {
  pdl_prologue();
  constexpr int NH = F32 ? 1 : kHeads;
  constexpr int kRow = DM + 4, kPart = NH * kRow;
  constexpr int kSlot = 32 * DM, kSlots = kRingBytes / kSlot;
  // [warps][kRingBytes] rings; [warps][kPart] partial results; [warps][kSlots] barriers; the units before every sequence
  extern __shared__ uint8_t smem_raw[];
  static_assert(NH * (kMaxDecCtas + 2) <= kDecWarps * kPart, "weights of a join");
  const uint32_t raw = smem_u32(smem_raw), ring0 = (raw + 1023u) & ~1023u;
  float *sm = reinterpret_cast<float *>(smem_raw + (ring0 - raw) + kDecWarps * kRingBytes);
  const uint32_t bars = ring0 + kDecWarps * (kRingBytes + kPart * 4);
  long long *before = reinterpret_cast<long long *>(smem_raw + (bars - raw) + kDecWarps * kSlots * 8);   // n_seqs + 1
  __shared__ long long warp_total[kDecWarps];
  __shared__ int last;
  __shared__ volatile int abort_flag;
  const CacheView &c = P.c;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int pairs_per_seq = c.Hkv * P.chunks;
  const uint32_t ring = ring0 + warp * kRingBytes, full = bars + warp * kSlots * 8;
  if (lane == 0) {
    for (int i = 0; i < kSlots; ++i) mbar_init(full + 8 * i, 1);
    fence_barrier_init();
  }
  if (tid == 0) abort_flag = 0;

  // ---- units before every sequence: an exclusive scan over the lengths, the same in every CTA
  auto seq_range = [&](int seq, int &first, int &len) {
    len = c.seq_lens[seq];
    const long long room = (long long)c.max_blocks * c.bt;
    if (len < 0 || len > room) {
      if (tid == 0) report(c.status, kWhereLength);
      len = len < 0 ? 0 : (int)room;
    }
    first = P.window > 0 && len > P.window ? len - P.window : 0;
  };
  const int per = (c.n_seqs + kDecThreads - 1) / kDecThreads;
  long long mine = 0;
  for (int s = tid * per; s < min(c.n_seqs, (tid + 1) * per); ++s) {
    int first, len = c.seq_lens[s];
    const long long room = (long long)c.max_blocks * c.bt;
    if (len < 0 || len > room) { report(c.status, kWhereLength); len = len < 0 ? 0 : (int)room; }
    first = P.window > 0 && len > P.window ? len - P.window : 0;
    before[s] = mine;
    mine += (long long)((len - (first & ~15) + kUnit - 1) / kUnit) * pairs_per_seq;
  }
  long long sum = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long up = __shfl_up_sync(0xffffffffu, sum, o);
    if (lane >= o) sum += up;
  }
  if (lane == 31) warp_total[warp] = sum;
  __syncthreads();
  long long base = sum - mine, total = 0;
#pragma unroll
  for (int w = 0; w < kDecWarps; ++w) {
    if (w < warp) base += warp_total[w];
    total += warp_total[w];
  }
  for (int s = tid * per; s < min(c.n_seqs, (tid + 1) * per); ++s) before[s] += base;
  if (tid == 0) before[c.n_seqs] = total;
  __syncthreads();

  // ---- sequences without tokens have no unit: their rows are written here
  for (int s = blockIdx.x; s < c.n_seqs; s += gridDim.x)
    if (before[s + 1] == before[s])
      for (int e = tid; e < P.H * (DM / 4); e += kDecThreads)
        decode_store<DM, F32>(P, s, e / (DM / 4), 4 * (e % (DM / 4)), make_float4(0.f, 0.f, 0.f, 0.f), 0.f, 0.f);

  // No more than kMaxPieces CTAs to a pair on the average, since one CTA joins what a pair's leave.  One long sequence among short
  // ones can have more, up to the whole grid: the join has room for as many.
  const long long G = min(min((long long)gridDim.x, total), (long long)kMaxPieces * c.n_seqs * pairs_per_seq);
  if (blockIdx.x >= G) return;

  // ---- this CTA's share.  Where pairs are few, whole CTAs to each pair, ceil(units / T) of them with the smallest T that the
  // grid allows: a second piece costs a CTA another start, join and end.  T may be this much above the even share (8 units and a
  // sixteenth: about a piece's fixed cost); otherwise the list is cut evenly.  (16 sequences of up to 4096 tokens, 8 kv heads: even
  // cuts 45 us.)  One lane holds a sequence, one a candidate for T.
  int my_seq = 0, my_pair = 0, my_part = 0, my_parts = 0;     // parts 0: cut evenly
  if (c.n_seqs <= 32 && c.n_seqs * pairs_per_seq <= G && total < (1 << 23)) {
    const int grid = (int)G;
    const int n_s = lane < c.n_seqs ? (int)(before[lane + 1] - before[lane]) / pairs_per_seq : 0;
    const int even = ((int)total + grid - 1) / grid, T = even + (even / 16 + 8) * lane / 31;
    const float rcp_T = 1.f / (float)T;
    auto parts_of = [&](int units, int t, float r) { return units == 0 ? 0 : max(1, (int)((float)(units + t - 1) * r)); };
    int ctas = 0;
    for (int s = 0; s < c.n_seqs; ++s) ctas += parts_of(__shfl_sync(0xffffffffu, n_s, s), T, rcp_T);
    const unsigned fits = __ballot_sync(0xffffffffu, (long long)ctas * pairs_per_seq <= grid);
    if (fits) {
      const int best = __ffs(fits) - 1;
      const int k = parts_of(n_s, __shfl_sync(0xffffffffu, T, best), __shfl_sync(0xffffffffu, rcp_T, best));
      int upto = k * pairs_per_seq;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int up = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += up;
      }
      const unsigned behind = __ballot_sync(0xffffffffu, upto > (int)blockIdx.x);
      if (!behind) return;            // fewer CTAs than the grid has
      my_seq = __ffs(behind) - 1;
      my_parts = __shfl_sync(0xffffffffu, k, my_seq);
      const int at = (int)blockIdx.x - (__shfl_sync(0xffffffffu, upto, my_seq) - my_parts * pairs_per_seq);
      my_pair = at / my_parts;
      my_part = at - my_pair * my_parts;
    }
  }
  long long u0, u1;
  int seq = my_seq;
  if (my_parts > 0) {
    const int n = (int)(before[seq + 1] - before[seq]) / pairs_per_seq;      // times the CTAs below 2^32
    const long long at = before[seq] + (long long)n * my_pair;
    u0 = at + (unsigned)n * (unsigned)my_part / (unsigned)my_parts;
    u1 = at + (unsigned)n * (unsigned)(my_part + 1) / (unsigned)my_parts;
  } else {
    u0 = total * blockIdx.x / G;
    u1 = total * (blockIdx.x + 1) / G;
    int a = 0, b = c.n_seqs;          // last sequence with before[seq] <= u0
    while (b - a > 1) {
      const int mid = (a + b) >> 1;
      if (before[mid] <= u0) a = mid; else b = mid;
    }
    seq = a;
  }
  // A piece: this CTA's units of one pair.  Its tokens are dealt to the warps in steps of 16: step i of a warp is step
  // warp + kDecWarps i of the piece, n of them.  What is needed only when it is done waits in shared memory.
  struct Piece { int seq, first, len, hk, j_begin, n; };
  struct Rest {
    int h0, nh;
    int slot;                         // 1: the pair that starts in this CTA's share and goes on; 0: one that started before it
    int c_first, parts;               // the pair's first CTA, and how many work on it
  };
  __shared__ Rest rest[2];
  const bool whole_ctas = my_parts > 0;
  if (tid == 0) { rest[0].c_first = (int)blockIdx.x - my_part; rest[0].parts = my_parts; }
  int h0, nh;                         // heads of the piece located last
  auto locate = [&](long long u, Piece &p, Rest &r) {      // returns where the piece ends
    while (before[seq + 1] <= u) ++seq;
    p.seq = seq;
    seq_range(seq, p.first, p.len);
    const int t_base = p.first & ~15;
    const int n_units = (p.len - t_base + kUnit - 1) / kUnit;
    const long long local = u - before[seq];
    const int pair = total < (1 << 30) ? (int)local / n_units : (int)(local / n_units), unit = (int)(local - (long long)pair * n_units);
    const long long pair_u0 = u - unit, pair_u1 = pair_u0 + n_units, end = min(u1, pair_u1);
    p.hk = pair / P.chunks;
    p.j_begin = t_base + unit * kUnit;
    const int steps = (min(t_base + (unit + (int)(end - u)) * kUnit, p.len) - p.j_begin + 15) / 16;
    p.n = steps > warp ? (steps - warp + kDecWarps - 1) / kDecWarps : 0;
    h0 = p.hk * P.group + (pair - p.hk * P.chunks) * NH;
    nh = min(NH, (p.hk + 1) * P.group - h0);
    if (tid == 0) {
      r.h0 = h0;
      r.nh = nh;
      r.slot = unit == 0;
      if (!whole_ctas) {
        r.c_first = (int)(((pair_u0 + 1) * G - 1) / total);
        r.parts = (int)((pair_u1 * G - 1) / total) - r.c_first + 1;
      }
    }
    return end;
  };
  // Codes are requested kSlots steps ahead, and before the piece ahead of theirs is written out; lanes look up the blocks of 32 steps
  // at a time, half of that ahead, and their scales as soon as the blocks are known.
  int ids = -1, next_ids = -1, cur_ids = -1;
  float ks = 0.f, vs = 0.f, next_ks = 0.f, next_vs = 0.f;
  unsigned turn = 0;                  // copies of earlier pieces
  auto look_up = [&](const Piece &p, int i) {
    return i < p.n ? cache_block(c, p.seq, (p.j_begin + 16 * (warp + kDecWarps * i)) >> c.bt_log2) : -1;
  };
  auto scales = [&](const Piece &p) {
    const long long at = (long long)ids * c.Hkv + p.hk;
    next_ks = ids >= 0 ? c.k_scale[at] : 0.f;
    next_vs = ids >= 0 ? c.v_scale[at] : 0.f;
  };
  auto request = [&](const Piece &p, int i) {
    if ((i & 31) == 0 && i > 0) {
      ids = next_ids;
      scales(p);
    }
    const int id = __shfl_sync(0xffffffffu, ids, i & 31);
    if (lane == 0) {
      const unsigned k = (turn + i) % kSlots;
      if (id >= 0) {
        const int tok = (p.j_begin + 16 * (warp + kDecWarps * i)) & (c.bt - 1);
        mbar_arrive_expect_tx(full + 8 * k, kSlot);
        tma_load_3d(ring + k * kSlot, &P.tk, full + 8 * k, 0, tok, id * c.Hkv + p.hk);
        tma_load_3d(ring + k * kSlot + kSlot / 2, &P.tv, full + 8 * k, 0, tok, id * c.Hkv + p.hk);
      } else {
        mbar_arrive(full + 8 * k);
      }
    }
    if ((i & 31) == 16) next_ids = look_up(p, i + 16 + lane);
  };
  int asked = 0;
  typename WarpState<DM, F32>::Query query;
  auto begin = [&](const Piece &p, int h0, int nh) {
    ids = cur_ids = look_up(p, lane);
    WarpState<DM, F32>::ask(P, p.seq, h0, nh, lane, query);
    for (asked = 0; asked < min(p.n, kSlots); ++asked) request(p, asked);
    scales(p);
  };

  Piece p;
  long long u = locate(u0, p, rest[0]);
  begin(p, h0, nh);
  __syncthreads();
  for (int turn_of = 0;; turn_of ^= 1) {
    WarpState<DM, F32> state;
    state.start(P, query, rest[turn_of].h0, rest[turn_of].nh, lane);
    query = {};                       // its registers are free until the next piece
    for (int i = 0; i < p.n; ++i) {
      if ((i & 31) == 0) {
        if (i > 0) cur_ids = ids;
        ks = next_ks;
        vs = next_vs;
      }
      const unsigned k = (turn + i) % kSlots;
      const bool ok = mbar_wait_fast(full + 8 * k, ((turn + i) / kSlots) & 1, &abort_flag, c.status, kWhereCodes);
      if (!__all_sync(0xffffffffu, ok)) {
        for (int j = i; j < asked; ++j) drain_copies(full + 8 * ((turn + j) % kSlots), ((turn + j) / kSlots) & 1);
        break;
      }
      const bool there = __shfl_sync(0xffffffffu, cur_ids, i & 31) >= 0;
      Codes<DM> r;
      read_codes<DM>(ring + k * kSlot, r, lane);
      __syncwarp();                   // every lane has its codes
      if (asked < p.n) request(p, asked++);
      if (there)
        state.step(P, r, __shfl_sync(0xffffffffu, ks, i & 31), __shfl_sync(0xffffffffu, vs, i & 31),
                   p.j_begin + 16 * (warp + kDecWarps * i), p.first, p.len, lane);
    }
    turn += asked;
    asked = 0;
    state.finish(sm + warp * kPart, lane);
    const Rest &r = rest[turn_of];
    const int done = p.seq;
    const bool more = u < u1;
    if (more) {
      u = locate(u, p, rest[turn_of ^ 1]);
      begin(p, h0, nh);
    }
    __syncthreads();
    float *slot = P.part + ((long long)blockIdx.x * 2 + r.slot) * kPart;
    const bool whole = r.parts == 1;
    for (int e = tid; e < r.nh * (DM / 4); e += kDecThreads) {
      const int h = e / (DM / 4), d = 4 * (e % (DM / 4));
      const float *at = sm + h * kRow;
      float m = -INFINITY, l = 0.f;
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int i = 0; i < kDecWarps; ++i) m = fmaxf(m, at[i * kPart + DM]);
      const float lift = m == -INFINITY ? 0.f : m;
#pragma unroll
      for (int i = 0; i < kDecWarps; ++i) {
        const float a = exp2f(at[i * kPart + DM] - lift);
        const float4 x = *reinterpret_cast<const float4 *>(at + i * kPart + d);
        v.x = fmaf(a, x.x, v.x); v.y = fmaf(a, x.y, v.y); v.z = fmaf(a, x.z, v.z); v.w = fmaf(a, x.w, v.w);
        l = fmaf(a, at[i * kPart + DM + 1], l);
      }
      if (whole) {
        decode_store<DM, F32>(P, done, r.h0 + h, d, v, m, l);
      } else {
        *reinterpret_cast<float4 *>(slot + h * kRow + d) = v;
        if (d == 0) *reinterpret_cast<float2 *>(slot + h * kRow + DM) = make_float2(m, l);
      }
    }
    __syncthreads();                  // partial results read; those of this CTA written
    if (!whole) {
      if (tid == 0) {
        const int shift = 16 * (r.c_first & 1);
        __threadfence();
        const unsigned old = atomicAdd(P.arrived + (r.c_first >> 1), 1u << shift);
        last = (int)((old >> shift) & 0xffffu) == r.parts - 1;
        if (last) atomicSub(P.arrived + (r.c_first >> 1), (unsigned)r.parts << shift);   // armed for the next launch
        __threadfence();
      }
      __syncthreads();
      if (last) {
        join_parts<DM, F32>(P, r.c_first, r.parts, done, r.h0, r.nh, sm);
        __syncthreads();
      }
    }
    if (!more) break;
  }
}

// ------------------------------------------------------------------ host side
templora_status_t check_decode(const templora_attn_t *a, const templora_kv_cache_t *c, bool pointers) {
  TL_TRY(attn_check_desc(a));
  TL_TRY(check_cache(c, pointers));
  if (a->n_kv_heads != c->n_kv_heads || a->head_dim != c->head_dim) return TEMPLORA_ERR_INVALID_ARG;
  if (a->n_docs != 0 || a->prefix_lens) return TEMPLORA_ERR_UNSUPPORTED;
  return TEMPLORA_OK;
}
// The partial results' room does not depend on the device: the most CTAs any launch may have.
size_t decode_need(const templora_attn_t *a) {
  const int dm = a->head_dim <= 64 ? 64 : 128, nh = a->dtype == TEMPLORA_F32 ? 1 : kHeads;
  return kStatusBytes + align_up((size_t)kMaxDecCtas * 2 * nh * (dm + 4) * sizeof(float), kWsAlign);
}

template <int DM, bool F32>
templora_status_t launch_decode(DecodeParams &p, cudaStream_t st) {
  const size_t rings = 1024 + (size_t)kDecWarps * (kRingBytes + (F32 ? 1 : kHeads) * (DM + 4) * 4 + kRingBytes / (32 * DM) * 8);
  const size_t smem = rings + (size_t)(p.c.n_seqs + 1) * sizeof(long long);
  TL_TRY((allow_smem<decode_attention_kernel<DM, F32>>(rings + (kMaxSeqs + 1) * sizeof(long long))));
  const long long planes = (long long)p.c.n_blocks * p.c.Hkv;
  if (!make_map_codes(&p.tk, p.c.k, p.c.D, p.c.bt, planes, DM) || !make_map_codes(&p.tv, p.c.v, p.c.D, p.c.bt, planes, DM))
    return TEMPLORA_ERR_CUDA;
  int sms = 0;
  TL_TRY(stream_sms(st, &sms));
  int ctas = sms * kDecCtasPerSm;
  if (ctas > kMaxDecCtas) ctas = kMaxDecCtas;
  // no more CTAs than units there could be
  const long long most = (long long)p.c.n_seqs * p.c.Hkv * p.chunks * (((long long)p.c.max_blocks * p.c.bt + 15) / kUnit + 1);
  if (ctas > most) ctas = (int)most;
  LaunchScope scope(kKindKvCache, st);
  TL_CUDA_CHECK(launch_pdl(decode_attention_kernel<DM, F32>, dim3(ctas), dim3(kDecThreads), smem, st, p));
  return TEMPLORA_OK;
}

template <typename T, int NV>
templora_status_t launch_append(const CacheView &c, const int *offsets, int n_new, const void *k, const void *v, long long lk,
                                long long lv, int rows, dim3 grid, cudaStream_t st) {
  LaunchScope scope(kKindKvCache, st);
  TL_CUDA_CHECK(launch_pdl(kv_append_kernel<T, NV>, grid, dim3(kAppendThreads), 0, st, c, offsets, n_new, (const T *)k, (const T *)v,
                           lk, lv, rows));
  return TEMPLORA_OK;
}
template <typename T>
templora_status_t launch_append(const CacheView &c, const int *offsets, int n_new, const void *k, const void *v, long long lk,
                                long long lv, int rows, dim3 grid, cudaStream_t st) {
  const int vecs = (c.bt * c.D / 16 + kAppendThreads - 1) / kAppendThreads;     // 1 to 4
  if (vecs == 1) return launch_append<T, 1>(c, offsets, n_new, k, v, lk, lv, rows, grid, st);
  if (vecs == 2) return launch_append<T, 2>(c, offsets, n_new, k, v, lk, lv, rows, grid, st);
  return launch_append<T, 4>(c, offsets, n_new, k, v, lk, lv, rows, grid, st);
}

}  // namespace
}  // namespace templora

using namespace templora;

extern "C" {

size_t templora_kv_cache_append_workspace_bytes(const templora_kv_cache_t *cache) {
  return check_cache(cache, false) == TEMPLORA_OK ? kStatusBytes : 0;
}

templora_status_t templora_kv_cache_append(const templora_kv_cache_t *cache, const int32_t *seq_lens,
                                           const int32_t *new_offsets, int32_t n_new, int32_t dtype, const void *k_new,
                                           const void *v_new, int64_t ld_k, int64_t ld_v, void *ws, size_t ws_bytes,
                                           void *stream) {
  TL_TRY(check_cache(cache, true));
  if (!seq_lens || !k_new || !v_new || n_new <= 0 || !aligned16(k_new) || !aligned16(v_new)) return TEMPLORA_ERR_INVALID_ARG;
  if (!word_aligned(seq_lens) || !word_aligned(new_offsets)) return TEMPLORA_ERR_INVALID_ARG;
  if (!new_offsets && n_new != cache->n_seqs) return TEMPLORA_ERR_INVALID_ARG;
  if (dtype != TEMPLORA_F32 && dtype != TEMPLORA_BF16) return TEMPLORA_ERR_UNSUPPORTED;
  const long long width = (long long)cache->n_kv_heads * cache->head_dim;
  const long long lk = row_stride(ld_k, width), lv = row_stride(ld_v, width);
  if (lk < 0 || lv < 0) return TEMPLORA_ERR_INVALID_ARG;
  TL_TRY(check_workspace(ws, ws_bytes, kStatusBytes));
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  const CacheView c = view(cache, seq_lens, ws);
  // a CTA looks at as many rows as a block holds, fewer while that leaves SMs idle (single tokens of many sequences)
  int rows = cache->block_tokens;
  while (rows > 1 && (long long)((n_new + rows - 1) / rows) * cache->n_kv_heads < 512) rows >>= 1;
  const dim3 grid((n_new + rows - 1) / rows, cache->n_kv_heads, 2);
  if (dtype == TEMPLORA_F32) return launch_append<float>(c, new_offsets, n_new, k_new, v_new, lk, lv, rows, grid, st);
  return launch_append<__nv_bfloat16>(c, new_offsets, n_new, k_new, v_new, lk, lv, rows, grid, st);
}

size_t templora_attention_decode_workspace_bytes(const templora_attn_t *attn, const templora_kv_cache_t *cache) {
  return check_decode(attn, cache, false) == TEMPLORA_OK ? decode_need(attn) : 0;
}

templora_status_t templora_attention_decode_fwd(const templora_attn_t *attn, const templora_kv_cache_t *cache,
                                                const int32_t *seq_lens, const void *q, int64_t ld_q, void *o,
                                                int64_t ld_o, float *lse, void *ws, size_t ws_bytes, void *stream) {
  TL_TRY(check_decode(attn, cache, true));
  if (!seq_lens || !q || !o || !aligned16(q) || !aligned16(o)) return TEMPLORA_ERR_INVALID_ARG;
  if (!word_aligned(seq_lens) || !word_aligned(lse)) return TEMPLORA_ERR_INVALID_ARG;
  const long long width = (long long)attn->n_heads * attn->head_dim;
  const long long lq = row_stride(ld_q, width), lo = row_stride(ld_o, width);
  if (lq < 0 || lo < 0) return TEMPLORA_ERR_INVALID_ARG;
  TL_TRY(check_workspace(ws, ws_bytes, decode_need(attn)));
  const bool f32 = attn->dtype == TEMPLORA_F32;
  DecodeParams p{};
  p.c = view(cache, seq_lens, ws);
  p.q = q; p.o = o; p.lse = lse; p.ldq = lq; p.ldo = lo;
  p.part = reinterpret_cast<float *>(reinterpret_cast<uint8_t *>(ws) + kStatusBytes);
  p.arrived = reinterpret_cast<unsigned *>(reinterpret_cast<uint8_t *>(ws) + sizeof(DeviceStatus));
  p.slopes = attn->slopes;
  p.H = attn->n_heads; p.group = attn->n_heads / attn->n_kv_heads;
  p.chunks = f32 ? p.group : (p.group + kHeads - 1) / kHeads;
  p.window = attn->window; p.scale = attn->scale; p.softcap = attn->softcap;
  if (attn->softcap >= kNoCap) p.softcap = 0.f;
  p.cap_in = p.softcap > 0.f ? fminf(1.f / p.softcap, 3e38f) : 0.f;      // finite for the smallest caps too
  p.cap_out = p.softcap * kLog2e;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  if (f32) return attn->head_dim <= 64 ? launch_decode<64, true>(p, st) : launch_decode<128, true>(p, st);
  return attn->head_dim <= 64 ? launch_decode<64, false>(p, st) : launch_decode<128, false>(p, st);
}

}  // extern "C"
