// k_pages.hip - the paged MXFP4 token store: quantising tokens into pages,
// reading them back, sharing and copying pages, and the MaxSim of queries with
// stored documents (Sec. 2.1, Def. 1) straight from the codes.
//
// MXFP4 (the OCP microscaling format): a block of 32 values x shares a scale
// X = 2^(s - 127), s an 8-bit exponent, and holds 32 elements of 4 bits (sign,
// two exponent bits, one mantissa bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6).  With E the
// exponent field of the largest |x| as a float, s = max(E - 2, 0), so the
// largest element lies in [4, 8) and is 4 or 6 after rounding; elements round
// to nearest, ties to even, and saturate at 6.  A block with an infinity or a
// NaN (E = 255) gets s = 255, the format's NaN.
//
// A page is 16 tokens, 1088 bytes, in the order in which the matrix
// instruction takes them (32 x 32 x 64: a lane holds 32 values, one block, of
// one token): codes [block 4][token 16][16 bytes], then scales
// [block % 2][token 16][block / 2].  Free slots of a page have the scale 255:
// their products are NaN, which a maximum passes over, so the scoring has no
// lengths to compare within a page, and a token with a value that is not
// finite is never a best match, for the same reason.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "device_common.h"
#include "internal.h"

namespace chimera {

typedef int v8i32 __attribute__((ext_vector_type(8)));
typedef unsigned v6u32 __attribute__((ext_vector_type(6)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr int CODE_BYTES = 1024;  // of a page; 64 bytes of scales follow
static_assert(kPageBytes == CODE_BYTES + 64, "16 tokens of 64 + 4 bytes");

// Where block b of a page's token t has its codes and its scale.
__device__ __forceinline__ int code_at(int b, int t) { return (b * 16 + t) * 16; }
__device__ __forceinline__ int scale_at(int b, int t) { return CODE_BYTES + ((b & 1) * 16 + t) * 2 + (b >> 1); }

// 2^(s - 127) as a float, s < 255 (s = 0: a subnormal).
__device__ __forceinline__ float scale_float(uint32_t s) { return __uint_as_float(s ? s << 23 : 0x00400000u); }

// ------------------------------------------------------------ plans
// A plan on its way from host memory: whole lines in order, which the bus takes
// at 38 GB/s, where items read one a wave come at 14.
__global__ __launch_bounds__(256) void k_pages_plan(const uint4 *__restrict__ host, uint4 *__restrict__ dev,
                                                    int64_t n) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i < n) dev[i] = host[i];
}

void launch_pages_plan(const void *host, void *dev, size_t bytes, hipStream_t s) {
  const int64_t n = (int64_t)(bytes / 16);
  hipLaunchKernelGGL(k_pages_plan, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, (const uint4 *)host,
                     (uint4 *)dev, n);
}

// ------------------------------------------------------------ quantising
// A workgroup takes one item of the plan (up to 16 pages of one document), a
// wave a page at a time, a lane one block of one token: 32 values, their
// largest in registers, 16 bytes of codes, one byte of scale.  Bound by memory, 256
// or 512 bytes read and 68 written a token: 8,000 documents of 70 bf16 tokens in 42
// us (4.3 TB/s), 501 of 320 float32 tokens in 20.7 us (4.4 TB/s).
template <bool F32>
__global__ __launch_bounds__(256) void k_pages_append(const PageItem *__restrict__ items,
                                                      const int32_t *__restrict__ ids, const void *__restrict__ X,
                                                      int64_t ld, uint8_t *__restrict__ pool,
                                                      int32_t *__restrict__ table, int stride,
                                                      int32_t *__restrict__ lens) {
  const PageItem w = items[blockIdx.x];
  const int lane = lane_id(), t = lane & 15, b = lane >> 4;
  for (int p = (int)(threadIdx.x >> 6); p < w.npages; p += 4) {
    const int32_t id = ids[w.pages + p];
    uint8_t *page = pool + (int64_t)id * kPageBytes;
    const int i = p * 16 + t - w.fill;  // token of the item; below 0: there before
    if (i >= 0 && i < w.ntok) {
      float x[32];
      if constexpr (F32) {
        const float4 *src = (const float4 *)((const float *)X + (w.row + i) * ld + b * 32);
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const float4 v = src[u];
          x[4 * u] = v.x, x[4 * u + 1] = v.y, x[4 * u + 2] = v.z, x[4 * u + 3] = v.w;
        }
      } else {
        const uint4 *src = (const uint4 *)((const uint16_t *)X + (w.row + i) * ld + b * 32);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const uint4 v = src[u];
          const uint32_t y[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            x[8 * u + 2 * k] = __uint_as_float(y[k] << 16);
            x[8 * u + 2 * k + 1] = __uint_as_float(y[k] & 0xFFFF0000u);
          }
        }
      }
      uint32_t top = 0;  // the largest magnitude; as bits, a NaN is larger than any number
#pragma unroll
      for (int k = 0; k < 32; ++k) top = max(top, __float_as_uint(x[k]) & 0x7FFFFFFFu);
      const uint32_t e = top >> 23;
      const uint32_t s = e == 255 ? 255 : e > 2 ? e - 2 : 0;
      uint32_t c[4] = {0, 0, 0, 0};
      if (s != 255) {
        const float sc = scale_float(s);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          c[u] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c[u], x[8 * u], x[8 * u + 1], sc, 0);
          c[u] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c[u], x[8 * u + 2], x[8 * u + 3], sc, 1);
          c[u] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c[u], x[8 * u + 4], x[8 * u + 5], sc, 2);
          c[u] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c[u], x[8 * u + 6], x[8 * u + 7], sc, 3);
        }
      }
      *(uint4 *)(page + code_at(b, t)) = make_uint4(c[0], c[1], c[2], c[3]);
      page[scale_at(b, t)] = (uint8_t)s;
    } else if (i >= w.ntok) {
      page[scale_at(b, t)] = 255;
    }
    if (lane == 0) table[(int64_t)w.doc * stride + w.first + p] = id;
  }
  if (threadIdx.x == 0 && w.len >= 0) lens[w.doc] = w.len;
}

// ------------------------------------------------------------ reading back
// A lane takes 8 values of a token, so that a wave writes whole rows: 4 rows
// of bf16 at a time.  Every value (2 significant bits, exponents from -128) is
// exact in bf16 and in float32.  Bound by memory, 68 bytes read and 256 or 512
// written a token: 8,000 documents of 70 tokens as bf16 in 34 us (5.4 TB/s).
template <bool F32>
__global__ __launch_bounds__(256) void k_pages_read(const PageItem *__restrict__ items,
                                                    const uint8_t *__restrict__ pool,
                                                    const int32_t *__restrict__ table, int stride,
                                                    void *__restrict__ out) {
  const PageItem w = items[blockIdx.x];
  const int lane = lane_id(), seg = lane & 15, b = seg >> 2;
  for (int p = (int)(threadIdx.x >> 6); p < w.npages; p += 4) {
    const uint8_t *page = pool + (int64_t)table[(int64_t)w.doc * stride + w.first + p] * kPageBytes;
#pragma unroll
    for (int it = 0; it < 4; ++it) {
      const int t = it * 4 + (lane >> 4), i = p * 16 + t;
      if (i >= w.ntok) continue;
      const uint32_t c = *(const uint32_t *)(page + code_at(b, t) + 4 * (seg & 3));
      const uint32_t s = page[scale_at(b, t)];
      const float sc = scale_float(s);
      const f32x2 v[4] = {
          __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, sc, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, sc, 1),
          __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, sc, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, sc, 3)};
      uint32_t y[8];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        y[2 * k] = s == 255 ? 0x7FC00000u : __float_as_uint(v[k][0]);
        y[2 * k + 1] = s == 255 ? 0x7FC00000u : __float_as_uint(v[k][1]);
      }
      if constexpr (F32) {
        uint4 *o = (uint4 *)((float *)out + (w.row + i) * CHIMERA_DIM + seg * 8);
        o[0] = make_uint4(y[0], y[1], y[2], y[3]);
        o[1] = make_uint4(y[4], y[5], y[6], y[7]);
      } else {
        uint4 *o = (uint4 *)((uint16_t *)out + (w.row + i) * CHIMERA_DIM + seg * 8);
        *o = make_uint4(y[0] >> 16 | y[1], y[2] >> 16 | y[3], y[4] >> 16 | y[5], y[6] >> 16 | y[7]);
      }
    }
  }
}

// ------------------------------------------------------------ sharing and copying
// A wave a document: its page ids, then the partly filled page behind the
// shared ones, with free slots behind its ntok tokens (4,099 documents: 5.3 us,
// bound by the dependent reads of item, page id and page).
__global__ __launch_bounds__(64) void k_pages_fork(const PageItem *__restrict__ items, uint8_t *__restrict__ pool,
                                                   int32_t *__restrict__ table, int stride,
                                                   int32_t *__restrict__ lens) {
  const PageItem w = items[blockIdx.x];
  const int lane = lane_id(), t = lane & 15, b = lane >> 4;
  const int32_t *from = table + (int64_t)w.src * stride;
  int32_t *to = table + (int64_t)w.doc * stride;
  for (int p = lane; p < w.first; p += 64) to[p] = from[p];
  if (w.ntok) {
    const uint8_t *s = pool + (int64_t)from[w.first] * kPageBytes;
    uint8_t *d = pool + (int64_t)w.pages * kPageBytes;
    *(uint4 *)(d + code_at(b, t)) = *(const uint4 *)(s + code_at(b, t));
    d[scale_at(b, t)] = t < w.ntok ? s[scale_at(b, t)] : 255;
    if (lane == 0) to[w.first] = w.pages;
  }
  if (lane == 0) lens[w.doc] = w.len;
}

// Tokens by position into pages of their own; a lane one block of one token.
// Bound by memory, 68 bytes read and written a token (314,000 tokens of 8,192
// documents: 13 us, 3.3 TB/s), and for one document by the few workgroups.
// publish: also the page ids and the length, where no item reads a document
// that another one writes (else k_pages_publish does, behind it).
template <class Pos>
__global__ __launch_bounds__(256) void k_pages_copy(const PageItem *__restrict__ items,
                                                    const int32_t *__restrict__ ids, const Pos *__restrict__ pos,
                                                    const uint8_t *__restrict__ from,
                                                    const int32_t *__restrict__ from_table, int from_stride,
                                                    uint8_t *__restrict__ pool, int32_t *__restrict__ table,
                                                    int stride, int32_t *__restrict__ lens, int publish) {
  const PageItem w = items[blockIdx.x];
  const int lane = lane_id(), t = lane & 15, b = lane >> 4;
  const int32_t *row = from_table + (int64_t)w.src * from_stride;
  for (int p = (int)(threadIdx.x >> 6); p < w.npages; p += 4) {
    const int32_t id = ids[w.pages + p];
    uint8_t *d = pool + (int64_t)id * kPageBytes;
    const int i = p * 16 + t;
    if (i < w.ntok) {
      const int at = pos ? (int)pos[w.row + i] : (int)w.row + i;
      const uint8_t *s = from + (int64_t)row[at >> 4] * kPageBytes;
      *(uint4 *)(d + code_at(b, t)) = *(const uint4 *)(s + code_at(b, at & 15));
      d[scale_at(b, t)] = s[scale_at(b, at & 15)];
    } else {
      d[scale_at(b, t)] = 255;
    }
    if (publish && lane == 0) table[(int64_t)w.doc * stride + w.first + p] = id;
  }
  if (publish && threadIdx.x == 0 && w.len >= 0) lens[w.doc] = w.len;
}

__global__ __launch_bounds__(64) void k_pages_publish(const PageItem *__restrict__ items,
                                                      const int32_t *__restrict__ ids, int32_t *__restrict__ table,
                                                      int stride, int32_t *__restrict__ lens) {
  const PageItem w = items[blockIdx.x];
  const int p = (int)threadIdx.x;
  if (p < w.npages) table[(int64_t)w.doc * stride + w.first + p] = ids[w.pages + p];
  if (p == 0 && w.len >= 0) lens[w.doc] = w.len;
}

__global__ __launch_bounds__(256) void k_pages_drop(const int64_t *__restrict__ ids, int64_t n,
                                                    int32_t *__restrict__ lens) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i < n) lens[ids[i]] = 0;
}

// ------------------------------------------------------------ scoring
// Operand of the query tokens.  A query value on the grid is an integer
// k = 2048 q.  The 6-bit floats of the format e2m3 are, times 8, all whole
// numbers up to 16, the even ones up to 32 and the multiples of 4 up to 60, and
// their products with 4-bit floats run at twice the rate of 8-bit ones.  Where a
// block's |k| stay up to 1024 (|q| <= 1/2) two digits of base 32 hold it exactly,
// k = 32 d1 + d0: up to 512 |d0| <= 16, and above, where bf16 has every fourth k
// only, d1 is even and d0 a multiple of 4, at most 32.  Larger blocks take three
// digits |d| <= 16, k = 1024 d2 + 32 d1 + d0; the third one's products are left
// out for a query that has none.  Blocks whose largest value is 8 or more are
// shifted right until its k is below 2^14, and rounded: half a unit, where the
// largest k is 2^13 units or more, so at most 2^-14 of the block's largest value.
// The largest finite bf16 shifts by 125, and the third digit's exponent is then
// the last one that a scale holds.  Lane l holds query token l % 32 of a block of 32, dimensions
// 64 step + 32 (l / 32) .. + 31.
struct QueryOperand {
  v6u32 digit[2][2];
  int scale[2];  // byte j: exponent of digit j
};

// In LDS, of 32 query tokens: digits 0 and 1 [step][digit][lane][6] (dead once
// they are in registers), digit 2 [step][lane][6], exponents [step][lane].
constexpr int LOW_WORDS = 2 * 2 * 64 * 6, HIGH_WORDS = 2 * 64 * 6 + 2 * 64;

// A thread makes half a block: 16 values of one token.  Its values as they lie in
// memory, for each of NB blocks of 32 tokens: token g of the blocks is token
// g % 2^slot of query g >> slot, `next` values a query; zero where that is at or
// past Tq, or the query past the `have` there are.
template <int NB, bool F32>
struct QueryRaw {
  uint4 v[NB][F32 ? 4 : 2];
};
__device__ __forceinline__ int half_step() { return (int)threadIdx.x >> 7; }
__device__ __forceinline__ int half_lane() { return ((int)threadIdx.x >> 1) & 63; }
template <int NB, bool F32>
__device__ __forceinline__ void fetch_query(const char *__restrict__ Q, int64_t next, int slot, int have, int Tq,
                                            QueryRaw<NB, F32> &raw) {
  const int d0 = 64 * half_step() + 32 * (half_lane() >> 5) + 16 * ((int)threadIdx.x & 1);
#pragma unroll
  for (int blk = 0; blk < NB; ++blk) {
    const int g = blk * 32 + (half_lane() & 31), u = g >> slot, j = g & ((1 << slot) - 1);
    const uint4 *src = (const uint4 *)(Q + (u * next + (int64_t)j * CHIMERA_DIM + d0) * (F32 ? 4 : 2));
    const bool on = j < Tq && u < have;
#pragma unroll
    for (int i = 0; i < (F32 ? 4 : 2); ++i) raw.v[blk][i] = on ? src[i] : make_uint4(0, 0, 0, 0);
  }
}

// All 256 threads: the operands of the blocks into LDS, low [NB][LOW_WORDS] and
// high [NB][HIGH_WORDS].  Returns whether one of this thread's has a third digit.
template <int NB, bool F32>
__device__ __forceinline__ bool prepare_query(const QueryRaw<NB, F32> &raw, uint32_t *low0, uint32_t *high0) {
  const int half = (int)threadIdx.x & 1, l = half_lane(), step = half_step();
  bool any = false;
#pragma unroll
  for (int blk = 0; blk < NB; ++blk) {
    float q[16];
#pragma unroll
    for (int i = 0; i < (F32 ? 4 : 2); ++i) {
      const uint4 v = raw.v[blk][i];
      const uint32_t y[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        if constexpr (F32) {
          q[4 * i + m] = __uint_as_float((uint32_t)grid_bf16_bits(__uint_as_float(y[m])) << 16);
        } else {
          // above 1/16 every bf16 is on the grid; below it k is rounded onto it
          q[8 * i + 2 * m] = __uint_as_float(y[m] << 16);
          q[8 * i + 2 * m + 1] = __uint_as_float(y[m] & 0xFFFF0000u);
        }
      }
    }
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) top = fmaxf(top, fabsf(q[i]));
    top = fmaxf(top, shfl_xor(top, 1));  // of the block's other half
    f32x16 dig[3][2] = {};  // even and odd dimensions, as the conversion takes them, and as many zeros
    int shift = 0;
    if (top <= 0.25f) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float k = rintf(q[i] * 2048.0f), a1 = rintf(k * (1.0f / 32.0f));
        dig[1][i & 1][i >> 1] = a1;
        dig[0][i & 1][i >> 1] = k - 32.0f * a1;
      }
    } else {
      const bool wide = top > 0.5f;
      any |= wide;
      shift = min(max((int)(__float_as_uint(top) >> 23) - 127 - 2, 0), 125);
      // x = k shifted.  A large k is no float, so from 9 bits on the shift comes
      // first: values below 1/16 are rounded to 0 either way, others are on the grid.
      const int first = shift > 8 ? shift : 0;
      const float up = __uint_as_float((uint32_t)(127 + 11 - first) << 23);
      const float down = __uint_as_float((uint32_t)(127 + first - shift) << 23);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float x = rintf(rintf(q[i] * up) * down);
        const float a2 = wide ? rintf(x * (1.0f / 1024.0f)) : 0.0f, r = x - 1024.0f * a2;
        const float a1 = fabsf(r) > 512.0f ? 2.0f * rintf(r * (1.0f / 64.0f)) : rintf(r * (1.0f / 32.0f));
        dig[2][i & 1][i >> 1] = a2;
        dig[1][i & 1][i >> 1] = a1;
        dig[0][i & 1][i >> 1] = r - 32.0f * a1;
      }
    }
    uint32_t *low = low0 + blk * LOW_WORDS, *high = high0 + blk * HIGH_WORDS;
#pragma unroll
    for (int m = 0; m < 3; ++m) {
      const v6u32 c = __builtin_amdgcn_cvt_scalef32_2xpk16_fp6_f32(dig[m][0], dig[m][1], 8.0f);
      // The conversion reads its sources while it writes: they are kept alive behind
      // it, so that the compiler does not put the result in their registers.
      asm volatile("" ::"v"(dig[m][0]), "v"(dig[m][1]), "v"(c));
      uint32_t *o = (m < 2 ? low + ((step * 2 + m) * 64 + l) * 6 : high + (step * 64 + l) * 6) + 3 * half;
#pragma unroll
      for (int i = 0; i < 3; ++i) o[i] = c[i];  // the first 16 of 32
    }
    // digit m counts 8 * 32^m / 2048 * 2^shift
    const uint32_t e = (uint32_t)(127 + 3 - 11 + shift);
    if (half == 0) high[2 * 64 * 6 + step * 64 + l] = e | (e + 5) << 8 | (e + 10) << 16;
  }
  return any;
}

__device__ __forceinline__ void load_query(const uint32_t *low, const uint32_t *high, QueryOperand &q) {
  const int l = lane_id();
#pragma unroll
  for (int step = 0; step < 2; ++step) {
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int i = 0; i < 6; ++i) q.digit[step][m][i] = low[((step * 2 + m) * 64 + l) * 6 + i];
    q.scale[step] = (int)high[2 * 64 * 6 + step * 64 + l];
  }
}

// This lane's part of two pages: the codes of its token's blocks of both steps
// and their scales (byte = step).
struct PageOperand {
  uint4 code[2];
  int scale;
};
// Pages a (rows 0 .. 15, lanes with bit 4 clear) and b (rows 16 .. 31), as units of
// 64 bytes from the pool's start; codes, scales: this lane's place in page 0.
struct PageBase {
  const uint8_t *codes, *scales;
  __device__ explicit PageBase(const uint8_t *pool) {
    const int t = lane_id() & 15, h = lane_id() >> 5;
    codes = pool + code_at(h, t);
    scales = pool + scale_at(h, t);
  }
};
constexpr uint32_t kPageUnits = kPageBytes / 64;
static_assert(kPageUnits * 64 == kPageBytes && kPagesMaxPages == 0xFFFFFFFFu / kPageUnits, "units in 32 bits");
__device__ __forceinline__ PageOperand load_pages(const PageBase &base, uint32_t a, uint32_t b) {
  const uint64_t at = (uint64_t)(lane_id() & 16 ? b : a) << 6;
  PageOperand o;
  o.code[0] = *(const uint4 *)(base.codes + at);
  o.code[1] = *(const uint4 *)(base.codes + at + (code_at(2, 0) - code_at(0, 0)));
  o.scale = *(const uint16_t *)(base.scales + at);
  return o;
}

// <document token, query token> of 32 x 32 pairs: register v of lane l is row
// 8 (v / 4) + 4 (l / 32) + v % 4, query token l % 32; so v < 8 are the rows of
// the first page.
// The digits in rising order: small sums first.
__device__ __forceinline__ f32x16 digit_products(const PageOperand &a, const v6u32 (&digit)[2], const int (&scale)[2],
                                                 f32x16 acc, int m) {
#define CHIMERA_MX(STEP, M)                                                                                   \
  acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(                                                      \
      v8i32{(int)a.code[STEP].x, (int)a.code[STEP].y, (int)a.code[STEP].z, (int)a.code[STEP].w, 0, 0, 0, 0}, \
      v8i32{(int)digit[STEP][0], (int)digit[STEP][1], (int)digit[STEP][2], (int)digit[STEP][3],              \
            (int)digit[STEP][4], (int)digit[STEP][5], 0, 0},                                                 \
      acc, 4, 2, STEP, a.scale, M, scale[STEP]);
  if (m == 0) {
    CHIMERA_MX(0, 0) CHIMERA_MX(1, 0)
  } else if (m == 1) {
    CHIMERA_MX(0, 1) CHIMERA_MX(1, 1)
  } else {
    CHIMERA_MX(0, 2) CHIMERA_MX(1, 2)
  }
#undef CHIMERA_MX
  return acc;
}
// third: the digit's words of this lane in LDS, or null where there is none.
__device__ __forceinline__ f32x16 page_products(const PageOperand &a, const QueryOperand &q, const uint32_t *third) {
  f32x16 acc = {0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    const v6u32 d[2] = {q.digit[0][m], q.digit[1][m]};
    acc = digit_products(a, d, q.scale, acc, m);
  }
  if (third) {
    v6u32 d[2];
#pragma unroll
    for (int step = 0; step < 2; ++step)
#pragma unroll
      for (int i = 0; i < 6; ++i) d[step][i] = third[step * 64 * 6 + i];
    acc = digit_products(a, d, q.scale, acc, 2);
  }
  return acc;
}

// Key of a score, as the searches rank them: rint(F * 2^22), saturated at the
// largest floats inside the range, +-(2^31 - 128), so that the lowest key, -2^31,
// means -infinity alone.
__device__ __forceinline__ int32_t score_key(float F) {
  const float x = rintf(F * KEY_SCALE);
  return F == -INFINITY ? INT32_MIN : (int32_t)fminf(fmaxf(x, -2147483520.0f), 2147483520.0f);
}

__global__ __launch_bounds__(256) void k_pages_unscored(int32_t *__restrict__ ids, float *__restrict__ scores,
                                                        int64_t n) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i < n && scores[i] == -512.0f) {  // -2^31 * 2^-22
    ids[i] = -1;
    scores[i] = -INFINITY;
  }
}

// MaxSim.  A wave scores list entries one after the other, up to 64 of them, for
// NB blocks of 32 query tokens: one query of up to 32 NB tokens or, PACK, several
// that share the list, each in 2^slot >= Tq places of the blocks: a page is loaded
// and multiplied once for all of them (64 queries x 30,000 documents of 64 tokens:
// 36, 85, 148 and 264 us with 1, 4, 8 and 16 query tokens; 371, 381, 410 and 477
// with two queries at a time).  PACK 2 is two queries of 32 places, known when it
// is compiled (1.2% faster there).  The queries stay in registers and the documents
// stream through, since a query's operand (6 KB a block) is larger than an average
// document's pages.  The entries' pages are strung together: lane j of a window has
// the place of its j-th page, a tile is two neighbouring pages whatever documents
// they belong to, and DEPTH tiles are under way (2, 3 and 4 are as fast, 6 is 4 to
// 12% slower).  A document's maxima over its rows stay in registers until its last
// page, then go to a ring in LDS; 16 documents at a time are summed over the query
// tokens, four lanes each, in the same order whatever NB and PACK are.  SPLIT: a
// workgroup takes one entry, its waves a quarter of the pages each, and their
// maxima meet in LDS.
//
// What it measured, and what is known of its bound.  With a list for each query:
// reads that miss L2 (256 x 2048 entries of 50,000 documents of 64 tokens: 245 us,
// 1.79 GB at 7.3 TB/s).  With one list for many (64 queries x 30,000 documents:
// 520 to 545 us, 1.9 PFLOP/s of useful work): the matrix cores are busy 52% of the
// cycles, at a clock of about 1.9 GHz.  What keeps them idle for the rest is not
// established: other vector instructions take about a third of the cycles, there
// are 2.5 waves a SIMD, and a wave waits 43% of its time to issue and 23% for data.
// For few entries: the chain of list, length, page table and page (100 documents: 7
// us).
constexpr int DEPTH = 2, FLUSH = 16, RING = 32;
static_assert(FLUSH + 2 * DEPTH <= RING, "documents that end within DEPTH tiles have room");

// Entries: ids [nq][ld] (null: documents 0 .. n - 1), below n_valid[q] where that
// is given; out [nq][n], float scores or (KEYS) int32 keys.  An entry that names
// no document, and a document without a finite token, score -infinity.
template <int NB, int PACK, bool SPLIT, bool F32, bool KEYS>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(NB == 1 ? 4 : 3))) void k_pages_score(
    const void *__restrict__ Q, int Tq, int q_stride, const int32_t *__restrict__ ids, int64_t ld,
    const int32_t *__restrict__ n_valid, int n, int nq, int any_slot, int per_wave, int chunks,
    const uint8_t *__restrict__ pool, const int32_t *__restrict__ table, int stride, const int32_t *__restrict__ lens,
    int64_t ndocs, void *__restrict__ out) {
  constexpr int ROW = NB * 32 + 1;  // of the maxima in LDS
  const int slot = PACK == 2 ? 5 : any_slot;
  const int per = PACK ? NB * 32 >> slot : 1;  // queries of a workgroup
  static_assert(4 * RING * ROW >= NB * LOW_WORDS, "the maxima take the first digits' place");
  __shared__ uint32_t high[NB * HIGH_WORDS], low[4 * RING * ROW];
  const int lane = lane_id(), wave = (int)(threadIdx.x >> 6);
  // Workgroups are dealt to the 8 XCDs in turn.  A chunk of the lists (per_wave
  // entries for each wave) stays with one XCD, all queries' workgroups for it one
  // behind the other: lists that ascend name about the same documents there,
  // some of which its L2 still holds.
  const int groups = PACK ? (nq + per - 1) / per : nq, wg = (int)blockIdx.x;
  const bool dealt = chunks % 8 == 0;
  const int k = dealt ? wg >> 3 : wg;
  const int chunk = dealt ? k / groups * 8 + (wg & 7) : k / groups;
  const int64_t q = (int64_t)(k % groups) * per;
  const int last = !PACK && n_valid ? min(n, n_valid[q]) : n;
  if (chunk * (SPLIT ? 1 : 4) * per_wave >= last) return;  // the whole workgroup
  const int have = PACK ? min(per, nq - (int)q) : 1;
  const int64_t step = (int64_t)q_stride * CHIMERA_DIM;
  QueryRaw<NB, F32> raw;  // under way while the list and the page table are read
  fetch_query<NB, F32>((const char *)Q + q * step * (F32 ? 4 : 2), step, PACK ? slot : 6, have, Tq, raw);
  const int c0 = (SPLIT ? chunk : chunk * 4 + wave) * per_wave;
  // lane e: entry c0 + e, its document's row of the page table and its pages
  const bool on = lane < per_wave && c0 + lane < last;
  int64_t row = 0;
  uint32_t np = 0;
  if (on) {
    const int64_t doc = ids ? ids[(PACK ? 0 : q * ld) + c0 + lane] : c0 + lane;
    if (doc >= 0 && doc < ndocs) {
      row = doc * stride;
      np = (uint32_t)(lens[doc] + 15) >> 4;
    }
  }
  const bool none = np == 0;
  const uint64_t full = __ballot(!none);  // entries that have pages
  if constexpr (SPLIT) {
    const uint32_t quarter = (np + 3) >> 2, first = min(wave * quarter, np);
    row += first;
    np = min(np - first, quarter);
  }
  const uint64_t some = __ballot(np > 0);
  const uint32_t end = wave_incl_scan(np);
  const uint32_t total = (uint32_t)__builtin_amdgcn_readlane((int)end, 63);
  row -= (int64_t)(end - np);  // + position in the string of pages
  // lane r: the r-th entry that has pages
  const int rank = __builtin_popcountll(some & ((1ull << lane) - 1));
  const int entry = __builtin_amdgcn_ds_permute((np ? rank : 63 - (lane - rank)) * 4, lane);

  // lane j: where page w0 + j of the string is, in units, and whether a document ends there
  auto window = [&](uint32_t w0, uint64_t &ends) -> uint32_t {
    const uint32_t at = w0 + lane;
    int e = 0;  // entries that end at or before it
#pragma unroll
    for (int step = 32; step >= 1; step >>= 1) {
      const uint32_t x = (uint32_t)__shfl((int)end, e + step - 1, 64);
      if (x <= at) e += step;
    }
    e = min(e, 63);
    const int64_t r = ((int64_t)__shfl((int)(row >> 32), e, 64) << 32) | (uint32_t)__shfl((int)(uint32_t)row, e, 64);
    const uint32_t stop = (uint32_t)__shfl((int)end, e, 64);  // by every lane: lane e may have no page here
    ends = __ballot(at < total && at + 1 == stop);
    return at < total ? (uint32_t)table[r + at] * kPageUnits : 0;
  };

  uint64_t ends, next_ends = 0;
  uint32_t page = window(0, ends), next_page = 0;  // under way while the query is prepared

  const bool wide = __syncthreads_or(prepare_query<NB, F32>(raw, low, high));
  QueryOperand op[NB];
#pragma unroll
  for (int u = 0; u < NB; ++u) load_query(low + u * LOW_WORDS, high + u * HIGH_WORDS, op[u]);
  __syncthreads();
  float *best_of = (float *)low + wave * RING * ROW;

  void *const out_q = (uint32_t *)out + q * n;
  auto put = [&](int c, int u, float F) {
    const int64_t at = (PACK ? (int64_t)u * n : 0) + c;
    if constexpr (KEYS) ((int32_t *)out_q)[at] = score_key(F);
    else ((float *)out_q)[at] = F;
  };
  if (on && none && !(SPLIT && wave))
    for (int u = 0; u < have; ++u) put(c0 + lane, u, -INFINITY);
  if (full == 0) return;  // SPLIT: the whole workgroup
  if constexpr (SPLIT) {
    for (int i = lane; i < ROW; i += 64) best_of[i] = -INFINITY;  // a wave may have no page
    __builtin_amdgcn_wave_barrier();
  }

  const PageBase base(pool);
  float m[NB];
#pragma unroll
  for (int u = 0; u < NB; ++u) m[u] = -INFINITY;
  int ended = 0, summed = 0;  // documents whose maxima are, or were, in LDS; those of them that are summed up
  auto sum_up = [&]() {
    __builtin_amdgcn_wave_barrier();
    constexpr int LANES = 64 / FLUSH, EACH = NB * 32 / LANES;  // lanes of a document, query tokens of a lane
    const int i = summed + lane / LANES, part = lane % LANES;  // the i-th entry that has pages
    const bool on = i < (SPLIT ? 1 : ended);
    const int c = c0 + (SPLIT ? 0 : __shfl(entry, i & 63, 64));
    const int places = PACK ? 1 << slot : NB * 32, u0 = PACK ? part * EACH >> slot : 0;  // of a query; this lane's first query
    auto best = [&](int j) {  // the maximum of this lane's j-th token, 0 for one past its query's
      const int tok = part * EACH + j;
      float x = best_of[(i % RING) * ROW + tok];
      if constexpr (SPLIT)
#pragma unroll
        for (int w = 1; w < 4; ++w) x = fmaxf(x, best_of[(w * RING + i) * ROW + tok]);
      return (tok & (places - 1)) < Tq ? x : 0.0f;
    };
    if (PACK && places < 8) {
#pragma unroll 1
      for (int j0 = 0; j0 < EACH; j0 += 4) {
        const float x[4] = {best(j0), best(j0 + 1), best(j0 + 2), best(j0 + 3)};
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          sum += x[j];
          const int u = u0 + ((j0 + j) >> slot);
          if ((j & (places - 1)) == places - 1) {
            if (on && u < have) put(c, u, sum);
            sum = 0.0f;
          }
        }
      }
    } else {
      float s8[2] = {0.0f, 0.0f};
#pragma unroll
      for (int j = 0; j < EACH; ++j) s8[j / 8] += best(j);
      float sum = s8[0];
      if (EACH == 16 && places >= 16) sum += s8[1];
      if (places >= 2 * EACH) sum += shfl_xor(sum, 1);
      if (places >= 4 * EACH) sum += shfl_xor(sum, 2);
      if (on && (part * EACH & (places - 1)) == 0 && u0 < have) put(c, u0, sum);
      if (EACH == 16 && places == 8 && on && u0 + 1 < have) put(c, u0 + 1, s8[1]);
    }
    __builtin_amdgcn_wave_barrier();
    summed = min(summed + FLUSH, ended);
  };
  auto page_done = [&]() {  // the document's last page: its maxima go to LDS
    const int slot = ended % RING;
#pragma unroll
    for (int u = 0; u < NB; ++u) {
      const float x = fmaxf(m[u], shfl_xor(m[u], 32));
      if (lane < 32) best_of[slot * ROW + u * 32 + lane] = x;
      m[u] = -INFINITY;
    }
    ++ended;
  };

  for (uint32_t w0 = 0; w0 < total; w0 += 64) {
    const int cnt = (int)min(total - w0, 64u), tiles = (cnt + 1) >> 1;
    if (w0 + 64 < total) next_page = window(w0 + 64, next_ends);
    // behind the last page that one stands again
    auto fetch = [&](int t) {
      return load_pages(base, (uint32_t)__builtin_amdgcn_readlane((int)page, min(2 * t, cnt - 1)),
                        (uint32_t)__builtin_amdgcn_readlane((int)page, min(2 * t + 1, cnt - 1)));
    };
    PageOperand a[DEPTH];
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) {
      a[d] = fetch(d);
      __builtin_amdgcn_sched_barrier(0);  // in this order: the first tile waits for its own loads alone
    }
    for (int t0 = 0; t0 < tiles; t0 += DEPTH) {
#pragma unroll
      for (int d = 0; d < DEPTH; ++d) {
        const int t = t0 + d;
        if (t < tiles) {
          // an odd number of pages: the last tile's second half has free slots
          if (2 * t + 1 == cnt && (lane & 16)) a[d].scale = 0xFFFF;
          f32x16 s[NB];
#pragma unroll
          for (int u = 0; u < NB; ++u)
            s[u] = page_products(a[d], op[u], wide ? high + u * HIGH_WORDS + lane * 6 : nullptr);
#pragma unroll
          for (int u = 0; u < NB; ++u)
#pragma unroll
            for (int v = 0; v < 8; ++v) m[u] = fmaxf(m[u], s[u][v]);
          if ((ends >> (2 * t)) & 1) page_done();
#pragma unroll
          for (int u = 0; u < NB; ++u)
#pragma unroll
            for (int v = 8; v < 16; ++v) m[u] = fmaxf(m[u], s[u][v]);
          if ((ends >> (2 * t + 1)) & 1) page_done();
        }
        // behind the branch, so that the registers of a tile stay where they are
        a[d] = fetch(t + DEPTH);
      }
      if (!SPLIT && ended - summed >= FLUSH) sum_up();
    }
    page = next_page;
    ends = next_ends;
  }
  if constexpr (SPLIT) {
    __syncthreads();
    if (wave == 0) sum_up();
  } else {
    while (summed < ended) sum_up();
  }
}

// ------------------------------------------------------------ launchers
void launch_pages_append(const PageItem *items, int64_t nitems, const int32_t *ids, const void *X, int x_dtype,
                         int64_t ld, uint8_t *pool, int32_t *table, int stride, int32_t *lens, hipStream_t s) {
  if (nitems <= 0) return;
  const dim3 grid((unsigned)nitems);
  if (x_dtype == CHIMERA_F32)
    hipLaunchKernelGGL(k_pages_append<true>, grid, dim3(256), 0, s, items, ids, X, ld, pool, table, stride, lens);
  else
    hipLaunchKernelGGL(k_pages_append<false>, grid, dim3(256), 0, s, items, ids, X, ld, pool, table, stride, lens);
}

void launch_pages_read(const PageItem *items, int64_t nitems, const uint8_t *pool, const int32_t *table, int stride,
                       void *out, int dtype, hipStream_t s) {
  if (nitems <= 0) return;
  const dim3 grid((unsigned)nitems);
  if (dtype == CHIMERA_F32)
    hipLaunchKernelGGL(k_pages_read<true>, grid, dim3(256), 0, s, items, pool, table, stride, out);
  else
    hipLaunchKernelGGL(k_pages_read<false>, grid, dim3(256), 0, s, items, pool, table, stride, out);
}

void launch_pages_fork(const PageItem *items, int64_t nitems, uint8_t *pool, int32_t *table, int stride, int32_t *lens,
                       hipStream_t s) {
  if (nitems <= 0) return;
  hipLaunchKernelGGL(k_pages_fork, dim3((unsigned)nitems), dim3(64), 0, s, items, pool, table, stride, lens);
}

void launch_pages_copy(const PageItem *items, int64_t nitems, const int32_t *ids, const void *pos, bool short_pos,
                       const uint8_t *from, const int32_t *from_table, int from_stride, uint8_t *pool, int32_t *table,
                       int stride, int32_t *lens, bool in_place, hipStream_t s) {
  if (nitems <= 0) return;
  const dim3 grid((unsigned)nitems);
  const int publish = in_place ? 0 : 1;
  if (short_pos)
    hipLaunchKernelGGL(k_pages_copy<uint16_t>, grid, dim3(256), 0, s, items, ids, (const uint16_t *)pos, from,
                       from_table, from_stride, pool, table, stride, lens, publish);
  else
    hipLaunchKernelGGL(k_pages_copy<int32_t>, grid, dim3(256), 0, s, items, ids, (const int32_t *)pos, from,
                       from_table, from_stride, pool, table, stride, lens, publish);
  if (in_place) hipLaunchKernelGGL(k_pages_publish, grid, dim3(64), 0, s, items, ids, table, stride, lens);
}

void launch_pages_drop(const int64_t *ids, int64_t n, int32_t *lens, hipStream_t s) {
  if (n <= 0) return;
  hipLaunchKernelGGL(k_pages_drop, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, ids, n, lens);
}

void launch_pages_unscored(int32_t *ids, float *scores, int64_t n, hipStream_t s) {
  if (n <= 0) return;
  hipLaunchKernelGGL(k_pages_unscored, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, ids, scores, n);
}

// List entries of a wave: enough waves to fill the chip first (16 a CU), then as
// many entries as a wave can take (64) where all queries share the list, 16 where
// each has its own: short chunks keep more of what the queries of a chunk read in
// an XCD's L2 (256 x 2048 entries of 50,000 documents: 258, 249 and 297 us with 8,
// 16 and 24 entries; 64 queries x 30,000 documents: 635, 565, 533 and 527 us with 8,
// 16, 32 and 64).
static int score_entries(int64_t n, int64_t groups, bool shared) {
  return (int)std::max<int64_t>(1, std::min<int64_t>(shared ? 64 : 16, n * groups / 4096));
}

template <int NB, int PACK, bool SPLIT>
static void launch_score_t(const void *Q, int q_dtype, int64_t nq, int Tq, int q_stride, const int32_t *ids,
                           int64_t ld, const int32_t *n_valid, int64_t n, const PagesView &pg, int slot, void *out,
                           bool keys, hipStream_t s) {
  const int per = PACK ? NB * 32 >> slot : 1;
  const int64_t groups = (nq + per - 1) / per;
  const int per_wave = SPLIT ? 1 : score_entries(n, groups, !ids || ld == 0), per_group = SPLIT ? 1 : 4 * per_wave;
  int64_t chunks = (n + per_group - 1) / per_group;
  if (chunks >= 8) chunks = (chunks + 7) / 8 * 8;
  const dim3 grid((unsigned)(chunks * groups));
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, Q, Tq, q_stride, ids, ld, n_valid, (int)n, (int)nq, slot, per_wave,
                       (int)chunks,
                       pg.pool, pg.table, pg.stride, pg.lens, pg.ndocs, out);
  };
  if constexpr (!PACK)
    if (keys) return go(k_pages_score<NB, PACK, SPLIT, false, true>);
  if (q_dtype == CHIMERA_F32) go(k_pages_score<NB, PACK, SPLIT, true, false>);
  else go(k_pages_score<NB, PACK, SPLIT, false, false>);
}

void launch_pages_score(const void *Q, int q_dtype, int64_t nq, int Tq, int q_stride, const int32_t *ids, int64_t ld,
                        const int32_t *n_valid, int64_t n, const PagesView &pg, void *out, bool keys, hipStream_t s) {
  if (nq <= 0 || n <= 0) return;
  // no more entries than CUs: a workgroup each (1 x 256 documents of 64, 512 and 2000
  // tokens: 6.8, 7.2 and 10.2 us, 6.8, 9.2 and 19.6 with a wave each; 1 x 1000
  // documents: 9.6, 11.1 and 25.9 against 7.0, 10.5 and 26.5)
  const bool split = n * nq <= 256;
  // queries that share the list lie side by side in the blocks, in one block if
  // that holds them all
  const bool pack = !split && Tq <= 32 && nq > 1 && (!ids || ld == 0) && !keys;
  int slot = 0;
  while (1 << slot < Tq) ++slot;
  const bool one = nq << slot <= 32;
  const int group = pack ? (one ? 32 : 64) >> slot : 1;
  // a launch counts its work-items in 32 bits: whole groups of queries
  const int64_t few = n / 64 + 8;  // workgroups of a group where there are more than 4096 waves, at most
  const int64_t per = std::max<int64_t>(1, ((int64_t)1 << 23) / few) * group;
  for (int64_t q0 = 0; q0 < nq; q0 += per) {
    const int64_t nb = std::min(per, nq - q0);
    const char *Qb = (const char *)Q + (size_t)q0 * q_stride * CHIMERA_DIM * (q_dtype == CHIMERA_F32 ? 4 : 2);
    const int32_t *idb = ids ? ids + q0 * ld : nullptr;
    const int32_t *nv = n_valid ? n_valid + q0 : nullptr;
    char *o = (char *)out + (size_t)q0 * n * 4;
    auto go = [&](auto launch) { launch(Qb, q_dtype, nb, Tq, q_stride, idb, ld, nv, n, pg, slot, o, keys, s); };
    if (split && Tq <= 32) go(launch_score_t<1, 0, true>);
    else if (split) go(launch_score_t<2, 0, true>);
    else if (pack && one) go(launch_score_t<1, 1, false>);
    else if (pack && slot == 5) go(launch_score_t<2, 2, false>);
    else if (pack) go(launch_score_t<2, 1, false>);
    else if (Tq <= 32) go(launch_score_t<1, 0, false>);
    else go(launch_score_t<2, 0, false>);
  }
}

}  // namespace chimera
