// kv4_rows.cuh — what the kernels that write rows into the paged 4-bit cache share: blocks of 16 values to
// codes and scale, and where a row of a step lives.
#pragma once
#include "kv4.cuh"

namespace semkv {

template <bool BF16>
__device__ __forceinline__ float2 unpack2(uint32_t w) {
  if (BF16) return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
  __half2 h;
  *reinterpret_cast<uint32_t*>(&h) = w;
  return __half22float2(h);
}
template <bool BF16>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  uint32_t w;
  if (BF16)
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
  else
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
  return w;
}
// max of magnitudes, pairwise; a NaN stays one
template <bool BF16>
__device__ __forceinline__ uint32_t absmax2(uint32_t a, uint32_t b) {
  uint32_t d;
  b &= 0x7FFF7FFFu;
  if (BF16)
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  else
    asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
// eight values as four bytes of codes
__device__ __forceinline__ uint32_t to_e2m1x8(const float (&y)[8]) {
  uint32_t r;
  asm("{\n .reg .b8 a, b, c, d;\n cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n"
      " cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n"
      " cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n mov.b32 %0, {a, b, c, d};\n}"
      : "=r"(r)
      : "f"(y[0]), "f"(y[1]), "f"(y[2]), "f"(y[3]), "f"(y[4]), "f"(y[5]), "f"(y[6]), "f"(y[7]));
  return r;
}
__device__ __forceinline__ uint32_t to_e4m3(float x) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(0.f), "f"(x));
  return r & 0xFFu;
}

__device__ __forceinline__ float max_nan(float a, float b) {
  float d;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}

// A block's 16 values two at a time, and their largest magnitude (a NaN if one is): from 16-bit words, or
// binary32 values as they were computed.
template <bool BF16>
struct PackedBlock {
  uint32_t w[8];
  __device__ __forceinline__ explicit PackedBlock(const uint4 (&in)[2])
      : w{in[0].x, in[0].y, in[0].z, in[0].w, in[1].x, in[1].y, in[1].z, in[1].w} {}
  __device__ __forceinline__ float2 two(int i) const { return unpack2<BF16>(w[i]); }
  __device__ __forceinline__ float largest() const {
    uint32_t m = w[0] & 0x7FFF7FFFu;
#pragma unroll
    for (int i = 1; i < 8; ++i) m = absmax2<BF16>(m, w[i]);
    const float2 m2 = unpack2<BF16>(m);
    return max_nan(m2.x, m2.y);
  }
};
struct FloatBlock {
  float x[16];
  __device__ __forceinline__ float2 two(int i) const { return make_float2(x[2 * i], x[2 * i + 1]); }
  __device__ __forceinline__ float largest() const {
    float m = fabsf(x[0]);
#pragma unroll
    for (int i = 1; i < 16; ++i) m = max_nan(m, fabsf(x[i]));
    return m;
  }
};

// One block: its scale byte and eight bytes of codes.  x / d is the quotient rounded to
// nearest: a product with the reciprocal, and one step of correction by the remainder
// (Markstein), which is exact where x is a multiple of half a grid step times d, so
// that ties fall as the format says.  Returns false for a NaN or an infinity.
template <typename Block>
__device__ __forceinline__ bool quantize_block(const Block& in, float g, uint32_t& scale, uint2& codes) {
  const float a = in.largest();
  const float t = __fdiv_rn(a, 6.f * g);
  uint32_t c[2];
  if (t <= 448.f) {
    scale = to_e4m3(t);
    const float s = __half2float(__ushort_as_half((uint16_t)e4m3x2_to_half2(scale)));
    const float d = __fmul_rn(s, g);
    const float r = scale ? __frcp_rn(d) : 0.f;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float y[8];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 x = in.two(4 * i + j);
        const float p = __fmul_rn(x.x, r), q = __fmul_rn(x.y, r);
        y[2 * j] = __fmaf_rn(__fmaf_rn(-p, d, x.x), r, p);
        y[2 * j + 1] = __fmaf_rn(__fmaf_rn(-q, d, x.y), r, q);
      }
      c[i] = to_e2m1x8(y);
    }
    // (with scale 0 the quotients are zeros of either sign: the format's codes are 0)
    codes = scale ? make_uint2(c[0], c[1]) : make_uint2(0, 0);
    return true;
  }
  // a NaN, an infinity, or values past the top of the grid: one value at a time
  float top = 0.f;
  bool fine = true;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float2 x = in.two(i);
    top = fmaxf(top, fmaxf(fabsf(x.x), fabsf(x.y)));  // (fmaxf drops a NaN)
    fine = fine && isfinite(x.x) && isfinite(x.y);
  }
  scale = to_e4m3(fminf(__fdiv_rn(top, 6.f * g), 448.f));
  const float d = __fmul_rn(__half2float(__ushort_as_half((uint16_t)e4m3x2_to_half2(scale))), g);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    float y[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 x = in.two(4 * i + j);
      y[2 * j] = scale && x.x == x.x ? __fdiv_rn(x.x, d) : 0.f;
      y[2 * j + 1] = scale && x.y == x.y ? __fdiv_rn(x.y, d) : 0.f;
    }
    c[i] = to_e2m1x8(y);
  }
  codes = make_uint2(c[0], c[1]);
  return fine;
}

// Where row `row` of the step lives: the byte offset of its (layer, page, head 0) record and
// its position in the sequence; false if it has no place.
__device__ __forceinline__ bool place_of(const Kv4Cache& c, const Kv4Batch& b, int layer, int row,
                                         int64_t& record, int64_t& pos) {
  if (row >= b.total) return false;
  int i = row;
  if (b.cu) {
    // the last i with cu[i] <= row: rows from cu[n] on are nobody's
    int lo = 0, hi = b.n;  // cu[lo] <= row (cu[0] is 0), the answer in [lo, hi]
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (b.cu[mid] <= row) lo = mid; else hi = mid - 1;
    }
    i = lo;
  }
  if (i >= b.n) return false;
  int begin, count;
  if (!kv4_range(b, i, begin, count)) {
    raise_error(c.err, kDevIndex);
    return false;
  }
  if (row < begin || row - begin >= count) return false;  // (a range that is not ascending)
  const int first = b.start[i];
  if (first < 0) return false;
  const int seq = b.seqs ? b.seqs[i] : i;
  pos = (int64_t)first + (row - begin);
  const int64_t column = pos >> c.page_shift;
  int page = -1;
  if (seq >= 0 && seq < c.max_seqs && column < c.max_pages)
    page = c.table[(int64_t)seq * c.max_pages + column];
  if (page < 0 || page >= c.num_pages) {
    raise_error(c.err, kDevIndex);
    return false;
  }
  record = kv4_record(c, layer, page, 0);
  return true;
}

}  // namespace semkv
