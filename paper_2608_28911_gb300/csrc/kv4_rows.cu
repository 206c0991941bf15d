// kv4_rows.cu — rows into a layer's pages of the paged 4-bit cache, and back.
//
// Both kernels are bound by memory: a row pair of head_dim 128 moves 512 bytes on the 16-bit
// side and 144 on the 4-bit side.  61K rows of 8 heads take 103 us there and back, 92% of the copy rate.  A warp holds whole rows of consecutive tokens, so that its accesses
// are whole rows and neighbouring tokens run on in the tile; it looks its tokens up once for all heads.
#include "kernels.h"
#include "kv4.cuh"

namespace semkv {
namespace {

constexpr int kRowThreads = 256;

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

// One block: its scale byte and eight bytes of codes.  x / d is the quotient rounded to
// nearest: a product with the reciprocal, and one step of correction by the remainder
// (Markstein), which is exact where x is a multiple of half a grid step times d, so
// that ties fall as the format says.  Returns false for a NaN or an infinity.
template <bool BF16>
__device__ __forceinline__ bool quantize_block(const uint4 (&in)[2], float g, uint32_t& scale,
                                               uint2& codes) {
  const uint32_t w[8] = {in[0].x, in[0].y, in[0].z, in[0].w, in[1].x, in[1].y, in[1].z, in[1].w};
  uint32_t m = w[0] & 0x7FFF7FFFu;
#pragma unroll
  for (int i = 1; i < 8; ++i) m = absmax2<BF16>(m, w[i]);
  const float2 m2 = unpack2<BF16>(m);
  float a;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(a) : "f"(m2.x), "f"(m2.y));
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
        const float2 x = unpack2<BF16>(w[4 * i + j]);
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
    const float2 x = unpack2<BF16>(w[i]);
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
      const float2 x = unpack2<BF16>(w[4 * i + j]);
      y[2 * j] = scale && x.x == x.x ? __fdiv_rn(x.x, d) : 0.f;
      y[2 * j + 1] = scale && x.y == x.y ? __fdiv_rn(x.y, d) : 0.f;
    }
    c[i] = to_e2m1x8(y);
  }
  codes = make_uint2(c[0], c[1]);
  return fine;
}

// Where row `row` of the step lives: the byte offset of its (layer, page, head 0) record and
// its position in the page; false if it has no place.
__device__ __forceinline__ bool place_of(const Kv4Cache& c, const Kv4Batch& b, int layer, int row,
                                         int64_t& record, int& in_page) {
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
  const int64_t pos = (int64_t)first + (row - begin);
  const int64_t column = pos >> c.page_shift;
  int page = -1;
  if (seq >= 0 && seq < c.max_seqs && column < c.max_pages)
    page = c.table[(int64_t)seq * c.max_pages + column];
  if (page < 0 || page >= c.num_pages) {
    raise_error(c.err, kDevIndex);
    return false;
  }
  record = kv4_record(c, layer, page, 0);
  in_page = (int)pos & (c.P - 1);
  return true;
}

// A lane has one block of 16 values of K and the same of V.
template <int D, bool BF16>
__global__ void __launch_bounds__(kRowThreads) kv4_write_kernel(Kv4Cache c, Kv4Batch b, int layer, const uint16_t* k,
                                                                int64_t k_stride, const uint16_t* v, int64_t v_stride) {
  constexpr int kBlocks = D / 16, kTokens = 32 / kBlocks;
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31;
  const int warp = blockIdx.x * (kRowThreads / 32) + (threadIdx.x >> 5);
  const int blk = lane % kBlocks, row = warp * kTokens + lane / kBlocks;
  int64_t record;
  int in_page;
  if (!place_of(c, b, layer, row, record, in_page)) return;
  const int64_t head_bytes = (int64_t)kv4_tile_bytes(D) << (c.page_shift - 4);
  uint8_t* tile = c.pages + record + (int64_t)(in_page >> 4) * kv4_tile_bytes(D);
  const int r = in_page & 15;
  const int at_codes = r * (D / 2) + blk * 8, at_scale = 16 * D + r * kBlocks + blk;
  const uint16_t* kr = k + row * k_stride + blk * 16;
  const uint16_t* vr = v + row * v_stride + blk * 16;
#pragma unroll 2
  for (int h = blockIdx.y; h < c.H; h += gridDim.y) {
    uint8_t* t = tile + h * head_bytes;
    const float gk = c.k_scale ? c.k_scale[layer * c.H + h] : 1.f;
    const float gv = c.v_scale ? c.v_scale[layer * c.H + h] : 1.f;
    const uint4* kp = reinterpret_cast<const uint4*>(kr + h * D);
    const uint4* vp = reinterpret_cast<const uint4*>(vr + h * D);
    const uint4 kx[2] = {__ldcs(kp), __ldcs(kp + 1)};
    const uint4 vx[2] = {__ldcs(vp), __ldcs(vp + 1)};
    uint32_t sk, sv;
    uint2 ck, cv;
    const bool fk = quantize_block<BF16>(kx, gk, sk, ck);
    const bool fv = quantize_block<BF16>(vx, gv, sv, cv);
    *reinterpret_cast<uint2*>(t + at_codes) = ck;
    *reinterpret_cast<uint2*>(t + 8 * D + at_codes) = cv;
    t[at_scale] = (uint8_t)sk;
    t[at_scale + D] = (uint8_t)sv;
    if (!fk || !fv) raise_error(c.err, kDevNonFinite);
  }
}

// A lane has half a block, so that its 16 bytes of result and its neighbours' are one run of a row (with
// whole blocks each store wrote half of every sector: 69 us for 5 prompts of 12K).
template <int D, bool BF16>
__global__ void __launch_bounds__(kRowThreads) kv4_read_kernel(Kv4Cache c, Kv4Batch b, int layer, uint16_t* k, int64_t k_stride,
                                                               uint16_t* v, int64_t v_stride) {
  constexpr int kLanes = D / 8, kTokens = 32 / kLanes;
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31;
  const int warp = blockIdx.x * (kRowThreads / 32) + (threadIdx.x >> 5);
  const int x = lane % kLanes, row = warp * kTokens + lane / kLanes;
  int64_t record;
  int in_page;
  if (!place_of(c, b, layer, row, record, in_page)) return;
  const int64_t head_bytes = (int64_t)kv4_tile_bytes(D) << (c.page_shift - 4);
  const uint8_t* tile = c.pages + record + (int64_t)(in_page >> 4) * kv4_tile_bytes(D);
  const int r = in_page & 15;
  const uint8_t* codes = tile + r * (D / 2) + x * 4;
  const uint8_t* scales = tile + 16 * D + r * (D / 16) + x / 2;
  uint16_t* kr = k + row * k_stride + x * 8;
  uint16_t* vr = v + row * v_stride + x * 8;
#pragma unroll 4
  for (int h = blockIdx.y; h < c.H; h += gridDim.y) {
    const uint8_t* t = codes + h * head_bytes;
    const uint8_t* s = scales + h * head_bytes;
    const uint32_t ck = __ldcs(reinterpret_cast<const uint32_t*>(t)), cv = __ldcs(reinterpret_cast<const uint32_t*>(t + 8 * D));
    const uint32_t s2 = e4m3x2_to_half2((uint32_t)s[0] | (uint32_t)s[D] << 8);
    const float gk = c.k_scale ? c.k_scale[layer * c.H + h] : 1.f;
    const float gv = c.v_scale ? c.v_scale[layer * c.H + h] : 1.f;
    auto put = [](uint32_t code, uint32_t scale, float g, uint16_t* to) {
      uint32_t w[4];
      e2m1x8_to_half2(code, w);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 f = unpack2<false>(hmul2_bits(w[j], scale));
        w[j] = pack2<BF16>(f.x * g, f.y * g);
      }
      __stcs(reinterpret_cast<uint4*>(to), make_uint4(w[0], w[1], w[2], w[3]));
    };
    put(ck, __byte_perm(s2, 0, 0x1010), gk, kr + h * D);
    put(cv, __byte_perm(s2, 0, 0x3232), gv, vr + h * D);
  }
}

template <int D, bool BF16, bool WRITE>
cudaError_t launch_rows(const Kv4Cache& c, const Kv4Batch& b, int layer, void* k, int64_t k_stride,
                        void* v, int64_t v_stride, int sms, cudaStream_t stream) {
  constexpr int kRowsPerCta = (kRowThreads / 32) * (WRITE ? 32 / (D / 16) : 32 / (D / 8));
  const int x = (b.total + kRowsPerCta - 1) / kRowsPerCta;
  // a few rows: a CTA for every head; many: the heads in a loop, which looks a row up once
  int y = 1;
  while (y < c.H && (int64_t)x * y < 4 * sms) y *= 2;
  if (y > c.H) y = c.H;
  uint16_t* const kp = static_cast<uint16_t*>(k);
  uint16_t* const vp = static_cast<uint16_t*>(v);
  return WRITE ? launch_pdl(kv4_write_kernel<D, BF16>, dim3(x, y), dim3(kRowThreads), 0, stream, c, b, layer, kp, k_stride, vp, v_stride)
               : launch_pdl(kv4_read_kernel<D, BF16>, dim3(x, y), dim3(kRowThreads), 0, stream, c, b, layer, kp, k_stride, vp, v_stride);
}

}  // namespace

cudaError_t launch_kv4_rows(const Kv4Cache& c, const Kv4Batch& b, bool write, int layer, int dtype,
                            void* k, int64_t k_stride, void* v, int64_t v_stride, int sms,
                            cudaStream_t stream) {
  if (b.total == 0) return cudaSuccess;
#define SEMKV_ROWS(D, BF, W) launch_rows<D, BF, W>(c, b, layer, k, k_stride, v, v_stride, sms, stream)
  const bool bf = dtype == SEMKV_BF16;
  if (c.D == 128)
    return write ? (bf ? SEMKV_ROWS(128, true, true) : SEMKV_ROWS(128, false, true))
                 : (bf ? SEMKV_ROWS(128, true, false) : SEMKV_ROWS(128, false, false));
  return write ? (bf ? SEMKV_ROWS(64, true, true) : SEMKV_ROWS(64, false, true))
               : (bf ? SEMKV_ROWS(64, true, false) : SEMKV_ROWS(64, false, false));
#undef SEMKV_ROWS
}

}  // namespace semkv
