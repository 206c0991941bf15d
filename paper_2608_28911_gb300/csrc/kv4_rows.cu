// kv4_rows.cu — rows into a layer's pages of the paged 4-bit cache, and back.
//
// Both kernels are bound by memory: a row pair of head_dim 128 moves 512 bytes on the 16-bit
// side and 144 on the 4-bit side.  61K rows of 8 heads take 103 us there and back, 92% of the copy rate.  A warp holds whole rows of consecutive tokens, so that its accesses
// are whole rows and neighbouring tokens run on in the tile; it looks its tokens up once for all heads.
#include "kernels.h"
#include "kv4_rows.cuh"

namespace semkv {
namespace {

constexpr int kRowThreads = 256;

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
  int64_t record, pos;
  if (!place_of(c, b, layer, row, record, pos)) return;
  const int in_page = (int)pos & (c.P - 1);
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
    const bool fk = quantize_block(PackedBlock<BF16>(kx), gk, sk, ck);
    const bool fv = quantize_block(PackedBlock<BF16>(vx), gv, sv, cv);
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
  int64_t record, pos;
  if (!place_of(c, b, layer, row, record, pos)) return;
  const int in_page = (int)pos & (c.P - 1);
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
