// kv4_rotate.cu — new rows of a step: queries and keys turned by their positions, keys and values into
// the pages of the paged 4-bit cache.
//
// A pair (a, b) of a head's dims at a position with cosine c and sine s of its angle becomes
// (a c - b s, b c + a s).  Every product, sum and difference is rounded to binary32 by itself (no fused
// multiply-add), so that a table of cosines and sines fixes every bit; K's blocks are quantized from these
// binary32 values.  Memory-bound: a row of 32 query and 8 KV heads of 128 dims moves 23 KB.
#include "kernels.h"
#include "kv4_rows.cuh"

namespace semkv {
namespace {

constexpr int kTurnThreads = 256;

// The 16-byte pieces (8 values) that make pairs with one another, and the angles they need: with halves piece
// e < rot / 16 goes with e + rot / 16, with neighbouring pairs a piece has its own.
struct Angles {
  float c[8], s[8];
};

template <bool PAIRS>
__device__ __forceinline__ Angles angles_of(const Kv4Rotation& t, int64_t position, int piece) {
  const float* at = t.cos_sin + position * t.rot + piece * (PAIRS ? 4 : 8);
  Angles a;
#pragma unroll
  for (int i = 0; i < (PAIRS ? 1 : 2); ++i) {
    const float4 c = __ldg(reinterpret_cast<const float4*>(at) + i);
    const float4 s = __ldg(reinterpret_cast<const float4*>(at + t.rot / 2) + i);
    a.c[4 * i] = c.x, a.c[4 * i + 1] = c.y, a.c[4 * i + 2] = c.z, a.c[4 * i + 3] = c.w;
    a.s[4 * i] = s.x, a.s[4 * i + 1] = s.y, a.s[4 * i + 2] = s.z, a.s[4 * i + 3] = s.w;
  }
  return a;
}

template <bool BF16>
__device__ __forceinline__ void unpack8(const uint4& w, float (&x)[8]) {
  const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = unpack2<BF16>(v[i]);
    x[2 * i] = f.x;
    x[2 * i + 1] = f.y;
  }
}
template <bool BF16>
__device__ __forceinline__ uint4 pack8(const float (&x)[8]) {
  return make_uint4(pack2<BF16>(x[0], x[1]), pack2<BF16>(x[2], x[3]), pack2<BF16>(x[4], x[5]), pack2<BF16>(x[6], x[7]));
}
__device__ __forceinline__ float turn_first(float a, float b, float c, float s) {
  return __fsub_rn(__fmul_rn(a, c), __fmul_rn(b, s));
}
__device__ __forceinline__ float turn_second(float a, float b, float c, float s) {
  return __fadd_rn(__fmul_rn(b, c), __fmul_rn(a, s));
}
// a piece of neighbouring pairs
__device__ __forceinline__ void turn_pairs(float (&x)[8], const Angles& t) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float a = x[2 * j], b = x[2 * j + 1];
    x[2 * j] = turn_first(a, b, t.c[j], t.s[j]);
    x[2 * j + 1] = turn_second(a, b, t.c[j], t.s[j]);
  }
}

// A lane has two pieces of a query head (those that make pairs, so that it may write where it read), and one
// block of 16 values of a KV head's K and V.  For K it also loads the pieces that its own make pairs with: they are in
// the lines that its neighbours load.
template <int D, bool BF16, bool PAIRS>
__global__ void __launch_bounds__(kTurnThreads) kv4_write_rotated_kernel(Kv4Cache c, Kv4Batch b, int layer, Kv4Rotation t,
                                                                         Kv4Rows q, Kv4Rows q_out, int q_heads, Kv4Rows k,
                                                                         Kv4Rows v) {
  constexpr int kBlocks = D / 16, kTokens = 32 / kBlocks;
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31;
  const int warp = blockIdx.x * (kTurnThreads / 32) + (threadIdx.x >> 5);
  const int blk = lane % kBlocks, row = warp * kTokens + lane / kBlocks;
  int64_t record, pos;
  if (!place_of(c, b, layer, row, record, pos)) return;
  const int in_page = (int)pos & (c.P - 1);
  const int64_t position = t.positions ? t.positions[row] : pos;
  if (position < 0 || position >= t.rows) {
    raise_error(c.err, kDevIndex);
    return;
  }
  const int half = t.rot / 16;  // pieces of half the turned dims
  if (q.p) {
    const bool turned = blk < half;
    const int p0 = PAIRS || !turned ? 2 * blk : blk, p1 = PAIRS || !turned ? 2 * blk + 1 : blk + half;
    Angles a0, a1;
    if (turned) {
      a0 = angles_of<PAIRS>(t, position, p0);
      if (PAIRS) a1 = angles_of<PAIRS>(t, position, p1);
    }
    const uint16_t* from = static_cast<const uint16_t*>(q.p) + row * q.stride;
    uint16_t* to = static_cast<uint16_t*>(q_out.p) + row * q_out.stride;
#pragma unroll 4
    for (int h = blockIdx.y; h < q_heads; h += gridDim.y) {
      uint4 w0 = *reinterpret_cast<const uint4*>(from + h * D + 8 * p0);
      uint4 w1 = *reinterpret_cast<const uint4*>(from + h * D + 8 * p1);
      if (turned) {
        float x[8], y[8];
        unpack8<BF16>(w0, x);
        unpack8<BF16>(w1, y);
        if (PAIRS) {
          turn_pairs(x, a0);
          turn_pairs(y, a1);
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float a = x[j], z = y[j];
            x[j] = turn_first(a, z, a0.c[j], a0.s[j]);
            y[j] = turn_second(a, z, a0.c[j], a0.s[j]);
          }
        }
        w0 = pack8<BF16>(x);
        w1 = pack8<BF16>(y);
      }
      *reinterpret_cast<uint4*>(to + h * D + 8 * p0) = w0;
      *reinterpret_cast<uint4*>(to + h * D + 8 * p1) = w1;
    }
  }
  const int64_t head_bytes = (int64_t)kv4_tile_bytes(D) << (c.page_shift - 4);
  uint8_t* tile = c.pages + record + (int64_t)(in_page >> 4) * kv4_tile_bytes(D);
  const int r = in_page & 15;
  const int at_codes = r * (D / 2) + blk * 8, at_scale = 16 * D + r * kBlocks + blk;
  const uint16_t* kr = static_cast<const uint16_t*>(k.p) + row * k.stride;
  const uint16_t* vr = static_cast<const uint16_t*>(v.p) + row * v.stride;
  // this block's pieces, the pieces they go with, and the angles
  bool turned[2], second[2];
  int mate[2];
  Angles a[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int p = 2 * blk + i;
    turned[i] = p < 2 * half;
    second[i] = !PAIRS && turned[i] && p >= half;
    mate[i] = PAIRS || !turned[i] ? p : second[i] ? p - half : p + half;
    if (turned[i]) a[i] = angles_of<PAIRS>(t, position, second[i] ? p - half : p);
  }
  for (int h = blockIdx.y; h < c.H; h += gridDim.y) {
    uint8_t* to = tile + h * head_bytes;
    const float gk = c.k_scale ? c.k_scale[layer * c.H + h] : 1.f;
    const float gv = c.v_scale ? c.v_scale[layer * c.H + h] : 1.f;
    const uint4* kp = reinterpret_cast<const uint4*>(kr + h * D);
    const uint4* vp = reinterpret_cast<const uint4*>(vr + h * D) + 2 * blk;
    const uint4 kx[2] = {kp[2 * blk], kp[2 * blk + 1]};
    uint4 kz[2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (!PAIRS) kz[i] = kp[mate[i]];
    const uint4 vx[2] = {__ldcs(vp), __ldcs(vp + 1)};
    FloatBlock block;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float x[8], z[8];
      unpack8<BF16>(kx[i], x);
      if (turned[i]) {
        if (PAIRS) {
          turn_pairs(x, a[i]);
        } else {
          unpack8<BF16>(kz[i], z);
#pragma unroll
          for (int j = 0; j < 8; ++j)
            x[j] = second[i] ? turn_second(z[j], x[j], a[i].c[j], a[i].s[j]) : turn_first(x[j], z[j], a[i].c[j], a[i].s[j]);
        }
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) block.x[8 * i + j] = x[j];
    }
    uint32_t sk, sv;
    uint2 ck, cv;
    const bool fk = quantize_block(block, gk, sk, ck);
    const bool fv = quantize_block(PackedBlock<BF16>(vx), gv, sv, cv);
    *reinterpret_cast<uint2*>(to + at_codes) = ck;
    *reinterpret_cast<uint2*>(to + 8 * D + at_codes) = cv;
    to[at_scale] = (uint8_t)sk;
    to[at_scale + D] = (uint8_t)sv;
    if (!fk || !fv) raise_error(c.err, kDevNonFinite);
  }
}

template <int D, bool BF16, bool PAIRS>
cudaError_t launch_rotated(const Kv4Cache& c, const Kv4Batch& b, int layer, const Kv4Rotation& t, const Kv4Rows& q,
                           const Kv4Rows& q_out, int q_heads, const Kv4Rows& k, const Kv4Rows& v, int sms, cudaStream_t stream) {
  constexpr int kRowsPerCta = (kTurnThreads / 32) * (32 / (D / 16));
  const int x = (b.total + kRowsPerCta - 1) / kRowsPerCta, most = q_heads > c.H ? q_heads : c.H;
  // a few rows: a CTA for every head; many: the heads in a loop, which looks a row up once
  int y = 1;
  while (y < most && (int64_t)x * y < 4 * sms) y *= 2;
  if (y > most) y = most;
  return launch_pdl(kv4_write_rotated_kernel<D, BF16, PAIRS>, dim3(x, y), dim3(kTurnThreads), 0, stream, c, b, layer, t, q, q_out,
                    q_heads, k, v);
}

}  // namespace

cudaError_t launch_kv4_write_rotated(const Kv4Cache& c, const Kv4Batch& b, int layer, const Kv4Rotation& t, int dtype,
                                     const Kv4Rows& q, const Kv4Rows& q_out, int q_heads, const Kv4Rows& k, const Kv4Rows& v,
                                     int sms, cudaStream_t stream) {
#define SEMKV_TURN(D, BF, PA) launch_rotated<D, BF, PA>(c, b, layer, t, q, q_out, q_heads, k, v, sms, stream)
  const bool bf = dtype == SEMKV_BF16;
  if (c.D == 128)
    return t.pairs ? (bf ? SEMKV_TURN(128, true, true) : SEMKV_TURN(128, false, true))
                   : (bf ? SEMKV_TURN(128, true, false) : SEMKV_TURN(128, false, false));
  return t.pairs ? (bf ? SEMKV_TURN(64, true, true) : SEMKV_TURN(64, false, true))
                 : (bf ? SEMKV_TURN(64, true, false) : SEMKV_TURN(64, false, false));
#undef SEMKV_TURN
}

}  // namespace semkv
