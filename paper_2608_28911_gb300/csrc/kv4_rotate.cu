// kv4_rotate.cu — new rows of a step: queries and keys turned by their positions, keys and values into
// the pages of the paged 4-bit cache.
//
// A pair (a, b) of a head's dims at a position with cosine c and sine s of its angle becomes
// (a c - b s, b c + a s).  Every product, sum and difference is rounded to binary32 by itself (no fused
// multiply-add), so that a table of cosines and sines fixes every bit; K's blocks are quantized from these
// binary32 values.  Memory-bound: a row of 32 query and 8 KV heads of 128 dims moves 23 KB, 61K rows take 224 us,
// 6.2 TB/s (with their read back 278 us, 97% of the copy rate).  CTAs are for queries or for keys and values: together in
// one they took 87 registers and 302 us; with 4 CTAs on an SM 278, with 3 318, with 2 373 (the read back among them).
// Neighbouring pairs take the same (61K rows 230 us without the read back, halves 232; 20K rows 91 both); halves of an odd
// number of pieces, whose keys read their mates as well, have 2 CTAs on an SM and take 298 us (20K rows 111, 2.5K 25 against 21).
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

enum { kHalves, kPairs, kOddHalves };  // kOddHalves: halves of an odd number of pieces

// Two pieces that make pairs with one another, or each its own.
template <int MODE>
__device__ __forceinline__ void turn_pieces(float (&x)[8], float (&y)[8], const Angles& a0, const Angles& a1) {
  if constexpr (MODE == kPairs) {
    turn_pairs(x, a0);
    turn_pairs(y, a1);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float a = x[j], b = y[j];
      x[j] = turn_first(a, b, a0.c[j], a0.s[j]);
      y[j] = turn_second(a, b, a0.c[j], a0.s[j]);
    }
  }
}

// Where a row lives and the position it is turned by; false if it has no place or no angle.
__device__ __forceinline__ bool turned_place(const Kv4Cache& c, const Kv4Batch& b, int layer, const Kv4Rotation& t, int row,
                                             int64_t& record, int64_t& pos, int64_t& position) {
  if (!place_of(c, b, layer, row, record, pos)) return false;
  position = t.positions ? t.positions[row] : pos;
  if (position >= 0 && position < t.rows) return true;
  raise_error(c.err, kDevIndex);
  return false;
}


// A lane has two pieces of a head, those that make pairs (or neighbours), so that a query may be written where it was
// read.  Rows of CTAs: `q_slices` for the query heads, the others for the KV heads; a lane goes over every so many
// heads, the next one's pieces on their way.
template <int D, bool BF16, int MODE>
__device__ __forceinline__ void turn_queries(const Kv4Cache& c, const Kv4Batch& b, int layer, const Kv4Rotation& t, const Kv4Rows& q,
                                             const Kv4Rows& q_out, int q_heads, int slice, int slices, int row, int lane_piece) {
  const int half = t.rot / 16;  // pieces of half the turned dims
  const bool turned = lane_piece < half, apart = MODE != kPairs && turned;
  const int p0 = apart ? lane_piece : 2 * lane_piece, p1 = apart ? lane_piece + half : 2 * lane_piece + 1;
  const uint16_t* from = static_cast<const uint16_t*>(q.p) + row * q.stride;
  uint16_t* to = static_cast<uint16_t*>(q_out.p) + row * q_out.stride;
  uint4 next[2];
  auto load = [&](int h) {
    next[0] = *reinterpret_cast<const uint4*>(from + h * D + 8 * p0);
    next[1] = *reinterpret_cast<const uint4*>(from + h * D + 8 * p1);
  };
  if (row < b.total) load(slice);
  int64_t record, pos, position;
  if (!turned_place(c, b, layer, t, row, record, pos, position)) return;
  Angles a0, a1;
  if (turned) {
    a0 = angles_of<MODE == kPairs>(t, position, p0);
    if (MODE == kPairs) a1 = angles_of<true>(t, position, p1);
  }
  for (int h = slice; h < q_heads; h += slices) {
    uint4 w0 = next[0], w1 = next[1];
    if (h + slices < q_heads) load(h + slices);
    if (turned) {
      float x[8], y[8];
      unpack8<BF16>(w0, x);
      unpack8<BF16>(w1, y);
      turn_pieces<MODE>(x, y, a0, a1);
      w0 = pack8<BF16>(x);
      w1 = pack8<BF16>(y);
    }
    *reinterpret_cast<uint4*>(to + h * D + 8 * p0) = w0;
    *reinterpret_cast<uint4*>(to + h * D + 8 * p1) = w1;
  }
}

// Keys are turned as queries are.  Then lanes of two pieces each that belong to two blocks (of 16 values, two pieces)
// hand one piece to their neighbour and take one, so that each has a block.  With an odd number of pieces in half the turned
// dims that does not come out even: there a lane loads what its block's pieces make pairs with as well.
template <int D, bool BF16, int MODE>
__device__ __forceinline__ void turn_keys(const Kv4Cache& c, const Kv4Batch& b, int layer, const Kv4Rotation& t, const Kv4Rows& k,
                                          const Kv4Rows& v, int slice, int slices, int row, int lane_piece) {
  constexpr int kBlocks = D / 16;
  const int half = t.rot / 16;
  const bool turned = lane_piece < half, apart = MODE == kHalves && turned;
  // the pieces it loads, the block it stores, and whether it takes the second of what a pair makes
  const bool odd = lane_piece & 1;
  const int p0 = apart ? lane_piece : 2 * lane_piece, p1 = apart ? lane_piece + half : 2 * lane_piece + 1;
  const int blk = apart ? (odd ? lane_piece - 1 + half : lane_piece) / 2 : lane_piece;
  const uint16_t* kr = static_cast<const uint16_t*>(k.p) + row * k.stride;
  const uint16_t* vr = static_cast<const uint16_t*>(v.p) + row * v.stride;
  uint4 next_k[2], next_v[2];
  auto load = [&](int h) {
    const uint4* kp = reinterpret_cast<const uint4*>(kr + h * D);
    const uint4* vp = reinterpret_cast<const uint4*>(vr + h * D) + 2 * blk;
    next_k[0] = kp[p0], next_k[1] = kp[p1];
    next_v[0] = __ldcs(vp), next_v[1] = __ldcs(vp + 1);
  };
  if (row < b.total) load(slice);
  int64_t record = 0, pos = 0, position = 0;
  const bool fine = turned_place(c, b, layer, t, row, record, pos, position);
  if (!__any_sync(~0u, fine)) return;
  if (!fine) position = 0;  // (its lanes go along with the others, and store nothing)
  const int in_page = (int)pos & (c.P - 1);
  const int64_t head_bytes = (int64_t)kv4_tile_bytes(D) << (c.page_shift - 4);
  uint8_t* tile = c.pages + record + (int64_t)(in_page >> 4) * kv4_tile_bytes(D);
  const int r = in_page & 15;
  const int at_codes = r * (D / 2) + blk * 8, at_scale = 16 * D + r * kBlocks + blk;
  Angles a0, a1;
  bool second[2] = {false, false}, mated[2] = {false, false};
  int mate[2] = {0, 0};
  if (MODE == kOddHalves) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int p = 2 * blk + i;
      mated[i] = p < 2 * half;
      second[i] = mated[i] && p >= half;
      mate[i] = second[i] ? p - half : p + half;
      if (mated[i]) (i ? a1 : a0) = angles_of<false>(t, position, second[i] ? p - half : p);
    }
  } else if (turned) {
    a0 = angles_of<MODE == kPairs>(t, position, p0);
    if (MODE == kPairs) a1 = angles_of<true>(t, position, p1);
  }
  for (int h = slice; h < c.H; h += slices) {
    const uint4 k0 = next_k[0], k1 = next_k[1];
    const uint4 vx[2] = {next_v[0], next_v[1]};
    uint4 z[2];
    if (MODE == kOddHalves) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (mated[i] && row < b.total) z[i] = reinterpret_cast<const uint4*>(kr + h * D)[mate[i]];
    }
    if (h + slices < c.H && row < b.total) load(h + slices);
    const float gk = c.k_scale ? c.k_scale[layer * c.H + h] : 1.f;
    const float gv = c.v_scale ? c.v_scale[layer * c.H + h] : 1.f;
    float x[8], y[8];
    unpack8<BF16>(k0, x);
    unpack8<BF16>(k1, y);
    if (MODE == kOddHalves) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float (&w)[8] = i ? y : x;
        const Angles& a = i ? a1 : a0;
        if (!mated[i]) continue;
        float m[8];
        unpack8<BF16>(z[i], m);
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = second[i] ? turn_second(m[j], w[j], a.c[j], a.s[j]) : turn_first(w[j], m[j], a.c[j], a.s[j]);
      }
    } else {
      if (turned) turn_pieces<MODE>(x, y, a0, a1);
      if (MODE == kHalves) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float got = __shfl_xor_sync(~0u, odd ? x[j] : y[j], 1);
          if (apart) (odd ? x[j] : y[j]) = got;
        }
      }
    }
    FloatBlock block;
#pragma unroll
    for (int j = 0; j < 8; ++j) block.x[j] = x[j], block.x[8 + j] = y[j];
    uint32_t sk, sv;
    uint2 ck, cv;
    const bool fk = quantize_block(block, gk, sk, ck);
    const bool fv = quantize_block(PackedBlock<BF16>(vx), gv, sv, cv);
    if (!fine) continue;
    uint8_t* to = tile + h * head_bytes;
    *reinterpret_cast<uint2*>(to + at_codes) = ck;
    *reinterpret_cast<uint2*>(to + 8 * D + at_codes) = cv;
    to[at_scale] = (uint8_t)sk;
    to[at_scale + D] = (uint8_t)sv;
    if (!fk || !fv) raise_error(c.err, kDevNonFinite);
  }
}

template <int D, bool BF16, int MODE>
__global__ void __launch_bounds__(kTurnThreads, MODE == kOddHalves ? 2 : 4)
    kv4_write_rotated_kernel(Kv4Cache c, Kv4Batch b, int layer, Kv4Rotation t, Kv4Rows q, Kv4Rows q_out, int q_heads, int q_slices,
                             Kv4Rows k, Kv4Rows v) {
  constexpr int kLanes = D / 16;  // of a row
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31, warp = blockIdx.x * (kTurnThreads / 32) + (threadIdx.x >> 5);
  const int lane_piece = lane % kLanes, row = warp * (32 / kLanes) + lane / kLanes;
  if ((int)blockIdx.y < q_slices)
    turn_queries<D, BF16, MODE>(c, b, layer, t, q, q_out, q_heads, blockIdx.y, q_slices, row, lane_piece);
  else
    turn_keys<D, BF16, MODE>(c, b, layer, t, k, v, blockIdx.y - q_slices, gridDim.y - q_slices, row, lane_piece);
}

template <int D, bool BF16, int MODE>
cudaError_t launch_rotated(const Kv4Cache& c, const Kv4Batch& b, int layer, const Kv4Rotation& t, const Kv4Rows& q,
                           const Kv4Rows& q_out, int q_heads, const Kv4Rows& k, const Kv4Rows& v, int sms, cudaStream_t stream) {
  constexpr int kRowsPerCta = (kTurnThreads / 32) * (32 / (D / 16));
  const int x = (b.total + kRowsPerCta - 1) / kRowsPerCta;
  // few rows: a CTA for every head (one row 6.5 us with its read back, in a loop over the heads 22); many: the heads in a loop,
  // which looks a row up once (61K rows: with four slices of the queries 4% longer)
  int q_slices = q.p ? 1 : 0, k_slices = 1;
  while ((int64_t)x * (q_slices + k_slices) < 4 * sms) {
    if (2 * q_slices <= q_heads && q_slices > 0) q_slices *= 2;
    else if (2 * k_slices <= c.H) k_slices *= 2;
    else break;
    if (2 * k_slices <= c.H && q_slices >= 4 * k_slices) k_slices *= 2;
  }
  return launch_pdl(kv4_write_rotated_kernel<D, BF16, MODE>, dim3(x, q_slices + k_slices), dim3(kTurnThreads), 0, stream, c, b, layer,
                    t, q, q_out, q_heads, q_slices, k, v);
}

}  // namespace

cudaError_t launch_kv4_write_rotated(const Kv4Cache& c, const Kv4Batch& b, int layer, const Kv4Rotation& t, int dtype,
                                     const Kv4Rows& q, const Kv4Rows& q_out, int q_heads, const Kv4Rows& k, const Kv4Rows& v,
                                     int sms, cudaStream_t stream) {
#define SEMKV_TURN(D, BF, MODE) launch_rotated<D, BF, MODE>(c, b, layer, t, q, q_out, q_heads, k, v, sms, stream)
#define SEMKV_TURN_MODE(D, BF) \
  (t.pairs ? SEMKV_TURN(D, BF, kPairs) : t.rot / 16 % 2 ? SEMKV_TURN(D, BF, kOddHalves) : SEMKV_TURN(D, BF, kHalves))
  const bool bf = dtype == SEMKV_BF16;
  if (c.D == 128) return bf ? SEMKV_TURN_MODE(128, true) : SEMKV_TURN_MODE(128, false);
  return bf ? SEMKV_TURN_MODE(64, true) : SEMKV_TURN_MODE(64, false);
#undef SEMKV_TURN_MODE
#undef SEMKV_TURN
}

}  // namespace semkv
