// kv4_attend.cu — attention over the paged 4-bit cache for few query rows (single tokens,
// drafted tokens), bound by reading the cache.
//
// For a tile of 16 tokens, on mma.sync m16n8k16 with fp16 operands and fp32 sums:
//   S^T = K Q^T      M = 16 tokens, N = 8 query rows, K = head dim
//   P   = 2^(S - e)  e: the row's reference exponent, moved only when a weight would pass 2^15
//   O^T += V^T P^T   M = head dim, N = 8 query rows, K = 16 tokens
// The tokens and the head dim are the M side, so eight rows (a GQA group, a few drafted
// tokens) fill N, and more rows are further N tiles of the same dequantized operands.  The order of
// the head dim inside the K products and of the tokens is free: lane (g, t) takes dims t D/4 ..
// of token g, one 16-byte load, as the A fragments of all its k steps, and Q's fragments follow that
// order.  For V, lane (g, t) holds the dims of block g (D 128) for four tokens; a shift and a merge
// put the nibbles of two tokens into one byte, so that the conversion leaves the pair (token a,
// token b) that the A fragment wants.  Tokens are taken in the order {0, 3, 1, 2, 4, 7, 5, 6} of
// every eight, which leaves K's loads without bank conflicts and V's two-way.
// S^T's accumulators become P^T's B fragments by one 8x8 transposition (movmatrix).
//
// Each warp streams its own units (32 tokens, two tiles) through a ring of bulk copies.
#include "kernels.h"
#include "kv4_attend.cuh"

namespace semkv {
namespace {

constexpr int kUnit = 32;       // tokens of a unit
constexpr int kWarps = 8;
constexpr int kThreads = kWarps * 32;
constexpr float kNone = -1e30f;  // reference exponent of a row without tokens
constexpr float kHead = 8.f;     // a moved reference puts the largest weight at 2^8
constexpr float kMost = 15.f;    // largest exponent of a weight

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
  uint32_t w;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
  return w;
}

// token of the tile at place x of the order: {0, 3, 1, 2} and the same four further, ...
__device__ __forceinline__ int token_at(int x) {
  const int t = (x & 7) >> 1, base = (x & 8) + t + (t & 2);
  return x & 1 ? base ^ 3 : base;
}

template <int D, int NT>
struct Layout {
  static constexpr int kTile = kv4_tile_bytes(D);
  static constexpr int kRows = 8 * NT;
  static constexpr int kStage = 2 * kTile;
  static constexpr int kStages = 3;
  static constexpr int kSums = D + 4;  // padded row of the merge area
  static constexpr int ring_bytes() { return kWarps * kStages * kStage; }
  static constexpr int merge_bytes() { return kWarps * kRows * (kSums + 2) * 4; }
  // the merge area lies over the ring, which is empty between items
  static constexpr int data_bytes() { return ring_bytes() > merge_bytes() ? ring_bytes() : merge_bytes(); }
  static constexpr int q_bytes() { return NT * (D / 16) * 32 * 8; }
  static constexpr int bytes() { return data_bytes() + q_bytes() + NT * 8 * 4 + kWarps * kStages * 8 + (kThreads + 1) * 8 + kWarps * 8; }
};

// Q's fragments of an item into shared memory, [n tile][k step][lane]: rows of the step's q for
// one KV head; bf16 rows are scaled by a power of two, which leaves their values exact in
// fp16 but for those 2^-24 and less of the row's largest.  scale[row]: what undoes it.
template <int D, int NT, bool BF16>
__device__ __forceinline__ void load_queries(const Kv4Attend& a, const Kv4Seq& s, int head, int tile, uint2* qf,
                                             float* scale) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int g = lane >> 2, t = lane & 3;
  if (warp >= NT) return;
  const int row = tile * 8 * NT + warp * 8 + g;
  const int j = row / a.group, h = head * a.group + row % a.group;
  uint32_t w[D / 8];
  float most = 0.f;
  if (j < s.count) {
    const uint4* p = reinterpret_cast<const uint4*>(a.q + (int64_t)(s.begin + j) * a.q_stride + h * D + t * (D / 4));
#pragma unroll
    for (int k = 0; k < D / 32; ++k) {
      const uint4 x = p[k];
      w[4 * k] = x.x, w[4 * k + 1] = x.y, w[4 * k + 2] = x.z, w[4 * k + 3] = x.w;
    }
  } else {
#pragma unroll
    for (int k = 0; k < D / 8; ++k) w[k] = 0;
  }
  float undo = 1.f;
  if (BF16) {
#pragma unroll
    for (int k = 0; k < D / 8; ++k) {
      most = fmaxf(most, fabsf(__uint_as_float(w[k] << 16)));
      most = fmaxf(most, fabsf(__uint_as_float(w[k] & 0xFFFF0000u)));
    }
    most = fmaxf(most, __shfl_xor_sync(~0u, most, 1));
    most = fmaxf(most, __shfl_xor_sync(~0u, most, 2));
    // the row's largest to [2^0, 2^1); rows of zeros, infinities or NaN as they are
    int e = (int)(__float_as_uint(most) >> 23) - 127;
    if (most == 0.f || !(most < INFINITY)) e = 0;
    e = e < -126 ? -126 : e;
    const float by = __uint_as_float((uint32_t)(127 - e) << 23);  // 2^-e (e = 127: 0, below)
    undo = e == 127 ? 0x1p127f : __uint_as_float((uint32_t)(127 + e) << 23);
    const float mul = e == 127 ? 0x1p-127f : by;
#pragma unroll
    for (int k = 0; k < D / 8; ++k)
      w[k] = pack_half2(__uint_as_float(w[k] << 16) * mul, __uint_as_float(w[k] & 0xFFFF0000u) * mul);
  }
#pragma unroll
  for (int k = 0; k < D / 16; ++k) qf[(warp * (D / 16) + k) * 32 + lane] = make_uint2(w[2 * k], w[2 * k + 1]);
  if (t == 0) scale[warp * 8 + g] = undo;
}

template <int D, int NT, bool BF16>
__global__ void __launch_bounds__(kThreads, NT == 1 ? 2 : 1) kv4_attend_kernel(Kv4Attend a) {
  using L = Layout<D, NT>;
  constexpr int kSteps = D / 16;   // k steps of S
  constexpr int kM = D / 16;       // m tiles of O
  extern __shared__ __align__(128) uint8_t smem[];
  uint8_t* data = smem;
  uint2* qf = reinterpret_cast<uint2*>(data + L::data_bytes());
  int64_t* prefix = reinterpret_cast<int64_t*>(reinterpret_cast<uint8_t*>(qf) + L::q_bytes());
  int64_t* sums = prefix + kThreads + 1;
  uint64_t* bars = reinterpret_cast<uint64_t*>(sums + kWarps);
  float* q_scale = reinterpret_cast<float*>(bars + kWarps * L::kStages);

  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int g = lane >> 2, t = lane & 3;
  uint8_t* ring = data + warp * (L::kStages * L::kStage);
  uint64_t* bar = bars + warp * L::kStages;
  if (lane == 0) {
    for (int s = 0; s < L::kStages; ++s)
      asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(smem_addr(bar + s)) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  pdl_wait();
  pdl_trigger();
  kv4_plan<L::kRows, kUnit, kThreads>(a, prefix, sums, blockIdx.x == 0);
  const int64_t W = prefix[kThreads];
  const int ctas = kv4_ctas(W, gridDim.x);
  if (W == 0 || (int)blockIdx.x >= ctas) return;
  const int64_t begin = kv4_range_begin(W, blockIdx.x, ctas), end = kv4_range_begin(W, blockIdx.x + 1, ctas);

  const int row_a = token_at(g), tok_v = token_at(2 * t);  // K row of lane group g; V's first token
  const int64_t page_bytes = (int64_t)L::kTile << (a.c.page_shift - 4);
  uint32_t phase = 0;  // parity of each stage's barrier, a bit each
  bool lost = false;   // a wait ran out

  for (int64_t cur = begin; cur < end;) {
    // the sequence that holds unit `cur`, the item and the part of it that is this CTA's
    int64_t before;
    const Kv4Seq s = kv4_find<L::kRows, kUnit, kThreads>(a, prefix, cur, before);
    const int64_t in_seq = cur - before;
    const int item = (int)(in_seq / s.units), u0 = (int)(in_seq - (int64_t)item * s.units);
    const int head = item / s.tiles, tile = item - head * s.tiles;
    const int64_t left = end - cur;
    const int u1 = s.units - u0 < left ? s.units : u0 + (int)left;

    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // the merge area becomes a ring again
    __syncthreads();  // the item before is done with the shared areas
    load_queries<D, NT, BF16>(a, s, head, tile, qf, q_scale);
    __syncthreads();

    // what this lane's query rows (columns 2t, 2t+1 of each n tile) see
    int see_lo[2 * NT], see_hi[2 * NT];
    float mul[2 * NT];
    int most_lo = 0, least_hi = 0x7FFFFFFF;
    const float gk = a.c.k_scale ? a.c.k_scale[a.layer * a.c.H + head] : 1.f;
#pragma unroll
    for (int x = 0; x < 2 * NT; ++x) {
      const int col = (x >> 1) * 8 + 2 * t + (x & 1);
      kv4_sight(a, s, tile * L::kRows + col, see_lo[x], see_hi[x]);
      mul[x] = a.scale_log2 * gk * q_scale[col];
      if (see_hi[x] >= 0 || (tile * L::kRows + col) / a.group < s.count) {
        most_lo = max(most_lo, see_lo[x]);
        least_hi = min(least_hi, see_hi[x]);
      }
    }
    most_lo = __reduce_max_sync(~0u, most_lo);
    least_hi = __reduce_min_sync(~0u, least_hi);

    float O[NT][kM][4];
    float ref[2 * NT], sum[2 * NT];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int m = 0; m < kM; ++m)
#pragma unroll
        for (int x = 0; x < 4; ++x) O[n][m][x] = 0.f;
#pragma unroll
    for (int x = 0; x < 2 * NT; ++x) ref[x] = kNone, sum[x] = 0.f;

    // this warp's units: u0 + warp, + kWarps, ...
    const int mine = u1 - u0 > warp ? (u1 - u0 - warp + kWarps - 1) / kWarps : 0;
    const uint8_t* head_base = a.c.pages + kv4_record(a.c, a.layer, 0, head);
    const int64_t page_stride = page_bytes * a.c.H;
    const int32_t* table = a.c.table + (int64_t)s.seq * a.c.max_pages;
    // lane l keeps the pages of the warp's unit k0 + l (with pages of 16 tokens: of both halves)
    int page_x = 0, page_y = 0, k0 = 0;
    auto fetch_pages = [&](int k) {
      k0 = k;
      const int kk = k + lane;
      if (kk < mine) {
        const int token = (s.u_first + u0 + warp + kk * kWarps) * kUnit;
        page_x = table[token >> a.c.page_shift];
        page_y = a.c.page_shift == 4 && token + 16 < s.length ? table[(token >> 4) + 1] : 0;
        if ((unsigned)page_x >= (unsigned)a.c.num_pages || (unsigned)page_y >= (unsigned)a.c.num_pages) {
          raise_error(a.c.err, kDevIndex);
          if ((unsigned)page_x >= (unsigned)a.c.num_pages) page_x = 0;
          if ((unsigned)page_y >= (unsigned)a.c.num_pages) page_y = 0;
        }
      }
    };
    auto issue = [&](int k, int stage) {
      if (k >= k0 + 32) fetch_pages(k);
      const int px = __shfl_sync(~0u, page_x, k - k0), py = __shfl_sync(~0u, page_y, k - k0);
      if (lane == 0) {
        const int token = (s.u_first + u0 + warp + k * kWarps) * kUnit;
        const bool two = token + 16 < s.length;
        const uint32_t dst = smem_addr(ring + stage * L::kStage), b = smem_addr(bar + stage);
        const uint8_t* src = head_base + px * page_stride + (int64_t)((token & (a.c.P - 1)) >> 4) * L::kTile;
        const uint32_t bytes = two ? 2 * L::kTile : L::kTile;
        const bool whole = a.c.page_shift > 4;
        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(b), "r"(bytes) : "memory");
        asm volatile(
            "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src),
            "r"(whole ? bytes : (uint32_t)L::kTile), "r"(b)
            : "memory");
        if (!whole && two)
          asm volatile(
              "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst + L::kTile),
              "l"(head_base + py * page_stride), "r"((uint32_t)L::kTile), "r"(b)
              : "memory");
      }
    };
    fetch_pages(0);
    const int ahead = mine < L::kStages ? mine : L::kStages;
    for (int k = 0; k < ahead; ++k) issue(k, k);

    int stage = 0;
    for (int k = 0; k < mine; ++k) {
      if (!lost && !mbar_wait_bounded(bar + stage, phase >> stage & 1)) {
        lost = true;
        if (lane == 0) raise_error(a.c.err, kDevWaitTimeout);
      }
      lost = __any_sync(~0u, lost);
      if (lost) {
        // the copies still in flight are waited for, as long again
        const int issued = min(mine, k + L::kStages);
        for (int j = k + 1; j < issued; ++j) {
          stage = stage + 1 == L::kStages ? 0 : stage + 1;
          mbar_wait_bounded(bar + stage, phase >> stage & 1);
        }
        break;
      }
      phase ^= 1u << stage;
      const int token = (s.u_first + u0 + warp + k * kWarps) * kUnit;
#pragma unroll 1
      for (int half = 0; half < 2; ++half) {
        const int t0 = token + 16 * half;
        if (t0 >= s.length) break;
        const uint8_t* tl = ring + stage * L::kStage + half * L::kTile;
        // ---- S^T = K Q^T
        float S[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n) S[n][0] = S[n][1] = S[n][2] = S[n][3] = 0.f;
        {
          uint32_t ka[D / 32], kb[D / 32];
          const uint8_t* pa = tl + row_a * (D / 2) + t * (D / 8);
          if constexpr (D == 128) {
            const uint4 x = *reinterpret_cast<const uint4*>(pa), y = *reinterpret_cast<const uint4*>(pa + 8 * (D / 2));
            ka[0] = x.x, ka[1] = x.y, ka[2] = x.z, ka[3] = x.w;
            kb[0] = y.x, kb[1] = y.y, kb[2] = y.z, kb[3] = y.w;
          } else {
            const uint2 x = *reinterpret_cast<const uint2*>(pa), y = *reinterpret_cast<const uint2*>(pa + 8 * (D / 2));
            ka[0] = x.x, ka[1] = x.y;
            kb[0] = y.x, kb[1] = y.y;
          }
          uint32_t sa[D / 64], sb[D / 64];  // a scale twice, for each 16 dims of the lane
          const uint8_t* ps = tl + 16 * D + row_a * (D / 16) + t * (D / 64);
          if constexpr (D == 128) {
            const uint32_t ha = e4m3x2_to_half2(*reinterpret_cast<const uint16_t*>(ps));
            const uint32_t hb = e4m3x2_to_half2(*reinterpret_cast<const uint16_t*>(ps + 8 * (D / 16)));
            sa[0] = __byte_perm(ha, 0, 0x1010), sa[1] = __byte_perm(ha, 0, 0x3232);
            sb[0] = __byte_perm(hb, 0, 0x1010), sb[1] = __byte_perm(hb, 0, 0x3232);
          } else {
            const uint32_t h = e4m3x2_to_half2((uint32_t)ps[0] | (uint32_t)ps[8 * (D / 16)] << 8);
            sa[0] = __byte_perm(h, 0, 0x1010);
            sb[0] = __byte_perm(h, 0, 0x3232);
          }
#pragma unroll
          for (int w = 0; w < D / 32; ++w) {
            uint32_t xa[4], xb[4];
            e2m1x8_to_half2(ka[w], xa);
            e2m1x8_to_half2(kb[w], xb);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              xa[i] = hmul2_bits(xa[i], sa[w / 2]);
              xb[i] = hmul2_bits(xb[i], sb[w / 2]);
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              const uint2 q0 = qf[(n * kSteps + 2 * w) * 32 + lane], q1 = qf[(n * kSteps + 2 * w + 1) * 32 + lane];
              mma16816(S[n], xa[0], xb[0], xa[1], xb[1], q0.x, q0.y);
              mma16816(S[n], xa[2], xb[2], xa[3], xb[3], q1.x, q1.y);
            }
          }
        }
        // ---- weights
        const bool open = t0 >= most_lo && t0 + 15 <= least_hi;  // every row sees the whole tile
        const int pos_a = t0 + row_a, pos_b = pos_a + 8;
        bool over = false;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const int i = 2 * n + x;
            S[n][x] *= mul[i];
            S[n][2 + x] *= mul[i];
            if (!open) {
              if (pos_a < see_lo[i] || pos_a > see_hi[i]) S[n][x] = -INFINITY;
              if (pos_b < see_lo[i] || pos_b > see_hi[i]) S[n][2 + x] = -INFINITY;
            }
            over = over || S[n][x] > ref[i] + kMost || S[n][2 + x] > ref[i] + kMost;
          }
        if (__any_sync(~0u, over)) {
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              const int i = 2 * n + x;
              float top = fmaxf(S[n][x], S[n][2 + x]);
              top = fmaxf(top, __shfl_xor_sync(~0u, top, 4));
              top = fmaxf(top, __shfl_xor_sync(~0u, top, 8));
              top = fmaxf(top, __shfl_xor_sync(~0u, top, 16));
              if (top > ref[i] + kMost) {
                const float to = top - kHead, f = exp2_approx(ref[i] - to);
                ref[i] = to;
                sum[i] *= f;
#pragma unroll
                for (int m = 0; m < kM; ++m) {
                  O[n][m][x] *= f;
                  O[n][m][2 + x] *= f;
                }
              }
            }
        }
        uint32_t pb[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            S[n][x] = exp2_approx(S[n][x] - ref[2 * n + (x & 1)]);
            sum[2 * n + (x & 1)] += S[n][x];
          }
          pb[n][0] = transpose8x8(pack_half2(S[n][0], S[n][1]));
          pb[n][1] = transpose8x8(pack_half2(S[n][2], S[n][3]));
        }
        // ---- O^T += V^T P^T: tokens a = tok_v and a ^ 3 (places 2t, 2t+1), and both + 8
        {
          const int ta = tok_v, tb = tok_v ^ 3;
          const uint8_t* pv = tl + 8 * D + g * (D / 16);
          const uint8_t* ps = tl + 17 * D + (D == 128 ? g : g >> 1);
          uint32_t s01 = (uint32_t)ps[ta * (D / 16)] | (uint32_t)ps[tb * (D / 16)] << 8;
          uint32_t s23 = (uint32_t)ps[(ta + 8) * (D / 16)] | (uint32_t)ps[(tb + 8) * (D / 16)] << 8;
          if (t0 + 16 > s.length) {
            // rows behind the last token hold anything: their scale is 0
            const int over_end = s.length - t0;
            if (ta >= over_end) s01 &= 0xFF00u;
            if (tb >= over_end) s01 &= 0x00FFu;
            if (ta + 8 >= over_end) s23 &= 0xFF00u;
            if (tb + 8 >= over_end) s23 &= 0x00FFu;
          }
          const uint32_t h01 = e4m3x2_to_half2(s01), h23 = e4m3x2_to_half2(s23);
#pragma unroll
          for (int w = 0; w < D / 64; ++w) {
            const uint32_t va = *reinterpret_cast<const uint32_t*>(pv + ta * (D / 2) + 4 * w);
            const uint32_t vb = *reinterpret_cast<const uint32_t*>(pv + tb * (D / 2) + 4 * w);
            const uint32_t vc = *reinterpret_cast<const uint32_t*>(pv + (ta + 8) * (D / 2) + 4 * w);
            const uint32_t vd = *reinterpret_cast<const uint32_t*>(pv + (tb + 8) * (D / 2) + 4 * w);
            uint32_t e01[4], o01[4], e23[4], o23[4];  // even and odd dims of the byte, token pairs
            e2m1x8_to_half2((va & 0x0F0F0F0Fu) | ((vb << 4) & 0xF0F0F0F0u), e01);
            e2m1x8_to_half2(((va >> 4) & 0x0F0F0F0Fu) | (vb & 0xF0F0F0F0u), o01);
            e2m1x8_to_half2((vc & 0x0F0F0F0Fu) | ((vd << 4) & 0xF0F0F0F0u), e23);
            e2m1x8_to_half2(((vc >> 4) & 0x0F0F0F0Fu) | (vd & 0xF0F0F0F0u), o23);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t a0 = hmul2_bits(e01[i], h01), a1 = hmul2_bits(o01[i], h01);
              const uint32_t a2 = hmul2_bits(e23[i], h23), a3 = hmul2_bits(o23[i], h23);
#pragma unroll
              for (int n = 0; n < NT; ++n) mma16816(O[n][4 * w + i], a0, a1, a2, a3, pb[n][0], pb[n][1]);
            }
          }
        }
      }
      __syncwarp();
      if (k + L::kStages < mine) {
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        issue(k + L::kStages, stage);
      }
      stage = stage + 1 == L::kStages ? 0 : stage + 1;
    }
    // ---- the warps' sums are put together
#pragma unroll
    for (int x = 0; x < 2 * NT; ++x) {
      sum[x] += __shfl_xor_sync(~0u, sum[x], 4);
      sum[x] += __shfl_xor_sync(~0u, sum[x], 8);
      sum[x] += __shfl_xor_sync(~0u, sum[x], 16);
    }
    const bool broken = __syncthreads_or(lost);  // every warp is done with its ring
    if (broken) return;
    float* area = reinterpret_cast<float*>(data);
    float* heads = area + kWarps * L::kRows * L::kSums;  // [warp][row]: reference, then sum
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int col = n * 8 + 2 * t + x;
        float* o = area + (warp * L::kRows + col) * L::kSums;
#pragma unroll
        for (int m = 0; m < kM; ++m)
          *reinterpret_cast<float2*>(o + g * (D / 8) + 2 * m) = make_float2(O[n][m][x], O[n][m][2 + x]);
        if (g == 0) {
          heads[(warp * L::kRows + col) * 2] = ref[2 * n + x];
          heads[(warp * L::kRows + col) * 2 + 1] = sum[2 * n + x];
        }
      }
    }
    __syncthreads();
    const bool done = u0 == 0 && u1 == s.units;
    const int slot = 2 * (int)blockIdx.x + (cur == begin ? 0 : 1);
    const float gv = a.c.v_scale ? a.c.v_scale[a.layer * a.c.H + head] : 1.f;
    const int rows = min(L::kRows, s.count * a.group - tile * L::kRows);
    for (int x = threadIdx.x; x < rows * (D / 4); x += kThreads) {
      const int col = x / (D / 4), d4 = x % (D / 4) * 4;
      float top = kNone;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) top = fmaxf(top, heads[(w * L::kRows + col) * 2]);
      float total = 0.f;
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float f = exp2_approx(heads[(w * L::kRows + col) * 2] - top);
        total += f * heads[(w * L::kRows + col) * 2 + 1];
        const float4 y = *reinterpret_cast<const float4*>(area + (w * L::kRows + col) * L::kSums + d4);
        o.x += f * y.x, o.y += f * y.y, o.z += f * y.z, o.w += f * y.w;
      }
      if (done) {
        const int row = tile * L::kRows + col;
        const int64_t at = (int64_t)(s.begin + row / a.group) * a.q_heads + head * a.group + row % a.group;
        const float inv = total == 0.f ? 0.f : gv / total;
        uint2 packed;
        if (BF16) {
          asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(packed.x) : "f"(o.y * inv), "f"(o.x * inv));
          asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(packed.y) : "f"(o.w * inv), "f"(o.z * inv));
        } else {
          packed = make_uint2(pack_half2(o.x * inv, o.y * inv), pack_half2(o.z * inv, o.w * inv));
        }
        *reinterpret_cast<uint2*>(a.out + at * D + d4) = packed;
        if (a.lse && d4 == 0) a.lse[at] = total == 0.f ? -INFINITY : (top + log2f(total)) * 0.6931471805599453f;
      } else {
        float* part = a.parts + ((int64_t)slot * L::kRows + col) * (D + 2);
        part[d4] = o.x, part[d4 + 1] = o.y, part[d4 + 2] = o.z, part[d4 + 3] = o.w;
        if (d4 == 0) part[D] = top, part[D + 1] = total;
      }
    }
    cur += u1 - u0;
  }
}

// Joins the parts of the items that several CTAs share, and fills the rows that see nothing.
// A CTA per (sequence, head and tile of rows), a thread per dim and several rows.
template <int D, bool BF16>
__global__ void __launch_bounds__(128) kv4_join_kernel(Kv4Attend a, int rows_tile, int unit, int grid) {
  pdl_wait();
  pdl_trigger();
  const int i = blockIdx.x;
  Kv4Seq s;
  {
    s.seq = a.b.seqs ? a.b.seqs[i] : i;
    if (!kv4_range(a.b, i, s.begin, s.count) || s.seq < 0 || s.seq >= a.c.max_seqs) return;
    s.tiles = (s.count * a.group + rows_tile - 1) / rows_tile;
  }
  const int64_t W = a.prefix[a.b.n], p0 = a.prefix[i], p1 = a.prefix[i + 1];
  const int ctas = kv4_ctas(W, grid);
  constexpr int kGroups = 128 / (D / 2);  // rows at a time, two dims to a thread
  const int d2 = threadIdx.x % (D / 2) * 2;
  for (int it = blockIdx.y; it < s.tiles * a.c.H; it += gridDim.y) {
    const int head = it / s.tiles, tile = it - head * s.tiles;
    const int64_t units = (p1 - p0) / ((int64_t)s.tiles * a.c.H), u0 = p0 + it * units, u1 = u0 + units;
    int c0 = 0, c1 = -1;
    if (units > 0) {
      c0 = kv4_owner(W, u0, ctas);
      c1 = kv4_owner(W, u1 - 1, ctas);
      if (c0 == c1) continue;  // finished where it ran
    }
    const float gv = a.c.v_scale ? a.c.v_scale[a.layer * a.c.H + head] : 1.f;
    const int rows = min(rows_tile, s.count * a.group - tile * rows_tile);
    const int first_slot = 2 * c0 + (units > 0 && kv4_range_begin(W, c0, ctas) < u0 ? 1 : 0);
    for (int col = threadIdx.x / (D / 2); col < rows; col += kGroups) {
      float top = kNone, total = 0.f, x = 0.f, y = 0.f;
      for (int c = c0; c <= c1; ++c)
        top = fmaxf(top, a.parts[((int64_t)(c == c0 ? first_slot : 2 * c) * rows_tile + col) * (D + 2) + D]);
#pragma unroll 4
      for (int c = c0; c <= c1; ++c) {
        const float* part = a.parts + ((int64_t)(c == c0 ? first_slot : 2 * c) * rows_tile + col) * (D + 2);
        const float f = exp2_approx(part[D] - top);
        const float2 o = *reinterpret_cast<const float2*>(part + d2);
        total += f * part[D + 1];
        x += f * o.x;
        y += f * o.y;
      }
      const int row = tile * rows_tile + col;
      const int64_t at = (int64_t)(s.begin + row / a.group) * a.q_heads + head * a.group + row % a.group;
      const float inv = total == 0.f ? 0.f : gv / total;
      uint32_t packed;
      if (BF16)
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(packed) : "f"(y * inv), "f"(x * inv));
      else
        packed = pack_half2(x * inv, y * inv);
      *reinterpret_cast<uint32_t*>(a.out + at * D + d2) = packed;
      if (a.lse && d2 == 0) a.lse[at] = total == 0.f ? -INFINITY : (top + log2f(total)) * 0.6931471805599453f;
    }
  }
}

template <int D, int NT, bool BF16>
cudaError_t launch_few(const Kv4Attend& a, int ctas, cudaStream_t stream) {
  using L = Layout<D, NT>;
  auto kernel = kv4_attend_kernel<D, NT, BF16>;
  static bool done[kAttrDevices];
  const cudaError_t e = once_per_device(done, [&] {
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, L::bytes());
  });
  if (e != cudaSuccess) return e;
  return launch_pdl(kernel, dim3(ctas), dim3(kThreads), L::bytes(), stream, a);
}

template <int D, bool BF16>
cudaError_t launch_few_rows(const Kv4Attend& a, int n_tiles, int ctas, cudaStream_t stream) {
  return n_tiles == 1 ? launch_few<D, 1, BF16>(a, ctas, stream)
                      : n_tiles == 2 ? launch_few<D, 2, BF16>(a, ctas, stream) : launch_few<D, 4, BF16>(a, ctas, stream);
}

// n tiles of 8 rows for the step's most rows: the fewest that hold them, up to four
int few_tiles(const Kv4Batch& b, int group) {
  const int64_t rows = (int64_t)b.max_count * group;
  return rows <= 8 ? 1 : rows <= 16 ? 2 : 4;
}
int few_ctas(int n_tiles, int sms) { return n_tiles == 1 ? 2 * sms : sms; }

}  // namespace

cudaError_t launch_kv4_join(const Kv4Attend& a, int rows, int unit, int ctas, int dtype, cudaStream_t stream) {
  const int64_t items = ((int64_t)a.b.max_count * a.group + rows - 1) / rows * a.c.H;
  const dim3 grid(a.b.n, (unsigned)(items < 1024 ? items : 1024));
  auto kernel = a.c.D == 128 ? (dtype == SEMKV_BF16 ? kv4_join_kernel<128, true> : kv4_join_kernel<128, false>)
                             : (dtype == SEMKV_BF16 ? kv4_join_kernel<64, true> : kv4_join_kernel<64, false>);
  return launch_pdl(kernel, grid, dim3(128), 0, stream, a, rows, unit, ctas);
}

static size_t prefix_bytes(int n) { return ((size_t)n + 1) * 8 + 15 & ~(size_t)15; }

size_t kv4_attention_workspace(const Kv4Cache& c, const Kv4Batch& b, int q_heads, int sms) {
  const int n = few_tiles(b, q_heads / c.H);
  return (size_t)2 * few_ctas(n, sms) * 8 * n * (c.D + 2) * 4 + prefix_bytes(b.n);
}

cudaError_t launch_kv4_attention(const Kv4Cache& c, const Kv4Batch& b, int layer, int dtype, const void* q, int64_t q_stride,
                                 int q_heads, void* out, float* lse, float softmax_scale, int window, void* ws, int sms,
                                 cudaStream_t stream) {
  Kv4Attend a;
  a.c = c;
  a.b = b;
  a.layer = layer;
  a.group = q_heads / c.H;
  a.q_heads = q_heads;
  a.window = window;
  a.q = static_cast<const uint16_t*>(q);
  a.q_stride = q_stride;
  a.out = static_cast<uint16_t*>(out);
  a.lse = lse;
  a.scale_log2 = softmax_scale * 1.4426950408889634f;
  a.prefix = static_cast<int64_t*>(ws);
  a.parts = reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + prefix_bytes(b.n));
  const int n = few_tiles(b, a.group), ctas = few_ctas(n, sms);
  const bool bf = dtype == SEMKV_BF16;
  const cudaError_t e =
      c.D == 128 ? (bf ? launch_few_rows<128, true>(a, n, ctas, stream) : launch_few_rows<128, false>(a, n, ctas, stream))
                 : (bf ? launch_few_rows<64, true>(a, n, ctas, stream) : launch_few_rows<64, false>(a, n, ctas, stream));
  if (e != cudaSuccess) return e;
  return launch_kv4_join(a, 8 * n, kUnit, ctas, dtype, stream);
}

}  // namespace semkv
