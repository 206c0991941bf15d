// kv4_attend.cu — attention over the paged 4-bit cache for few query rows (single tokens,
// drafted tokens), bound by reading the cache and by turning it into operands: 16 sequences of 64K
// with 8 KV heads in groups of 4 take 215 us, 83% of the copy rate, at 52% of the issue slots (337
// instructions for a tile of 16 tokens) and 19% of the tensor pipe.
//
// For a tile of 16 tokens, on mma.sync m16n8k16 with fp16 operands and fp32 sums:
//   S^T = K Q^T      M = 16 tokens, N = 8 query rows, K = head dim
//   P   = 2^(S - e)  e: the row's reference exponent, moved only when a weight would pass 2^15
//                    (far logits: kFar)
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
// Every warp is a worker of its own (kv4_attend.cuh): it streams its range, 32 tokens at a time,
// through a ring of bulk copies and meets no other warp.
#include "kernels.h"
#include "kv4_attend.cuh"

namespace semkv {
namespace {

constexpr int kUnit = 32;       // tokens of a unit
constexpr int kWarps = 8;
constexpr int kThreads = kWarps * 32;

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
  static constexpr int ring_bytes() { return kWarps * kStages * kStage; }
  // Q's fragments lie in registers where there are eight rows, else in shared memory
  static constexpr int q_bytes() { return NT == 1 ? 0 : kWarps * NT * (D / 16) * 32 * 8; }
  static constexpr int bytes() { return ring_bytes() + q_bytes() + kWarps * kStages * 8 + (kThreads + 1) * 8 + kWarps * 8; }
};

// An item's start counts for two units (with one, ragged batches end 15% later; with three or four it is the
// same); a range has four at least (fewer cost the join what they save).
__host__ __device__ constexpr Kv4FewCut few_cut(int n_tiles) { return Kv4FewCut{8 * n_tiles, kUnit, 2, 4}; }

// The fragments of eight query rows (row0 + g) for one KV head, w[2k], w[2k + 1] those of k step k.
template <int D>
__device__ __forceinline__ void load_queries(const Kv4Attend& a, const Kv4Seq& s, int head, int row0, uint32_t (&w)[D / 8]) {
  const int lane = threadIdx.x & 31;
  const int g = lane >> 2, t = lane & 3;
  const int row = row0 + g;
  const int j = row / a.group, h = head * a.group + row % a.group;
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
}
// bf16 rows as fp16, times their factor; returns what undoes it.
template <int D, bool BF16>
__device__ __forceinline__ float turn_queries(uint32_t (&w)[D / 8]) {
  float undo = 1.f;
  if (BF16) {
    float most = 0.f;
#pragma unroll
    for (int k = 0; k < D / 8; ++k) {
      most = fmaxf(most, fabsf(__uint_as_float(w[k] << 16)));
      most = fmaxf(most, fabsf(__uint_as_float(w[k] & 0xFFFF0000u)));
    }
    most = fmaxf(most, __shfl_xor_sync(~0u, most, 1));
    most = fmaxf(most, __shfl_xor_sync(~0u, most, 2));
    const float mul = query_factor(most, undo);
#pragma unroll
    for (int k = 0; k < D / 8; ++k)
      w[k] = pack_half2(__uint_as_float(w[k] << 16) * mul, __uint_as_float(w[k] & 0xFFFF0000u) * mul);
  }
  return undo;
}

// Rows of sequences without tokens, and their items' spans.
template <int D>
__device__ __forceinline__ void fill_empty(const Kv4Attend& a, Kv4FewCut cut) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (int i0 = warp * 32; i0 < a.b.n; i0 += kThreads) {
    const Kv4Seq mine = i0 + lane < a.b.n ? cut.seq(a, i0 + lane, false) : Kv4Seq{};
    // (a sequence that is left out has count 0)
    for (uint32_t m = __ballot_sync(~0u, mine.count > 0 && mine.units == 0); m; m &= m - 1) {
      const int x = __ffs(m) - 1, count = __shfl_sync(~0u, mine.count, x), tiles = __shfl_sync(~0u, mine.tiles, x);
      const int64_t row0 = (int64_t)__shfl_sync(~0u, mine.begin, x) * a.q_heads;
      for (int64_t y = lane; y < (int64_t)count * a.q_heads * (D / 8); y += 32)
        reinterpret_cast<uint4*>(a.out + row0 * D)[y] = make_uint4(0, 0, 0, 0);
      for (int64_t y = lane; a.lse && y < (int64_t)count * a.q_heads; y += 32) a.lse[row0 + y] = -INFINITY;
      for (int y = lane; y < a.c.H * tiles; y += 32)
        a.spans[((int64_t)(i0 + x) * a.c.H + y / tiles) * a.tiles + y % tiles].x = -1;
    }
  }
}

template <int D, int NT, bool BF16>
__global__ void __launch_bounds__(kThreads, NT == 1 ? 2 : 1) kv4_attend_kernel(Kv4Attend a) {
  using L = Layout<D, NT>;
  constexpr Kv4FewCut cut = few_cut(NT);
  constexpr int kSteps = D / 16;   // k steps of S
  constexpr int kM = D / 16;       // m tiles of O
  extern __shared__ __align__(128) uint8_t smem[];
  int64_t* prefix = reinterpret_cast<int64_t*>(smem + L::ring_bytes() + L::q_bytes());
  int64_t* sums = prefix + kThreads + 1;
  uint64_t* bars = reinterpret_cast<uint64_t*>(sums + kWarps);

  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int g = lane >> 2, t = lane & 3;
  uint8_t* ring = smem + warp * (L::kStages * L::kStage);
  uint2* qf = reinterpret_cast<uint2*>(smem + L::ring_bytes()) + warp * (NT * kSteps * 32);
  uint64_t* bar = bars + warp * L::kStages;
  if (lane == 0) {
    for (int s = 0; s < L::kStages; ++s)
      asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(smem_addr(bar + s)) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  pdl_wait();
  pdl_trigger();
  kv4_plan<kThreads, false>(a, cut, prefix, sums, blockIdx.x == 0);
  if (blockIdx.x == 0) fill_empty<D>(a, cut);
  const int64_t W = prefix[kThreads];
  const Kv4Ranges ranges(W, cut.least, gridDim.x * kWarps);
  const int worker = warp * gridDim.x + blockIdx.x;  // few workers: spread over the SMs
  if (W == 0 || worker >= ranges.count) return;
  const int64_t end = ranges.begin(worker + 1);

  const int row_a = token_at(g), tok_v = token_at(2 * t);  // K row of lane group g; V's first token
  const int64_t head_bytes = (int64_t)L::kTile << (a.c.page_shift - 4);
  const int64_t page_stride = head_bytes * a.c.H;
  uint32_t phase = 0;  // parity of each stage's barrier, a bit each; kFarBit: a reference of the item is far (kFar)
  constexpr uint32_t kFarBit = 0x80000000u;  // (a variable of its own made the eight-row kernel spill)
  int stage = 0;       // of the next unit

  for (int64_t place = ranges.begin(worker); place < end;) {
    int64_t before;
    int which;
    const Kv4Seq s = kv4_find<kThreads>(a, cut, prefix, place, before, which);
    const int per = s.units + cut.start;
    const int64_t in_seq = place - before;
    const int item = (int)kv4_div(in_seq, per), off = (int)(in_seq - (int64_t)item * per);
    const int take = (int)min((int64_t)(per - off), end - place);
    place += take;
    const int u0 = max(0, off - cut.start), u1 = off + take - cut.start;
    if (u1 <= u0) continue;
    const int head = s.tiles == 1 ? item : item / s.tiles, tile = item - head * s.tiles;

    // the pages of units u0 + k0 .. u0 + k0 + 31, a lane each (with pages of 16 tokens: of both halves)
    const int mine = u1 - u0, token0 = (s.u_first + u0) * kUnit;
    const uint8_t* head_base = a.c.pages + kv4_record(a.c, a.layer, 0, head);
    const int32_t* table = a.c.table + (int64_t)s.seq * a.c.max_pages;
    int page_x = 0, page_y = 0, k0 = 0;
    auto fetch_pages = [&](int k) {
      k0 = k;
      const int kk = k + lane;
      if (kk < mine) {
        const int token = token0 + kk * kUnit;
        page_x = table[token >> a.c.page_shift];
        page_y = a.c.page_shift == 4 && token + 16 < s.length ? table[(token >> 4) + 1] : 0;
        if ((unsigned)page_x >= (unsigned)a.c.num_pages || (unsigned)page_y >= (unsigned)a.c.num_pages) {
          raise_error(a.c.err, kDevIndex);
          if ((unsigned)page_x >= (unsigned)a.c.num_pages) page_x = 0;
          if ((unsigned)page_y >= (unsigned)a.c.num_pages) page_y = 0;
        }
      }
    };
    auto issue = [&](int k, int to) {
      if (k >= k0 + 32) fetch_pages(k);
      const int px = __shfl_sync(~0u, page_x, k - k0), py = __shfl_sync(~0u, page_y, k - k0);
      if (lane == 0) {
        const int token = token0 + k * kUnit;
        const bool two = token + 16 < s.length;
        const uint32_t dst = smem_addr(ring + to * L::kStage), b = smem_addr(bar + to);
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

    // ---- the (first) queries on their way before the copies, which they would queue behind
    uint32_t q1[D / 8];
    load_queries<D>(a, s, head, tile * L::kRows, q1);
    fetch_pages(0);
    {
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // (the item before has read its stages)
      const int ahead = min(mine, L::kStages);
      int to = stage;
      for (int k = 0; k < ahead; ++k) {
        issue(k, to);
        to = to + 1 == L::kStages ? 0 : to + 1;
      }
    }

    float undo[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      if (n > 0) load_queries<D>(a, s, head, tile * L::kRows + 8 * n, q1);
      undo[n] = turn_queries<D, BF16>(q1);
      if (NT > 1) {
#pragma unroll
        for (int k = 0; k < kSteps; ++k) qf[(n * kSteps + k) * 32 + lane] = make_uint2(q1[2 * k], q1[2 * k + 1]);
      }
    }

    // what this lane's query rows (columns 2t, 2t+1 of each n tile) see
    int see_lo[2 * NT], see_hi[2 * NT];
    float mul[2 * NT];
    int most_lo = 0, least_hi = 0x7FFFFFFF;
    const float gk = a.c.k_scale ? a.c.k_scale[a.layer * a.c.H + head] : 1.f;
#pragma unroll
    for (int x = 0; x < 2 * NT; ++x) {
      const int row = tile * L::kRows + (x >> 1) * 8 + 2 * t + (x & 1);
      kv4_sight(a, s, row, see_lo[x], see_hi[x]);
      mul[x] = a.scale_log2 * gk * __shfl_sync(~0u, undo[x >> 1], 4 * (2 * t + (x & 1)));
      if (row / a.group < s.count) {
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
    phase &= ~kFarBit;
    __syncwarp();  // Q's fragments are there

    // S^T += K Q^T of a tile
    auto scores = [&](const uint8_t* tl, float(&S)[NT][4]) {
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
          const uint2 b0 = NT == 1 ? make_uint2(q1[4 * w], q1[4 * w + 1]) : qf[(n * kSteps + 2 * w) * 32 + lane];
          const uint2 b1 = NT == 1 ? make_uint2(q1[4 * w + 2], q1[4 * w + 3]) : qf[(n * kSteps + 2 * w + 1) * 32 + lane];
          mma16816(S[n], xa[0], xb[0], xa[1], xb[1], b0.x, b0.y);
          mma16816(S[n], xa[2], xb[2], xa[3], xb[3], b1.x, b1.y);
        }
      }
    };
    // O^T += V^T P^T of a tile with `left` tokens: a = tok_v and a ^ 3 (places 2t, 2t+1), and both + 8
    auto values = [&](const uint8_t* tl, int left, const uint32_t(&pb)[NT][2]) {
      const int ta = tok_v, tb = tok_v ^ 3;
      const uint8_t* pv = tl + 8 * D + g * (D / 16);
      const uint8_t* ps = tl + 17 * D + (D == 128 ? g : g >> 1);
      uint32_t s01 = (uint32_t)ps[ta * (D / 16)] | (uint32_t)ps[tb * (D / 16)] << 8;
      uint32_t s23 = (uint32_t)ps[(ta + 8) * (D / 16)] | (uint32_t)ps[(tb + 8) * (D / 16)] << 8;
      if (left < 16) {
        // rows behind the last token hold anything: their scale is 0
        if (ta >= left) s01 &= 0xFF00u;
        if (tb >= left) s01 &= 0x00FFu;
        if (ta + 8 >= left) s23 &= 0xFF00u;
        if (tb + 8 >= left) s23 &= 0x00FFu;
      }
      const uint32_t h01 = e4m3x2_to_half2(s01), h23 = e4m3x2_to_half2(s23);
      uint32_t va[D / 64], vb[D / 64], vc[D / 64], vd[D / 64];
      if constexpr (D == 128) {
        const uint2 xa = *reinterpret_cast<const uint2*>(pv + ta * (D / 2)), xb = *reinterpret_cast<const uint2*>(pv + tb * (D / 2));
        const uint2 xc = *reinterpret_cast<const uint2*>(pv + (ta + 8) * (D / 2)), xd = *reinterpret_cast<const uint2*>(pv + (tb + 8) * (D / 2));
        va[0] = xa.x, va[1] = xa.y, vb[0] = xb.x, vb[1] = xb.y;
        vc[0] = xc.x, vc[1] = xc.y, vd[0] = xd.x, vd[1] = xd.y;
      } else {
        va[0] = *reinterpret_cast<const uint32_t*>(pv + ta * (D / 2));
        vb[0] = *reinterpret_cast<const uint32_t*>(pv + tb * (D / 2));
        vc[0] = *reinterpret_cast<const uint32_t*>(pv + (ta + 8) * (D / 2));
        vd[0] = *reinterpret_cast<const uint32_t*>(pv + (tb + 8) * (D / 2));
      }
#pragma unroll
      for (int w = 0; w < D / 64; ++w) {
        uint32_t e01[4], o01[4], e23[4], o23[4];  // even and odd dims of the byte, token pairs
        e2m1x8_to_half2((va[w] & 0x0F0F0F0Fu) | ((vb[w] << 4) & 0xF0F0F0F0u), e01);
        e2m1x8_to_half2(((va[w] >> 4) & 0x0F0F0F0Fu) | (vb[w] & 0xF0F0F0F0u), o01);
        e2m1x8_to_half2((vc[w] & 0x0F0F0F0Fu) | ((vd[w] << 4) & 0xF0F0F0F0u), e23);
        e2m1x8_to_half2(((vc[w] >> 4) & 0x0F0F0F0Fu) | (vd[w] & 0xF0F0F0F0u), o23);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t a0 = hmul2_bits(e01[i], h01), a1 = hmul2_bits(o01[i], h01);
          const uint32_t a2 = hmul2_bits(e23[i], h23), a3 = hmul2_bits(o23[i], h23);
#pragma unroll
          for (int n = 0; n < NT; ++n) mma16816(O[n][4 * w + i], a0, a1, a2, a3, pb[n][0], pb[n][1]);
        }
      }
    };

    for (int k = 0; k < mine; ++k) {
      if (!__all_sync(~0u, mbar_wait_bounded(bar + stage, phase >> stage & 1))) {
        if (lane == 0) raise_error(a.c.err, kDevWaitTimeout);
        // the copies still in flight are waited for, as long again
        for (int j = k + 1; j < min(mine, k + L::kStages); ++j) {
          stage = stage + 1 == L::kStages ? 0 : stage + 1;
          mbar_wait_bounded(bar + stage, phase >> stage & 1);
        }
        return;
      }
      phase ^= 1u << stage;
      const int token = token0 + k * kUnit;
      // a unit's two tiles together (up to 16 rows: registers), so that their products and conversions overlap
      // and one vote serves both; what lies behind the last token is masked, whatever the stage holds there
      constexpr int kTogether = NT * D <= 256 ? 2 : 1;
#pragma unroll 1
      for (int half = 0; half < 2; half += kTogether) {
        const int t0 = token + 16 * half;
        if (t0 >= s.length) break;
        const uint8_t* tl = ring + stage * L::kStage + half * L::kTile;
        float S[kTogether][NT][4];
#pragma unroll
        for (int h = 0; h < kTogether; ++h) {
#pragma unroll
          for (int n = 0; n < NT; ++n) S[h][n][0] = S[h][n][1] = S[h][n][2] = S[h][n][3] = 0.f;
          scores(tl + h * L::kTile, S[h]);
        }
        // ---- weights: exponents S mul - ref, two rows of a lane at a time
        const bool open = t0 >= most_lo && t0 + 16 * kTogether - 1 <= least_hi;  // every row sees all of it
        float E[kTogether][NT][4];
        float top = -INFINITY;
        auto exponents = [&](bool rounded) {
#pragma unroll
          for (int h = 0; h < kTogether; ++h) {
            const int pos_a = t0 + 16 * h + row_a, pos_b = pos_a + 8;
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              const uint64_t m2 = pair(mul[2 * n], mul[2 * n + 1]), r2 = pair(-ref[2 * n], -ref[2 * n + 1]);
              float(&e)[4] = E[h][n];
              if (rounded) {  // (scalar: of a packed product and a packed sum one fused operation was made)
#pragma unroll
                for (int x = 0; x < 4; ++x) e[x] = __fsub_rn(__fmul_rn(S[h][n][x], mul[2 * n + (x & 1)]), ref[2 * n + (x & 1)]);
              } else {
                unpair(pair_fma(pair(S[h][n][0], S[h][n][1]), m2, r2), e[0], e[1]);
                unpair(pair_fma(pair(S[h][n][2], S[h][n][3]), m2, r2), e[2], e[3]);
              }
              if (!open) {
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                  if (pos_a < see_lo[2 * n + x] || pos_a > see_hi[2 * n + x]) e[x] = -INFINITY;
                  if (pos_b < see_lo[2 * n + x] || pos_b > see_hi[2 * n + x]) e[2 + x] = -INFINITY;
                }
              }
              asm("max.f32 %0, %0, %1, %2;" : "+f"(top) : "f"(e[0]), "f"(e[1]));
              asm("max.f32 %0, %0, %1, %2;" : "+f"(top) : "f"(e[2]), "f"(e[3]));
            }
          }
        };
        exponents(false);
        if (__any_sync(~0u, top > kMost || (phase & kFarBit))) {
          // references move to 2^8 below their rows' largest, and the sums with them
          bool far = false;
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              const int i = 2 * n + x;
              // (a first reference is so far from the logits that E says nothing of them)
              float l = -INFINITY;
#pragma unroll
              for (int h = 0; h < kTogether; ++h) {
                if (E[h][n][x] > -INFINITY) l = fmaxf(l, S[h][n][x] * mul[i]);
                if (E[h][n][2 + x] > -INFINITY) l = fmaxf(l, S[h][n][2 + x] * mul[i]);
              }
              l = fmaxf(l, __shfl_xor_sync(~0u, l, 4));
              l = fmaxf(l, __shfl_xor_sync(~0u, l, 8));
              l = fmaxf(l, __shfl_xor_sync(~0u, l, 16));
              if (l - ref[i] > kMost) {
                const float to = reference_for(l), f = exp2_approx(ref[i] - to);
                ref[i] = to;
                sum[i] *= f;
#pragma unroll
                for (int m = 0; m < kM; ++m) {
                  O[n][m][x] *= f;
                  O[n][m][2 + x] *= f;
                }
              }
              far = far || is_far(ref[i]);
            }
          far = __any_sync(~0u, far);
          phase = far ? phase | kFarBit : phase & ~kFarBit;
          exponents(far);
        }
#pragma unroll
        for (int h = 0; h < kTogether; ++h) {
          uint32_t pb[NT][2];
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            float(&e)[4] = E[h][n];
#pragma unroll
            for (int x = 0; x < 4; ++x) e[x] = exp2_approx(e[x]);
            unpair(pair_add(pair(sum[2 * n], sum[2 * n + 1]), pair_add(pair(e[0], e[1]), pair(e[2], e[3]))), sum[2 * n], sum[2 * n + 1]);
            pb[n][0] = transpose8x8(pack_half2(e[0], e[1]));
            pb[n][1] = transpose8x8(pack_half2(e[2], e[3]));
          }
          values(tl + h * L::kTile, s.length - t0 - 16 * h, pb);
        }
      }
      __syncwarp();
      if (k + L::kStages < mine) {
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        issue(k + L::kStages, stage);
      }
      stage = stage + 1 == L::kStages ? 0 : stage + 1;
    }

    // ---- the item's rows, or this range's part of them: lane g holds dims g D/8 .. of columns 2t, 2t+1
#pragma unroll
    for (int x = 0; x < 2 * NT; ++x) {
      sum[x] += __shfl_xor_sync(~0u, sum[x], 4);
      sum[x] += __shfl_xor_sync(~0u, sum[x], 8);
      sum[x] += __shfl_xor_sync(~0u, sum[x], 16);
    }
    const bool done = u0 == 0 && u1 == s.units;
    const int rows = min(L::kRows, s.count * a.group - tile * L::kRows);
    const float gv = a.c.v_scale ? a.c.v_scale[a.layer * a.c.H + head] : 1.f;
    if (lane == 0) {
      int2* span = a.spans + ((int64_t)which * a.c.H + head) * a.tiles + tile;
      if (u0 == 0) span->x = done ? -1 : worker;
      else if (u1 == s.units) span->y = worker;
    }
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int col = n * 8 + 2 * t + x;
        if (col >= rows) continue;
        const float total = sum[2 * n + x];
        if (done) {
          const int row = tile * L::kRows + col;
          const int64_t at = (int64_t)(s.begin + row / a.group) * a.q_heads + head * a.group + row % a.group;
          const float inv = total == 0.f ? 0.f : gv / total;
          uint32_t w[kM];
#pragma unroll
          for (int m = 0; m < kM; ++m) w[m] = pack_out<BF16>(O[n][m][x] * inv, O[n][m][2 + x] * inv);
          uint4* to = reinterpret_cast<uint4*>(a.out + at * D + g * (D / 8));
#pragma unroll
          for (int m = 0; m < kM; m += 4) to[m / 4] = make_uint4(w[m], w[m + 1], w[m + 2], w[m + 3]);
          if (a.lse && g == 0) a.lse[at] = total == 0.f ? -INFINITY : (ref[2 * n + x] + log2f(total)) * 0.6931471805599453f;
        } else {
          float* part = a.parts + ((int64_t)(2 * worker + (u0 == 0 ? 1 : 0)) * L::kRows + col) * kv4_part_floats(D);
          float4* to = reinterpret_cast<float4*>(part + g * (D / 8));
#pragma unroll
          for (int m = 0; m < kM; m += 2)
            to[m / 2] = make_float4(O[n][m][x], O[n][m][2 + x], O[n][m + 1][x], O[n][m + 1][2 + x]);
          if (g == 0) *reinterpret_cast<float2*>(part + D) = make_float2(ref[2 * n + x], total);
        }
      }
  }
}

// Joins the parts of the items that several workers share: a CTA for each query row, whose warps take
// the parts in turn: eight where the CTAs of all rows are then resident at once, else four (the long
// sequences of a ragged batch have fifty parts).  One session at 4K takes 16.1, 13.6, 11.8 us in all with
// 2, 4, 8 warps, 61 ragged sequences 42.0, 39.8, 41.0.
template <int D, bool BF16, int kJoinWarps>
__global__ void __launch_bounds__(kJoinWarps * 32) kv4_join_kernel(Kv4Attend a, int rows_tile, int workers) {
  __shared__ float acc[kJoinWarps][D];
  __shared__ float2 sums[kJoinWarps];  // reference exponent, weight sum
  pdl_wait();
  pdl_trigger();
  const int i = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  constexpr int kDims = D / 32;
  // y: row of the sequence (token j, query head), head by head of the cache, as if it had the most tokens,
  // so that the loads below do not wait for one another
  const int most_rows = a.b.max_count * a.group;
  for (int64_t y = blockIdx.y; y < (int64_t)most_rows * a.c.H; y += gridDim.y) {
    const int head = (int)kv4_div(y, most_rows), row = (int)(y - (int64_t)head * most_rows);
    const int tile = row / rows_tile, col = row - tile * rows_tile;
    const int2 span = a.spans[((int64_t)i * a.c.H + head) * a.tiles + tile];
    const int seq = a.b.seqs ? a.b.seqs[i] : i;
    const float gv = a.c.v_scale ? a.c.v_scale[a.layer * a.c.H + head] : 1.f;
    int begin, count;
    const bool ok = kv4_range(a.b, i, begin, count) && seq >= 0 && seq < a.c.max_seqs;
    // (a row that is not there, or that was finished where it ran; a worker whose wait ran out left no span)
    if (!ok || row >= count * a.group || span.x < 0 || span.x > span.y || span.y >= workers) continue;
    const int parts = span.y - span.x + 1;
    const int64_t size = (int64_t)rows_tile * kv4_part_floats(D);
    // the first part begins the item (slot 2 w + 1), the others continue it (slot 2 w)
    const float* base = a.parts + 2 * span.x * size + col * kv4_part_floats(D) + kDims * lane;
    float ref = kNone, total = 0.f, o[kDims] = {};
#pragma unroll 4
    for (int p = warp; p < parts; p += kJoinWarps) {
      const float* part = base + (2 * p + (p == 0)) * size;
      const float2 rs = *reinterpret_cast<const float2*>(part + D - kDims * lane);
      float x[kDims];
      if constexpr (kDims == 4) {
        const float4 v = *reinterpret_cast<const float4*>(part);
        x[0] = v.x, x[1] = v.y, x[2] = v.z, x[3] = v.w;
      } else {
        const float2 v = *reinterpret_cast<const float2*>(part);
        x[0] = v.x, x[1] = v.y;
      }
      const float to = fmaxf(ref, rs.x), f = exp2_approx(ref - to), g = exp2_approx(rs.x - to);
      ref = to;
      total = total * f + rs.y * g;
#pragma unroll
      for (int d = 0; d < kDims; ++d) o[d] = o[d] * f + x[d] * g;
    }
    __syncthreads();  // the row before is done with the shared sums
#pragma unroll
    for (int d = 0; d < kDims; ++d) acc[warp][kDims * lane + d] = o[d];
    if (lane == 0) sums[warp] = make_float2(ref, total);
    __syncthreads();
    if (warp > 0) continue;
#pragma unroll
    for (int w = 1; w < kJoinWarps; ++w) {
      const float to = fmaxf(ref, sums[w].x), f = exp2_approx(ref - to), g = exp2_approx(sums[w].x - to);
      ref = to;
      total = total * f + sums[w].y * g;
#pragma unroll
      for (int d = 0; d < kDims; ++d) o[d] = o[d] * f + acc[w][kDims * lane + d] * g;
    }
    const int64_t at = (int64_t)(begin + row / a.group) * a.q_heads + head * a.group + row % a.group;
    const float inv = total == 0.f ? 0.f : gv / total;
    uint32_t* to = reinterpret_cast<uint32_t*>(a.out + at * D) + kDims / 2 * lane;
#pragma unroll
    for (int d = 0; d < kDims / 2; ++d) to[d] = pack_out<BF16>(o[2 * d] * inv, o[2 * d + 1] * inv);
    if (a.lse && lane == 0) a.lse[at] = total == 0.f ? -INFINITY : (ref + log2f(total)) * 0.6931471805599453f;
  }
}

template <bool BF16, int WARPS>
cudaError_t launch_join_of(const Kv4Attend& a, int rows_tile, int workers, cudaStream_t stream) {
  const int64_t rows = (int64_t)a.b.max_count * a.q_heads;
  auto kernel = a.c.D == 128 ? kv4_join_kernel<128, BF16, WARPS> : kv4_join_kernel<64, BF16, WARPS>;
  return launch_pdl(kernel, dim3(a.b.n, (unsigned)(rows < 4096 ? rows : 4096)), dim3(WARPS * 32), 0, stream, a, rows_tile,
                    workers);
}
template <bool BF16>
cudaError_t launch_join(const Kv4Attend& a, int rows_tile, int workers, int64_t warps, cudaStream_t stream) {
  return warps >= 8 ? launch_join_of<BF16, 8>(a, rows_tile, workers, stream)
                    : launch_join_of<BF16, 4>(a, rows_tile, workers, stream);
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
  switch (n_tiles) {
    case 1: return launch_few<D, 1, BF16>(a, ctas, stream);
    case 2: return launch_few<D, 2, BF16>(a, ctas, stream);
    case 3: return launch_few<D, 3, BF16>(a, ctas, stream);
    default: return launch_few<D, 4, BF16>(a, ctas, stream);
  }
}

// n tiles of 8 rows for the step's most rows: the fewest that hold them, up to what the registers hold
// (O takes D / 4 of them for each)
int few_tiles(const Kv4Batch& b, int group) {
  const int64_t rows = (int64_t)b.max_count * group;
  return rows <= 8 ? 1 : rows <= 16 ? 2 : rows <= 24 ? 3 : 4;
}
int few_ctas(int n_tiles, int sms) { return n_tiles == 1 ? 2 * sms : sms; }

}  // namespace

// Workspace: the parts, behind the lengths before each sequence and the joins (many rows) or the items' spans (few).
static int few_items(const Kv4Batch& b, int group, int n_tiles) {
  return (int)(((int64_t)b.max_count * group + 8 * n_tiles - 1) / (8 * n_tiles));
}
static size_t front_bytes(const Kv4Cache& c, const Kv4Batch& b, int group, int sms) {
  if (kv4_many(b, group)) return kv4_many_front_bytes(b, sms);
  const size_t spans = (size_t)b.n * c.H * few_items(b, group, few_tiles(b, group));
  return (spans * 8 + 15) & ~(size_t)15;
}

size_t kv4_attention_workspace(const Kv4Cache& c, const Kv4Batch& b, int q_heads, int sms) {
  const int group = q_heads / c.H, n = few_tiles(b, group);
  const size_t floats = kv4_many(b, group) ? kv4_many_part_floats(c.D, sms)
                                           : (size_t)2 * few_ctas(n, sms) * kWarps * 8 * n * kv4_part_floats(c.D);
  return floats * 4 + front_bytes(c, b, group, sms);
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
  a.spans = static_cast<int2*>(ws);
  a.parts = reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + front_bytes(c, b, a.group, sms));
  a.joins = reinterpret_cast<int4*>(a.parts) - sms;
  if (kv4_many(b, a.group)) return launch_kv4_many(a, dtype, sms, stream);
  const int n = few_tiles(b, a.group), ctas = few_ctas(n, sms);
  a.tiles = few_items(b, a.group, n);
  const bool bf = dtype == SEMKV_BF16;
  const cudaError_t e =
      c.D == 128 ? (bf ? launch_few_rows<128, true>(a, n, ctas, stream) : launch_few_rows<128, false>(a, n, ctas, stream))
                 : (bf ? launch_few_rows<64, true>(a, n, ctas, stream) : launch_few_rows<64, false>(a, n, ctas, stream));
  if (e != cudaSuccess) return e;
  const int64_t rows = (int64_t)b.max_count * q_heads, warps = (int64_t)80 * sms / (rows * b.n);
  return bf ? launch_join<true>(a, 8 * n, ctas * kWarps, warps, stream)
            : launch_join<false>(a, 8 * n, ctas * kWarps, warps, stream);
}

}  // namespace semkv
