// kv4_attend.cuh — how a step's attention over the paged 4-bit cache is split over CTAs, shared
// by the kernels that do it and the one that joins their parts.
//
// An item is (sequence, KV head, tile of `rows` query rows); a query row is (token j, head
// g of the group) with index j * group + g.  An item's units are `unit` consecutive positions
// each, from the unit of the first position that any row of the sequence sees to its last.  The
// units of all items, in order, are cut into equal contiguous ranges, one per CTA, so ragged
// lengths balance by themselves; every CTA finds its range from the lengths on the device.
// A CTA walks its range item by item.  An item that lies in one CTA is finished there; of
// the others each CTA writes a part, of which a range has at most two: its first and its last.
#pragma once
#include "kv4.cuh"

namespace semkv {

struct Kv4Attend {
  Kv4Cache c;
  Kv4Batch b;
  int layer, group, q_heads, window;
  const uint16_t* q;
  int64_t q_stride;
  uint16_t* out;
  float* lse;
  float scale_log2;  // softmax scale * log2(e)
  float* parts;      // [2 * CTAs][rows][D + 2]: sums, then reference exponent and weight sum
  int64_t* prefix;   // [b.n + 1]: units before each sequence (written by CTA 0, for the join)
};

// One sequence's share of the plan.
struct Kv4Seq {
  int seq, begin, count, length;  // its rows of the step and its tokens
  int tiles;                      // tiles of query rows
  int u_first, units;             // units of each item: u_first .. u_first + units - 1
};

template <int ROWS, int UNIT>
__device__ __forceinline__ Kv4Seq kv4_seq(const Kv4Attend& a, int i, bool report) {
  Kv4Seq s;
  s.seq = a.b.seqs ? a.b.seqs[i] : i;
  s.tiles = s.units = s.u_first = s.length = 0;
  bool ok = kv4_range(a.b, i, s.begin, s.count);
  if (ok && (s.seq < 0 || s.seq >= a.c.max_seqs)) ok = false;
  if (!ok) {
    if (report) raise_error(a.c.err, kDevIndex);
    s.count = 0;
    return s;
  }
  const int64_t cap = (int64_t)a.c.max_pages << a.c.page_shift;
  const int t = a.c.length[s.seq];
  s.length = t < 0 ? 0 : t > cap ? (int)cap : t;
  if (report && t > cap) raise_error(a.c.err, kDevIndex);
  s.tiles = (s.count * a.group + ROWS - 1) / ROWS;
  if (s.count > 0 && s.length > 0) {
    // the first row's first position
    const int64_t lo = a.window ? (int64_t)s.length - s.count + 1 - a.window : 0;
    s.u_first = lo > 0 ? (int)(lo / UNIT) : 0;
    s.units = (s.length + UNIT - 1) / UNIT - s.u_first;
  }
  return s;
}

// The plan: thread x of the block counts the units of sequences x * per .. (x + 1) * per - 1, with
// per = ceil(n / THREADS); prefix[x] = the units before them, prefix[THREADS] = all.
template <int ROWS, int UNIT, int THREADS>
__device__ __forceinline__ void kv4_plan(const Kv4Attend& a, int64_t* prefix, int64_t* sums, bool first_cta) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int per = (a.b.n + THREADS - 1) / THREADS;
  const int i0 = threadIdx.x * per, i1 = min(a.b.n, i0 + per);
  int64_t sum = 0;
  for (int i = i0; i < i1; ++i) {
    const Kv4Seq s = kv4_seq<ROWS, UNIT>(a, i, first_cta);
    sum += (int64_t)s.units * s.tiles * a.c.H;
  }
  int64_t y = sum;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int64_t o = __shfl_up_sync(~0u, y, d);
    if (lane >= d) y += o;
  }
  if (lane == 31) sums[warp] = y;
  __syncthreads();
  int64_t at = y - sum;
  for (int w = 0; w < warp; ++w) at += sums[w];
  prefix[threadIdx.x] = at;
  if (threadIdx.x == THREADS - 1) prefix[THREADS] = at + sum;
  if (first_cta) {
    for (int i = i0; i < i1; ++i) {
      a.prefix[i] = at;
      const Kv4Seq s = kv4_seq<ROWS, UNIT>(a, i, false);
      at += (int64_t)s.units * s.tiles * a.c.H;
    }
    if (threadIdx.x == THREADS - 1) a.prefix[a.b.n] = at;
  }
  __syncthreads();
}

// The sequence that holds unit `cur` (below prefix[THREADS]); `at`: the units before it.
template <int ROWS, int UNIT, int THREADS>
__device__ __forceinline__ Kv4Seq kv4_find(const Kv4Attend& a, const int64_t* prefix, int64_t cur, int64_t& at) {
  int lo = 0, hi = THREADS - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (prefix[mid] <= cur) lo = mid; else hi = mid - 1;
  }
  const int per = (a.b.n + THREADS - 1) / THREADS;
  at = prefix[lo];
  Kv4Seq s = kv4_seq<ROWS, UNIT>(a, lo * per, false);
  for (int k = 1; k < per; ++k) {
    const int64_t units = (int64_t)s.units * s.tiles * a.c.H;
    if (cur < at + units || lo * per + k >= a.b.n) break;
    at += units;
    s = kv4_seq<ROWS, UNIT>(a, lo * per + k, false);
  }
  return s;
}

// CTA c's range of W units on `ctas` CTAs (no more than W) begins at W c / ctas.
__device__ __forceinline__ int64_t kv4_range_begin(int64_t W, int c, int ctas) { return W * c / ctas; }
// the CTA whose range holds unit u
__device__ __forceinline__ int kv4_owner(int64_t W, int64_t u, int ctas) {
  return (int)(((u + 1) * ctas - 1) / W);
}
__device__ __forceinline__ int kv4_ctas(int64_t W, int ctas) { return W < ctas ? (int)W : ctas; }

// Which positions a query row sees: [lo, hi]; hi < 0 for a row that is not there.
template <typename S>
__device__ __forceinline__ void kv4_sight(const Kv4Attend& a, const S& s, int row, int& lo, int& hi) {
  const int j = row / a.group;
  hi = j < s.count ? s.length - s.count + j : -1;
  lo = a.window && hi >= a.window ? hi - a.window + 1 : 0;
}

__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

cudaError_t launch_kv4_join(const Kv4Attend& a, int rows, int unit, int ctas, int dtype, cudaStream_t stream);

}  // namespace semkv
