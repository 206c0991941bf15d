// kv4_attend.cuh — how a step's attention over the paged 4-bit cache is split over workers, shared
// by the kernels that do it and the one that joins their parts.
//
// An item is (sequence, KV head, tile of query rows); a query row is (token j, head g of the
// group) with index j * group + g.  An item's units are `unit` consecutive positions each, from
// the unit of the first position that any row of the sequence sees to its last.  Each item also
// counts as a few units of its own before them, the time that starting one costs.  These
// lengths, item after item, are cut into equal contiguous ranges, one for each worker (a warp or
// a CTA), so ragged lengths balance by themselves; every worker finds its range from the lengths
// on the device.  An item that lies in one worker's range is finished there; of the others each
// worker writes a part: one that begins its item and does not end it (its range's last) or one that
// continues an item (its range's first), so two slots for each worker hold them.
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
  float* parts;      // [2 * workers][rows][D + 4]: sums, then reference exponent and weight sum
  int64_t* prefix;   // [b.n + 1]: length before each sequence (written by CTA 0, for the join)
};

// How a kernel's items are cut: rows of a tile, positions of a unit, units that an item's start
// counts for, and the least length of a range.
struct Kv4Cut {
  int rows, unit, start, least;
};

__host__ __device__ constexpr int kv4_part_floats(int D) { return D + 4; }

// One sequence's share of the plan.
struct Kv4Seq {
  int seq, begin, count, length;  // its rows of the step and its tokens
  int tiles;                      // tiles of query rows
  int u_first, units;             // units of each item: u_first .. u_first + units - 1
};

__device__ __forceinline__ Kv4Seq kv4_seq(const Kv4Attend& a, Kv4Cut cut, int i, bool report) {
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
  s.tiles = (s.count * a.group + cut.rows - 1) / cut.rows;
  if (s.count > 0 && s.length > 0) {
    // the first row's first position
    const int64_t lo = a.window ? (int64_t)s.length - s.count + 1 - a.window : 0;
    s.u_first = lo > 0 ? (int)(lo / cut.unit) : 0;
    s.units = (s.length + cut.unit - 1) / cut.unit - s.u_first;
  }
  return s;
}
__device__ __forceinline__ int64_t kv4_weight(const Kv4Attend& a, Kv4Cut cut, const Kv4Seq& s) {
  return s.units ? (int64_t)(s.units + cut.start) * s.tiles * a.c.H : 0;
}

// The plan: thread x of the block adds up sequences x * per .. (x + 1) * per - 1, with
// per = ceil(n / THREADS); prefix[x] = the length before them, prefix[THREADS] = all.
template <int THREADS>
__device__ __forceinline__ void kv4_plan(const Kv4Attend& a, Kv4Cut cut, int64_t* prefix, int64_t* sums,
                                         bool first_cta) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int per = (a.b.n + THREADS - 1) / THREADS;
  const int i0 = threadIdx.x * per, i1 = min(a.b.n, i0 + per);
  int64_t sum = 0;
  for (int i = i0; i < i1; ++i) sum += kv4_weight(a, cut, kv4_seq(a, cut, i, first_cta));
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
      at += per == 1 ? sum : kv4_weight(a, cut, kv4_seq(a, cut, i, false));
    }
    if (threadIdx.x == THREADS - 1) a.prefix[a.b.n] = at;
  }
  __syncthreads();
}

// The sequence that place `v` (below prefix[THREADS]) lies in; `at`: the length before it.
template <int THREADS>
__device__ __forceinline__ Kv4Seq kv4_find(const Kv4Attend& a, Kv4Cut cut, const int64_t* prefix, int64_t v,
                                           int64_t& at) {
  int lo = 0, hi = THREADS - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (prefix[mid] <= v) lo = mid; else hi = mid - 1;
  }
  const int per = (a.b.n + THREADS - 1) / THREADS;
  at = prefix[lo];
  Kv4Seq s = kv4_seq(a, cut, lo * per, false);
  for (int k = 1; k < per; ++k) {
    const int64_t w = kv4_weight(a, cut, s);
    if (v < at + w || lo * per + k >= a.b.n) break;
    at += w;
    s = kv4_seq(a, cut, lo * per + k, false);
  }
  return s;
}

// Workers that take part: no range shorter than cut.least.  Worker w's range of the length W begins
// at W w / workers.
__device__ __forceinline__ int kv4_workers(int64_t W, Kv4Cut cut, int most) {
  const int64_t w = W / cut.least;
  return w < 1 ? 1 : w < most ? (int)w : most;
}
__device__ __forceinline__ int64_t kv4_range_begin(int64_t W, int w, int workers) { return W * w / workers; }
// the worker whose range holds place v
__device__ __forceinline__ int kv4_owner(int64_t W, int64_t v, int workers) {
  return (int)(((v + 1) * workers - 1) / W);
}

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

cudaError_t launch_kv4_join(const Kv4Attend& a, Kv4Cut cut, int workers, int dtype, cudaStream_t stream);

}  // namespace semkv
