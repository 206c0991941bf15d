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
  int64_t* prefix;   // (many rows) [b.n + 1]: length before each sequence
  int4* joins;       // (many rows) [workers]: the item that each begins and does not end (Kv4Join)
  int2* spans;       // (few rows) [b.n][heads][tiles]: first and last worker of each item; first -1: it was
  int tiles;         //   finished by one
};

__host__ __device__ constexpr int kv4_part_floats(int D) { return D + 4; }

// One sequence's rows of the step and its tokens.
struct Kv4Seq {
  int seq, begin, count, length;
  int tiles;           // tiles of query rows
  int u_first, units;  // (Kv4FewCut) units of each item: u_first .. u_first + units - 1
  int hidden, level;   // (Kv4ManyCut) tiles at the front that see nothing; the first that sees `cap`
};

__device__ __forceinline__ Kv4Seq kv4_seq(const Kv4Attend& a, int rows, int i, bool report) {
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
  s.tiles = (int)(((int64_t)s.count * a.group + rows - 1) / rows);
  return s;
}

// Cut for few rows: lengths in units of `unit` tokens; the items of a sequence are alike, from the
// unit of the first row's first position to the last.
struct Kv4FewCut {
  int rows, unit, start, least;
  __device__ __forceinline__ Kv4Seq seq(const Kv4Attend& a, int i, bool report) const {
    Kv4Seq s = kv4_seq(a, rows, i, report);
    if (s.count > 0 && s.length > 0) {
      const int64_t lo = a.window ? (int64_t)s.length - s.count + 1 - a.window : 0;
      s.u_first = lo > 0 ? (int)(lo / unit) : 0;
      s.units = (s.length + unit - 1) / unit - s.u_first;
    }
    return s;
  }
  __device__ __forceinline__ int64_t weight(const Kv4Attend& a, const Kv4Seq& s) const {
    return s.units ? (int64_t)(s.units + start) * s.tiles * a.c.H : 0;
  }
};

// Cut for many rows: lengths in tokens.  A tile holds `tokens` whole tokens of the sequence (its rows are
// tokens * group); tile x sees the positions below e = p0 + (x + 1) tokens, p0 the first row's, and
// of them the last `cap` (all, without a window), so lengths add up in closed form.
struct Kv4ManyCut {
  static constexpr int unit = 128, start = 448, least = 256;
  int rows, tokens;
  uint64_t magic;  // 2^32 / group, rounded up: x / group = x * magic >> 32 for the rows x of a tile
  __device__ __forceinline__ int token_of(int x) const { return (int)((uint64_t)x * magic >> 32); }
  __device__ __forceinline__ Kv4Seq seq(const Kv4Attend& a, int i, bool report) const {
    Kv4Seq s = kv4_seq(a, rows, i, report);
    const int p0 = s.length - s.count;
    s.hidden = p0 < 0 ? -p0 / tokens : 0;
    s.level = 0x7FFFFFFF;
    if (a.window) {
      const int64_t x = (cap(a) - p0 + tokens - 1) / tokens - 1;  // (rare, so 64 bits)
      s.level = x < s.hidden ? s.hidden : x < s.level ? (int)x : s.level;
    }
    return s;
  }
  __device__ __forceinline__ int64_t cap(const Kv4Attend& a) const {
    return a.window ? (int64_t)a.window + tokens : (int64_t)1 << 40;
  }
  // the tile that a place of one head lies in
  __device__ __forceinline__ int find(const Kv4Attend& a, const Kv4Seq& s, int64_t place) const {
    int lo = 0, hi = s.tiles - 1;  // the last that begins at or before it
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (before(a, s, mid) <= place) lo = mid; else hi = mid - 1;
    }
    return lo;
  }
  // length of one head's tiles before tile k
  __device__ __forceinline__ int64_t before(const Kv4Attend& a, const Kv4Seq& s, int64_t k) const {
    if (s.length == 0) return 0;
    if (k <= s.hidden) return 0;
    const int64_t p0 = (int64_t)s.length - s.count, k0 = s.hidden;
    const int64_t x = k < s.level ? k : s.level;
    const int64_t ramp = (x - k0) * p0 + tokens * ((x * (x + 1) - k0 * (k0 + 1)) >> 1);
    return ramp + (k > x ? (k - x) * cap(a) : 0) + (k - k0) * start;
  }
  // a tile's own length (positions end at 2^30, a tile at 256 more)
  __device__ __forceinline__ int length(const Kv4Attend& a, const Kv4Seq& s, int tile) const {
    const int e = s.length - s.count + (tile + 1) * tokens;
    if (s.length == 0 || e <= 0) return 0;
    return (a.window && e - tokens > a.window ? a.window + tokens : e) + start;
  }
  __device__ __forceinline__ int64_t weight(const Kv4Attend& a, const Kv4Seq& s) const {
    return before(a, s, s.tiles) * a.c.H;
  }
  // a tile's units [first, last) and the position `from` of its length's first token
  __device__ __forceinline__ void units(const Kv4Attend& a, const Kv4Seq& s, int tile, int& first, int& last,
                                        int& from) const {
    const int e = s.length - s.count + (tile + 1) * tokens;
    from = a.window && e - tokens > a.window ? e - tokens - a.window : 0;
    first = from / unit;
    const int to = e < s.length ? e : s.length;
    last = to > 0 ? (to + unit - 1) / unit : first;
  }
  // places, from the sequence's first, of an item's first and last unit; false if it has none
  __device__ __forceinline__ bool ends(const Kv4Attend& a, const Kv4Seq& s, int head, int tile, int64_t& first,
                                       int64_t& last) const {
    int u0, u1, from;
    units(a, s, tile, u0, u1, from);
    if (s.length == 0 || u1 <= u0) return false;
    first = head * before(a, s, s.tiles) + before(a, s, tile) + start;
    const int at = (u1 - 1) * unit - from;
    last = first + (at > 0 ? at : 0);
    return true;
  }
};

// The plan: thread x of the block adds up sequences x * per .. (x + 1) * per - 1, with
// per = ceil(n / THREADS); prefix[x] = the length before them, prefix[THREADS] = all.
// KEEP: CTA 0 leaves each sequence's in a.prefix.
template <int THREADS, bool KEEP, class Cut>
__device__ __forceinline__ void kv4_plan(const Kv4Attend& a, Cut cut, int64_t* prefix, int64_t* sums,
                                         bool first_cta) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int per = (a.b.n + THREADS - 1) / THREADS;
  const int i0 = threadIdx.x * per, i1 = min(a.b.n, i0 + per);
  int64_t sum = 0;
  for (int i = i0; i < i1; ++i) sum += cut.weight(a, cut.seq(a, i, first_cta));
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
  if (KEEP && first_cta) {
    for (int i = i0; i < i1; ++i) {
      a.prefix[i] = at;
      at += per == 1 ? sum : cut.weight(a, cut.seq(a, i, false));
    }
    if (threadIdx.x == THREADS - 1) a.prefix[a.b.n] = at;
  }
  __syncthreads();
}

// The sequence that place `v` (below prefix[THREADS]) lies in; `at`: the length before it, `i`: which.
template <int THREADS, class Cut>
__device__ __forceinline__ Kv4Seq kv4_find(const Kv4Attend& a, Cut cut, const int64_t* prefix, int64_t v,
                                           int64_t& at, int& i) {
  // the last entry at or below v: of every THREADS / 32-th by one vote, of those behind it by another (the
  // whole warp asks for one place)
  constexpr int kStep = THREADS / 32;
  static_assert(kStep <= 32 && THREADS % 32 == 0, "two votes find an entry");
  const int lane = threadIdx.x & 31;
  int lo = (31 - __clz(__ballot_sync(~0u, prefix[lane * kStep] <= v))) * kStep;
  lo += 31 - __clz(__ballot_sync(~0u, lane < kStep && prefix[lo + (lane < kStep ? lane : 0)] <= v));
  const int per = (a.b.n + THREADS - 1) / THREADS;
  at = prefix[lo];
  i = lo * per;
  Kv4Seq s = cut.seq(a, i, false);
  for (int k = 1; k < per; ++k) {
    const int64_t w = cut.weight(a, s);
    if (v < at + w || i + 1 >= a.b.n) break;
    at += w;
    s = cut.seq(a, ++i, false);
  }
  return s;
}

// a / b; most dividends fit 32 bits, and a 64-bit division is a few hundred cycles of code that a
// short kernel first has to fetch
__device__ __forceinline__ int64_t kv4_div(int64_t a, int64_t b) {
  return ((a | b) >> 32) == 0 ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b;
}

// The length W cut into ranges: as many as there are workers, but none shorter than `least`; the first
// W % count are one longer.
struct Kv4Ranges {
  int count, longer;
  int64_t each;
  __device__ __forceinline__ Kv4Ranges(int64_t W, int least, int most) {
    const int64_t w = W / least;
    count = w < 1 ? 1 : w < most ? (int)w : most;
    each = kv4_div(W, count);
    longer = (int)(W - each * count);
  }
  __device__ __forceinline__ int64_t begin(int w) const { return w * each + min(w, longer); }
  // the range that holds place v
  __device__ __forceinline__ int owner(int64_t v) const {
    const int64_t front = longer * (each + 1);
    return v < front ? (int)kv4_div(v, each + 1) : longer + (int)kv4_div(v - front, each);
  }
};

// two binary32 values in a register pair
__device__ __forceinline__ uint64_t pair(float x, float y) {
  uint64_t p;
  asm("mov.b64 %0, {%1, %2};" : "=l"(p) : "f"(x), "f"(y));
  return p;
}
__device__ __forceinline__ void unpair(uint64_t p, float& x, float& y) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(p));
}
__device__ __forceinline__ uint64_t pair_fma(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ uint64_t pair_mul(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint64_t pair_add(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}

__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
  uint32_t w;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
  return w;
}
template <bool BF16>
__device__ __forceinline__ uint32_t pack_out(float lo, float hi) {
  if (!BF16) return pack_half2(lo, hi);
  uint32_t w;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
  return w;
}

// bf16 query rows meet the cache as fp16, scaled by a power of two that brings the row's largest
// value into [1, 2): exact but for values below 2^-14 of it (their last bits, 2^-25 of the largest).
// The factor from the largest magnitude, and what undoes it.
__device__ __forceinline__ float query_factor(float most, float& undo) {
  int e = (int)(__float_as_uint(most) >> 23) - 127;
  if (most == 0.f || !(most < INFINITY)) e = 0;  // rows of zeros and rows with an infinity as they are
  e = e < -126 ? -126 : e;
  // (2^-127, the inverse for e = 127, is not a normal number)
  undo = e == 127 ? 0x1p127f : __uint_as_float((uint32_t)(127 + e) << 23);
  return e == 127 ? 0x1p-127f : __uint_as_float((uint32_t)(127 - e) << 23);
}

constexpr float kNone = -0x1.fffffep127f;  // reference exponent of a row without tokens: below every finite logit
constexpr float kHead = 8.f;     // a moved reference puts the largest weight at 2^8
constexpr float kMost = 15.f;    // largest exponent of a weight
// A logit past 2^22 has steps of a half and more in binary32.  The exponent as one fused product and sum would hold up
// to half a step of what the reference was rounded by, so that far out equal logits all had weight 0 or infinity; there
// the product is rounded first, and where kHead is no longer exact beside it the reference is the largest itself.
constexpr float kFar = 0x1p22f;
__device__ __forceinline__ float reference_for(float top) { return fabsf(top) > 0x1p26f ? top : top - kHead; }
__device__ __forceinline__ bool is_far(float ref) { return fabsf(ref) > kFar && ref != kNone; }

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

// The kernel for many rows (kv4_chunk.cu): whether a step takes it, its parts, its launch.
bool kv4_many(const Kv4Batch& b, int group);
size_t kv4_many_part_floats(int D, int sms);
size_t kv4_many_front_bytes(const Kv4Batch& b, int sms);  // prefix, then joins
cudaError_t launch_kv4_many(const Kv4Attend& a, int dtype, int sms, cudaStream_t stream);

}  // namespace semkv
