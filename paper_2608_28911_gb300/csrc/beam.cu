// beam.cu — one step of beam search: the k best of a group's beams * vocab continuations.
//
// Two kernels.  The scan streams the rows once.  Each thread keeps sum exp(x - m) of its logits, the largest of
// them, and in which of its tiles it saw one above a floor, a logit that k of the piece are known to reach.  The merge has a
// CTA for each group: the rows' normalizers from the sums; then a score that k of the scan's threads reach with
// their largest logits; and of those threads alone, k or a few more, the marked tiles once more, logit by logit.
// So the scan sorts nothing and writes little, whatever k is; a piece has up to 262144 logits (131072 of 32 bits).
//
// Bound by memory where the rows are many: 64 x 16 rows of 131072 bf16 logits, k 32, take 55 us, the scan 47 of them
// (5.7 TB/s; reading alone takes 40), with rows of 131071, which do not begin on multiples of 16 bytes, 62 us, in f32 87.  Few
// rows are bound by the latency of two kernels: 4 rows of 32768, k 8, 11 us, 25 of 50003 in f32 13 us.  What took longer:
// lists of the best kept by the CTA as it streams (171 us for the scan), candidates put aside where they are met (93),
// tiles brought by bulk copies (102), a warp that settles what the others stream (72).
//
// A candidate is a key: a number whose order is the candidates', and all keys differ.  A key T that k or a few more of
// the threads' largest keys reach is found bit by bit, a barrier that counts for each, from the first bit in which the keys
// differ.
//
// A sum's terms are 2^(x log2 e - c) with a whole number c, so that sums of different c are brought together exactly.
// They are binary32, with a bound on their error.  If that leaves open which of two rows' candidates
// comes first, the merge sums the rows in question again, in pairs of binary32 numbers: 44 us for a row of 131072, one after
// the other (16 beams that are alike 0.7 ms; rows of equal logits, which are looked at key by key as well, 1.7 ms).
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <float.h>
#include <math.h>

#include "common.cuh"
#include "kernels.h"

namespace semkv {
namespace {

constexpr int kScanThreads = 256, kMergeThreads = 1024;
constexpr int kSlack = 16;       // keys that a threshold may let through beside the k best
constexpr int kRanked = 512;     // keys that the merge puts in order without cutting them down first
constexpr float kLog2e = 1.4426950408889634f;
constexpr double kLn2 = 0.69314718055994530942;
// Past this logits are too coarse for x log2 e in one rounding: rows with a largest logit beyond it are summed exactly.
constexpr float kFar = 1048576.f;
constexpr float kNone = -INFINITY;

// ------------------------------------------------------------------ keys ------

// A float as an unsigned number of the same order; -0 as +0.
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return b ^ ((int32_t)b < 0 ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t u) {
  return __uint_as_float(u ^ ((int32_t)u < 0 ? 0x80000000u : 0xFFFFFFFFu));
}
// In a group: the score (a binary32 number and what it lacks), then the lower beam, the larger logit and the lower
// token.  a = 0: none.
struct GroupKey {
  uint64_t a, b;
  static constexpr int kBits = 128;
  __device__ __forceinline__ static GroupKey none() { return {0, 0}; }
  __device__ __forceinline__ static GroupKey of(float score, float rest, int beam, float x, int token) {
    return {(uint64_t)ordered(score) << 32 | ordered(rest),
            (uint64_t)(SEMKV_BEAM_MAX - 1 - beam) << 56 | (uint64_t)ordered(x) << 24 | (0xFFFFFFu - (uint32_t)token)};
  }
  __device__ __forceinline__ static GroupKey of_word(uint32_t w) { return {(uint64_t)w << 32, 0}; }
  __device__ __forceinline__ uint32_t word() const { return (uint32_t)(a >> 32); }
  __device__ __forceinline__ float score() const { return unordered((uint32_t)(a >> 32)); }
  __device__ __forceinline__ float rest() const { return unordered((uint32_t)a); }
  __device__ __forceinline__ int beam() const { return SEMKV_BEAM_MAX - 1 - (int)(b >> 56); }
  __device__ __forceinline__ float logit() const { return unordered((uint32_t)(b >> 24)); }
  __device__ __forceinline__ int token() const { return (int)(0xFFFFFFu - (uint32_t)(b & 0xFFFFFFu)); }
  __device__ __forceinline__ bool valid() const { return a != 0; }
  __device__ __forceinline__ bool operator>=(const GroupKey& o) const { return a > o.a || (a == o.a && b >= o.b); }
  __device__ __forceinline__ GroupKey with(int bit) const {
    return bit >= 64 ? GroupKey{a | 1ull << (bit - 64), b} : GroupKey{a, b | 1ull << bit};
  }
};

// A number alone.
struct WordKey {
  uint32_t a;
  static constexpr int kBits = 32;
  __device__ __forceinline__ static WordKey of_word(uint32_t w) { return {w}; }
  __device__ __forceinline__ uint32_t word() const { return a; }
  __device__ __forceinline__ WordKey with(int bit) const { return {a | 1u << bit}; }
};

// The least and the largest of the CTA's words.
struct Extent {
  uint32_t least, most;
};
template <int THREADS>
__device__ __forceinline__ Extent extent_of(Extent mine, Extent* shared) {
  constexpr int kWarps = THREADS / 32;
  const int lane = threadIdx.x & 31;
  mine = {__reduce_min_sync(~0u, mine.least), __reduce_max_sync(~0u, mine.most)};
  __syncthreads();  // what the call before left has been read
  if (lane == 0) shared[threadIdx.x >> 5] = mine;
  __syncthreads();
  mine = shared[lane % kWarps];
  return {__reduce_min_sync(~0u, mine.least), __reduce_max_sync(~0u, mine.most)};
}

// A key that k or a few more of the keys reach (k exactly, or all that are equal, where no key tells the others
// apart).  count(x): how many reach x, for all threads; there are k or more.  e: of their words.
template <typename Key, typename Count>
__device__ __forceinline__ Key threshold(int k, Extent e, Count count) {
  const int same = __clz(e.least ^ e.most);  // bits that all keys share
  Key t = Key::of_word(same == 32 ? e.least : e.least & ~(0xFFFFFFFFu >> same));
  for (int bit = Key::kBits - 1 - same; bit >= 0; --bit) {
    const Key up = t.with(bit);
    if (up.word() > e.most) continue;
    const int c = count(up);
    if (c < k) continue;
    t = up;
    if (c <= k + kSlack) break;
  }
  return t;
}

// The best keys of a CTA so far, in shared memory: at least the k best of all that were offered.
template <typename Key, int THREADS>
struct Best {
  Key* list;    // [cap]
  Key* spare;   // [k + kSlack]
  int* count;   // keys in the list
  Extent* extents;
  int k, cap;
  Key floor;    // k keys of this or more are in the list (or have been): a key below does not matter

  // For all threads at once, behind a barrier: the list's n keys are cut down to the k best and up to kSlack more.
  __device__ __forceinline__ void cut(int n) {
    Extent e{0xFFFFFFFFu, 0u};
    for (int i = threadIdx.x; i < n; i += THREADS) e = {min(e.least, list[i].word()), max(e.most, list[i].word())};
    e = extent_of<THREADS>(e, extents);
    const Key t = threshold<Key>(k, e, [&](const Key& up) {
      int c = 0;
      for (int i = 0; i < n; i += THREADS) c += __syncthreads_count(i + (int)threadIdx.x < n && list[i + threadIdx.x] >= up);
      return c;
    });
    __syncthreads();
    if (threadIdx.x == 0) *count = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += THREADS)
      if (list[i] >= t) spare[atomicAdd(count, 1)] = list[i];
    __syncthreads();
    for (int i = threadIdx.x; i < *count; i += THREADS) list[i] = spare[i];
    __syncthreads();
    floor = t;
  }
  // Threads bring a few keys each; `top` is the largest of the thread's own and collect(bound) puts those from the
  // bound on.  The list holds k + kSlack threads' keys beside its own k + kSlack.
  template <int PER, typename Collect>
  __device__ __forceinline__ void offer(const Key& top, Collect collect) {
    // (a key equal to the floor is in the list already)
    bool hot = top.valid() && top >= floor;
    int n = __syncthreads_count(hot);
    if (n == 0) return;
    const int held = *count;
    __syncthreads();
    const bool full = held + n * PER > cap;
    if (full && held > k + kSlack) {
      cut(held);
      hot = top.valid() && top >= floor;
      n = __syncthreads_count(hot);
    }
    if (full && n > k + kSlack) {
      const Extent e = extent_of<THREADS>(hot ? Extent{top.word(), top.word()} : Extent{0xFFFFFFFFu, 0u}, extents);
      floor = threshold<Key>(k, e, [&](const Key& up) { return __syncthreads_count(hot && top >= up); });
      hot = hot && top >= floor;
    }
    if (hot) collect(floor);
  }
  __device__ __forceinline__ void put(const Key& x) { list[atomicAdd(count, 1)] = x; }
};

// ------------------------------------------------------------------ rows ------

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// 2^d for a whole number d <= 0 (or minus infinity)
__device__ __forceinline__ float pow2(float d) {
  return d < -126.f ? 0.f : __uint_as_float((uint32_t)((int)d + 127) << 23);
}
// The whole number that terms beside a largest logit m are scaled by: their sum is at least 1/2.
__device__ __forceinline__ float scale_of(float m) { return ceilf(fminf(fmaxf(m, -kFar), kFar) * kLog2e); }
// a + b = s + e exactly
__device__ __forceinline__ void two_sum(float a, float b, float& s, float& e) {
  s = __fadd_rn(a, b);
  const float z = __fsub_rn(s, a);
  e = __fadd_rn(__fsub_rn(a, __fsub_rn(s, z)), __fsub_rn(b, z));
}

// sum + low with the lane's whose number differs in bit d
__device__ __forceinline__ void add_pair(float& sum, float& low, int d) {
  float err;
  const float other = __shfl_xor_sync(~0u, sum, d);
  low += __shfl_xor_sync(~0u, low, d);
  two_sum(sum, other, sum, err);
  low += err;
}

// Eight 16-bit or four 32-bit logits as they lie in memory.
template <int DTYPE>
struct alignas(16) Vec {
  static constexpr int kSize = DTYPE == SEMKV_F32 ? 4 : 2, kCount = 16 / kSize;
  uint32_t w[4];

  __device__ __forceinline__ static uint32_t none() {
    return DTYPE == SEMKV_F32 ? 0xFF800000u : DTYPE == SEMKV_BF16 ? 0xFF80FF80u : 0xFC00FC00u;
  }
  __device__ __forceinline__ void fill_none() { w[0] = w[1] = w[2] = w[3] = none(); }
  __device__ __forceinline__ float at(int i) const {
    if (DTYPE == SEMKV_F32) return __uint_as_float(w[i]);
    if (DTYPE == SEMKV_BF16) return __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
    return __half2float(__ushort_as_half((uint16_t)(i & 1 ? w[i / 2] >> 16 : w[i / 2])));
  }
  __device__ __forceinline__ static float pick(const uint32_t (&x)[4], int i) {
    const int of = DTYPE == SEMKV_F32 ? i : i / 2;
    const uint32_t two = of & 2 ? (of & 1 ? x[3] : x[2]) : (of & 1 ? x[1] : x[0]);
    if (DTYPE == SEMKV_F32) return __uint_as_float(two);
    const uint32_t half = i & 1 ? two >> 16 : two & 0xFFFFu;
    return DTYPE == SEMKV_BF16 ? __uint_as_float(half << 16) : __half2float(__ushort_as_half((uint16_t)half));
  }
  __device__ __forceinline__ void set(int i, uint32_t bits) {
    if (DTYPE == SEMKV_F32) w[i] = bits;
    else w[i / 2] = i & 1 ? (w[i / 2] & 0xFFFFu) | bits << 16 : (w[i / 2] & 0xFFFF0000u) | (bits & 0xFFFFu);
  }
  // the largest, a NaN if one is
  __device__ __forceinline__ static uint32_t max2(uint32_t a, uint32_t b) {
    uint32_t d;
    if (DTYPE == SEMKV_F32) asm("max.NaN.f32 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    else if (DTYPE == SEMKV_BF16) asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    else asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
  }
  // the largest of each half of the words, and of both halves
  __device__ __forceinline__ uint32_t largest2() const { return max2(max2(w[0], w[1]), max2(w[2], w[3])); }
  __device__ __forceinline__ static float larger(uint32_t two) {
    if (DTYPE == SEMKV_F32) return __uint_as_float(two);
    Vec v;
    v.w[0] = two;
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(v.at(0)), "f"(v.at(1)));
    return d;
  }
  // NaN and +infinity become -infinity
  __device__ __forceinline__ void clean() {
#pragma unroll
    for (int i = 0; i < kCount; ++i)
      if (!(at(i) < INFINITY)) set(i, none());
  }
};

// The 16 bytes that begin `lead` bytes into x and y.
template <int DTYPE>
__device__ __forceinline__ Vec<DTYPE> join_vec(const uint4& x, const uint4& y, int lead) {
  const uint32_t t[7] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z};
  uint32_t a[5], b[5];
#pragma unroll
  for (int i = 0; i < 5; ++i) a[i] = lead & 8 ? t[i + 2] : t[i];
#pragma unroll
  for (int i = 0; i < 4; ++i) b[i] = lead & 4 ? a[i + 1] : a[i];
  b[4] = lead & 4 ? (lead & 8 ? y.w : y.y) : a[4];
  Vec<DTYPE> v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v.w[i] = DTYPE == SEMKV_F32 ? b[i] : __funnelshift_r(b[i], b[i + 1], 8 * (lead & 2));
  return v;
}
// Logits first .. first + count of a row, the others -infinity.  The vectors lie `lead` bytes behind a multiple of
// 16; those inside the row are brought by whole aligned loads all the same, two for one of them (its neighbour's
// other half is in the cache).  So a thread's logits, and the order of the sum, do not depend on where a row lies.
template <int DTYPE>
__device__ __forceinline__ Vec<DTYPE> load_vec(const char* row, int first, int vocab, int lead) {
  using V = Vec<DTYPE>;
  const char* at = row + (int64_t)first * V::kSize;
  const int room = V::kCount + (lead ? V::kCount : 0);  // logits that the loads below may touch
  V v;
  if (first + room <= vocab && (lead == 0 || first >= V::kCount)) {
    const uint4* from = reinterpret_cast<const uint4*>(at - lead);
    return join_vec<DTYPE>(__ldg(from), lead ? __ldg(from + 1) : make_uint4(0, 0, 0, 0), lead);
  }
  v.fill_none();
#pragma unroll
  for (int i = 0; i < V::kCount; ++i)
    if (first + i < vocab)
      v.set(i, DTYPE == SEMKV_F32 ? reinterpret_cast<const uint32_t*>(at)[i] : (uint32_t)reinterpret_cast<const uint16_t*>(at)[i]);
  return v;
}

// ------------------------------------------------------------------ scan ------

constexpr int kScanWarps = kScanThreads / 32, kVecs = 4, kMarkTiles = 32;  // vectors of a thread in a tile, tiles of a piece
// How a call's rows are cut.  Each is `units` units of a vector for each of a CTA's threads; a CTA has `share`
// units, of one row behind the other, up to 32 tiles, so a row lies in up to `splits` pieces.
struct Pieces {
  int units, share, splits;
  bool aligned;
  uint32_t per_split;  // 2^32 / splits, rounded up: a product's upper half is the quotient (0: splits is 1)
  // [rows][splits] the largest logit, the sum of 2^(x log2 e - scale_of(it)) as two numbers, and the floor
  float4* sums;
  // [rows][splits][threads] ordered(the largest logit) of the threads that reach the floor, in no order, then zeros
  uint32_t* words;
  uint2* marks;  // beside those that reach it: the tiles to look at, and the thread
  float ln_vocab;
  // Shares begin anywhere in a row: `offset` units before it is where the share that holds its first unit begins.
  __device__ __forceinline__ int offset_of(int row) const {
    const uint32_t n = share;
    return (int)((uint32_t)row % n * ((uint32_t)units % n) % n);
  }
  __device__ __forceinline__ int pieces_of(int offset) const { return (offset + units - 1) / share + 1; }
  __device__ __forceinline__ int begin_unit(int offset, int split) const { return max(0, split * share - offset); }
  __device__ __forceinline__ int end_unit(int offset, int split) const { return min(units, (split + 1) * share - offset); }
};

// A row that is read: neither done nor without a chance.
__device__ __forceinline__ bool row_counts(const BeamArgs& a, int row) {
  const float s = a.scores[row];
  return (!a.done || !a.done[row]) && s > -INFINITY && s < INFINITY;
}

template <int DTYPE>
__device__ __forceinline__ const char* row_at(const BeamArgs& a, int row) {
  return static_cast<const char*>(a.logits) + (int64_t)row * a.stride * Vec<DTYPE>::kSize;
}

// A row as vectors that lie on multiples of 16 bytes: it begins `shift` logits into the first, whose others are not
// its own.  Logits are counted from there.
struct RowView {
  const char* base;
  int shift, size;
};
template <int DTYPE>
__device__ __forceinline__ RowView row_view(const BeamArgs& a, int row, bool aligned = false) {
  const char* at = row_at<DTYPE>(a, row);
  if (aligned) return {at, 0, a.vocab};
  const int lead = (int)((uintptr_t)at & 15), shift = lead / Vec<DTYPE>::kSize;
  return {at - lead, shift, a.vocab + shift};
}
// The vector from logit `first` on; outside the row, or from `end` on, -infinity.
template <int DTYPE>
__device__ __forceinline__ Vec<DTYPE> load_one(const RowView& r, int first, int end) {
  using V = Vec<DTYPE>;
  const char* at = r.base + (int64_t)first * V::kSize;
  V v;
  if (first + V::kCount <= end && (first > 0 || r.shift == 0)) {
    const uint4 x = __ldg(reinterpret_cast<const uint4*>(at));
    v.w[0] = x.x, v.w[1] = x.y, v.w[2] = x.z, v.w[3] = x.w;
    return v;
  }
  v.fill_none();
#pragma unroll
  for (int i = 0; i < V::kCount; ++i)
    if (first + i >= r.shift && first + i < end)
      v.set(i, DTYPE == SEMKV_F32 ? reinterpret_cast<const uint32_t*>(at)[i] : (uint32_t)reinterpret_cast<const uint16_t*>(at)[i]);
  return v;
}
// A thread's vectors of a tile, the first of them from logit `first` on.
template <int DTYPE>
__device__ __forceinline__ void load_vecs(Vec<DTYPE> (&v)[kVecs], const RowView& r, int first, int end) {
  using V = Vec<DTYPE>;
  constexpr int kUnit = kScanThreads * V::kCount;
  if (first + (kVecs - 1) * kUnit + V::kCount <= end && (first > 0 || r.shift == 0)) {
    const uint4* from = reinterpret_cast<const uint4*>(r.base + (int64_t)first * V::kSize);
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      const uint4 x = __ldcs(from + i * kScanThreads);
      v[i].w[0] = x.x, v[i].w[1] = x.y, v[i].w[2] = x.z, v[i].w[3] = x.w;
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < kVecs; ++i) v[i] = load_one<DTYPE>(r, first + i * kUnit, end);
}

// ALIGNED: all rows begin on a multiple of 16 bytes, which saves the registers that shifts take (64 x 16 x 131072: 55 us
// in all, 57 with them).
template <int DTYPE, bool ALIGNED>
__global__ void __launch_bounds__(kScanThreads, 4) beam_scan_kernel(BeamArgs a, Pieces p) {
  using V = Vec<DTYPE>;
  constexpr int kUnit = kScanThreads * V::kCount, kTile = kVecs * kUnit;
  __shared__ uint32_t warp_words[2][kScanWarps];
  __shared__ float4 warp_sums[2][kScanWarps];
  __shared__ int reaching[2], others[2];  // (of this piece, and the one behind it)
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_wait();
  pdl_trigger();
  int64_t unit = (int64_t)blockIdx.x * p.share;
  const int64_t past = min((int64_t)a.groups * a.beams * p.units, unit + p.share);
  int row = (int)(unit / p.units), first_unit = (int)(unit - (int64_t)row * p.units), raised = 0, turn = 0;
  if (tid < 2) reaching[tid] = others[tid] = 0;
  for (; unit < past; ++row, first_unit = 0) {
    const int offset = p.offset_of(row), split = (first_unit + offset) / p.share, end_unit = p.end_unit(offset, split);
    const int begin = first_unit * kUnit;
    unit += end_unit - first_unit;
    if (!row_counts(a, row)) continue;
    const RowView r = row_view<DTYPE>(a, row, ALIGNED);
    const int end = min(r.size, end_unit * kUnit);  // (not above `begin` where only rows that lie otherwise go on)
    // of this thread's logits; k logits of `floor` or more have been seen: the same or less does not matter any more
    float m = kNone, c = -4 * kFar, sum = 0.f, low = 0.f, floor = kNone;
    uint32_t seen = 0;
    int tile = 0;
    // The threads' largest so far tell of a floor: of every warp the n-th, n k's share, the lowest of which k threads reach.
    auto raise = [&]() {
      const int want = (a.k + kScanWarps - 1) / kScanWarps;
      uint32_t mine = m > kNone ? ordered(m) : 0u, word;
      for (int have = 0;;) {
        word = __reduce_max_sync(~0u, mine);
        have += __popc(__ballot_sync(~0u, mine == word));
        if (have >= want || word == 0) break;
        if (mine == word) mine = 0;
      }
      uint32_t* words = warp_words[raised++ & 1];
      if (lane == 0) words[warp] = word;
      __syncthreads();
      // (the counts of the piece before, which all have left behind: the one behind this begins with them)
      if (tid == 0) reaching[~turn & 1] = others[~turn & 1] = 0;
      word = __reduce_min_sync(~0u, words[lane % kScanWarps]);
      if (word) floor = fmaxf(floor, unordered(word));
    };
    // One tile, whose vectors make room for those two tiles on.
    auto step = [&](V (&v)[kVecs], int t0) {
      auto largest = [&]() {
        uint32_t two = v[0].largest2();
#pragma unroll
        for (int i = 1; i < kVecs; ++i) two = V::max2(two, v[i].largest2());
        return V::larger(two);
      };
      float top = largest();
      if (!(top < INFINITY)) {
#pragma unroll
        for (int i = 0; i < kVecs; ++i) v[i].clean();
        top = largest();
        raise_error(a.err, kDevNonFinite);
      }
      m = fmaxf(m, top);
      if (__fmaf_rn(m, kLog2e, -c) > 2.f) {
        const float up = scale_of(m), by = pow2(c - up);  // (0 the first time)
        sum *= by;
        low *= by;
        c = up;
      }
      float s[kVecs];
#pragma unroll
      for (int i = 0; i < kVecs; ++i) {
        float e[V::kCount];
#pragma unroll
        for (int j = 0; j < V::kCount; ++j) e[j] = exp2_fast(__fmaf_rn(v[i].at(j), kLog2e, -c));
#pragma unroll
        for (int w = V::kCount / 2; w > 0; w /= 2)
#pragma unroll
          for (int j = 0; j < w; ++j) e[j] += e[j + w];
        s[i] = e[0];
      }
      float err;
      two_sum(sum, (s[0] + s[1]) + (s[2] + s[3]), sum, err);
      low += err;
      if (t0 + 2 * kTile < end) load_vecs<DTYPE>(v, r, t0 + 2 * kTile + tid * V::kCount, end);
      seen |= (uint32_t)(top > floor) << tile++;
    };
    V v0[kVecs], v1[kVecs];
    load_vecs<DTYPE>(v0, r, begin + tid * V::kCount, end);
    if (begin + kTile < end) load_vecs<DTYPE>(v1, r, begin + kTile + tid * V::kCount, end);
    for (int t0 = begin; t0 < end; t0 += 2 * kTile) {
      step(v0, t0);
      if (t0 + kTile < end) step(v1, t0 + kTile);
      if (t0 + 2 * kTile >= end || (tile & (tile - 1)) != 0) continue;
      raise();  // (behind the second tile, the fourth, the eighth ...: a tile further on has less and less above it)
    }
    const int64_t piece = (int64_t)row * p.splits + split;
    // the warp's sum, a pair of numbers
    float most = m;
#pragma unroll
    for (int d = 16; d > 0; d /= 2) most = fmaxf(most, __shfl_xor_sync(~0u, most, d));
    const float by = m > kNone ? pow2(c - scale_of(most)) : 0.f;
    sum *= by;
    low *= by;
#pragma unroll
    for (int d = 16; d > 0; d /= 2) add_pair(sum, low, d);
    if (lane == 0) warp_sums[turn & 1][warp] = make_float4(most, sum, low, 0.f);
    raise();
    {
      const bool in = m >= floor && m > kNone;
      const uint32_t ins = __ballot_sync(~0u, in);
      int at_in = 0, at_out = 0;
      if (lane == 0) {
        at_in = atomicAdd(reaching + (turn & 1), __popc(ins));
        at_out = atomicAdd(others + (turn & 1), 32 - __popc(ins));
      }
      at_in = __shfl_sync(~0u, at_in, 0);
      at_out = __shfl_sync(~0u, at_out, 0);
      const int64_t to = piece * kScanThreads + (in ? at_in + __popc(ins & ((1u << lane) - 1))
                                                    : kScanThreads - 1 - at_out - __popc(~ins & ((1u << lane) - 1)));
      p.words[to] = in ? ordered(m) : 0u;
      if (in) p.marks[to] = make_uint2(seen, tid);
    }
    if (warp == 0) {
      // the warps' sums together
      float all = lane < kScanWarps ? warp_sums[turn & 1][lane].x : kNone;
      const float4 x = lane < kScanWarps ? warp_sums[turn & 1][lane] : make_float4(kNone, 0.f, 0.f, 0.f);
#pragma unroll
      for (int d = kScanWarps / 2; d > 0; d /= 2) all = fmaxf(all, __shfl_xor_sync(~0u, all, d));
      const float by = x.x > kNone ? pow2(scale_of(x.x) - scale_of(all)) : 0.f;
      sum = x.y * by;
      low = x.z * by;
#pragma unroll
      for (int d = kScanWarps / 2; d > 0; d /= 2) add_pair(sum, low, d);
      if (lane == 0) p.sums[piece] = make_float4(all, sum, low, floor);
    }
    ++turn;
  }
}

// ------------------------------------------------------- the exact sums ------

// 2^(j/256) for j = 0 .. 255 as pairs of binary32 numbers, to 2^-44: products of the root in 64 bits.
constexpr int kPowerCount = 256;
struct Powers {
  float2 at[kPowerCount];
};
constexpr Powers make_powers() {
  Powers p{};
  double x = 1.0;
  for (int j = 0; j < kPowerCount; ++j) {
    p.at[j].x = (float)x;
    p.at[j].y = (float)(x - (double)(float)x);
    x *= 1.0027112750502024854;
  }
  return p;
}
__constant__ const Powers kPowers = make_powers();

// sum + low grows by exp(x + xl) for -64 < x <= 0 and an |xl| of half a step of x at most: 2^(j/256) * exp(t) with x log2 e
// in two numbers, a whole j, |t| <= ln 2 / 512, and exp(t) - 1 = t + t^2 / 2 + t^3 / 6.  2^-40 of it off: the fourth power is
// 2^-42.6, t^2 / 2 below 2^-20, so that its roundings are 2^-44 each, and what x log2 e and t lack is carried along.
// (Restated on the CPU, the worst of 2 million arguments is 2^-40.7 off, of those above -30 2^-41.2.)
__device__ __forceinline__ void add_exp(float x, float xl, const float2* powers, float& sum, float& low) {
  constexpr float kLow = (float)(1.4426950408889634074 - (double)kLog2e), kWhole = 12582912.f;  // 1.5 * 2^23: the last bit is 1
  constexpr float kBig = (float)kLn2, kSmall = (float)(kLn2 - (double)kBig);
  const float p = __fmul_rn(x, kLog2e);
  float e = __fmaf_rn(x, kLow, __fmaf_rn(xl, kLog2e, __fmaf_rn(x, kLog2e, -p)));
  const float z = __fmaf_rn(p, (float)kPowerCount, kWhole), r0 = __fmaf_rn(__fsub_rn(z, kWhole), -1.f / kPowerCount, p);
  const int j = __float_as_int(z) - __float_as_int(kWhole);
  const float r = __fadd_rn(r0, e);
  e = __fadd_rn(__fsub_rn(r0, r), e);
  const float t = __fmul_rn(r, kBig);
  const float tl = __fmaf_rn(e, kBig, __fmaf_rn(r, kSmall, __fmaf_rn(r, kBig, -t)));
  // exp(t + tl) - 1 = h + hl
  const float q = __fmaf_rn(__fmul_rn(t, t), __fmaf_rn(t, 1.f / 6, 0.5f), tl);
  const float h = __fadd_rn(t, q), hl = __fadd_rn(__fsub_rn(t, h), q);
  const float2 w = powers[j & (kPowerCount - 1)];
  const float a = __fmul_rn(w.x, h);
  const float b = __fmaf_rn(w.x, hl, __fmaf_rn(w.y, h, __fadd_rn(__fmaf_rn(w.x, h, -a), w.y)));
  const float s = __int_as_float(((j >> 8) + 127) << 23);
  const float high = __fadd_rn(w.x, a), rest = __fadd_rn(__fadd_rn(__fsub_rn(w.x, high), a), b);
  float err;
  two_sum(sum, __fmul_rn(high, s), sum, err);
  low += __fmaf_rn(rest, s, err);
}

// ln sum exp(x - most) of a row, by a whole CTA, to 2^-38, for its first warp.  `most` is the row's largest logit.
template <int DTYPE>
__device__ __noinline__ double exact_normalizer(const BeamArgs& a, int row, float most, float2* powers, double* parts) {
  using V = Vec<DTYPE>;
  const char* at = row_at<DTYPE>(a, row);
  const int lead = (int)((uintptr_t)at & 15);
  double total = 0.0;
  if (threadIdx.x < kPowerCount) powers[threadIdx.x] = kPowers.at[threadIdx.x];
  __syncthreads();
  // 32 logits at a time in two numbers: `low` is off by 2^-25 of itself with each, and up to 32 steps of 2^-25 of the sum,
  // so 2^-40 of it at most.  (All of a row's in one pair, equal logits' errors add up: 2^21 of them were 2^-34 off.)
  constexpr int kBlock = 32 / V::kCount, kStep = kMergeThreads * V::kCount;
  for (int begin = threadIdx.x * V::kCount; begin < a.vocab; begin += kBlock * kStep) {
    float sum = 0.f, low = 0.f;
#pragma unroll 1
    for (int i = 0, first = begin; i < kBlock && first < a.vocab; ++i, first += kStep) {
      const V v = load_vec<DTYPE>(at, first, a.vocab, lead);
      // (what lies 64 below the largest is less than 2^-92 of it: past every bit that counts.  A NaN is left out here, too.)
#pragma unroll
      for (int j = 0; j < V::kCount; ++j) {
        float d, dl;
        two_sum(v.at(j), -most, d, dl);
        if (d <= 0.f && d > -64.f) add_exp(d, dl, powers, sum, low);
      }
    }
    total += (double)sum + (double)low;
  }
#pragma unroll
  for (int d = 16; d > 0; d /= 2) total += __shfl_xor_sync(~0u, total, d);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) parts[threadIdx.x >> 5] = total;
  __syncthreads();
  if (threadIdx.x >= 32) return 0.0;
  total = threadIdx.x < kMergeThreads / 32 ? parts[threadIdx.x] : 0.0;
#pragma unroll
  for (int d = 16; d > 0; d /= 2) total += __shfl_xor_sync(~0u, total, d);
  return log(total);
}

// ----------------------------------------------------------------- merge ------

// What a row's logits need to become scores: value + rest + (logit - most).
struct Base {
  float value, rest;
  float most;   // the row's largest logit
  float error;  // how far value + rest may be off
  float cut;    // no score below this (as rough() gives it) is among the k best
  int kind;     // kNobody, kLogits, kDone
  int pieces, offset;
};
enum { kNobody, kLogits, kDone };

// (value is the sum's rounding, so that what goes by it alone is off by no more than that: norm_low grows with a row's
// largest logit, 0.07 at a million)
__device__ __forceinline__ void set_value(Base& r, float score, float norm, float norm_low) {
  float value, rest;
  two_sum(score, -norm, value, rest);
  two_sum(value, rest - norm_low, r.value, r.rest);
}
// A logit's score by rounded numbers.  What lies below binary32's range counts as its lowest number: -infinity is for what
// is no candidate.
__device__ __forceinline__ float rough(float value, float most, float x) { return fmaxf(value + (x - most), -FLT_MAX); }
__device__ __forceinline__ GroupKey score_of(const Base& r, int beam, float x, int token) {
  float d, dl, s, e;
  two_sum(x, -r.most, d, dl);
  two_sum(r.value, d, s, e);
  e += r.rest + dl;
  const float score = __fadd_rn(s, e);
  if (!(score > kNone)) return GroupKey::of(-FLT_MAX, -FLT_MAX, beam, x, token);  // (behind those that are in the range)
  return GroupKey::of(score, __fadd_rn(__fsub_rn(s, score), e), beam, x, token);
}

constexpr int kPlaces = 2048, kTable = 1024, kFew = 32, kBatch = 4;
__host__ __device__ constexpr int log_sets_of(int k) { return k <= 16 ? 1 : k <= 48 ? 2 : 3; }
// The list holds what offer() asks of it: k + kSlack threads' keys, a vector each, beside its own k + kSlack.
__host__ __device__ constexpr int merge_cap(int k, int dtype) {
  return (k + kSlack) * (dtype == SEMKV_F32 ? 5 : 9) > 2 * kRanked ? (k + kSlack) * (dtype == SEMKV_F32 ? 5 : 9) : 2 * kRanked;
}
__host__ __device__ constexpr int merge_bytes(int k, int dtype) {
  return (merge_cap(k, dtype) + k + kSlack) * (int)sizeof(GroupKey) + kPlaces * (int)sizeof(int2) + kTable * (int)sizeof(float3);
}

// MANY: a group has more sets of threads to look at than two steps of its warps, so that it pays to tell first which
// pieces matter (1 x 64 x 200000, k 128: 54 us with, 89 without; 4 x 32768: 11.3 with, 10.4 without).
template <int DTYPE, bool MANY>
__global__ void __launch_bounds__(kMergeThreads) beam_merge_kernel(BeamArgs a, Pieces p) {
  using V = Vec<DTYPE>;
  constexpr int kUnit = kScanThreads * V::kCount, kTile = kVecs * kUnit;
  extern __shared__ __align__(16) unsigned char shared[];
  __shared__ int count, place_count, live;
  __shared__ double parts[kMergeThreads / 32];
  __shared__ Extent extents[kMergeThreads / 32];
  __shared__ uint32_t worst_error, top_score, lowest_cut, best_floor;  // (as ordered numbers)
  __shared__ Base base[SEMKV_BEAM_MAX];
  __shared__ uint32_t again[SEMKV_BEAM_MAX / 32];  // rows to be summed once more
  __shared__ float2 powers[kPowerCount];
  __shared__ GroupKey out[SEMKV_BEAM_MAX];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int group = blockIdx.x, row0 = group * a.beams;
  Best<GroupKey, kMergeThreads> best;
  best.list = reinterpret_cast<GroupKey*>(shared);
  best.spare = best.list + merge_cap(a.k, DTYPE);
  best.count = &count;
  best.extents = extents;
  best.k = a.k;
  best.cap = merge_cap(a.k, DTYPE);
  int2* places = reinterpret_cast<int2*>(best.spare + a.k + kSlack);  // beam and split, the first token of a thread's vectors
  float3* table = reinterpret_cast<float3*>(places + kPlaces);  // of pieces: which, and what makes their logits scores
  if (tid < SEMKV_BEAM_MAX / 32) again[tid] = 0;
  if (tid == 0) count = place_count = 0, worst_error = best_floor = 0u, top_score = ordered(0.f), lowest_cut = 0xFFFFFFFFu;
  __syncthreads();
  pdl_wait();
  pdl_trigger();
  const int pieces = a.beams * p.splits;
  const float4* sums = p.sums + (int64_t)row0 * p.splits;
  const uint32_t* words = p.words + (int64_t)row0 * p.splits * kScanThreads;
  const uint2* marks = p.marks + (int64_t)row0 * p.splits * kScanThreads;
  // The scan's threads, 32 at a time, go around the warps: of each piece the first few such sets (2^log_sets), which are
  // more than a piece of random logits fills, and where the last of these is full the others.
  constexpr int kWarps = kMergeThreads / 32;
  const int log_sets = log_sets_of(a.k), last_set = (1 << log_sets) - 1;
  // (the first are on their way while the sums are brought together: the pieces' largest, or the words themselves)
  float4 first_sums;
  uint32_t first_words[kBatch];
  if constexpr (MANY) {
    first_sums = tid < pieces ? sums[tid] : make_float4(kNone, 0.f, 0.f, kNone);
  } else {
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const int set = j * kWarps + warp;
      first_words[j] = set < pieces << log_sets ? words[(set >> log_sets) * kScanThreads + (set & last_set) * 32 + lane] : 0u;
    }
  }
  // a warp for each row: its pieces' sums together
  for (int b = warp; b < a.beams; b += kMergeThreads / 32) {
    const int row = row0 + b;
    const float4* s = p.sums + (int64_t)row * p.splits;
    const int offset = p.offset_of(row), pieces = p.pieces_of(offset);
    const float4 mine = lane < pieces ? s[lane] : make_float4(kNone, 0.f, 0.f, 0.f);
    const float score = a.scores[row];
    const bool is_done = a.done && a.done[row];
    Base r{score, 0.f, 0.f, 0.f, kNone, kNobody, pieces, offset};
    if (score != score || score == INFINITY) {
      if (lane == 0) raise_error(a.err, kDevNonFinite);
    } else if (score > kNone && is_done) {
      r.kind = kDone;
    } else if (score > kNone) {
      float m = mine.x;
      for (int i = lane + 32; i < pieces; i += 32) m = fmaxf(m, s[i].x);
#pragma unroll
      for (int d = 16; d > 0; d /= 2) m = fmaxf(m, __shfl_xor_sync(~0u, m, d));
      if (m > kNone) {
        const float c = scale_of(m);
        float sum = 0.f, low = 0.f, err;
        for (int i = lane; i < pieces; i += 32) {
          const float4 x = i == lane ? mine : s[i];
          const float by = x.x > kNone ? pow2(scale_of(x.x) - c) : 0.f;
          two_sum(sum, x.y * by, sum, err);
          low += x.z * by + err;
        }
#pragma unroll
        for (int d = 16; d > 0; d /= 2) add_pair(sum, low, d);
        r.most = m;
        r.kind = kLogits;
        // ln sum exp(x - m) = (c ln 2 - m) + ln(sum), the logarithm by the sum's exponent and a number from 3/4 to 3/2.
        // What the terms' log2 e lacks is made up for with the weighted mean of the logits, m - u at the
        // lowest with u = ln vocab - ln sum exp(x - m): m - u / 2 is taken, half the range is the error.
        constexpr float kBig = (float)kLn2, kSmall = (float)(kLn2 - (double)kBig);
        constexpr float kLack = (float)((double)kLog2e * kLn2 - 1.0);
        const int e = ((int)(__float_as_uint(sum) - 0x3F400000u)) >> 23;
        const float n = c + (float)e, h = __fmul_rn(n, kBig);
        float norm, rest;
        two_sum(h, -m, norm, rest);
        rest += __fmaf_rn(n, kBig, -h) + n * kSmall + __fdividef(low, sum);
        two_sum(norm, logf(__uint_as_float(__float_as_uint(sum) - ((uint32_t)e << 23))), norm, err);
        const float u = p.ln_vocab - norm;
        rest += err - kLack * (m - 0.5f * u);
        set_value(r, score, norm, rest);
        // In units of 2^-24: an exponent's argument is off by half a step, so 1 for each of |x - m| + 3 ln 2, on the average
        // over the terms u + 3 ln 2; exponentials by 4; sums of eight and of four numbers by 5; the logarithm by 1.
        r.error = fabsf(m) > kFar ? 0.f : (1.125f * fmaxf(u, 0.f) + 13.f) * 0x1p-24f;
      }
    }
    if (lane == 0) {
      base[b] = r;
      atomicMax(&worst_error, ordered(r.error));
      if (r.kind == kLogits) atomicMax(&top_score, ordered(score));  // (no value is above its beam's score)
      if (r.kind == kLogits && fabsf(r.most) > kFar) atomicOr(again + (b >> 5), 1u << (b & 31));
    }
  }
  __syncthreads();
  const float worst = unordered(worst_error);
  auto sum_again = [&](int b) {
    const double norm = exact_normalizer<DTYPE>(a, row0 + b, base[b].most, powers, parts);
    if (tid == 0) {
      set_value(base[b], a.scores[row0 + b], (float)norm, (float)(norm - (double)(float)norm));
      base[b].error = 0x1p-36f;
    }
    __syncthreads();
  };
  auto sum_marked = [&]() {
    for (int w = 0; w < SEMKV_BEAM_MAX / 32; ++w)
      for (uint32_t bits = again[w]; bits; bits &= bits - 1) {
        const int b = 32 * w + __ffs(bits) - 1;
        if (base[b].kind == kLogits) sum_again(b);
      }
  };
  sum_marked();  // (logits past what the scan's sums are made for)
  auto beam_of = [&](int i) { return p.per_split ? (int)__umulhi((uint32_t)i / kScanThreads, p.per_split) : i / kScanThreads; };
  // what(q, beam, the piece's largest logit, its floor) for this thread's pieces of those from q0 on that were read
  auto over_pieces = [&](int q0, int q1, auto what) {
    for (int q = q0 + tid; q < q1; q += kMergeThreads) {
      const int b = beam_of(q * kScanThreads);
      if (base[b].kind != kLogits || q - b * p.splits >= base[b].pieces) continue;  // (nothing was written)
      const float4 x = q == tid ? first_sums : sums[q];
      what(q, b, x.x, x.w);
    }
  };
  // A score below a beam's cut is surely none of the k best if k reach `reach`.  (2^-20 of the numbers that were added is
  // far more than their roundings.  Those of a score that reaches it, some beam's value v and a logit that takes
  // something off, are |v| and up to |v| + |score|: not more than the score itself unless v is above 0.)
  const float slack = 2.1f * worst + 0x1p-20f * unordered(top_score);
  auto cut_of = [&](float value, float reach) {
    return reach > kNone ? reach - slack - 0x1p-20f * (fabsf(value) + fabsf(reach)) : kNone;
  };
  float known = kNone;
  if constexpr (MANY) {
    // k reach each piece's floor: the best of these tells which pieces matter
    over_pieces(0, pieces, [&](int, int b, float, float floor) {
      if (floor > kNone) atomicMax(&best_floor, ordered(rough(base[b].value, base[b].most, floor)));
    });
    __syncthreads();
    known = best_floor ? unordered(best_floor) : kNone;
  }
  // The pieces from q0 on whose best reaches cut(its beam's value), as many as there is room for.
  auto fill_table = [&](int q0, auto cut) {
    __syncthreads();
    if (tid == 0) live = 0;
    __syncthreads();
    over_pieces(q0, min(pieces, q0 + kTable), [&](int q, int b, float most, float) {
      const Base& r = base[b];
      if (rough(r.value, r.most, most) >= cut(r.value)) table[atomicAdd(&live, 1)] = make_float3(__int_as_float(q), r.value, r.most);
    });
    __syncthreads();
  };
  // Scores of the largest logits that the words tell of, rounded, -infinity for none: what(i, score) for all of this
  // thread's in the table.  more(word): there are more in the piece (the same for a whole warp).
  auto over_table = [&](auto what, auto more) {
    const int sets = live << log_sets;
    for (int set0 = warp; set0 < sets; set0 += kBatch * kWarps) {
      uint32_t word[kBatch];
      float3 t[kBatch];
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const int set = set0 + j * kWarps;
        if (set < sets) {
          t[j] = table[set >> log_sets];
          if (!MANY && set0 == warp) word[j] = first_words[j];
          else word[j] = words[__float_as_int(t[j].x) * kScanThreads + (set & last_set) * 32 + lane];
        }
      }
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const int set = set0 + j * kWarps;
        if (set >= sets) break;
        if (!MANY && t[j].y == kNone) continue;  // (nothing was written)
        int i = __float_as_int(t[j].x) * kScanThreads + (set & last_set) * 32 + lane;
        what(i, word[j] ? rough(t[j].y, t[j].z, unordered(word[j])) : kNone);
        if ((set & last_set) == last_set && more(word[j]))
          for (int s = last_set + 1; s < kScanThreads / 32; ++s) {
            const uint32_t x = words[i += 32];
            what(i, x ? rough(t[j].y, t[j].z, unordered(x)) : kNone);
          }
      }
    }
  };
  // A score that k threads reach with theirs (-infinity: fewer have one), from the largest of each thread's.
  auto reached = [&](float mine) {
    const bool in = mine > kNone;
    const uint32_t word = ordered(mine);
    const int n = __syncthreads_count(in);
    if (n < a.k) return kNone;
    const Extent e = extent_of<kMergeThreads>(in ? Extent{word, word} : Extent{0xFFFFFFFFu, 0u}, extents);
    if (n <= a.k + kSlack) return unordered(e.least);
    return unordered(threshold<WordKey>(a.k, e, [&](const WordKey& up) { return __syncthreads_count(in && word >= up.a); }).a);
  };
  const auto more = [&](uint32_t x) { return __any_sync(~0u, lane == 31 && x != 0); };
  const auto by_known = [&](float value) { return cut_of(value, known); };
  if constexpr (MANY) {
    fill_table(0, by_known);
    if (pieces > kTable || live > 2 * kFew) {
      // very many pieces: first a score from the best of them alone
      float most = kNone;
      over_pieces(0, min(pieces, kTable), [&](int, int b, float x, float) { most = rough(base[b].value, base[b].most, x); });
      const bool in = most > kNone;
      const uint32_t word = ordered(most);
      float least = kNone;
      if (__syncthreads_count(in) > kFew + kSlack) {
        const Extent e = extent_of<kMergeThreads>(in ? Extent{word, word} : Extent{0xFFFFFFFFu, 0u}, extents);
        least = unordered(threshold<WordKey>(kFew, e, [&](const WordKey& up) { return __syncthreads_count(in && word >= up.a); }).a);
      }
      fill_table(0, [&](float) { return least; });
      most = kNone;
      over_table([&](int, float s) { most = fmaxf(most, s); }, more);
      known = fmaxf(known, reached(most));
      fill_table(0, by_known);
    }
  } else {
    for (int q = tid; q < pieces; q += kMergeThreads) {
      const int b = beam_of(q * kScanThreads);
      const bool is = base[b].kind == kLogits && q - b * p.splits < base[b].pieces;
      table[q] = make_float3(__int_as_float(q), is ? base[b].value : kNone, base[b].most);
    }
    if (tid == 0) live = pieces;
    __syncthreads();
  }
  // A score that k of all reach, and how far below it a candidate may stay and be among the k best all the same.
  float top = kNone, second = kNone;  // of this thread's
  int top_at = 0;
  for (int q0 = 0;;) {
    over_table(
        [&](int i, float s) {
          second = fmaxf(second, fminf(s, top));
          if (s > top) top = s, top_at = i;
        },
        more);
    if (!MANY || (q0 += kTable) >= pieces) break;
    fill_table(q0, by_known);
  }
  const float own = tid < a.beams && base[tid].kind == kDone ? base[tid].value : kNone;  // a beam that is done
  const float reach = fmaxf(known, reached(fmaxf(top, own)));
  // (a beam's scores are its value at most)
  if (tid < a.beams) {
    const float value = base[tid].value;
    const float cut = cut_of(value, reach);
    base[tid].cut = cut;
    if (base[tid].kind != kNobody && value >= cut) atomicMin(&lowest_cut, ordered(cut));
    if (own > kNone && own >= cut) best.put(score_of(base[tid], tid, 0.f, a.end_token));
  }
  __syncthreads();
  // the marked tiles of those that come near it
  auto look_at = [&](int i, uint32_t tiles) {
    const int b = beam_of(i), split = i / kScanThreads - b * p.splits;
    const uint2 mark = marks[i];
    tiles &= mark.x;
    int w = atomicAdd(&place_count, __popc(tiles));
    const int first = p.begin_unit(base[b].offset, split) * kUnit + (int)mark.y * V::kCount;
    for (uint32_t bits = tiles; bits && w < kPlaces; bits &= bits - 1)
      places[w++] = make_int2(i / kScanThreads, first + (__ffs(bits) - 1) * kTile);
  };
  const float lowest = unordered(lowest_cut);
  auto look = [&](uint32_t tiles) {
    const auto near = [&](int i, float s) { if (s > kNone && s >= base[beam_of(i)].cut) look_at(i, tiles); };
    if (MANY && pieces > kTable) {
      for (int q0 = 0; q0 < pieces; q0 += kTable) {
        fill_table(q0, by_known);
        over_table(near, more);
      }
    } else if (second > kNone && second >= lowest) {
      over_table(near, [&](uint32_t) { return true; });
    } else if (top > kNone && top >= lowest) {
      near(top_at, top);
    }
  };
  auto take = [&]() {
    for (int i = tid; i < place_count; i += kMergeThreads) {
      const int2 at = places[i];
      const int b = beam_of(at.x * kScanThreads), row = row0 + b;
      const Base& r = base[b];
      const RowView view = row_view<DTYPE>(a, row);
      const float floor = sums[at.x].w;
      V v[kVecs];
      load_vecs<DTYPE>(v, view, at.y, min(view.size, p.end_unit(r.offset, at.x - b * p.splits) * kUnit));
      uint32_t hits = 0;
#pragma unroll
      for (int i = 0; i < kVecs; ++i)
#pragma unroll
        for (int j = 0; j < V::kCount; ++j) {
          const float x = v[i].at(j);
          hits |= (uint32_t)(x > kNone && x < INFINITY && x >= floor && rough(r.value, r.most, x) >= r.cut) << (i * V::kCount + j);
        }
      int w = hits ? atomicAdd(&count, __popc(hits)) : 0;
      for (; hits && w < best.cap; hits &= hits - 1) {  // (one or two)
        const int n = __ffs(hits) - 1, i = n / V::kCount;
        uint32_t x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = i & 2 ? (i & 1 ? v[3].w[e] : v[2].w[e]) : (i & 1 ? v[1].w[e] : v[0].w[e]);
        best.list[w++] = score_of(r, b, V::pick(x, n % V::kCount), at.y - view.shift + i * kUnit + n % V::kCount);
      }
    }
  };
  // (all marked tiles, or, where there is no room for that many places, four tiles of each piece at a time)
  bool many = false;
  for (int part = -1; part < kMarkTiles / 4; ++part) {
    look(part < 0 ? ~0u : 15u << (4 * part));
    __syncthreads();
    many = place_count > kPlaces;
    if (!many) take();
    if (many != (part < 0)) break;  // all is done, or will not be
    __syncthreads();
    if (tid == 0) place_count = 0;
    __syncthreads();
  }
  __syncthreads();
  bool exact = many || count > kRanked;
  if (exact) {
    // Ties of very many.  All rows are summed again, so that a key says which is better, and the k best
    // are kept while the marked tiles go by.
    for (int b = 0; b < a.beams; ++b)
      if (base[b].kind == kLogits && base[b].value >= base[b].cut) sum_again(b);
    if (tid == 0) count = 0;
    best.floor = GroupKey::none();
    __syncthreads();
    const int marked = pieces * kScanThreads;
    for (int i0 = 0; i0 < marked; i0 += kMergeThreads) {
      const int i = i0 + tid, b = i < marked ? beam_of(i) : 0, split = i < marked ? i / kScanThreads - b * p.splits : 0;
      const uint32_t x = i < marked && base[b].kind == kLogits && split < base[b].pieces ? words[i] : 0u;
      const float s = x ? rough(base[b].value, base[b].most, unordered(x)) : kNone;
      const uint2 mark = s > kNone && s >= base[b].cut ? marks[i] : make_uint2(0u, 0u);
      uint32_t bits = mark.x;
      if (i0 == 0) {
        const GroupKey end_key = tid < a.beams && base[tid].kind == kDone ? score_of(base[tid], tid, 0.f, a.end_token) : GroupKey::none();
        best.template offer<1>(end_key, [&](const GroupKey&) { best.put(end_key); });
      }
      const int row = row0 + b;
      const RowView view = row_view<DTYPE>(a, row);
      const int end = min(view.size, p.end_unit(base[b].offset, split) * kUnit);
      const int first0 = p.begin_unit(base[b].offset, split) * kUnit + (int)mark.y * V::kCount;
      for (; __syncthreads_or(bits != 0); bits &= bits - 1)
        for (int j = 0; j < kVecs; ++j) {
          const int first = bits ? first0 + (__ffs(bits) - 1) * kTile + j * kUnit : end;
          V v;
          v.fill_none();
          if (first < end) v = load_one<DTYPE>(view, first, end);
          v.clean();
          GroupKey most = GroupKey::none();
#pragma unroll
          for (int e = 0; e < V::kCount; ++e)
            if (v.at(e) > kNone) {
              const GroupKey key = score_of(base[b], b, v.at(e), first - view.shift + e);
              if (key >= most) most = key;
            }
          best.template offer<V::kCount>(most, [&](const GroupKey& least) {
#pragma unroll
            for (int e = 0; e < V::kCount; ++e)
              if (v.at(e) > kNone) {
                const GroupKey key = score_of(base[b], b, v.at(e), first - view.shift + e);
                if (key >= least) best.put(key);
              }
          });
        }
    }
    __syncthreads();
    if (count > kRanked) best.cut(count);
  }
  // A warp for each key: its place among them.
  auto place_of_key = [&](int i, int all) {
    const GroupKey x = best.list[i];
    int before = 0;
    for (int j = lane; j < all; j += 32) before += best.list[j] >= x;
    return (int)__reduce_add_sync(~0u, before) - 1;
  };
  int held;
  for (;;) {
    const int all = count;
    for (int i = warp; i < all; i += kMergeThreads / 32) {
      const int place = place_of_key(i, all);
      if (place < a.k && lane == 0) out[place] = best.list[i];
      if (lane == 0) places[i].x = place;  // (the places are done with; there are as many at least)
    }
    held = min(all, a.k);
    __syncthreads();
    if (exact) break;
    // Is the order sure?  Neighbours of different rows, and whoever comes close to the last one.  (If two are as near as
    // the worst rows' errors, so are all between them, and the rows of both have a neighbour of another row there.)
    auto close = [&](const GroupKey& x, const GroupKey& y) {
      const int b = x.beam(), c = y.beam();
      if (b == c || fabsf((x.score() - y.score()) + (x.rest() - y.rest())) > 2.001f * worst) return false;
      atomicOr(again + (b >> 5), 1u << (b & 31));
      atomicOr(again + (c >> 5), 1u << (c & 31));
      return base[b].kind == kLogits || base[c].kind == kLogits;
    };
    bool open = false;
    for (int i = tid; i + 1 < held; i += kMergeThreads) open |= close(out[i], out[i + 1]);
    if (held == a.k)
      for (int i = tid; i < all; i += kMergeThreads)
        if (places[i].x >= a.k) open |= close(best.list[i], out[a.k - 1]);
    if (!__syncthreads_or(open)) break;
    sum_marked();
    for (int i = tid; i < all; i += kMergeThreads) {
      const GroupKey x = best.list[i];
      best.list[i] = score_of(base[x.beam()], x.beam(), x.logit(), x.token());
    }
    __syncthreads();
    exact = true;
  }
  for (int i = tid; i < a.k; i += kMergeThreads) {
    const int64_t at = (int64_t)group * a.k + i;
    const bool is = i < held;
    a.parent[at] = is ? row0 + out[i].beam() : -1;
    a.token[at] = is ? out[i].token() : -1;
    a.score[at] = is ? out[i].score() : kNone;
  }
}

int vec_logits(int dtype) { return dtype == SEMKV_F32 ? 4 : 8; }

// One CTA to each of the places that the SMs have for them (64 x 16 x 131072: 55 us; with twice as many CTAs 57, with half
// 59), whole tiles where a row has one, rows of less than two tiles whole (16 x 8 x 10000: 12 us, cut anywhere 15), and no
// more than a mark can tell apart.  The cut depends on the sizes and on whether all
// rows begin on a multiple of 16 bytes, so that equal calls give equal bits.
constexpr int kWantCtas = 152 * 4;
Pieces cut_rows(int rows, int vocab, int dtype, bool aligned) {
  const int unit = kScanThreads * vec_logits(dtype);
  Pieces p = {};
  p.aligned = aligned;
  p.units = (vocab + (aligned ? 0 : vec_logits(dtype) - 1) + unit - 1) / unit;
  int64_t share = ((int64_t)rows * p.units + kWantCtas - 1) / kWantCtas;
  if (p.units >= kVecs) share = (share + kVecs - 1) / kVecs * kVecs;
  if (share < p.units && p.units < 2 * kVecs) share = p.units;
  if (share > kVecs * kMarkTiles) share = kVecs * kMarkTiles;
  p.share = (int)share;
  p.splits = p.units % p.share == 0 ? p.units / p.share : (p.units + p.share - 2) / p.share + 1;
  p.ln_vocab = logf((float)vocab);
  p.per_split = p.splits > 1 ? 0xFFFFFFFFu / (uint32_t)p.splits + 1 : 0u;
  return p;
}

template <int DTYPE>
cudaError_t launch(const BeamArgs& a, const Pieces& p, cudaStream_t stream) {
  const unsigned ctas = (unsigned)(((int64_t)a.groups * a.beams * p.units + p.share - 1) / p.share);
  static bool ready[kAttrDevices] = {};
  cudaError_t e = once_per_device(ready, [] {
    const int bytes = merge_bytes(SEMKV_BEAM_MAX, DTYPE);
    const cudaError_t e = cudaFuncSetAttribute(beam_merge_kernel<DTYPE, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    return e == cudaSuccess ? cudaFuncSetAttribute(beam_merge_kernel<DTYPE, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) : e;
  });
  if (e != cudaSuccess) return e;
  e = launch_pdl(p.aligned ? beam_scan_kernel<DTYPE, true> : beam_scan_kernel<DTYPE, false>, dim3(ctas), dim3(kScanThreads), 0, stream, a, p);
  if (e != cudaSuccess) return e;
  const auto merge = (a.beams * p.splits) << log_sets_of(a.k) > 2 * kBatch * (kMergeThreads / 32) ? beam_merge_kernel<DTYPE, true> : beam_merge_kernel<DTYPE, false>;
  return launch_pdl(merge, dim3(a.groups), dim3(kMergeThreads), merge_bytes(a.k, DTYPE), stream, a, p);
}

}  // namespace

size_t beam_select_workspace(int groups, int beams, int vocab, int dtype, int k) {
  (void)k;
  const int rows = groups * beams;
  const int aligned = cut_rows(rows, vocab, dtype, true).splits, others = cut_rows(rows, vocab, dtype, false).splits;
  return (size_t)rows * (aligned > others ? aligned : others) * (sizeof(float4) + kScanThreads * (sizeof(uint2) + sizeof(uint32_t)));
}

cudaError_t launch_beam_select(const BeamArgs& a, int dtype, void* ws, cudaStream_t stream) {
  const int rows = a.groups * a.beams;
  const int64_t row_bytes = a.stride * (dtype == SEMKV_F32 ? 4 : 2);
  Pieces p = cut_rows(rows, a.vocab, dtype, (uintptr_t)a.logits % 16 == 0 && (rows == 1 || row_bytes % 16 == 0));
  p.sums = static_cast<float4*>(ws);
  p.marks = reinterpret_cast<uint2*>(p.sums + (size_t)rows * p.splits);
  p.words = reinterpret_cast<uint32_t*>(p.marks + (size_t)rows * p.splits * kScanThreads);
  if (dtype == SEMKV_F32) return launch<SEMKV_F32>(a, p, stream);
  return dtype == SEMKV_BF16 ? launch<SEMKV_BF16>(a, p, stream) : launch<SEMKV_F16>(a, p, stream);
}

}  // namespace semkv
