// kv4_pages.cu — page operations of the paged 4-bit cache: reserve, fork, free, compact.
//
// The state is three arrays: each sequence's table and length, and each page's reference
// count.  A page is free when its count is 0, so there is no free list to keep in step
// with it: a plan kernel of one CTA finds the lowest free pages with two passes over the counts
// (16 KB of L2 per 4096 pages) and hands them out by a prefix sum over the sequences'
// needs, in list order, so equal states give equal tables.  What moves rows runs after the
// plan in kernels over all SMs, bound by memory.  64 branches of 4 prompts take 21 us: free, fork, plan
// and 10 us for the 64 pages of 8 layers.  Pruning 4 sequences of about 28K to a quarter takes 81 us, of which
// the rows' move is 62, at 72% of the memory's rate: it brings whole lines of 128 bytes, twice what is kept.
#include "kernels.h"
#include "kv4.cuh"

namespace semkv {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kMoveThreads = 256;

// Workspace: [claim: max_seqs][offset: n + 1][kept: n][held: n][pairs: 2 n][counters: 4][list: num_pages]
// and for compact [old: n * max_pages][source: n * tokens], 32-bit words.
struct PagesWs {
  int32_t* claim;   // lowest list index that names the sequence
  int32_t* offset;  // first of the i-th sequence's new pages in the list; bit 31: copy its last page
  int32_t* kept;    // (compact) flagged tokens that stay, and all tokens that there were
  int32_t* held;
  int2* pairs;      // (reserve) pages to copy: from, to
  int32_t* counters;  // [0] pages to copy, [1] new pages (-1: refused)
  int32_t* list;    // new pages, ascending
  int32_t* old;     // (compact) [n][max_pages] the sequences' pages before the call
  int32_t* source;  // (compact) [n][tokens] position of each flagged token that stays
};

__host__ __device__ inline int64_t pad4(int64_t words) { return (words + 3) & ~(int64_t)3; }

int64_t ws_words(const Kv4Cache& c, int64_t n, int64_t tokens, bool compact) {
  return pad4(c.max_seqs) + pad4(n + 1) + 2 * pad4(n) + pad4(2 * n) + 4 + pad4(c.num_pages) +
         (compact ? pad4(n * c.max_pages) + pad4(n * tokens) : 0);
}

PagesWs carve(const Kv4Cache& c, int n, void* ws) {
  PagesWs w;
  int32_t* p = static_cast<int32_t*>(ws);
  w.claim = p;
  p += pad4(c.max_seqs);
  w.offset = p;
  p += pad4((int64_t)n + 1);
  w.kept = p;
  p += pad4(n);
  w.held = p;
  p += pad4(n);
  w.pairs = reinterpret_cast<int2*>(p);
  p += pad4(2 * (int64_t)n);
  w.counters = p;
  p += 4;
  w.list = p;
  p += pad4(c.num_pages);
  w.old = p;
  p += pad4((int64_t)n * c.max_pages);
  w.source = p;
  return w;
}

// ------------------------------------------------------- block helpers ------

// Exclusive prefix sum over a block of kPlanThreads; `total` for every thread.
__device__ __forceinline__ int64_t block_exclusive(int64_t x, int64_t* sums, int64_t& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int64_t y = x;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int64_t o = __shfl_up_sync(~0u, y, d);
    if (lane >= d) y += o;
  }
  __syncthreads();  // the sums of the call before have been read
  if (lane == 31) sums[warp] = y;
  __syncthreads();
  if (warp == 0) {
    int64_t z = sums[lane];
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int64_t o = __shfl_up_sync(~0u, z, d);
      if (lane >= d) z += o;
    }
    sums[lane] = z;
  }
  __syncthreads();
  total = sums[31];
  return y - x + (warp ? sums[warp - 1] : 0);
}

__device__ __forceinline__ int4 refs_at(const Kv4Cache& c, int p) {
  if (p + 3 < c.num_pages) return *reinterpret_cast<const int4*>(c.refs + p);
  int4 r = make_int4(1, 1, 1, 1);
  if (p < c.num_pages) r.x = c.refs[p];
  if (p + 1 < c.num_pages) r.y = c.refs[p + 1];
  if (p + 2 < c.num_pages) r.z = c.refs[p + 2];
  return r;
}

// The lowest `want` free pages, ascending, into `list`; returns how many there are (want or
// fewer).  Each warp counts the free pages of its own stretch, then writes them at its place.
__device__ int64_t find_free(const Kv4Cache& c, int64_t want, int32_t* list, int64_t* sums) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int stretch = ((c.num_pages + 32 * 128 - 1) / (32 * 128)) * 128;
  const int64_t begin = (int64_t)warp * stretch;
  int mine = 0;
  for (int s = 4 * lane; s < stretch && begin + s < c.num_pages; s += 128) {
    const int4 r = refs_at(c, (int)begin + s);
    mine += (r.x == 0) + (r.y == 0) + (r.z == 0) + (r.w == 0);
  }
  mine = __reduce_add_sync(~0u, mine);
  __syncthreads();
  if (lane == 0) sums[warp] = mine;
  __syncthreads();
  int64_t at = 0, total = 0;
  for (int w = 0; w < 32; ++w) {
    if (w < warp) at += sums[w];
    total += sums[w];
  }
  for (int s = 0; s < stretch && begin + s < c.num_pages && at < want; s += 128) {
    const int p = (int)begin + s + 4 * lane;
    const int4 r = p < c.num_pages ? refs_at(c, p) : make_int4(1, 1, 1, 1);
    const int z[4] = {r.x == 0, r.y == 0, r.z == 0, r.w == 0};
    const int n = z[0] + z[1] + z[2] + z[3];
    int incl = n;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int o = __shfl_up_sync(~0u, incl, d);
      if (lane >= d) incl += o;
    }
    int64_t to = at + incl - n;
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (z[k]) {
        if (to < want) list[to] = p + k;
        ++to;
      }
    at += __shfl_sync(~0u, incl, 31);
  }
  __syncthreads();
  return total < want ? total : want;
}

// claim[seq] = the lowest list index that names it
__device__ __forceinline__ void claim_all(const Kv4Cache& c, int n, const int32_t* seqs, int32_t* claim) {
  if (!seqs) return;
  for (int i = threadIdx.x; i < n; i += kPlanThreads) {
    const int s = seqs[i];
    if (s >= 0 && s < c.max_seqs) claim[s] = 0x7FFFFFFF;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += kPlanThreads) {
    const int s = seqs[i];
    if (s >= 0 && s < c.max_seqs) atomicMin(claim + s, i);
  }
  __syncthreads();
}
__device__ __forceinline__ int claimed_seq(const Kv4Cache& c, int i, const int32_t* seqs,
                                           const int32_t* claim) {
  const int s = seqs ? seqs[i] : i;
  return s >= 0 && s < c.max_seqs && (!seqs || claim[s] == i) ? s : -1;
}

__device__ __forceinline__ int tokens_of(const Kv4Cache& c, int seq) {
  // a length never reaches past its table
  const int64_t cap = (int64_t)c.max_pages << c.page_shift;
  const int t = c.length[seq];
  return t < 0 ? 0 : t > cap ? (int)cap : t;
}
__device__ __forceinline__ int pages_for(const Kv4Cache& c, int64_t tokens) {
  return (int)((tokens + c.P - 1) >> c.page_shift);
}
__device__ __forceinline__ bool page_ok(const Kv4Cache& c, int page) {
  return page >= 0 && page < c.num_pages;
}

// ------------------------------------------------------------- reserve ------

constexpr uint32_t kCopyFlag = 0x80000000u;

__global__ void __launch_bounds__(kPlanThreads) kv4_reserve_kernel(Kv4Cache c, Kv4Batch b, PagesWs w) {
  __shared__ int64_t sums[32];
  __shared__ int too_long;
  pdl_wait();
  pdl_trigger();
  if (threadIdx.x == 0) {
    too_long = 0;
    w.counters[0] = 0;
  }
  claim_all(c, b.n, b.seqs, w.claim);
  __syncthreads();
  // needs, and where each sequence's pages begin in the list
  int64_t carry = 0;
  for (int i0 = 0; i0 < b.n; i0 += kPlanThreads) {
    const int i = i0 + threadIdx.x;
    int64_t need = 0;
    bool copy = false;
    if (i < b.n) {
      const int s = claimed_seq(c, i, b.seqs, w.claim);
      int begin, count;
      if (s >= 0 && kv4_range(b, i, begin, count) && count > 0) {
        const int old = tokens_of(c, s);
        const int64_t after = (int64_t)old + count;
        if (after > (int64_t)c.max_pages << c.page_shift) {
          too_long = 1;
        } else {
          if (old & (c.P - 1)) {
            const int last = c.table[(int64_t)s * c.max_pages + (old >> c.page_shift)];
            copy = page_ok(c, last) && c.refs[last] > 1;
          }
          need = pages_for(c, after) - pages_for(c, old) + copy;
        }
      }
    }
    int64_t total;
    const int64_t at = carry + block_exclusive(need, sums, total);
    // (a sum that passes the pool's size is refused below, so 31 bits hold every used one)
    if (i < b.n) w.offset[i] = (int)((uint32_t)at | (copy ? kCopyFlag : 0u));
    carry += total;
    if (carry > c.num_pages) break;  // the same for every thread
  }
  __syncthreads();
  bool fits = !too_long && carry <= c.num_pages;
  if (fits && carry > 0) fits = find_free(c, carry, w.list, sums) == carry;
  if (threadIdx.x == 0) {
    w.counters[1] = fits ? (int)carry : -1;
    if (fits) w.offset[b.n] = (int)carry;
    if (!fits) raise_error(c.err, kDevCapacity);
  }
  __syncthreads();
  if (!fits) {
    for (int i = threadIdx.x; i < b.n; i += kPlanThreads) b.start[i] = -1;
    return;
  }
  const int lane = threadIdx.x & 31;
  for (int i = threadIdx.x >> 5; i < b.n; i += kPlanThreads / 32) {
    const int s = claimed_seq(c, i, b.seqs, w.claim);
    int begin, count;
    if (s < 0 || !kv4_range(b, i, begin, count)) {
      if (lane == 0) {
        b.start[i] = -1;
        raise_error(c.err, kDevIndex);
      }
      continue;
    }
    const int old = tokens_of(c, s);
    const uint32_t word = (uint32_t)w.offset[i];
    const int at = (int)(word & ~kCopyFlag), copy = word >> 31;
    const int need = (int)((uint32_t)w.offset[i + 1] & ~kCopyFlag) - at;
    const int column = pages_for(c, old) - copy;
    int32_t* row = c.table + (int64_t)s * c.max_pages + column;
    if (copy && lane == 0) {
      const int from = row[0];
      atomicSub(c.refs + from, 1);
      w.pairs[atomicAdd(w.counters, 1)] = make_int2(from, w.list[at]);
    }
    __syncwarp();
    for (int k = lane; k < need; k += 32) {
      const int page = w.list[at + k];
      row[k] = page;
      c.refs[page] = 1;
    }
    __syncwarp();
    if (lane == 0) {
      b.start[i] = old;
      c.length[s] = old + count;
    }
  }
}

// Whole pages, every layer: units of (pair, layer, 8 KB).
__global__ void __launch_bounds__(kMoveThreads) kv4_copy_kernel(Kv4Cache c, PagesWs w) {
  pdl_wait();
  pdl_trigger();
  if (w.counters[1] < 0) return;
  const int pairs = w.counters[0];
  const int64_t bytes = (int64_t)c.H * (kv4_tile_bytes(c.D) << (c.page_shift - 4));
  constexpr int kUnit = kMoveThreads * 16 * 2;
  const int units_per_page = (int)((bytes + kUnit - 1) / kUnit);
  const int64_t units = (int64_t)pairs * c.layers * units_per_page;
  for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
    const int part = (int)(u % units_per_page);
    const int64_t pl = u / units_per_page;
    const int layer = (int)(pl % c.layers);
    const int2 pair = w.pairs[pl / c.layers];
    const uint4* from = reinterpret_cast<const uint4*>(c.pages + kv4_record(c, layer, pair.x, 0));
    uint4* to = reinterpret_cast<uint4*>(c.pages + kv4_record(c, layer, pair.y, 0));
    const int words = (int)(bytes / 16);
    const int a = part * (kUnit / 16) + threadIdx.x, b2 = a + kMoveThreads;
    uint4 x, y;
    if (a < words) x = __ldcs(from + a);
    if (b2 < words) y = __ldcs(from + b2);
    if (a < words) to[a] = x;
    if (b2 < words) to[b2] = y;
  }
}

// ---------------------------------------------------------- fork, free ------

__global__ void __launch_bounds__(128) kv4_fork_kernel(Kv4Cache c, int n, const int32_t* src, const int32_t* dst) {
  pdl_wait();
  pdl_trigger();
  const int i = blockIdx.x;
  const int from = src[i], to = dst[i];
  // the entry's own reasons to be left out
  int wrong = from < 0 || from >= c.max_seqs || to < 0 || to >= c.max_seqs;
  for (int j = threadIdx.x; j < n; j += blockDim.x) {
    const int d = dst[j];
    wrong |= src[j] == to || d == from || (j != i && d == to);
  }
  if (__syncthreads_or(wrong)) {
    if (threadIdx.x == 0) raise_error(c.err, kDevIndex);
    return;
  }
  if (__syncthreads_or(c.length[to] != 0)) {
    if (threadIdx.x == 0) raise_error(c.err, kDevCapacity);
    return;
  }
  const int tokens = tokens_of(c, from), used = pages_for(c, tokens);
  const int32_t* a = c.table + (int64_t)from * c.max_pages;
  int32_t* z = c.table + (int64_t)to * c.max_pages;
  for (int k = threadIdx.x; k < used; k += blockDim.x) {
    const int page = a[k];
    z[k] = page;
    if (page_ok(c, page)) atomicAdd(c.refs + page, 1);
    else raise_error(c.err, kDevIndex);
  }
  if (threadIdx.x == 0) c.length[to] = tokens;
}

__global__ void __launch_bounds__(128) kv4_free_kernel(Kv4Cache c, int n, const int32_t* seqs) {
  __shared__ int held;
  pdl_wait();
  pdl_trigger();
  const int s = seqs ? seqs[blockIdx.x] : blockIdx.x;
  if (s < 0 || s >= c.max_seqs) {
    if (threadIdx.x == 0) raise_error(c.err, kDevIndex);
    return;
  }
  if (threadIdx.x == 0) {
    // whoever takes the length gives the pages back: a sequence listed twice is freed once
    const int64_t cap = (int64_t)c.max_pages << c.page_shift;
    const int t = atomicExch(c.length + s, 0);
    held = pages_for(c, t < 0 ? 0 : t > cap ? cap : t);
  }
  __syncthreads();
  const int32_t* row = c.table + (int64_t)s * c.max_pages;
  for (int k = threadIdx.x; k < held; k += blockDim.x) {
    const int page = row[k];
    if (page_ok(c, page)) atomicSub(c.refs + page, 1);
    else raise_error(c.err, kDevIndex);
  }
}

// ------------------------------------------------------------- compact ------

// Positions of the flagged tokens of one sequence, in order, and its pages as they were: the kernels
// behind read these, so that the table may change while the rows are still on their way.
__global__ void __launch_bounds__(kPlanThreads) kv4_keep_kernel(Kv4Cache c, const int32_t* seqs, const uint8_t* keep,
                                                                int tokens, PagesWs w) {
  __shared__ int64_t sums[32];
  pdl_wait();
  pdl_trigger();
  const int i = blockIdx.x, s = seqs ? seqs[i] : i;
  if (s < 0 || s >= c.max_seqs) return;
  const int held = tokens_of(c, s), flagged = held < tokens ? held : tokens;
  for (int k = threadIdx.x; k < pages_for(c, held); k += kPlanThreads)
    w.old[(int64_t)i * c.max_pages + k] = c.table[(int64_t)s * c.max_pages + k];
  const uint8_t* flags = keep + (int64_t)i * tokens;
  int32_t* source = w.source + (int64_t)i * tokens;
  const bool wide = ((uintptr_t)flags & 15) == 0;
  int64_t carry = 0;
  constexpr int kPer = 16;
  for (int t0 = 0; t0 < flagged; t0 += kPlanThreads * kPer) {
    const int t = t0 + threadIdx.x * kPer;
    uint32_t bits = 0;
    if (wide && t + kPer <= flagged) {
      const uint4 x = *reinterpret_cast<const uint4*>(flags + t);
      const uint32_t word[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
      for (int k = 0; k < kPer; ++k)
        if ((word[k / 4] >> (8 * (k % 4))) & 0xFFu) bits |= 1u << k;
    } else {
      for (int k = 0; k < kPer; ++k)
        if (t + k < flagged && flags[t + k]) bits |= 1u << k;
    }
    int64_t total;
    int64_t at = carry + block_exclusive(__popc(bits), sums, total);
    for (; bits; bits &= bits - 1) source[at++] = t + __ffs(bits) - 1;
    carry += total;
  }
  if (threadIdx.x == 0) {
    w.kept[i] = (int)carry;
    w.held[i] = held;
  }
}

// tokens that stay: the flagged ones, then all behind the flags
__device__ __forceinline__ int left_of(const PagesWs& w, int i, int tokens) {
  const int held = w.held[i];
  return w.kept[i] + (held > tokens ? held - tokens : 0);
}

__global__ void __launch_bounds__(kPlanThreads) kv4_compact_plan_kernel(Kv4Cache c, int n, const int32_t* seqs,
                                                                        int tokens, PagesWs w) {
  __shared__ int64_t sums[32];
  pdl_wait();
  pdl_trigger();
  claim_all(c, n, seqs, w.claim);
  int64_t carry = 0;
  for (int i0 = 0; i0 < n; i0 += kPlanThreads) {
    const int i = i0 + threadIdx.x;
    int64_t need = 0;
    if (i < n) {
      const int s = claimed_seq(c, i, seqs, w.claim);
      if (s >= 0) need = pages_for(c, left_of(w, i, tokens));
      else raise_error(c.err, kDevIndex);
    }
    int64_t total;
    const int64_t at = carry + block_exclusive(need, sums, total);
    if (i < n) w.offset[i] = (int)(at < c.num_pages ? at : c.num_pages);
    carry += total;
  }
  bool fits = carry <= c.num_pages;
  if (fits && carry > 0) fits = find_free(c, carry, w.list, sums) == carry;
  if (threadIdx.x == 0) {
    w.counters[1] = fits ? (int)carry : -1;
    w.offset[n] = fits ? (int)carry : 0;
    if (!fits) raise_error(c.err, kDevCapacity);
  }
}

// One piece of heads h0, h0 + step, ...: N loads on their way before the first store.
template <typename T, int N>
__device__ __forceinline__ void copy_heads(uint8_t* dst, const uint8_t* src, int64_t stride, int h0, int step, int H) {
  for (int h = h0; h < H; h += N * step) {
    T x[N];
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (h + i * step < H) x[i] = *reinterpret_cast<const T*>(src + (h + i * step) * stride);
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (h + i * step < H) *reinterpret_cast<T*>(dst + (h + i * step) * stride) = x[i];
  }
}

// The first n CTAs put a sequence's new pages in the old ones' place; the others move rows, a unit of
// one new page of one layer at a time.  A thread has a row, K or V, and a 16-byte piece of its codes for
// all heads, so that its addresses are worked out once and the heads' loads follow one another.
template <int D>
__global__ void __launch_bounds__(kMoveThreads) kv4_move_kernel(Kv4Cache c, int n, const int32_t* seqs, int tokens, PagesWs w) {
  pdl_wait();
  pdl_trigger();
  const int pages = w.counters[1];
  if (pages < 0) return;
  if ((int)blockIdx.x < n) {
    const int i = blockIdx.x, s = claimed_seq(c, i, seqs, w.claim);
    if (s < 0) return;
    const int left = left_of(w, i, tokens), used = pages_for(c, w.held[i]), need = pages_for(c, left), at = w.offset[i];
    int32_t* row = c.table + (int64_t)s * c.max_pages;
    for (int k = threadIdx.x; k < used; k += kMoveThreads) {  // (need <= used)
      const int old = w.old[(int64_t)i * c.max_pages + k];
      if (page_ok(c, old)) atomicSub(c.refs + old, 1);
      else raise_error(c.err, kDevIndex);
      if (k < need) {
        const int page = w.list[at + k];
        row[k] = page;
        c.refs[page] = 1;
      }
    }
    if (threadIdx.x == 0) c.length[s] = left;
    return;
  }
  constexpr int kTile = kv4_tile_bytes(D);
  constexpr int kCodes = D / 2 / 16;  // 16-byte pieces of a row's codes
  using Scales = typename std::conditional<D == 128, uint2, uint32_t>::type;
  const int64_t head_bytes = (int64_t)kTile << (c.page_shift - 4);
  for (int64_t u = blockIdx.x - n; u < (int64_t)pages * c.layers; u += gridDim.x - n) {
    const int k = (int)(u / c.layers), layer = (int)(u - (int64_t)k * c.layers);
    int lo = 0, hi = n - 1;  // the sequence whose new pages k is among: the last with offset <= k
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (w.offset[mid] <= k) lo = mid; else hi = mid - 1;
    }
    const int first = (k - w.offset[lo]) << c.page_shift, kept = w.kept[lo];
    const int rows = min(c.P, left_of(w, lo, tokens) - first);
    uint8_t* to = c.pages + kv4_record(c, layer, w.list[k], 0);
    // where row r of the page was, in its head 0 record
    auto from = [&](int r, int& in_tile) {
      const int j = first + r;
      const int old = j < kept ? w.source[(int64_t)lo * tokens + j] : tokens + (j - kept);
      int page = w.old[(int64_t)lo * c.max_pages + (old >> c.page_shift)];
      if (!page_ok(c, page)) {
        raise_error(c.err, kDevIndex);
        page = 0;
      }
      const int in_page = old & (c.P - 1);
      in_tile = in_page & 15;
      return c.pages + kv4_record(c, layer, page, 0) + (in_page >> 4) * kTile;
    };
    // pieces of codes, then of scales; with fewer of them than threads the heads are shared out
    auto pieces = [&](int total, auto body) {
      const int share = total >= kMoveThreads ? 1 : kMoveThreads / total;
      if ((int)threadIdx.x >= total * share && share > 1) return;
      const int h0 = share > 1 ? threadIdx.x / total : 0;
      for (int x = share > 1 ? threadIdx.x - h0 * total : threadIdx.x; x < total; x += kMoveThreads) body(x, h0, share);
    };
    pieces(rows * 2 * kCodes, [&](int x, int h0, int step) {
      const int piece = x % kCodes, v = x / kCodes & 1, r = x / (2 * kCodes);
      int in_tile;
      const uint8_t* src = from(r, in_tile);
      src += v * 8 * D + in_tile * (D / 2) + piece * 16;
      uint8_t* dst = to + (r >> 4) * kTile + v * 8 * D + (r & 15) * (D / 2) + piece * 16;
      copy_heads<uint4, 8>(dst, src, head_bytes, h0, step, c.H);
    });
    pieces(rows * 2, [&](int x, int h0, int step) {
      const int v = x & 1, r = x >> 1;
      int in_tile;
      const uint8_t* src = from(r, in_tile);
      src += 16 * D + v * D + in_tile * (D / 16);
      uint8_t* dst = to + (r >> 4) * kTile + 16 * D + v * D + (r & 15) * (D / 16);
      copy_heads<Scales, 8>(dst, src, head_bytes, h0, step, c.H);
    });
  }
}

}  // namespace

size_t kv4_pages_workspace(const Kv4Cache& c, int n, int tokens, bool compact) {
  return (size_t)ws_words(c, n, tokens, compact) * 4;
}

cudaError_t launch_kv4_reserve(const Kv4Cache& c, const Kv4Batch& b, void* ws, int sms, cudaStream_t stream) {
  const PagesWs w = carve(c, b.n, ws);
  cudaError_t e = launch_pdl(kv4_reserve_kernel, dim3(1), dim3(kPlanThreads), 0, stream, c, b, w);
  if (e != cudaSuccess) return e;
  const int64_t bytes = (int64_t)c.H * (kv4_tile_bytes(c.D) << (c.page_shift - 4));
  const int64_t most = (int64_t)b.n * c.layers * ((bytes + 8191) / 8192), grid = most < 4 * sms ? most : 4 * sms;
  return launch_pdl(kv4_copy_kernel, dim3((unsigned)grid), dim3(kMoveThreads), 0, stream, c, w);
}

cudaError_t launch_kv4_fork(const Kv4Cache& c, int n, const int32_t* src, const int32_t* dst, cudaStream_t stream) {
  return launch_pdl(kv4_fork_kernel, dim3(n), dim3(128), 0, stream, c, n, src, dst);
}

cudaError_t launch_kv4_free(const Kv4Cache& c, int n, const int32_t* seqs, cudaStream_t stream) {
  return launch_pdl(kv4_free_kernel, dim3(n), dim3(128), 0, stream, c, n, seqs);
}

cudaError_t launch_kv4_compact(const Kv4Cache& c, int n, const int32_t* seqs, const uint8_t* keep, int tokens, void* ws,
                               int sms, cudaStream_t stream) {
  const PagesWs w = carve(c, n, ws);
  cudaError_t e = launch_pdl(kv4_keep_kernel, dim3(n), dim3(kPlanThreads), 0, stream, c, seqs, keep, tokens, w);
  if (e != cudaSuccess) return e;
  e = launch_pdl(kv4_compact_plan_kernel, dim3(1), dim3(kPlanThreads), 0, stream, c, n, seqs, tokens, w);
  if (e != cudaSuccess) return e;
  auto move = c.D == 128 ? kv4_move_kernel<128> : kv4_move_kernel<64>;
  return launch_pdl(move, dim3(n + 6 * sms), dim3(kMoveThreads), 0, stream, c, n, seqs, tokens, w);
}

}  // namespace semkv
