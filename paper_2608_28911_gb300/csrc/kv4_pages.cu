// kv4_pages.cu — page operations of the paged 4-bit cache: reserve, fork, free, reorder, compact.
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
// and for compact and reorder [old: n * max_pages][source: n * tokens][trades: 6 n], 32-bit words.
struct Trade;
struct PagesWs {
  int32_t* claim;   // lowest list index that names the sequence
  int32_t* offset;  // first of the i-th sequence's new pages in the list; bit 31: copy its last page
  int32_t* kept;    // (compact) flagged tokens that stay, and all tokens that there were
  int32_t* held;
  int2* pairs;      // (reserve) pages to copy: from, to
  int32_t* counters;  // [0] pages to copy, [1] new pages (-1: refused)
  int32_t* list;    // new pages, ascending
  int32_t* old;     // (compact, reorder) [n][max_pages] the sequences' pages before the call
  int32_t* source;  // (compact) [n][tokens] position of each flagged token that stays
  Trade* trades;    // (reorder) [n]
};

__host__ __device__ inline int64_t pad4(int64_t words) { return (words + 3) & ~(int64_t)3; }

int64_t ws_words(const Kv4Cache& c, int64_t n, int64_t tokens, bool compact) {
  return pad4(c.max_seqs) + pad4(n + 1) + 2 * pad4(n) + pad4(2 * n) + 4 + pad4(c.num_pages) +
         (compact ? pad4(n * c.max_pages) + pad4(n * tokens) + pad4(6 * n) : 0);
}

PagesWs carve(const Kv4Cache& c, int n, int tokens, void* ws) {
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
  p += pad4((int64_t)n * tokens);
  w.trades = reinterpret_cast<Trade*>(p);
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

// ------------------------------------------------------------- reorder ------

// Entry i of a list: the sequence that it changes, or -1 where it changes none, and what takes its place.
struct Trade {
  int seq, from;     // from: the parent's sequence, or -1
  int had, used;     // pages
  int tokens;
  int moves;         // what stood there before the call may not stand there after it
};

// `before`: the sequence was listed before.  Raises the error of an entry that is left out.
__device__ __forceinline__ Trade trade_of(const Kv4Cache& c, int n, const int32_t* seqs, const int32_t* parent, int i, bool before,
                                          bool raise) {
  const int s = seqs ? seqs[i] : i, p = parent[i];
  const int from = p >= 0 && p < n ? (seqs ? seqs[p] : p) : -1;
  const bool there = s >= 0 && s < c.max_seqs;
  const bool fine = there && !before && (p == -1 || (from >= 0 && from < c.max_seqs));
  if (!fine && raise) raise_error(c.err, kDevIndex);
  Trade t{-1, -1, 0, 0, 0, 0};
  if (there) t.had = pages_for(c, tokens_of(c, s));
  t.moves = there && (before || p != i);
  if (!fine || p == i) return t;
  t.seq = s;
  t.from = from;
  t.tokens = p >= 0 ? tokens_of(c, from) : 0;
  t.used = pages_for(c, t.tokens);
  return t;
}

// One column of a sequence's table: `mine` was there (-1: nothing), `theirs` comes.
__device__ __forceinline__ void trade_page(const Kv4Cache& c, const Trade& t, int column, int mine, int theirs) {
  const bool had = column < t.had, used = column < t.used;
  if ((had && !page_ok(c, mine)) || (used && !page_ok(c, theirs))) raise_error(c.err, kDevIndex);
  if (had && used && mine == theirs) return;  // a page that both had
  if (had && page_ok(c, mine)) atomicSub(c.refs + mine, 1);
  if (!used) return;
  c.table[(int64_t)t.seq * c.max_pages + column] = theirs;
  if (page_ok(c, theirs)) atomicAdd(c.refs + theirs, 1);
}

// Whoever becomes a branch of another takes its state before the call, whatever becomes of that one
// meanwhile.  Lists whose tables fit into the registers of one cluster: all of it is read, then the CTAs
// wait for one another, then all is written.  Latency: 3.1 us for four beams, 4.4 for 128 sequences of 240 columns; with the
// two kernels below 3.5 and 4.7, and 2 us more on the host.
constexpr int kTradeThreads = 1024, kTradeCtas = 8, kTradeHold = 8, kTradeEntries = 128;
__host__ __device__ constexpr bool trades_fit(int n, int max_pages) {
  return (n + kTradeCtas - 1) / kTradeCtas <= kTradeEntries &&
         (int64_t)((n + kTradeCtas - 1) / kTradeCtas) * max_pages <= kTradeThreads * kTradeHold;
}
__global__ void __launch_bounds__(kTradeThreads) kv4_trade_kernel(Kv4Cache c, int n, const int32_t* seqs, const int32_t* parent) {
  __shared__ Trade trades[kTradeEntries];
  pdl_wait();
  pdl_trigger();
  const int each = (n + gridDim.x - 1) / gridDim.x, first = blockIdx.x * each;
  const int count = max(0, min(each, n - first));
  for (int e = threadIdx.x >> 5; e < count; e += kTradeThreads / 32) {
    const int i = first + e, lane = threadIdx.x & 31;
    int before = 0;
    if (seqs)
      for (int j = lane; j < i; j += 32) before |= seqs[j] == seqs[i];
    before = __any_sync(~0u, before);
    const Trade t = trade_of(c, n, seqs, parent, i, before, lane == 0);
    if (lane == 0) trades[e] = t;
  }
  __syncthreads();
  int mine[kTradeHold], theirs[kTradeHold];
#pragma unroll
  for (int j = 0; j < kTradeHold; ++j) {
    const int at = j * kTradeThreads + threadIdx.x, e = at / c.max_pages, column = at - e * c.max_pages;
    mine[j] = theirs[j] = -1;
    if (e >= count || trades[e].seq < 0) continue;
    if (column < trades[e].had) mine[j] = c.table[(int64_t)trades[e].seq * c.max_pages + column];
    if (column < trades[e].used) theirs[j] = c.table[(int64_t)trades[e].from * c.max_pages + column];
  }
  asm volatile("barrier.cluster.arrive.release;\nbarrier.cluster.wait.acquire;" ::: "memory");
#pragma unroll
  for (int j = 0; j < kTradeHold; ++j) {
    const int at = j * kTradeThreads + threadIdx.x, e = at / c.max_pages, column = at - e * c.max_pages;
    if (e >= count || trades[e].seq < 0) continue;
    trade_page(c, trades[e], column, mine[j], theirs[j]);
  }
  for (int e = threadIdx.x; e < count; e += kTradeThreads)
    if (trades[e].seq >= 0) c.length[trades[e].seq] = trades[e].tokens;
}

// Longer lists take two kernels: the first notes the trades, and the tables that change as they were where somebody wants
// them.  1024 sequences of 2000 pages, half of them changed: 7 us.  Each entry looks through the whole list, so the time
// grows with its square in the end (one page each: 4096 sequences 38 us, 16384 0.25 ms, 65535 3.2 ms).
constexpr int kNoteThreads = 256;
__global__ void __launch_bounds__(kNoteThreads) kv4_note_kernel(Kv4Cache c, int n, const int32_t* seqs, const int32_t* parent, PagesWs w) {
  pdl_wait();
  pdl_trigger();
  const int i = blockIdx.x;
  int before = 0, wanted = 0;
  for (int j = threadIdx.x; j < n; j += blockDim.x) {
    wanted |= j != i && parent[j] == i;
    if (seqs) before |= j < i && seqs[j] == seqs[i];
  }
  before = __syncthreads_or(before);
  wanted = __syncthreads_or(wanted);
  const Trade t = trade_of(c, n, seqs, parent, i, before, threadIdx.x == 0);
  if (threadIdx.x == 0) w.trades[i] = t;
  if (!t.moves || !wanted) return;
  const int32_t* row = c.table + (int64_t)(seqs ? seqs[i] : i) * c.max_pages;
  int32_t* old = w.old + (int64_t)i * c.max_pages;
#pragma unroll 8
  for (int k = threadIdx.x; k < t.had; k += kNoteThreads) old[k] = row[k];
}

__global__ void __launch_bounds__(kNoteThreads) kv4_reorder_kernel(Kv4Cache c, const int32_t* parent, PagesWs w) {
  pdl_wait();
  pdl_trigger();
  const int i = blockIdx.x;
  const Trade t = w.trades[i];
  if (t.seq < 0) return;
  const int32_t* mine = c.table + (int64_t)t.seq * c.max_pages;
  const int32_t* theirs = nullptr;
  if (t.from >= 0) {
    const int p = parent[i];
    theirs = w.trades[p].moves ? w.old + (int64_t)p * c.max_pages : c.table + (int64_t)t.from * c.max_pages;
  }
  constexpr int kAhead = 8;  // of a thread's columns, all read before the first is dealt with
  for (int k0 = threadIdx.x; k0 < max(t.had, t.used); k0 += kAhead * kNoteThreads) {
    int a[kAhead], z[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int k = k0 + j * kNoteThreads;
      a[j] = k < t.had ? mine[k] : -1;
      z[j] = k < t.used ? theirs[k] : -1;
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) trade_page(c, t, k0 + j * kNoteThreads, a[j], z[j]);
  }
  if (threadIdx.x == 0) c.length[t.seq] = t.tokens;
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
  const PagesWs w = carve(c, b.n, 0, ws);
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

cudaError_t launch_kv4_reorder(const Kv4Cache& c, int n, const int32_t* seqs, const int32_t* parent, void* ws,
                               cudaStream_t stream) {
  if (trades_fit(n, c.max_pages)) {
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = n < kTradeCtas ? n : kTradeCtas;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(attr[1].val.clusterDim.x);
    cfg.blockDim = dim3(kTradeThreads);
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kv4_trade_kernel, c, n, seqs, parent);
  }
  const PagesWs w = carve(c, n, 0, ws);
  const cudaError_t e = launch_pdl(kv4_note_kernel, dim3(n), dim3(kNoteThreads), 0, stream, c, n, seqs, parent, w);
  if (e != cudaSuccess) return e;
  return launch_pdl(kv4_reorder_kernel, dim3(n), dim3(kNoteThreads), 0, stream, c, parent, w);
}

cudaError_t launch_kv4_compact(const Kv4Cache& c, int n, const int32_t* seqs, const uint8_t* keep, int tokens, void* ws,
                               int sms, cudaStream_t stream) {
  const PagesWs w = carve(c, n, tokens, ws);
  cudaError_t e = launch_pdl(kv4_keep_kernel, dim3(n), dim3(kPlanThreads), 0, stream, c, seqs, keep, tokens, w);
  if (e != cudaSuccess) return e;
  e = launch_pdl(kv4_compact_plan_kernel, dim3(1), dim3(kPlanThreads), 0, stream, c, n, seqs, tokens, w);
  if (e != cudaSuccess) return e;
  auto move = c.D == 128 ? kv4_move_kernel<128> : kv4_move_kernel<64>;
  return launch_pdl(move, dim3(n + 6 * sms), dim3(kMoveThreads), 0, stream, c, n, seqs, tokens, w);
}

}  // namespace semkv
