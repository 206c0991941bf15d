// kv4_chunk.cu — attention over the paged 4-bit cache for many query rows (chunks of prompts, whole
// prompts), bound by the tensor cores.
//
// One CTA per SM over its range of the batch's work (kv4_attend.cuh).  A tile is two blocks of 128
// query rows; for each unit of 128 tokens
//   S_t = Q_t K^T      tcgen05.mma, 128 x 128 x D, fp16, sums in tensor memory
//   P_t = 2^(S_t - e)  one thread per row; P_t (fp16) takes S_t's place in tensor memory
//   O_t += P_t V       tcgen05.mma with P_t read from tensor memory
// so that 256 rows share the work of turning a unit's codes into fp16, and one block's softmax runs
// while the other's products do.  Sixteen warps:
//   0-3, 4-7  the softmax of block 0 and 1 (a warp's tensor memory lanes are those of warp % 4)
//   8-11      the unit's codes to fp16 K and V in shared memory, two buffers each, the codes
//             loaded into registers a unit ahead and the page numbers two
//   12        issues the products
//   13-15     the query rows, those of the next item while the last unit of this one is at work
// One of the last walks the range and hands its items to all through a ring in shared memory.
// A softmax thread holds its row's 128 logits of a unit in registers, so tensor memory is read once
// for them: the warpgroups share the launch's 4 x 128 registers a thread as 184, 184, 80, 64.
// The core matrices (8 rows of 16 bytes) of a K or V unit lie 128 bytes apart along the head dim and
// 16 D bytes apart along the tokens.  That is K-major for S (head dim is its K) and MN-major for
// O (head dim is its N), so V needs no transposition, and eight lanes storing one 16-byte piece
// of eight tokens fill 128 bytes: no bank conflicts.
// The reference exponent e of a row moves only when a weight would pass 2^15; its thread then
// rescales its row of O, which no product touches at that time: the one before has completed
// (S_t's barrier, which follows it, tells) and the next waits for P_t.
// Two blocks and a unit of 128 take 3050 cycles of an SM, of which the products are 2350 at the rate of the
// peak and the operands' trips through shared memory 2050: 2048 tokens over 30K run at 1.49 PFLOP/s, 79% of a
// large library product, from a captured graph (655 us), and at 1.45, 77%, as calls among others (670 us).  An item
// costs about 10000 cycles besides, mostly for its results and the unit on its diagonal.
// A tile of one block only (a few tokens of a large group, the end of a chunk) has both halves work on it:
// they take its units in turn, and the first puts the two sums together, which halves its time.
// Tensor memory: S_0, S_1, O_0, O_1, 128 columns each.
#include "kernels.h"
#include "kv4_attend.cuh"

namespace semkv {
namespace {

constexpr int kUnit = Kv4ManyCut::unit;
constexpr int kThreads = 16 * 32;
constexpr int kBlock = 128;     // rows of a block

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

// A whole warp's wait with a limit: false after kWaitPolls polls, or soon after another wait of the CTA
// ran out.
__device__ __forceinline__ bool wait(uint64_t* bar, uint32_t parity, volatile int* failed) {
  const uint32_t at = smem_addr(bar);
  for (uint32_t i = 0; i < kWaitPolls; ++i) {
    uint32_t ok;
    asm volatile(
        "{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}"
        : "=r"(ok)
        : "r"(at), "r"(parity)
        : "memory");
    if (__all_sync(~0u, ok)) return true;
    if ((i & 255) == 255 && __any_sync(~0u, *failed)) return false;
  }
  *failed = 1;
  return false;
}
__device__ __forceinline__ void arrive(uint64_t* bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_addr(bar)) : "memory");
}

// Shared-memory matrix descriptors without swizzle: start (bits 0-13), leading (16-29) and stride
// (32-45) offsets in 16 bytes, version 1 (46).  K-major: leading = next core matrix along K,
// stride = next eight rows; MN-major: leading = next eight along K, stride = next core matrix along
// the rows.  The low word, to which a step along K is added, and the high word.
__device__ __forceinline__ uint32_t desc_low(uint32_t at, uint32_t leading) { return at >> 4 | leading >> 4 << 16; }
__device__ constexpr uint32_t desc_high(uint32_t stride) { return stride >> 4 | 1u << 14; }
// fp16 operands, fp32 sums, M = 128; bit 16: B is MN-major
__device__ constexpr uint32_t instr_desc(int n, bool b_mn) {
  return (1u << 4) | (b_mn ? 1u << 16 : 0u) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(kBlock >> 4) << 24);
}
// The products of one warp, which runs convergent so that their operands stay in uniform registers:
// `leader` holds in the one lane that issues them.  Issued from a branch of that lane alone,
// each took 120 cycles, twice what the product takes.
__device__ __forceinline__ void mma_ss(uint32_t leader, uint32_t d, uint32_t a, uint32_t b, uint32_t high, uint32_t idesc,
                                       uint32_t add) {
  asm volatile(
      "{\n .reg .pred p, l;\n .reg .b64 x, y;\n setp.ne.u32 l, %0, 0;\n setp.ne.u32 p, %6, 0;\n mov.b64 x, {%2, %4};\n"
      " mov.b64 y, {%3, %4};\n @l tcgen05.mma.cta_group::1.kind::f16 [%1], x, y, %5, p;\n}" ::"r"(leader),
      "r"(d), "r"(a), "r"(b), "r"(high), "r"(idesc), "r"(add)
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t leader, uint32_t d, uint32_t a, uint32_t b, uint32_t high, uint32_t idesc,
                                       uint32_t add) {
  asm volatile(
      "{\n .reg .pred p, l;\n .reg .b64 y;\n setp.ne.u32 l, %0, 0;\n setp.ne.u32 p, %6, 0;\n mov.b64 y, {%3, %4};\n"
      " @l tcgen05.mma.cta_group::1.kind::f16 [%1], [%2], y, %5, p;\n}" ::"r"(leader),
      "r"(d), "r"(a), "r"(b), "r"(high), "r"(idesc), "r"(add)
      : "memory");
}
__device__ __forceinline__ uint32_t elect() {
  uint32_t leader;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xFFFFFFFF;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(leader));
  return leader;
}
__device__ __forceinline__ void commit(uint32_t leader, uint64_t* bar) {
  asm volatile(
      "{\n .reg .pred l;\n setp.ne.u32 l, %1, 0;\n"
      " @l tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}" ::"r"(smem_addr(bar)),
      "r"(leader)
      : "memory");
}
#define SEMKV_R8(v, i) "=r"(v[i]), "=r"(v[i + 1]), "=r"(v[i + 2]), "=r"(v[i + 3]), "=r"(v[i + 4]), "=r"(v[i + 5]), "=r"(v[i + 6]), "=r"(v[i + 7])
#define SEMKV_U8(v, i) "+r"(v[i]), "+r"(v[i + 1]), "+r"(v[i + 2]), "+r"(v[i + 3]), "+r"(v[i + 4]), "+r"(v[i + 5]), "+r"(v[i + 6]), "+r"(v[i + 7])
#define SEMKV_I8(v, i) "r"(v[i]), "r"(v[i + 1]), "r"(v[i + 2]), "r"(v[i + 3]), "r"(v[i + 4]), "r"(v[i + 5]), "r"(v[i + 6]), "r"(v[i + 7])
// 32 columns of the warp's lanes, and the wait for them (which takes the registers, so that no use
// moves above it)
__device__ __forceinline__ void tmem_load(uint32_t at, uint32_t (&v)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,"
      "%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : SEMKV_R8(v, 0), SEMKV_R8(v, 8), SEMKV_R8(v, 16), SEMKV_R8(v, 24)
      : "r"(at));
}
__device__ __forceinline__ void tmem_wait(uint32_t (&v)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : SEMKV_U8(v, 0), SEMKV_U8(v, 8), SEMKV_U8(v, 16), SEMKV_U8(v, 24)
               :
               : "memory");
}
// 16 columns, waited for
__device__ __forceinline__ void tmem_load16(uint32_t at, uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n"
      "tcgen05.wait::ld.sync.aligned;"
      : SEMKV_R8(v, 0), SEMKV_R8(v, 8)
      : "r"(at)
      : "memory");
}
__device__ __forceinline__ void tmem_store16(uint32_t at, const uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};" ::SEMKV_I8(v, 0),
      SEMKV_I8(v, 8), "r"(at)
      : "memory");
}
__device__ __forceinline__ void tmem_store(uint32_t at, const uint32_t (&v)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,"
      "%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};" ::SEMKV_I8(v, 0),
      SEMKV_I8(v, 8), SEMKV_I8(v, 16), SEMKV_I8(v, 24), "r"(at)
      : "memory");
}
__device__ __forceinline__ void tmem_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

constexpr int kWalkBytes = 384, kBarBytes = 32 * 8;

template <int D>
struct Layout {
  static constexpr int kTile = kBlock * D * 2;        // a block of Q, or a unit of K or V, in fp16
  static constexpr int kChunk = 128;                  // next core matrix along the head dim
  static constexpr int kGroup = D / 8 * 128;          // next eight rows
  static constexpr int v(int b) { return b * kTile; }
  static constexpr int k(int b) { return (2 + b) * kTile; }
  static constexpr int q(int t) { return (4 + t) * kTile; }
  static constexpr int prefix() { return 6 * kTile; }
  static constexpr int undo() { return prefix() + (kThreads + 2) * 8; }
  static constexpr int other() { return undo() + 4 * kBlock * 4; }
  static constexpr int sums() { return other() + kBlock * 8; }
  static constexpr int bars() { return sums() + 16 * 8; }
  static constexpr int walk() { return bars() + kBarBytes; }
  static constexpr int bytes() { return walk() + kWalkBytes; }
};

constexpr int kItems = 4;  // of the ring that hands items from warp to warp

// The barriers, and the two words behind them.
struct Bars {
  uint64_t i_full[kItems], i_empty[kItems], q_full[2], q_empty[2], k_full[2], v_full[2], k_empty[2], v_empty[2], s_full[2], p_full[2], o_full[2], x_full, x_empty, drain;
  int failed;
  uint32_t tmem;
};
static_assert(sizeof(Bars) <= kBarBytes, "room for the barriers");

// An item and this CTA's part of it.
struct Item {
  int seq, begin, count, length;  // its sequence (Kv4Seq)
  int head, tile, rows;           // rows: of this tile
  int u0, u1;                     // units of this part
  int first, last;                // units of the item
  int parts;                      // workers that share it, where it begins and does not end here; else 0
};
// What the join has to know of an item that a worker begins and does not end: its first row (of those of all
// query heads), rows | parts << 16, V's scale.  (With the join looking for it six ragged prompts took 236 us, not the 232
// of that time.)
struct Kv4Join {
  int64_t first_row;
  uint32_t rows_parts;
  float gv;
};
static_assert(sizeof(Kv4Join) == sizeof(int4), "stored as one");

// A walk over the CTA's range: found once, then from item to item.  One warp walks and hands the items
// to the others through a ring in shared memory; an item without rows ends it.
struct Walk {
  Kv4Seq s;
  int i, head, tile;
  int off;       // places of the item that are behind the walk
  int64_t left;  // places of the range before it
  Kv4Ranges ranges;
  Item items[kItems];

  __device__ __forceinline__ void start(const Kv4Attend& a, const Kv4ManyCut& cut, const int64_t* prefix, const Kv4Ranges& all) {
    const int64_t place = all.begin(blockIdx.x), end = all.begin(blockIdx.x + 1);
    int64_t at;
    int which;
    const Kv4Seq q = kv4_find<kThreads>(a, cut, prefix, place, at, which);
    const int64_t head_length = cut.before(a, q, q.tiles);
    const int h = (int)kv4_div(place - at, head_length);
    const int64_t in_head = place - at - h * head_length;
    const int t = cut.find(a, q, in_head);
    if ((threadIdx.x & 31) == 0) {
      s = q;
      i = which;
      head = h;
      tile = t;
      off = (int)(in_head - cut.before(a, q, t));
      left = end - place;
      ranges = all;
    }
    __syncwarp();
  }

  // The next item with units in the range into x; without rows at the range's end.
  __device__ __forceinline__ void next(const Kv4Attend& a, const Kv4ManyCut& cut, Item& x) {
    Kv4Seq q = s;
    int which = i, h = head, t = tile, o = off;
    int64_t more = left;
    bool found = false;
    while (more > 0 && !found) {
      if (t == q.tiles) {
        t = 0;
        if (++h == a.c.H) {
          h = 0;
          do {
            if (++which >= a.b.n) break;
            q = cut.seq(a, which, false);
          } while (q.tiles == 0);
          if (which >= a.b.n) break;
        }
      }
      const int length = cut.length(a, q, t), take = more < length - o ? (int)more : length - o;
      int from;
      cut.units(a, q, t, x.first, x.last, from);
      // the unit whose place (that of its first token) is the first at or behind p
      auto unit_at = [&](int p) {
        return p <= cut.start ? x.first : min(x.last, (from + p - cut.start + kUnit - 1) / kUnit);
      };
      x.u0 = unit_at(o);
      x.u1 = o + take >= length ? x.last : unit_at(o + take);
      x.head = h;
      x.tile = t;
      x.rows = min(cut.rows, (q.count - t * cut.tokens) * a.group);
      x.parts = 0;
      if (x.u0 == x.first && x.u1 < x.last && x.u1 > x.u0) {
        // (the range ends in it) the range of its last unit's place
        const int last = cut.start + max(0, (x.last - 1) * kUnit - from);
        x.parts = ranges.owner(ranges.begin(blockIdx.x + 1) + (last - (o + take))) - (int)blockIdx.x + 1;
      }
      ++t;
      o = 0;
      more -= take;
      found = take > 0 && x.u1 > x.u0;
    }
    if (!found) x.rows = 0;
    x.seq = q.seq, x.begin = q.begin, x.count = q.count, x.length = q.length;
    __syncwarp();  // the lanes have read the fields
    if ((threadIdx.x & 31) == 0) {
      s = q;
      i = which, head = h, tile = t, off = o;
      left = more;
    }
    __syncwarp();
  }
};

// A warp's place in the ring of items.
struct Feed {
  Bars* bars;
  const Item* items;
  uint32_t n = 0;
  // the next item; null at the end, or when a wait ran out
  __device__ __forceinline__ const Item* next() {
    const uint32_t slot = n % kItems;
    if (!wait(&bars->i_full[slot], n / kItems & 1, &bars->failed)) return nullptr;
    return items[slot].rows ? items + slot : nullptr;
  }
  // this warp wants nothing more of it
  __device__ __forceinline__ void done() {
    __syncwarp();
    if ((threadIdx.x & 31) == 0) arrive(&bars->i_empty[n % kItems]);
    ++n;
  }
};

static_assert(sizeof(Walk) <= kWalkBytes, "room for the walks");

// ------------------------------------------------------------- queries ------

// Q's rows into shared memory as the first operand of S: eight rows at a time, a lane a quarter of
// row l % 8.  Two sets of factors, by the item's parity: the softmax of one item may still want
// its own while the next one's rows are put in place.
template <int D, bool BF16>
__device__ __forceinline__ void query_warps(const Kv4Attend& a, const Kv4ManyCut& cut, Walk& walk, uint8_t* smem, Bars* bars, float* undo) {
  using L = Layout<D>;
  constexpr int kPieces = D / 32;  // 16-byte pieces of a quarter
  const int lane = threadIdx.x & 31, warp = (threadIdx.x >> 5) - 13;
  const int r8 = lane & 7, q = lane >> 3;
  const uint32_t sign = a.scale_log2 < 0.f ? 0x80008000u : 0u;  // a negative scale goes into Q's signs: the largest
  volatile int* failed = &bars->failed;                            // logit is S's largest
  uint32_t n[2] = {0, 0}, published = 0;
  bool ended = false;
  // warp 2 walks, two items ahead of these warps' own
  auto publish = [&] {
    Item x;
    walk.next(a, cut, x);
    const uint32_t slot = published % kItems;
    if (!wait(&bars->i_empty[slot], (published / kItems & 1) ^ 1, failed)) return;
    if (lane == 0) {
      if (x.rows && x.parts) {
        const Kv4Join join{(int64_t)(x.begin + x.tile * cut.tokens) * a.q_heads + x.head * a.group,
                           (uint32_t)x.rows | (uint32_t)x.parts << 16,
                           a.c.v_scale ? a.c.v_scale[a.layer * a.c.H + x.head] : 1.f};
        a.joins[blockIdx.x] = *reinterpret_cast<const int4*>(&join);
      }
      walk.items[slot] = x;
      arrive(&bars->i_full[slot]);
    }
    __syncwarp();
    ++published;
    ended = x.rows == 0;
  };
  if (warp == 2) {
    publish();
    if (!ended) publish();
  }
  Feed feed{bars, walk.items};
  while (const Item* item = feed.next()) {
    const Item& it = *item;
    const uint16_t* base = a.q + (int64_t)(it.begin + it.tile * cut.tokens) * a.q_stride + it.head * a.group * D;
    // the rows come nearer while those before them are still wanted
    for (int x = warp * 32 + lane; x < it.rows * (D / 64); x += 96) {
      const int in_tile = x / (D / 64), j = cut.token_of(in_tile);
      const uint16_t* at = base + (int64_t)j * a.q_stride + (in_tile - j * a.group) * D + x % (D / 64) * 64;
      asm volatile("prefetch.global.L2 [%0];" ::"l"(at));
    }
    for (int t = 0; t < 2 && t * kBlock < it.rows; ++t) {
      if (!wait(&bars->q_empty[t], (n[t] & 1) ^ 1, failed)) return;
      ++n[t];
      // all rows on their way at once, straight to their places; a lane turns what it copied itself
      uint8_t* to = smem + L::q(t) + warp * L::kGroup + r8 * 16 + q * kPieces * L::kChunk;
#pragma unroll 2
      for (int group = warp; group < kBlock / 8; group += 3) {
        const int in_tile = t * kBlock + group * 8 + r8, j = cut.token_of(in_tile);
        const uint32_t bytes = in_tile < it.rows ? 16 : 0;  // (0: the piece is filled with zeros)
        const uint16_t* src = bytes ? base + (int64_t)j * a.q_stride + (in_tile - j * a.group) * D + q * (D / 4) : a.q;
        const uint32_t dst = smem_addr(to + (group - warp) * L::kGroup);
#pragma unroll
        for (int c = 0; c < kPieces; ++c)
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst + c * L::kChunk), "l"(src + 8 * c), "r"(bytes)
                       : "memory");
      }
      asm volatile("cp.async.wait_all;" ::: "memory");
      if (BF16 || sign) {
#pragma unroll 1
        for (int group = warp; group < kBlock / 8; group += 3) {
          uint4 x[kPieces];
          uint4* at = reinterpret_cast<uint4*>(to + (group - warp) * L::kGroup);
#pragma unroll
          for (int c = 0; c < kPieces; ++c) x[c] = at[c * (L::kChunk / 16)];
          uint64_t by2 = 0;
          if (BF16) {
            uint32_t m = 0;  // largest magnitudes, pairwise
#pragma unroll
            for (int c = 0; c < kPieces; ++c) {
              const uint32_t w[4] = {x[c].x, x[c].y, x[c].z, x[c].w};
#pragma unroll
              for (int i = 0; i < 4; ++i) asm("max.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(w[i] & 0x7FFF7FFFu));
            }
            float most = fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xFFFF0000u)), back;
            most = fmaxf(most, __shfl_xor_sync(~0u, most, 8));
            most = fmaxf(most, __shfl_xor_sync(~0u, most, 16));
            const float by = query_factor(most, back);
            by2 = sign ? pair(-by, -by) : pair(by, by);
            if (q == 0) undo[(feed.n & 1) * 2 * kBlock + t * kBlock + group * 8 + r8] = back;
          }
#pragma unroll
          for (int c = 0; c < kPieces; ++c) {
            uint32_t w[4] = {x[c].x, x[c].y, x[c].z, x[c].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              if (BF16) {
                float lo, hi;
                unpair(pair_mul(pair(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u)), by2), lo, hi);
                w[i] = pack_half2(lo, hi);
              } else {
                w[i] ^= sign;
              }
            }
            at[c * (L::kChunk / 16)] = make_uint4(w[0], w[1], w[2], w[3]);
          }
        }
      }
      fence_smem();
      __syncwarp();
      if (lane == 0) arrive(&bars->q_full[t]);
    }
    if (warp == 2 && !ended) publish();
    feed.done();
  }
  // the products have read the last rows (their barriers outlive the arrivals)
  for (int t = 0; t < 2; ++t)
    if (n[t] && !wait(&bars->q_empty[t], (n[t] & 1) ^ 1, failed)) return;
}

// ------------------------------------------------------------- softmax ------

// A row's state between the units of an item.
struct RowState {
  float ref, sum;
  uint32_t s_phase;
  bool ok;
};
// The rest of an item from its first far logit (kFar) on, the logits of unit u being in S: what the loop in
// softmax_warps does, with the products rounded first.  A function of its own, called where the largest logit
// is known: 2048 tokens over 30K take 656 us with it and 653 without, six ragged prompts 219 and 216; as a
// branch of the loop it cost 666 to 700 and 221 to 226.
template <int D>
__device__ __noinline__ RowState far_units(RowState x, uint32_t S, uint32_t O, float mul, int lo, int hi, int u, int u0, int u1, int step,
                                           uint64_t* s_full, uint64_t* p_full, volatile int* failed) {
  for (;;) {
    float top = -INFINITY;
#pragma unroll 1
    for (int c = 0; c < kUnit; c += 16) {
      uint32_t v[16];
      tmem_load16(S + c, v);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int pos = u * kUnit + c + i;
        top = fmaxf(top, pos < lo || pos > hi ? -INFINITY : __uint_as_float(v[i]));
      }
    }
    top *= mul;
    const bool over = top - x.ref > kMost;
    if (__any_sync(~0u, over)) {
      float f = 1.f;
      if (over) {
        const float to = reference_for(top);
        f = exp2_approx(x.ref - to);
        x.ref = to;
        x.sum *= f;
      }
      if (u != u0) {
#pragma unroll 1
        for (int c = 0; c < D; c += 16) {
          uint32_t o[16];
          tmem_load16(O + c, o);
#pragma unroll
          for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
          tmem_store16(O + c, o);
        }
      }
    }
#pragma unroll 1
    for (int c = 0; c < kUnit; c += 32) {
      uint32_t v[32], w[16];
      tmem_load(S + c, v);
      tmem_wait(v);
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        const int pos = u * kUnit + c + i;
        // (scalar: of a packed product and a packed sum one fused operation was made)
        const float e = exp2_approx(__fsub_rn(__fmul_rn(__uint_as_float(v[i]), mul), x.ref));
        v[i] = pos < lo || pos > hi ? 0u : __float_as_uint(e);
        x.sum += __uint_as_float(v[i]);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) w[i] = pack_half2(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1]));
      tmem_store16(S + c / 2, w);
    }
    tmem_stored();
    fence_before();
    __syncwarp();
    if ((threadIdx.x & 31) == 0) arrive(p_full);
    u += step;
    if (u >= u1) return x;
    x.ok = wait(s_full, x.s_phase, failed);
    x.s_phase ^= 1;
    if (!x.ok) return x;
    fence_after();
  }
}

template <int D, bool BF16>
__device__ __forceinline__ void softmax_warps(const Kv4Attend& a, const Kv4ManyCut& cut, Walk& walk, const float* undo, float2* other, Bars* bars, uint32_t tmem) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int t = warp >> 2, r = (warp & 3) * 32 + lane;
  const uint32_t lanes = (uint32_t)(warp & 3) << 21;  // the warp's tensor memory lanes
  const uint32_t S = tmem + lanes + 128 * t, O = tmem + lanes + 256 + 128 * t;
  volatile int* failed = &bars->failed;
  uint32_t s_phase = 0, o_phase = 0, x_phase = 0;
  Feed feed{bars, walk.items};
  for (; const Item* item = feed.next(); feed.done()) {
    const Item& it = *item;
    // with one block of rows both halves work on it, in turn unit by unit, and the first puts the two
    // results together
    const bool split = it.rows <= kBlock;
    const int u0 = it.u0 + (split ? t : 0), u1 = it.u1, step = split ? 2 : 1;
    if (u0 >= u1) continue;
    const int rr = split ? r : t * kBlock + r;  // this thread's row of the tile
    const float gk = a.c.k_scale ? a.c.k_scale[a.layer * a.c.H + it.head] : 1.f;
    const float gv = a.c.v_scale ? a.c.v_scale[a.layer * a.c.H + it.head] : 1.f;
    const float scale = fabsf(a.scale_log2) * gk;
    float mul = 0.f;
    // the positions that the row sees (a row that is not there sees all: its zeros are nobody's)
    auto sight = [&](int& lo, int& hi) {
      lo = 0, hi = 0x7FFFFFFF;
      if (rr < it.rows) {
        hi = it.length - it.count + it.tile * cut.tokens + cut.token_of(rr);
        lo = a.window && hi >= a.window ? hi - a.window + 1 : 0;
      }
    };
    int most_lo, least_hi;
    sight(most_lo, least_hi);
    most_lo = __reduce_max_sync(~0u, most_lo), least_hi = __reduce_min_sync(~0u, least_hi);
    float ref = kNone, sum = 0.f;
    bool ok = true;
    for (int u = u0; u < u1; u += step) {
      ok = wait(&bars->s_full[t], s_phase, failed);
      s_phase ^= 1;
      if (!ok) break;
      fence_after();
      // (S is there, so Q was; never 0: a masked logit stays -infinity)
      if (u == u0) mul = fmaxf(BF16 ? scale * undo[(feed.n & 1) * 2 * kBlock + rr] : scale, 0x1p-126f);
      const int pos = u * kUnit;
      const bool open = pos >= most_lo && pos + kUnit - 1 <= least_hi;
      // the reference exponent for a unit whose largest logit is `top`, and the sums with it
      auto settle = [&](float top) {
        const bool over = top > ref + kMost;
        if (!__any_sync(~0u, over)) return;
        float f = 1.f;
        if (over) {
          f = exp2_approx(ref - (top - kHead));
          ref = top - kHead;
          sum *= f;
        }
        if (u == u0) return;
#pragma unroll 1
        for (int c = 0; c < D / 16; ++c) {
          uint32_t o[16];
          tmem_load16(O + 16 * c, o);
#pragma unroll
          for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
          tmem_store16(O + 16 * c, o);
        }
      };
      // the weights of 32 logits: those of columns 2 i, 2 i + 1 into w[i]
      uint64_t sums[2] = {0, 0};
      auto turn = [&](const uint32_t(&v)[32], uint64_t mul2, uint64_t ref2, uint32_t(&w)[16]) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          float x, y;
          unpair(pair_fma(pair(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1])), mul2, ref2), x, y);
          x = exp2_approx(x);
          y = exp2_approx(y);
          sums[i & 1] = pair_add(sums[i & 1], pair(x, y));
          w[i] = pack_half2(x, y);
        }
      };
      auto largest = [](const uint32_t(&v)[32]) {
        float m[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int i = 0; i < 32; i += 2)
          asm("max.f32 %0, %0, %1, %2;" : "+f"(m[i >> 1 & 1]) : "f"(__uint_as_float(v[i])), "f"(__uint_as_float(v[i + 1])));
        return fmaxf(m[0], m[1]);
      };
      if (__builtin_expect(!open, 0)) {
        // a unit that some row sees a part of: what is hidden becomes -infinity where it lies.  A warp's rows are a
        // few tokens, so that of its groups of 32 positions one or two are hidden in part and need a look.
        // (With a loop of its own for such units, which took 6600 cycles, six ragged prompts took 239 us, not the 232 of
        // that time.)
        int lo, hi;
        sight(lo, hi);
#pragma unroll 1
        for (int c = 0; c < kUnit; c += 32) {
          const int from = lo - pos - c, to = hi - pos - c;  // this row sees from .. to of the 32
          if (__all_sync(~0u, from <= 0 && to >= 31)) continue;
          const uint32_t seen = from > 31 || to < 0 ? 0u : ~0u << max(from, 0) & ~0u >> (31 - min(to, 31));
          uint32_t v[32];
          tmem_load(S + c, v);
          tmem_wait(v);
#pragma unroll
          for (int i = 0; i < 32; ++i)
            if (!(seen >> i & 1)) v[i] = 0xFF800000u;
          tmem_store(S + c, v);
        }
        tmem_stored();
      }
      uint32_t v[kUnit / 32][32];
      float top = -INFINITY;
      tmem_load(S, v[0]);
#pragma unroll
      for (int c = 0; c < kUnit / 32; ++c) {
        tmem_wait(v[c]);
        if (c + 1 < kUnit / 32) tmem_load(S + 32 * (c + 1), v[c + 1]);  // on its way behind this one's maximum
        top = fmaxf(top, largest(v[c]));
      }
      if (__builtin_expect(__any_sync(~0u, fabsf(top * mul) > kFar && top > -INFINITY), 0)) {
        int lo, hi;
        sight(lo, hi);
        const RowState x = far_units<D>({ref, sum, s_phase, true}, S, O, mul, lo, hi, u, u0, u1, step, &bars->s_full[t], &bars->p_full[t], failed);
        ref = x.ref, sum = x.sum, s_phase = x.s_phase, ok = x.ok;
        break;
      }
      settle(top * mul);
      const uint64_t mul2 = pair(mul, mul), ref2 = pair(-ref, -ref);
#pragma unroll
      for (int c = 0; c < kUnit / 32; ++c) {
        uint32_t w[16];
        turn(v[c], mul2, ref2, w);
        tmem_store16(S + 16 * c, w);  // in S's place
      }
      {
        float x, y;
        unpair(pair_add(sums[0], sums[1]), x, y);
        sum += x + y;
      }
      tmem_stored();
      fence_before();
      __syncwarp();
      if (lane == 0) arrive(&bars->p_full[t]);
    }
    // ---- while the last products run: where the row goes, or this range's part of it
    const bool done = it.u0 == it.first && it.u1 == it.last;
    const int64_t at = (int64_t)(it.begin + it.tile * cut.tokens) * a.q_heads + it.head * a.group +
                       cut.token_of(rr) * (a.q_heads - a.group) + rr;
    float* part = a.parts + ((int64_t)(2 * blockIdx.x + (it.u0 == it.first ? 1 : 0)) * cut.rows + rr) * kv4_part_floats(D);
    uint4* to = done ? reinterpret_cast<uint4*>(a.out + at * D) : reinterpret_cast<uint4*>(part);
    ok = ok && wait(&bars->o_full[t], o_phase, failed);
    o_phase ^= 1;
    if (!ok) return;
    fence_after();
    const bool both = split && it.u1 - it.u0 > 1;
    if (both && t == 1) {
      other[r] = make_float2(ref, sum);
      fence_before();
      __syncwarp();
      if (lane == 0) arrive(&bars->x_full);
      // (its half of O is read before the next item may touch it)
      if (!wait(&bars->x_empty, x_phase, failed)) return;
      x_phase ^= 1;
      continue;
    }
    float f = 1.f, g = 0.f;  // factors of the halves' sums
    if (both) {
      if (!wait(&bars->x_full, x_phase, failed)) return;
      x_phase ^= 1;
      fence_after();
      const float2 o = other[r];
      const float top = fmaxf(ref, o.x);
      f = exp2_approx(ref - top);
      g = exp2_approx(o.x - top);
      ref = top;
      sum = sum * f + o.y * g;
    }
    const float inv = sum == 0.f ? 0.f : gv / sum;
    // (a loop: code that runs once an item is fetched anew each time, and unrolled it was 4% of a prompt slower)
#pragma unroll 1
    for (int c = 0; c < D / 32; ++c) {
      uint32_t v[32];
      tmem_load(O + 32 * c, v);
      tmem_wait(v);
      if (both) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          uint32_t y[16];
          tmem_load16(O + 128 + 32 * c + 16 * half, y);
#pragma unroll
          for (int i = 0; i < 16; ++i)
            v[16 * half + i] = __float_as_uint(__uint_as_float(v[16 * half + i]) * f + __uint_as_float(y[i]) * g);
        }
        if (c + 1 == D / 32) {
          fence_before();
          __syncwarp();
          if (lane == 0) arrive(&bars->x_empty);
        }
      }
      if (rr < it.rows && done) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t w[4];
#pragma unroll
          for (int x = 0; x < 4; ++x)
            w[x] = pack_out<BF16>(__uint_as_float(v[8 * i + 2 * x]) * inv, __uint_as_float(v[8 * i + 2 * x + 1]) * inv);
          to[4 * c + i] = make_uint4(w[0], w[1], w[2], w[3]);
        }
      } else if (rr < it.rows) {
#pragma unroll
        for (int i = 0; i < 8; ++i) to[8 * c + i] = make_uint4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
      }
      __syncwarp();
    }
    if (rr < it.rows) {
      if (done) {
        if (a.lse) a.lse[at] = sum == 0.f ? -INFINITY : (ref + log2f(sum)) * 0.6931471805599453f;
      } else {
        *reinterpret_cast<float2*>(part + D) = make_float2(ref, sum);
      }
    }
    fence_before();
  }
}

// ------------------------------------------------------- codes to fp16 ------

// Eight tokens' rows of K or V, a lane the quarter q of token l % 8: its codes and its scales.
template <int D>
struct Codes {
  static constexpr int kWords = D / 32;  // 32-bit words of codes in a quarter of a row
  uint32_t w[kWords];
  uint32_t scale;                        // D 128: two e4m3 bytes, D 64: one
};

template <int D>
__device__ __forceinline__ void load_codes(Codes<D>& x, const uint8_t* codes, const uint8_t* scales) {
  if constexpr (D == 128) {
    const uint4 v = *reinterpret_cast<const uint4*>(codes);
    x.w[0] = v.x, x.w[1] = v.y, x.w[2] = v.z, x.w[3] = v.w;
    x.scale = *reinterpret_cast<const uint16_t*>(scales);
  } else {
    const uint2 v = *reinterpret_cast<const uint2*>(codes);
    x.w[0] = v.x, x.w[1] = v.y;
    x.scale = *scales;
  }
}

// 16-byte pieces of fp16, a core matrix row each
template <int D>
__device__ __forceinline__ void store_values(const Codes<D>& x, uint8_t* to) {
  const uint32_t s2 = e4m3x2_to_half2(x.scale);
#pragma unroll
  for (int i = 0; i < Codes<D>::kWords; ++i) {
    const uint32_t s = __byte_perm(s2, 0, D == 128 && i >= 2 ? 0x3232 : 0x1010);
    uint32_t h[4];
    e2m1x8_to_half2(x.w[i], h);
    *reinterpret_cast<uint4*>(to + i * Layout<D>::kChunk) =
        make_uint4(hmul2_bits(h[0], s), hmul2_bits(h[1], s), hmul2_bits(h[2], s), hmul2_bits(h[3], s));
  }
}

template <int D>
__device__ __forceinline__ void code_warps(const Kv4Attend& a, const Kv4ManyCut& cut, Walk& walk, uint8_t* smem, Bars* bars) {
  using L = Layout<D>;
  const int lane = threadIdx.x & 31, warp = (threadIdx.x >> 5) - 8;
  const int r8 = lane & 7, q = lane >> 3;
  const int row = warp * 32 + r8;  // of the unit; the lane's further rows are 8, 16, 24 behind
  volatile int* failed = &bars->failed;
  const int64_t head_bytes = (int64_t)kv4_tile_bytes(D) << (a.c.page_shift - 4);
  const int at_codes = r8 * (D / 2) + q * (D / 8), at_scale = 16 * D + r8 * (D / 16) + q * (D / 64);
  uint8_t* to = smem + (row >> 3) * L::kGroup + r8 * 16 + q * (D / 32) * L::kChunk;
  const int64_t page_stride = head_bytes * a.c.H;
  // Two units ahead of the one in hand: of `next` the pages' numbers are on their way, of the one before it
  // the warp's two tiles are known and their codes are loaded.
  const uint8_t* base = nullptr;
  const int32_t* table = nullptr;
  int u = 0, u1 = 0, length = 0;
  int page[2], next_left = 0;           // left: tokens from the warp's first on
  const uint8_t* next_base = nullptr;
  int next_in_page = 0;
  const uint8_t* tile[2];
  int left = 0;
  Feed feed{bars, walk.items};
  // the next unit, this item's or the next one's: its pages' numbers are asked for
  auto step = [&] {
    if (++u >= u1) {
      const Item* it = feed.next();
      if (!it) return false;
      base = a.c.pages + kv4_record(a.c, a.layer, 0, it->head);
      table = a.c.table + (int64_t)it->seq * a.c.max_pages;
      u = it->u0, u1 = it->u1, length = it->length;
      feed.done();
    }
    const int token = u * kUnit + warp * 32;
    next_base = base;
    next_left = length - token;
    next_in_page = token & (a.c.P - 1);
    page[0] = next_left > 0 ? table[token >> a.c.page_shift] : 0;
    page[1] = next_left > 16 ? table[(token + 16) >> a.c.page_shift] : 0;
    return true;
  };
  // the numbers are there: its tiles
  auto find_tiles = [&] {
    left = next_left;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      if ((unsigned)page[x] >= (unsigned)a.c.num_pages) {
        raise_error(a.c.err, kDevIndex);
        page[x] = 0;
      }
      const int in_page = (next_in_page + 16 * x) & (a.c.P - 1);
      tile[x] = next_base + page[x] * page_stride + (in_page >> 4) * kv4_tile_bytes(D) + at_codes;
    }
  };
  auto load = [&](Codes<D>(&x)[4], bool is_v) {
#pragma unroll
    for (int half = 0; half < 2; ++half) {  // a tile: rows r8 and r8 + 8 of it
      const uint8_t* codes = tile[half] + (is_v ? 8 * D : 0);
      const uint8_t* scales = tile[half] + (is_v ? D : 0) + (at_scale - at_codes);
      const int here = left - 16 * half;
      // (rows behind the last token may be anything, a tile without tokens is not there at all)
      if (here > 0) {
        load_codes<D>(x[2 * half], codes, scales);
        load_codes<D>(x[2 * half + 1], codes + 8 * (D / 2), scales + 8 * (D / 16));
      }
      if (here < 16) {
        if (r8 >= here) x[2 * half] = Codes<D>{};
        if (r8 + 8 >= here) x[2 * half + 1] = Codes<D>{};
      }
    }
  };
  Codes<D> k[4], v[4];
  uint32_t n = 0;  // units so far
  bool more = step(), ahead = false;
  if (more) {
    find_tiles();
    load(k, false);
    load(v, true);
    ahead = step();
  }
  for (; more; ++n) {
    more = ahead;
    if (more) {
      find_tiles();
      ahead = step();
    }
    const int b = n & 1;
    const uint32_t free_phase = (n >> 1 & 1) ^ 1;
    if (!wait(&bars->k_empty[b], free_phase, failed)) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) store_values<D>(k[i], to + L::k(b) + i * L::kGroup);
    fence_smem();
    __syncwarp();
    if (lane == 0) arrive(&bars->k_full[b]);
    if (more) load(k, false);
    if (!wait(&bars->v_empty[b], free_phase, failed)) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) store_values<D>(v[i], to + L::v(b) + i * L::kGroup);
    fence_smem();
    __syncwarp();
    if (lane == 0) arrive(&bars->v_full[b]);
    if (more) load(v, true);
  }
  // the products have read the last buffers (their barriers outlive the arrivals)
  for (uint32_t m = n < 2 ? 0 : n - 2; m < n; ++m)
    if (!wait(&bars->k_empty[m & 1], m >> 1 & 1, failed) || !wait(&bars->v_empty[m & 1], m >> 1 & 1, failed)) return;
}

// ------------------------------------------------------------ products ------

template <int D>
__device__ __forceinline__ void product_warp(const Kv4Attend& a, const Kv4ManyCut& cut, Walk& walk, uint8_t* smem, Bars* bars, uint32_t tmem,
                                             uint32_t leader) {
  using L = Layout<D>;
  volatile int* failed = &bars->failed;
  const uint32_t at = smem_addr(smem);
  constexpr uint32_t kHigh = desc_high(L::kGroup), vHigh = desc_high(L::kChunk);
  const uint32_t k0 = desc_low(at + L::k(0), L::kChunk), q0 = desc_low(at + L::q(0), L::kChunk);
  const uint32_t v0 = desc_low(at + L::v(0), L::kGroup);
  auto scores = [&](int block, int t, uint32_t b) {  // S_t = Q_block K^T
    const uint32_t q = q0 + block * (L::kTile >> 4), k = k0 + b * (L::kTile >> 4);
#pragma unroll
    for (int x = 0; x < D / 16; ++x)
      mma_ss(leader, tmem + 128 * t, q + x * (2 * L::kChunk >> 4), k + x * (2 * L::kChunk >> 4), kHigh, instr_desc(kUnit, false),
             x > 0);
    commit(leader, &bars->s_full[t]);
  };
  uint32_t n = 0, q_phase = 0, p_phase = 0;  // units so far; a bit for each block
  Feed feed{bars, walk.items};
  auto values = [&](int t, uint32_t b, bool add) {  // O_t += P_t V
    const uint32_t v = v0 + b * (L::kTile >> 4);
#pragma unroll
    for (int x = 0; x < kUnit / 16; ++x)
      mma_ts(leader, tmem + 256 + 128 * t, tmem + 128 * t + 8 * x, v + x * (2 * L::kGroup >> 4), vHigh, instr_desc(D, true),
             (uint32_t)(add || x > 0));
  };
  auto queries = [&](int t) {
    const bool ok = wait(&bars->q_full[t], q_phase >> t & 1, failed);
    q_phase ^= 1u << t;
    return ok;
  };
  auto weights = [&](int t) {
    const bool ok = wait(&bars->p_full[t], p_phase >> t & 1, failed);
    p_phase ^= 1u << t;
    fence_after();
    return ok;
  };
  while (const Item* item = feed.next()) {
    const bool split = item->rows <= kBlock;
    const int units = item->u1 - item->u0;
    feed.done();
    if (!queries(0) || (!split && !queries(1))) return;
    if (split) {
      // the halves take units in turn: S_0 and S_1 are of neighbouring units
      for (int u = 0; u < units && u < 2; ++u) {
        const uint32_t m = n + u;
        if (!wait(&bars->k_full[m & 1], m >> 1 & 1, failed)) return;
        fence_after();
        scores(0, u, m & 1);
        commit(leader, &bars->k_empty[m & 1]);
        if (u + 1 == units) commit(leader, &bars->q_empty[0]);
      }
      for (int u = 0; u < units; ++u, ++n) {
        const uint32_t b = n & 1;
        const int t = u & 1;
        if (!wait(&bars->v_full[b], n >> 1 & 1, failed) || !weights(t)) return;
        values(t, b, u > 1);
        commit(leader, &bars->v_empty[b]);
        if (u + 2 < units) {
          if (!wait(&bars->k_full[b], (n + 2) >> 1 & 1, failed)) return;
          fence_after();
          scores(0, t, b);
          commit(leader, &bars->k_empty[b]);
          if (u + 3 == units) commit(leader, &bars->q_empty[0]);
        } else {
          commit(leader, &bars->o_full[t]);
        }
      }
      continue;
    }
    if (!wait(&bars->k_full[n & 1], n >> 1 & 1, failed)) return;
    fence_after();
    for (int t = 0; t < 2; ++t) {
      scores(t, t, n & 1);
      if (units == 1) commit(leader, &bars->q_empty[t]);
    }
    commit(leader, &bars->k_empty[n & 1]);
    for (int u = 0; u < units; ++u, ++n) {
      const uint32_t b = n & 1;
      if (!wait(&bars->v_full[b], n >> 1 & 1, failed)) return;
      for (int t = 0; t < 2; ++t) {
        if (!weights(t)) return;
        values(t, b, u > 0);
        if (t == 1) commit(leader, &bars->v_empty[b]);
        if (u + 1 < units) {
          if (t == 0) {
            if (!wait(&bars->k_full[b ^ 1], (n + 1) >> 1 & 1, failed)) return;
            fence_after();
          }
          scores(t, t, b ^ 1);
          if (u + 2 == units) commit(leader, &bars->q_empty[t]);
          if (t == 1) commit(leader, &bars->k_empty[b ^ 1]);
        } else {
          commit(leader, &bars->o_full[t]);
        }
      }
    }
  }
}

template <int D, bool BF16>
__global__ void __launch_bounds__(kThreads, 1) kv4_chunk_kernel(Kv4Attend a, Kv4ManyCut cut) {
  using L = Layout<D>;
  extern __shared__ __align__(128) uint8_t smem[];
  int64_t* prefix = reinterpret_cast<int64_t*>(smem + L::prefix());
  int64_t* sums = reinterpret_cast<int64_t*>(smem + L::sums());
  float* undo = reinterpret_cast<float*>(smem + L::undo());
  Bars* bars = reinterpret_cast<Bars*>(smem + L::bars());
  const int warp = threadIdx.x >> 5;
  if (threadIdx.x == 0) {
    auto init = [](uint64_t* bar, int count) {
      asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_addr(bar)), "r"(count) : "memory");
    };
    for (int x = 0; x < kItems; ++x) {
      init(&bars->i_full[x], 1);
      init(&bars->i_empty[x], kThreads / 32);
    }
    for (int x = 0; x < 2; ++x) {
      init(&bars->q_full[x], 3);
      init(&bars->q_empty[x], 1);
      init(&bars->k_full[x], 4);
      init(&bars->v_full[x], 4);
      init(&bars->k_empty[x], 1);
      init(&bars->v_empty[x], 1);
      init(&bars->s_full[x], 1);
      init(&bars->p_full[x], 4);
      init(&bars->o_full[x], 1);
    }
    init(&bars->x_full, 4);
    init(&bars->x_empty, 4);
    init(&bars->drain, 1);
    bars->failed = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 12) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(&bars->tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = bars->tmem;
  pdl_wait();
  pdl_trigger();
  kv4_plan<kThreads, true>(a, cut, prefix, sums, blockIdx.x == 0);
  const int64_t W = prefix[kThreads];
  const Kv4Ranges ranges(W, cut.least, gridDim.x);
  if (threadIdx.x == kThreads - 32) a.joins[blockIdx.x] = make_int4(0, 0, 0, 0);  // (the thread that may replace it)
  if (W > 0 && (int)blockIdx.x < ranges.count) {
    Walk& walk = *reinterpret_cast<Walk*>(smem + L::walk());
    if (warp == kThreads / 32 - 1) walk.start(a, cut, prefix, ranges);
    // 184 + 184 + 80 + 64 = 4 * 128, the registers of the launch.  2048 tokens over 30K took 653 us with these,
    // 712 with 176, 176, 88, 72, 700 with 184, 184, 72, 72 and 710 with 192, 192, 72, 56.  ptxas still spills a few
    // registers (40 bytes stored with f16 rows, 24 with bf16).
    if (warp < 8) {
      asm volatile("setmaxnreg.inc.sync.aligned.u32 184;");
      softmax_warps<D, BF16>(a, cut, walk, undo, reinterpret_cast<float2*>(smem + L::other()), bars, tmem);
    } else if (warp < 12) {
      asm volatile("setmaxnreg.dec.sync.aligned.u32 80;");
      code_warps<D>(a, cut, walk, smem, bars);
    } else {
      asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
      if (warp == 12) {
        const uint32_t leader = elect();
        product_warp<D>(a, cut, walk, smem, bars, tmem, leader);
        if (__any_sync(~0u, *(volatile int*)&bars->failed)) {
          // products still at work are waited for, as long again
          commit(leader, &bars->drain);
          mbar_wait_bounded(&bars->drain, 0);
        }
      } else
        query_warps<D, BF16>(a, cut, walk, smem, bars, undo);
    }
  }
  fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && bars->failed) raise_error(a.c.err, kDevWaitTimeout);
  if (warp == 12) {
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
}

// Joins the parts of the tiles that several CTAs share: CTA x takes the tile that range x begins and
// does not end, a warp for four rows.  CTAs behind those fill the rows that see nothing, one for each
// sequence.
constexpr int kJoinThreads = 256;
constexpr int kJoinSplit = 8;  // CTAs of a tile

template <int D, bool BF16>
__global__ void __launch_bounds__(kJoinThreads) kv4_chunk_join_kernel(Kv4Attend a, Kv4ManyCut cut, int most) {
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, x = blockIdx.x;
  constexpr int kDims = D / 32, kStep = kJoinSplit * kJoinThreads / 32;
  const int row0 = blockIdx.y * (kJoinThreads / 32) + warp;
  if (x >= most) {
    const Kv4Seq s = cut.seq(a, x - most, false);
    const int64_t hidden = s.length == 0 ? s.count : min((int64_t)s.count, (int64_t)s.hidden * cut.tokens);
    for (int64_t y = row0; y < hidden * a.q_heads; y += kStep) {
      const int64_t at = (int64_t)s.begin * a.q_heads + y;
#pragma unroll
      for (int d = 0; d < kDims; d += 2) *reinterpret_cast<uint32_t*>(a.out + at * D + kDims * lane + d) = 0;
      if (a.lse && lane == 0) a.lse[at] = -INFINITY;
    }
    return;
  }
  const int4 words = a.joins[x];
  const Kv4Join& join = *reinterpret_cast<const Kv4Join*>(&words);
  const int rows = join.rows_parts & 0xFFFF, parts = join.rows_parts >> 16;
  if (parts < 2) return;
  // a warp's rows together, so that their loads do not wait for one another
  constexpr int kRows = 2 * kBlock / kStep;
  float ref[kRows], total[kRows], o[kRows][kDims];
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    ref[k] = kNone, total[k] = 0.f;
#pragma unroll
    for (int d = 0; d < kDims; ++d) o[k][d] = 0.f;
  }
  for (int p = 0; p < parts; ++p) {
    // the first part begins the item (slot 2 w + 1), the others continue it (slot 2 w)
    const float* part = a.parts + ((int64_t)(2 * (x + p) + (p == 0)) * cut.rows + row0) * kv4_part_floats(D);
    float2 rs[kRows];
    float v[kRows][kDims];
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
      const float* of = part + (row0 + k * kStep < rows ? k * kStep : 0) * kv4_part_floats(D);
      rs[k] = row0 < rows ? *reinterpret_cast<const float2*>(of + D) : make_float2(kNone, 0.f);
      if constexpr (kDims == 4) {
        const float4 y = row0 < rows ? *reinterpret_cast<const float4*>(of + 4 * lane) : float4{};
        v[k][0] = y.x, v[k][1] = y.y, v[k][2] = y.z, v[k][3] = y.w;
      } else {
        const float2 y = row0 < rows ? *reinterpret_cast<const float2*>(of + 2 * lane) : float2{};
        v[k][0] = y.x, v[k][1] = y.y;
      }
    }
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
      const float to = fmaxf(ref[k], rs[k].x), f = exp2_approx(ref[k] - to), g = exp2_approx(rs[k].x - to);
      ref[k] = to;
      total[k] = total[k] * f + rs[k].y * g;
#pragma unroll
      for (int d = 0; d < kDims; ++d) o[k][d] = o[k][d] * f + v[k][d] * g;
    }
  }
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    const int col = row0 + k * kStep;
    if (col >= rows) continue;
    const int64_t at = join.first_row + cut.token_of(col) * (a.q_heads - a.group) + col;
    const float inv = total[k] == 0.f ? 0.f : join.gv / total[k];
    uint32_t* to = reinterpret_cast<uint32_t*>(a.out + at * D + kDims * lane);
#pragma unroll
    for (int d = 0; d < kDims; d += 2) to[d / 2] = pack_out<BF16>(o[k][d] * inv, o[k][d + 1] * inv);
    if (a.lse && lane == 0) a.lse[at] = total[k] == 0.f ? -INFINITY : (ref[k] + log2f(total[k])) * 0.6931471805599453f;
  }
}

// The same where a step has few tiles, each with many parts: a CTA for each row of a tile, whose warps
// take the parts in turn (one tile of 128 rows over 29K tokens has 114: 93 us with a warp for a row).
template <int D, bool BF16>
__global__ void __launch_bounds__(kJoinThreads) kv4_chunk_join_rows_kernel(Kv4Attend a, Kv4ManyCut cut, int most, int tiles) {
  constexpr int kWarps = kJoinThreads / 32, kDims = D / 32;
  __shared__ float acc[kWarps][D];
  __shared__ float2 sums[kWarps];  // reference exponent, weight sum
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int head = blockIdx.x / tiles % a.c.H, tile = blockIdx.x % tiles, i = blockIdx.x / tiles / a.c.H;
  const int64_t W = a.prefix[a.b.n], p0 = a.prefix[i];
  const Kv4Seq s = cut.seq(a, i, false);
  if (tile >= s.tiles) return;
  const Kv4Ranges ranges(W, cut.least, most);
  int w0 = 0, parts = 0;
  int64_t first, last;
  if (cut.ends(a, s, head, tile, first, last)) {
    w0 = ranges.owner(p0 + first);
    parts = ranges.owner(p0 + last) - w0 + 1;
    if (parts == 1) return;  // finished where it ran
  }
  const int rows = min(cut.rows, (s.count - tile * cut.tokens) * a.group);
  const float gv = a.c.v_scale ? a.c.v_scale[a.layer * a.c.H + head] : 1.f;
  for (int col = blockIdx.y; col < rows; col += gridDim.y) {
    float ref = kNone, total = 0.f, o[kDims] = {};
#pragma unroll 4
    for (int p = warp; p < parts; p += kWarps) {
      const float* part = a.parts + ((int64_t)(2 * (w0 + p) + (p == 0)) * cut.rows + col) * kv4_part_floats(D);
      const float2 rs = *reinterpret_cast<const float2*>(part + D);
      float x[kDims];
#pragma unroll
      for (int d = 0; d < kDims; ++d) x[d] = part[kDims * lane + d];
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
    for (int w = 1; w < kWarps; ++w) {
      const float to = fmaxf(ref, sums[w].x), f = exp2_approx(ref - to), g = exp2_approx(sums[w].x - to);
      ref = to;
      total = total * f + sums[w].y * g;
#pragma unroll
      for (int d = 0; d < kDims; ++d) o[d] = o[d] * f + acc[w][kDims * lane + d] * g;
    }
    const int row = tile * cut.rows + col;
    const int64_t at = (int64_t)(s.begin + row / a.group) * a.q_heads + head * a.group + row % a.group;
    const float inv = total == 0.f ? 0.f : gv / total;
#pragma unroll
    for (int d = 0; d < kDims; d += 2)
      *reinterpret_cast<uint32_t*>(a.out + at * D + kDims * lane + d) = pack_out<BF16>(o[d] * inv, o[d + 1] * inv);
    if (a.lse && lane == 0) a.lse[at] = total == 0.f ? -INFINITY : (ref + log2f(total)) * 0.6931471805599453f;
  }
}

// Tiles of whole tokens, as many as two blocks hold.
Kv4ManyCut many_cut(int group) {
  const int tokens = 2 * kBlock / group;
  return Kv4ManyCut{tokens * group, tokens, ((1ull << 32) + group - 1) / group};
}

template <int D, bool BF16>
cudaError_t launch_chunk(const Kv4Attend& a, const Kv4ManyCut& cut, int sms, cudaStream_t stream) {
  using L = Layout<D>;
  auto kernel = kv4_chunk_kernel<D, BF16>;
  static bool done[kAttrDevices];
  const cudaError_t e = once_per_device(done, [&] {
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, L::bytes());
  });
  if (e != cudaSuccess) return e;
  return launch_pdl(kernel, dim3(sms), dim3(kThreads), L::bytes(), stream, a, cut);
}

}  // namespace

bool kv4_many(const Kv4Batch& b, int group) {
  // one tile of the small kernel holds up to 32 rows; more would read the cache again.  8 sequences of 32K, head
  // dim 128: 20 and 24 rows 124 us there, 28 rows 145, 32 rows 149, here 194 each; one sequence of 32K: 40, 44 and 46
  // us there, 50 here; head dim 64, 8 sequences: 87, 104 and 104 there, 153 here.  With a second tile, 36 rows of 8
  // sequences took 261 us there and 184 here.  (A tile of 48 rows, which head dim 64 leaves registers for, was no
  // faster than this kernel: 36 rows of 8 sequences of 4K 32 us, 30 here.)
  return (int64_t)b.max_count * group > 32 && group <= 2 * kBlock;
}

size_t kv4_many_front_bytes(const Kv4Batch& b, int sms) {
  return (((size_t)b.n + 1) * 8 + 15 & ~(size_t)15) + (size_t)sms * sizeof(int4);
}
size_t kv4_many_part_floats(int D, int sms) { return (size_t)2 * sms * 2 * kBlock * kv4_part_floats(D); }

cudaError_t launch_kv4_many(const Kv4Attend& a, int dtype, int sms, cudaStream_t stream) {
  const Kv4ManyCut cut = many_cut(a.group);
  const bool bf = dtype == SEMKV_BF16;
  const cudaError_t e =
      a.c.D == 128 ? (bf ? launch_chunk<128, true>(a, cut, sms, stream) : launch_chunk<128, false>(a, cut, sms, stream))
                   : (bf ? launch_chunk<64, true>(a, cut, sms, stream) : launch_chunk<64, false>(a, cut, sms, stream));
  if (e != cudaSuccess) return e;
  const int64_t tiles = ((int64_t)a.b.max_count + cut.tokens - 1) / cut.tokens, items = tiles * a.b.n * a.c.H;
  if (items * 8 <= sms) {  // eight parts or more to a tile
    auto rows = a.c.D == 128 ? (bf ? kv4_chunk_join_rows_kernel<128, true> : kv4_chunk_join_rows_kernel<128, false>)
                             : (bf ? kv4_chunk_join_rows_kernel<64, true> : kv4_chunk_join_rows_kernel<64, false>);
    return launch_pdl(rows, dim3((unsigned)items, cut.rows), dim3(kJoinThreads), 0, stream, a, cut, sms, (int)tiles);
  }
  auto join = a.c.D == 128 ? (bf ? kv4_chunk_join_kernel<128, true> : kv4_chunk_join_kernel<128, false>)
                           : (bf ? kv4_chunk_join_kernel<64, true> : kv4_chunk_join_kernel<64, false>);
  return launch_pdl(join, dim3(sms + a.b.n, kJoinSplit), dim3(kJoinThreads), 0, stream, a, cut, sms);
}

}  // namespace semkv
