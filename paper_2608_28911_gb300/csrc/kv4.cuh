// kv4.cuh — the paged 4-bit cache's format, and what its kernels share.
//
// A tile is 16 tokens of one head: [K codes 16][D/2] [V codes 16][D/2] [K scales 16][D/16]
// [V scales 16][D/16], 18 D bytes.  One contiguous tile is one bulk copy for the attention
// kernels, whatever the page size, and a token's row is written without touching its
// neighbours' bytes.  Code times scale has at most six significant bits and lies in
// [2^-10, 2688], so it is exact in fp16: the matrix instructions see the cache's values
// without a rounding, and the head's binary32 scale is applied to their results.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include "../../include/semkv.h"
#include "common.cuh"

namespace semkv {

struct Kv4Cache {
  int layers, H, D, P, page_shift;  // P = 1 << page_shift
  int num_pages, max_seqs, max_pages;
  uint8_t* pages;
  const float* k_scale;
  const float* v_scale;
  int32_t* table;
  int32_t* length;
  int32_t* refs;
  int32_t* err;
};

struct Kv4Batch {
  int n, total, max_count;
  const int32_t* seqs;
  const int32_t* cu;
  int32_t* start;
};

__host__ __device__ constexpr int kv4_tile_bytes(int D) { return 18 * D; }

__device__ __forceinline__ int64_t kv4_record(const Kv4Cache& c, int layer, int page, int head) {
  // first byte of (layer, page, head): page_tokens / 16 tiles
  return (((int64_t)layer * c.num_pages + page) * c.H + head) *
         ((int64_t)kv4_tile_bytes(c.D) << (c.page_shift - 4));
}

// The i-th sequence's rows [begin, begin + count) of a step; false where the range is wrong.
__device__ __forceinline__ bool kv4_range(const Kv4Batch& b, int i, int& begin, int& count) {
  if (!b.cu) {
    begin = i;
    count = 1;
    return i < b.total;
  }
  begin = b.cu[i];
  const int end = b.cu[i + 1];
  count = end - begin;
  return begin >= 0 && end >= begin && end <= b.total && count <= b.max_count;
}

// ---------------------------------------------------------- conversions ------

// Four bytes of codes, two e2m1 values each, as four half2 (lower code in the lower half).
__device__ __forceinline__ void e2m1x8_to_half2(uint32_t w, uint32_t (&h)[4]) {
  asm("{\n .reg .b8 a, b, c, d;\n mov.b32 {a, b, c, d}, %4;\n"
      " cvt.rn.f16x2.e2m1x2 %0, a;\n cvt.rn.f16x2.e2m1x2 %1, b;\n"
      " cvt.rn.f16x2.e2m1x2 %2, c;\n cvt.rn.f16x2.e2m1x2 %3, d;\n}"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
      : "r"(w));
}
// Two e4m3 bytes as a half2 (exact).
__device__ __forceinline__ uint32_t e4m3x2_to_half2(uint32_t two) {
  uint32_t h;
  asm("{\n .reg .b16 t;\n cvt.u16.u32 t, %1;\n cvt.rn.f16x2.e4m3x2 %0, t;\n}" : "=r"(h) : "r"(two));
  return h;
}
__device__ __forceinline__ uint32_t hmul2_bits(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}

}  // namespace semkv
