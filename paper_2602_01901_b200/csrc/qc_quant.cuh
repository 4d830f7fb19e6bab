// The layout of 4-bit pages, as the kernels that write and read them see it.
//
// A pool holds one tensor (K or V) of one layer and stream.  A page of P tokens is first the codes
// [n_kv_heads][P / 16][8 * D bytes], then the parameters [n_kv_heads][P] of 4 bytes (lo as bf16 in the low
// half, r as bf16 in the high half).  A block of 16 tokens is laid out so that lane (g = lane / 4, t = lane % 4)
// of a warp reads its operands of the m16n8k16 products as whole 16-byte vectors, 512 bytes in lane order per
// load.  A word's low and high half then give two 16-bit operands at a time: bits 0-3 and 16-19 one pair, 4-7
// and 20-23 the next, and after a shift by 8 the other two.
//   K: lane (g, t) has elements t * D / 4 .. of tokens 2 g and 2 g + 1 (rows g and g + 8 of the product, the
//      element pairs (0, 4), (1, 5), (2, 6), (3, 7) of a word along its inner axis).
//   V: lane (g, t) has elements g * D / 8 .. of tokens 4 t .. 4 t + 3, a word holding two elements of the four
//      tokens, a byte per token (rows g and g + 8: the even and the odd element; token pairs (0, 2) and (1, 3)
//      along the inner axis).
#pragma once

#include <stdint.h>

namespace qc {

__host__ __device__ __forceinline__ int64_t quant_page_bytes(int n_kv_heads, int d, int page) {
  return static_cast<int64_t>(n_kv_heads) * page * (d / 2 + 4);
}

// The step 1 / r of a row: 0 where r is 0 (all its elements are lo).
__device__ __forceinline__ float quant_step(uint32_t params) {
  const float r = __uint_as_float(params & 0xffff0000u);
  return r == 0.f ? 0.f : __frcp_rn(r);
}

}  // namespace qc
