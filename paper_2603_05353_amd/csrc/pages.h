// What the kernels on 8-bit pages share: the byte order of a page's values and the way from rows to pages.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ifkv_internal.h"

namespace ifkv {

constexpr int kPageTokens = IFKV_PAGE_TOKENS;
static_assert(kPageTokens == 64, "a page is one wavefront's tile of tokens");

// Byte of token t within the 64 of a value row.  A 16x16 result of the first product leaves lane l with the probabilities of
// tokens 16 i + 4 (l / 16) .. + 3 of each of the four blocks i of 16 tokens: those sixteen are 16 bytes in a row, so a lane's
// operand of the second product is one 16-byte load and the probabilities never change lanes.
__host__ __device__ constexpr int value_byte(int t) { return ((t >> 2) & 3) << 4 | (t >> 5) << 3 | ((t >> 4) & 1) << 2 | (t & 3); }

// First row and end of sequence s, within the rows there are.
__device__ __forceinline__ void rows_of(const PageTable &t, int s, int &lo, int &hi) {
  if (t.row_start == nullptr) {
    lo = s;
    hi = s + 1;
    return;
  }
  const int n = static_cast<int>(t.n_rows);
  lo = min(max(t.row_start[s], 0), n);
  hi = min(max(t.row_start[s + 1], lo), n);
}

// The page that holds token block `logical` of sequence s, or -1.
__device__ __forceinline__ int page_of(const PageTable &t, int s, int logical, int n_pages) {
  const int p = t.table[static_cast<int64_t>(s) * t.width + logical];
  return p >= 0 && p < n_pages ? p : -1;
}

}  // namespace ifkv
