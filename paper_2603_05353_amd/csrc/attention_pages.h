// Attention over 8-bit pages: how a launch is divided among workgroups, and the pieces that its kernels share.
#pragma once

#include "ifkv_device.h"
#include "pages.h"

namespace ifkv {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kAttendThreads = 256;   // four wavefronts
constexpr int kAttendWaves = kAttendThreads / 64;
constexpr int kMaxItems = 1024;       // of a launch that is cut along the cache

// An item is a block of query columns (row, query head of the kv head) of one sequence; all kv heads have the same items.
// All pages of all items, kv head after kv head, make one long list, which is cut into equal shares, one for each unit of the
// launch (a workgroup): long sequences are spread over many units, short ones stay whole, and all units end
// together however uneven the lengths are.  Only the device knows those: every workgroup adds up the items' pages (their last
// rows' positions) and finds its share by itself.
struct AttendPlan {
  int n_blocks;       // column blocks of a sequence
  int columns;        // of a block
  int group;          // query heads of a kv head
  int units;          // at most; 0: not cut, a workgroup takes the item blockIdx.x of kv head blockIdx.y
  int least_pages;    // of a unit
  int start_pages;    // what beginning an item costs, in pages: so many stand before its own in the list, and nobody reads them
};

// Shares: unit u has the pages [edge(u), edge(u + 1)) of the list of n.
struct Shares {
  uint32_t n, units;
  __device__ __forceinline__ Shares(const AttendPlan &plan, uint32_t pages)
      : n(pages), units(min(static_cast<uint32_t>(plan.units), max(1u, (pages + plan.least_pages - 1) / plan.least_pages))) {}
  __device__ __forceinline__ uint32_t edge(uint32_t u) const { return static_cast<uint32_t>(static_cast<uint64_t>(u) * n / units); }
  // the unit that has page x: the last whose edge is not behind it
  __device__ __forceinline__ uint32_t unit_of(uint32_t x) const {
    return static_cast<uint32_t>((static_cast<uint64_t>(x + 1) * units + n - 1) / n) - 1;
  }
};

// An item's rows.
struct AttendItem {
  int seq, block, lo, hi;
  __device__ __forceinline__ AttendItem(const PageTable &t, const AttendPlan &plan, int max_rows, int item)
      : seq(item / plan.n_blocks), block(item - seq * plan.n_blocks) {
    rows_of(t, seq, lo, hi);
    hi = min(hi, lo + max_rows);
  }
};

// Pages up to the last token that any row of an item sees; 0: it has no rows, 1: or they see nothing.  `lanes` (a power of two, at
// most 64) neighbouring threads look at its rows together and all of them return the answer.
__device__ __forceinline__ int item_pages(const PageTable &t, const AttendPlan &plan, int max_rows, int index, int sub, int lanes) {
  const AttendItem i(t, plan, max_rows, index);
  const int64_t c0 = static_cast<int64_t>(i.block) * plan.columns;
  const int r0 = i.lo + static_cast<int>(c0 / plan.group);
  const int r1 = min(i.hi, i.lo + static_cast<int>((c0 + plan.columns + plan.group - 1) / plan.group));
  int n = r0 < r1 ? 1 : 0;
  for (int r = r0 + sub; r < r1; r += lanes) {
    const int p = t.row_pos[r];
    if (p >= 0 && (p >> 6) < t.width) n = max(n, (p >> 6) + 1);
  }
  for (int o = 1; o < lanes; o <<= 1) n = max(n, __shfl_xor(n, o, 64));
  return n;
}

// Threads that look at an item's rows together.
__device__ __forceinline__ int item_lanes(const AttendPlan &plan, int max_rows) {
  const int rows = min(max_rows, (plan.columns + plan.group - 1) / plan.group + 1);
  int lanes = 1;
  while (lanes < rows && lanes < 64) lanes <<= 1;
  return lanes;
}

struct AttendPlanMemory {
  int start[kMaxItems + 1];   // pages of a kv head in the list before an item
  int scan[kAttendWaves];
};

// All items' pages.  The first workgroup leaves the table for the kernel that joins.
__device__ __forceinline__ void add_up_items(const PageTable &t, const AttendPlan &plan, int max_rows, bool leave, int *table,
                                             AttendPlanMemory &mem) {
  const int n_items = t.n_seqs * plan.n_blocks;
  const int lanes = item_lanes(plan, max_rows);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  for (int i0 = 0; i0 < n_items; i0 += kAttendThreads / lanes) {
    const int i = i0 + tid / lanes;
    if (i >= n_items) continue;   // (the lanes of an item go together)
    const int n = item_pages(t, plan, max_rows, i, tid & (lanes - 1), lanes);
    if ((tid & (lanes - 1)) == 0) mem.start[i] = n > 0 ? n + plan.start_pages : 0;
  }
  __syncthreads();
  constexpr int PER = kMaxItems / kAttendThreads;   // neighbouring items of a thread
  int pages[PER], mine = 0;
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    const int i = tid * PER + u;
    pages[u] = i < n_items ? mem.start[i] : 0;
    mine += pages[u];
  }
  int before = mine;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int a = __shfl_up(before, o, 64);
    if (lane >= o) before += a;
  }
  if (lane == 63) mem.scan[wave] = before;
  __syncthreads();
  before -= mine;
  for (int w = 0; w < wave; ++w) before += mem.scan[w];
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    const int i = tid * PER + u;
    if (i <= n_items) {
      mem.start[i] = before;
      if (leave) table[i] = before;
    }
    before += pages[u];
  }
  if (tid == kAttendThreads - 1 && n_items == kMaxItems) {
    mem.start[kMaxItems] = before;
    if (leave) table[kMaxItems] = before;
  }
  __syncthreads();
}

// Eight e4m3 numbers of two words, times a power of two, as bf16: exact.
__device__ __forceinline__ bf16x8 widen(uint32_t a, uint32_t b, float scale) {
  const bf16x2 p = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, false), q = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, true);
  const bf16x2 r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, false), s = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, true);
  return bf16x8{p[0], p[1], q[0], q[1], r[0], r[1], s[0], s[1]};
}

// x as the sum of PARTS bf16 numbers, each the rest rounded to nearest even.
template <int PARTS>
__device__ __forceinline__ void split8(const float (&x)[8], bf16x8 (&out)[PARTS]) {
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    float a = x[e], b = x[e + 1];
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
      const bf16x2 pair = {static_cast<__bf16>(a), static_cast<__bf16>(b)};
      out[p][e] = pair[0];
      out[p][e + 1] = pair[1];
      const uint32_t w = __builtin_bit_cast(uint32_t, pair);
      a -= __uint_as_float(w << 16);
      b -= __uint_as_float(w & 0xFFFF0000u);
    }
  }
}

size_t attend_matrix_scratch_bytes(const ifkv_ctx *ctx);
hipError_t launch_attend_matrix(ifkv_ctx *ctx, const ifkv_page_cache &pages, const PageTable &t, int32_t max_rows, const void *q,
                                int64_t q_stride, void *out, float *lse_out);

}  // namespace ifkv
