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
// Pages of an item are cut into parts of the same number of pages throughout the launch, so that long sequences become many
// workgroups and short ones stay whole; a workgroup has one part.  How long a part is depends on lengths that only
// the device knows: every workgroup adds up the items' pages (their last rows' positions) and finds its part by itself.
struct AttendPlan {
  int n_blocks;       // column blocks of a sequence
  int columns;        // of a block
  int group;          // query heads of a kv head
  int target_parts;   // for all items of a kv head together, about; 0: items are not cut
  int least_pages;    // of a part
};

struct AttendPart {
  int seq, block;     // the item
  int first, last;    // its pages [first, last)
  int n_parts;        // of the item; 1: the workgroup writes the result itself
  int slot;           // partial results of this part, among those of the kv head
  int lo, hi;         // rows of the sequence
};

// Pages up to the last token that any row of an item sees.  `lanes` (a power of two, at most 64) neighbouring threads look at
// its rows together and all of them return the answer.
__device__ __forceinline__ int item_pages(const PageTable &t, const AttendPlan &plan, int max_rows, int item, int sub, int lanes) {
  const int s = item / plan.n_blocks, b = item - s * plan.n_blocks;
  int lo, hi;
  rows_of(t, s, lo, hi);
  hi = min(hi, lo + max_rows);
  const int r0 = lo + static_cast<int>(static_cast<int64_t>(b) * plan.columns / plan.group);
  const int r1 = min(hi, lo + static_cast<int>((static_cast<int64_t>(b + 1) * plan.columns + plan.group - 1) / plan.group));
  int n = 0;
  for (int r = r0 + sub; r < r1; r += lanes) {
    const int p = t.row_pos[r];
    if (p >= 0 && (p >> 6) < t.width) n = max(n, (p >> 6) + 1);
  }
  for (int o = 1; o < lanes; o <<= 1) n = max(n, __shfl_xor(n, o, 64));
  return n;
}

struct AttendPlanMemory {
  int pages[kMaxItems];
  int sum[kAttendWaves];
  int scan[2][kAttendWaves];
  int found[5];
};

// What this workgroup does; false: nothing.  meta (written by the workgroups of kv head 0): first slot and parts of each item.
__device__ __forceinline__ bool find_part(const PageTable &t, const AttendPlan &plan, int max_rows, int index, bool writes_meta, int2 *meta,
                                          AttendPlanMemory &mem, AttendPart &part) {
  const int n_items = t.n_seqs * plan.n_blocks;
  const int rows = min(max_rows, (plan.columns + plan.group - 1) / plan.group + 1);
  int lanes = 1;
  while (lanes < rows && lanes < 64) lanes <<= 1;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int item = index, pages = 0;
  part.n_parts = 1;
  part.slot = 0;
  part.first = 0;
  if (plan.target_parts == 0) {
    pages = item_pages(t, plan, max_rows, item, lane & (lanes - 1), lanes);
    part.last = pages;
  } else {
    int total = 0;
    for (int i0 = 0; i0 < n_items; i0 += kAttendThreads / lanes) {
      const int i = i0 + tid / lanes;
      if (i >= n_items) continue;   // (the lanes of an item go together)
      const int n = item_pages(t, plan, max_rows, i, tid & (lanes - 1), lanes);
      if ((tid & (lanes - 1)) == 0) {
        mem.pages[i] = n;
        total += n;
      }
    }
    total = wave_sum_i(total);
    if (lane == 0) mem.sum[wave] = total;
    if (tid == 0) mem.found[0] = -1;
    __syncthreads();
    total = 0;
#pragma unroll
    for (int w = 0; w < kAttendWaves; ++w) total += mem.sum[w];
    int step = max(plan.least_pages, (total + plan.target_parts - 1) / plan.target_parts);
    step = (step + kAttendWaves - 1) / kAttendWaves * kAttendWaves;
    // four items a thread: their parts, and the slots of those that have more than one
    constexpr int PER = kMaxItems / kAttendThreads;
    int parts[PER], mine = 0, slots = 0;
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      const int i = tid * PER + u;
      parts[u] = i < n_items ? max(1, (mem.pages[i] + step - 1) / step) : 0;
      mine += parts[u];
      slots += parts[u] > 1 ? parts[u] : 0;
    }
    int before = mine, slots_before = slots;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int a = __shfl_up(before, o, 64), b = __shfl_up(slots_before, o, 64);
      if (lane >= o) before += a, slots_before += b;
    }
    if (lane == 63) mem.scan[0][wave] = before, mem.scan[1][wave] = slots_before;
    __syncthreads();
    before -= mine;
    slots_before -= slots;
    for (int w = 0; w < wave; ++w) before += mem.scan[0][w], slots_before += mem.scan[1][w];
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      if (index >= before && index < before + parts[u]) {
        mem.found[0] = tid * PER + u;
        mem.found[1] = index - before;
        mem.found[2] = parts[u];
        mem.found[3] = slots_before + index - before;
      }
      before += parts[u];
      slots_before += parts[u] > 1 ? parts[u] : 0;
    }
    __syncthreads();
    item = mem.found[0];
    if (item < 0) return false;
    pages = mem.pages[item];
    part.n_parts = mem.found[2];
    part.slot = mem.found[3];
    part.first = mem.found[1] * step;
    part.last = min(pages, part.first + step);
    if (writes_meta && mem.found[1] == 0 && tid == 0) meta[item] = make_int2(part.slot, part.n_parts);
  }
  // the same in every lane: scalars
  item = __builtin_amdgcn_readfirstlane(item);
  part.first = __builtin_amdgcn_readfirstlane(part.first);
  part.last = __builtin_amdgcn_readfirstlane(part.last);
  part.n_parts = __builtin_amdgcn_readfirstlane(part.n_parts);
  part.slot = __builtin_amdgcn_readfirstlane(part.slot);
  part.seq = item / plan.n_blocks;
  part.block = item - part.seq * plan.n_blocks;
  rows_of(t, part.seq, part.lo, part.hi);
  part.hi = min(part.hi, part.lo + max_rows);
  // a block behind the sequence's rows
  return static_cast<int64_t>(part.block) * plan.columns < static_cast<int64_t>(part.hi - part.lo) * plan.group;
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
