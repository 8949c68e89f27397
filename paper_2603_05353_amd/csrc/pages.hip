// Writing rows into 8-bit pages and copying pages.
#include <algorithm>

#include "ifkv_device.h"
#include "pages.h"

namespace ifkv {

namespace {

constexpr int kThreads = 256;

// Four numbers as e4m3, rounded to nearest even (magnitudes at most 448, or NaN).
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true));
}

// Four e4m3 numbers times f, rounded again.
__device__ __forceinline__ uint32_t rescale_e4m3(uint32_t w, float f) {
  const int v = static_cast<int>(w);
  return pack_e4m3(__builtin_amdgcn_cvt_f32_fp8(v, 0) * f, __builtin_amdgcn_cvt_f32_fp8(v, 1) * f,
                   __builtin_amdgcn_cvt_f32_fp8(v, 2) * f, __builtin_amdgcn_cvt_f32_fp8(v, 3) * f);
}

// 2^e with the smallest e >= -100 for which amax <= 448 * 2^e: 448 = 1.75 * 2^8, so one more than the exponent of amax less 8
// where its mantissa is above 1.75.
__device__ __forceinline__ float scale_for(uint32_t amax_bits) {
  const int e = static_cast<int>((amax_bits + 0x1FFFFFu) >> 23) - 8;  // biased
  return __uint_as_float(static_cast<uint32_t>(max(e, 127 - 100)) << 23);
}

// Which sequence owns row r: the number of starts at or below it, counted by the whole workgroup.
__device__ __forceinline__ int sequence_of(const PageTable &t, int r, int *s_count) {
  if (t.row_start == nullptr) return r;
  if (threadIdx.x == 0) *s_count = 0;
  __syncthreads();
  int n = 0;
  for (int s = threadIdx.x; s < t.n_seqs; s += kThreads) n += t.row_start[s] <= r;
  n = wave_sum_i(n);
  if ((threadIdx.x & 63) == 0) atomicAdd(s_count, n);
  __syncthreads();
  n = *s_count;
  __syncthreads();
  return n - 1;
}

// ---------------------------------------------------------------------------
// Rows into pages.  Pages are what the work is divided by: all rows of a page decide its scale together, so the workgroup of
// the row that is the first of its sequence to go to a page takes that page's rows, at most 64 that follow each other.  A
// workgroup looks at rows_per_block rows (one kv head; keys or values) and does the pages that begin among them.
// The page's tile is made whole in LDS, in the order that it has in memory, and written with 16-byte stores.
// ---------------------------------------------------------------------------
template <typename Tag, int D>
__global__ __launch_bounds__(kThreads) void store_pages_kernel(PageTable t, const int32_t *__restrict__ kv_len, uint8_t *__restrict__ k_pages,
                                                               uint8_t *__restrict__ v_pages, float *__restrict__ k_scale,
                                                               float *__restrict__ v_scale, int n_pages, int n_kv_heads,
                                                               const char *__restrict__ k_new, const char *__restrict__ v_new,
                                                               int64_t k_row_bytes, int64_t v_row_bytes, int rows_per_block) {
  using E = Elem<Tag>;
  constexpr int VE = E::kVec;
  constexpr int VECS = D / VE;                               // 16-byte vectors of a row's head
  constexpr int ITEMS = kPageTokens * VECS / kThreads;       // of a full page, a thread
  constexpr int TILE = kPageTokens * D;
  __shared__ uint4 s_tile[TILE / 16];
  __shared__ int s_row[kPageTokens];                         // the row of a slot, or -1
  __shared__ int s_count;
  __shared__ uint32_t s_amax[kThreads / 64];
  uint8_t *tile = reinterpret_cast<uint8_t *>(s_tile);
  const int tid = threadIdx.x, lane = tid & 63;
  const int h = blockIdx.y;
  const bool values = blockIdx.z != 0;
  const char *src = (values ? v_new : k_new) + static_cast<int64_t>(h) * D * E::kBytes;
  const int64_t row_bytes = values ? v_row_bytes : k_row_bytes;

  const int r0 = static_cast<int>(blockIdx.x) * rows_per_block;
  const int r1 = static_cast<int>(min(static_cast<int64_t>(r0) + rows_per_block, t.n_rows));
  int seq = sequence_of(t, r0, &s_count);
  int lo = 0, hi = 0;
  if (seq >= 0) rows_of(t, seq, lo, hi);
  for (int r = r0; r < r1;) {
    while (r >= hi || seq < 0) {  // on to the row's sequence (sequences without rows are passed over)
      if (++seq >= t.n_seqs) return;
      rows_of(t, seq, lo, hi);
      if (r < lo) r = lo;
      if (r >= r1) return;
    }
    const int pos = t.row_pos[r];
    const int logical = pos >> 6;
    if (pos < 0 || logical >= t.width || (r > lo && (t.row_pos[r - 1] >> 6) == logical)) {
      ++r;  // no token, or a row of a page that began before
      continue;
    }
    // the rows of this page: those from r on which lie in it without a gap
    const int rl = r + lane;
    const int pl = rl < hi ? t.row_pos[rl] : -1;
    const uint64_t in = __ballot(rl < hi && pl >= 0 && (pl >> 6) == logical);
    const int count = in == ~0ull ? 64 : __builtin_ctzll(~in);
    const int page = page_of(t, seq, logical, n_pages);
    const int len = kv_len[seq];
    const int next = r + count;
    if (page < 0) {
      r = next;
      continue;
    }
    __syncthreads();  // the page before is written
    if (tid < kPageTokens) s_row[tid] = -1;
    __syncthreads();
    if (tid < count) s_row[pl & 63] = rl;
    __syncthreads();

    const int64_t at = static_cast<int64_t>(page) * n_kv_heads + h;
    float *scale_at = (values ? v_scale : k_scale) + at;
    uint4 *out = reinterpret_cast<uint4 *>((values ? v_pages : k_pages) + at * TILE);
    const int filled = s_row[lane];
    const bool kept = __ballot(filled < 0 && lane < len - logical * 64) != 0;

    // rows and their largest element (as bits: magnitudes order as whole numbers)
    v4u x[ITEMS];
    uint32_t amax = 0;
#pragma unroll
    for (int u = 0; u < ITEMS; ++u) {
      const int it = u * kThreads + tid, row = s_row[it / VECS];
      x[u] = v4u{0, 0, 0, 0};
      if (row >= 0) x[u] = *reinterpret_cast<const v4u *>(src + row * row_bytes + (it % VECS) * 16);
    }
#pragma unroll
    for (int u = 0; u < ITEMS; ++u) {
      float f[VE];
      E::unpack(x[u], f);
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        const uint32_t b = __float_as_uint(f[e]) & 0x7FFFFFFFu;
        amax = max(amax, b < 0x7F800000u ? b : 0u);
      }
    }
    amax = static_cast<uint32_t>(wave_max_i(static_cast<int>(amax)));
    if (lane == 0) s_amax[tid >> 6] = amax;
    const float before = kept ? *scale_at : 0.f;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) amax = max(amax, s_amax[w]);
    const float scale = kept ? fmaxf(before, scale_for(amax)) : scale_for(amax);
    const float back = kept ? before / scale : 0.f;  // a power of two, at most 1
    const float inverse = 1.f / scale;

    for (int i = tid; i < TILE / 16; i += kThreads) {
      uint4 w = make_uint4(0, 0, 0, 0);
      if (kept) {
        w = out[i];
        if (back != 1.f) w = make_uint4(rescale_e4m3(w.x, back), rescale_e4m3(w.y, back), rescale_e4m3(w.z, back), rescale_e4m3(w.w, back));
      }
      s_tile[i] = w;
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < ITEMS; ++u) {
      const int it = u * kThreads + tid, slot = it / VECS, c = (it % VECS) * VE;
      if (s_row[slot] < 0) continue;
      float f[VE];
      E::unpack(x[u], f);
#pragma unroll
      for (int e = 0; e < VE; ++e) f[e] = (__float_as_uint(f[e]) & 0x7F800000u) == 0x7F800000u ? __uint_as_float(0x7FC00000u) : f[e] * inverse;
#pragma unroll
      for (int e = 0; e < VE; e += 4) {
        const uint32_t w = pack_e4m3(f[e], f[e + 1], f[e + 2], f[e + 3]);
        if (values) {
#pragma unroll
          for (int b = 0; b < 4; ++b) tile[(c + e + b) * kPageTokens + value_byte(slot)] = static_cast<uint8_t>(w >> (8 * b));
        } else {
          *reinterpret_cast<uint32_t *>(tile + slot * D + c + e) = w;
        }
      }
    }
    __syncthreads();
    for (int i = tid; i < TILE / 16; i += kThreads) out[i] = s_tile[i];
    if (tid == 0) *scale_at = scale;
    r = next;
  }
}

// ---------------------------------------------------------------------------
// Pages onto pages: every workgroup moves kCopyBytes of one page's keys or values.
// ---------------------------------------------------------------------------
constexpr int kCopyVecs = 4;                                  // 16-byte loads in flight, a thread
constexpr int kCopyBytes = kThreads * kCopyVecs * 16;

__global__ __launch_bounds__(kThreads) void copy_pages_kernel(PagePairs pairs, char *__restrict__ k, char *__restrict__ v,
                                                              float *__restrict__ k_scale, float *__restrict__ v_scale, int64_t page_bytes,
                                                              int n_kv_heads) {
  const int64_t src = pairs.src[blockIdx.y], dst = pairs.dst[blockIdx.y];
  char *pool = blockIdx.z != 0 ? v : k;
  const int64_t at = static_cast<int64_t>(blockIdx.x) * kCopyBytes + threadIdx.x * 16;
  const char *from = pool + src * page_bytes;
  char *to = pool + dst * page_bytes;
  v4u x[kCopyVecs];
#pragma unroll
  for (int u = 0; u < kCopyVecs; ++u)
    if (at + u * kThreads * 16 < page_bytes) x[u] = __builtin_nontemporal_load(reinterpret_cast<const v4u *>(from + at + u * kThreads * 16));
#pragma unroll
  for (int u = 0; u < kCopyVecs; ++u)
    if (at + u * kThreads * 16 < page_bytes) __builtin_nontemporal_store(x[u], reinterpret_cast<v4u *>(to + at + u * kThreads * 16));
  if (blockIdx.x == 0) {
    float *scale = blockIdx.z != 0 ? v_scale : k_scale;
    for (int h = threadIdx.x; h < n_kv_heads; h += kThreads) scale[dst * n_kv_heads + h] = scale[src * n_kv_heads + h];
  }
}

}  // namespace

hipError_t launch_store_pages(ifkv_ctx *ctx, const ifkv_page_cache &pages, const PageTable &t, const int32_t *kv_len, const void *k_new,
                              const void *v_new, int64_t k_stride, int64_t v_stride) {
  const auto &d = ctx->desc;
  // rows a workgroup looks at: a page's worth where that still leaves the chip enough of them, fewer otherwise
  const int64_t rows_per_block =
      std::max<int64_t>({std::min<int64_t>(64, t.n_rows * d.n_kv_heads / 1024), (t.n_rows + (int64_t(1) << 20) - 1) >> 20, 1});
  const int64_t e = static_cast<int64_t>(dtype_size(d.dtype));
  dim3 grid(static_cast<unsigned>((t.n_rows + rows_per_block - 1) / rows_per_block), d.n_kv_heads, 2), block(kThreads);
#define IFKV_LAUNCH_STORE(TAG, D)                                                                                                      \
  hipLaunchKernelGGL((store_pages_kernel<TAG, D>), grid, block, 0, ctx->stream, t, kv_len, static_cast<uint8_t *>(pages.k),           \
                     static_cast<uint8_t *>(pages.v), pages.k_scale, pages.v_scale, static_cast<int>(pages.n_pages), d.n_kv_heads,    \
                     static_cast<const char *>(k_new), static_cast<const char *>(v_new), k_stride * e, v_stride * e,                  \
                     static_cast<int>(rows_per_block))
  if (d.dtype == IFKV_BF16) {
    if (d.head_dim == 128)
      IFKV_LAUNCH_STORE(BF16Tag, 128);
    else
      IFKV_LAUNCH_STORE(BF16Tag, 64);
  } else {
    if (d.head_dim == 128)
      IFKV_LAUNCH_STORE(F32Tag, 128);
    else
      IFKV_LAUNCH_STORE(F32Tag, 64);
  }
#undef IFKV_LAUNCH_STORE
  return hipGetLastError();
}

hipError_t launch_copy_pages(ifkv_ctx *ctx, const ifkv_page_cache &pages, const PagePairs &pairs, int n) {
  const auto &d = ctx->desc;
  const int64_t page_bytes = static_cast<int64_t>(d.n_kv_heads) * kPageTokens * d.head_dim;
  dim3 grid(static_cast<unsigned>((page_bytes + kCopyBytes - 1) / kCopyBytes), n, 2), block(kThreads);
  hipLaunchKernelGGL(copy_pages_kernel, grid, block, 0, ctx->stream, pairs, static_cast<char *>(pages.k), static_cast<char *>(pages.v),
                     pages.k_scale, pages.v_scale, page_bytes, d.n_kv_heads);
  return hipGetLastError();
}

}  // namespace ifkv
