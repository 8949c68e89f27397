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

// The sequence that owns row r and its rows, found by every wavefront for itself: the number of starts at or below r, less one
// (-1 and n_seqs: none does), the largest of those and the smallest of the others.
__device__ __forceinline__ int sequence_of(const PageTable &t, int r, int &lo, int &hi) {
  if (t.row_start == nullptr) {
    lo = r;
    hi = r + 1;
    return r;
  }
  int n = 0, below = 0, above = static_cast<int>(t.n_rows);
  for (int s = threadIdx.x & 63; s <= t.n_seqs; s += 64) {
    const int start = t.row_start[s];
    n += start <= r;
    below = start <= r ? max(below, start) : below;
    above = start <= r ? above : min(above, start);
  }
  lo = wave_max_i(below);
  hi = wave_min_i(above);
  return wave_reduce_i(n, [](int a, int b) __attribute__((always_inline)) { return a + b; }) - 1;
}

// Bits of all lanes, or-ed.
__device__ __forceinline__ uint64_t wave_or(uint64_t v) {
  const auto f = [](int a, int b) __attribute__((always_inline)) { return a | b; };
  const uint32_t lo = wave_reduce_i(static_cast<int>(v), f), hi = wave_reduce_i(static_cast<int>(v >> 32), f);
  return static_cast<uint64_t>(hi) << 32 | lo;
}

// ---------------------------------------------------------------------------
// Rows into pages.  Pages are what the work is divided by: all rows of a page decide its scale together, so the workgroup of
// the row that is the first of its sequence to go to a page takes that page's rows, at most 64 that follow each other.  A
// workgroup looks at rows_per_block rows (one kv head; keys or values) and does the pages that begin among them.
//
// Bytes go from registers straight to their places, and only those that change: a thread has eight (bf16) or four (fp32) elements of a
// token's key, or of four neighbouring tokens' values, which are four neighbouring bytes.  Which slots are filled is one
// 64-bit mask (rows ascend: the row of a slot is the number of filled slots before it), so the only thing that the wavefronts
// have to agree on is the largest element.  Memory bounds a finished context (32K tokens, 8 heads of 128 in bf16: 201 MB in
// 47 us, 41 at a copy's rate), the chain positions -> rows -> scale -> bytes a single token (one
// of each of 64 sequences 7 us; of 512 36 us, where a token's values change 4 bytes of 128 cache lines a head).
// ---------------------------------------------------------------------------
template <typename Tag, int D>
__global__ __launch_bounds__(kThreads, Elem<Tag>::kBytes == 2 ? 5 : 4) void store_pages_kernel(
    PageTable t, const int32_t *__restrict__ kv_len, uint8_t *__restrict__ k_pages, uint8_t *__restrict__ v_pages,
    float *__restrict__ k_scale, float *__restrict__ v_scale, int n_pages, int n_kv_heads, const char *__restrict__ k_new,
    const char *__restrict__ v_new, int64_t k_row_bytes, int64_t v_row_bytes, int rows_per_block) {
  using E = Elem<Tag>;
  constexpr int VE = E::kVec;
  constexpr int VECS = D / VE;                                              // 16-byte vectors of a row's head
  constexpr int QUADS = (kPageTokens / 4 * VECS + kThreads - 1) / kThreads;  // of a thread: four vectors each
  constexpr int TILE = kPageTokens * D;
  __shared__ uint32_t s_amax[2][kThreads / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int h = blockIdx.y;
  const bool values = blockIdx.z != 0;
  const char *src = (values ? v_new : k_new) + static_cast<int64_t>(h) * D * E::kBytes;
  const int64_t row_bytes = values ? v_row_bytes : k_row_bytes;
  // the four slots of a quad and its place within a row: four neighbouring tokens for values, the same vector of slots that lie
  // kSlotStep apart for keys (whose neighbours then write a row of bytes together)
  constexpr int kSlotStep = kThreads / VECS < 16 ? kThreads / VECS : 16;

  const int r0 = static_cast<int>(blockIdx.x) * rows_per_block;
  const int r1 = static_cast<int>(min(static_cast<int64_t>(r0) + rows_per_block, t.n_rows));
  const auto block_of = [&](int pos) __attribute__((always_inline)) { return pos >= 0 && (pos >> 6) < t.width ? pos >> 6 : -1; };
  int seq = -1, lo = 0, hi = 0, turn = 0;
  for (int r = r0; r < r1;) {
    // positions of the next rows (asked for before it is known whose they are) and of the one before them
    const int ahead = t.row_pos[min(static_cast<int64_t>(r) + lane, t.n_rows - 1)], behind = t.row_pos[max(r - 1, 0)];
    if (r == r0) {
      seq = sequence_of(t, r0, lo, hi);
      if (seq < 0) hi = 0;
    }
    while (r >= hi) {   // on to the row's sequence (sequences without rows are passed over)
      if (++seq >= t.n_seqs) return;
      rows_of(t, seq, lo, hi);
    }
    if (seq >= t.n_seqs) return;
    if (r < lo) {
      r = lo;
      continue;
    }
    // the next row that is the first of its page
    const int pl = lane < hi - r ? ahead : -1;
    const int mine = block_of(pl);
    int before = __shfl_up(mine, 1, 64);
    if (lane == 0) before = r > lo ? block_of(behind) : -1;
    const uint64_t begins = __ballot(mine >= 0 && mine != before && lane < r1 - r);
    const int skip = begins != 0 ? __builtin_ctzll(begins) : 64;
    if (skip > 0) {
      r += min(skip, hi - r);
      continue;
    }
    const int logical = __builtin_amdgcn_readfirstlane(mine);
    // (requests that need no other's answer go out together: the page, the length, the rows)
    const int page = page_of(t, seq, logical, n_pages);
    const int len = kv_len[seq];
    // the rows of this page: those from r on which lie in it without a gap
    const uint64_t in = __ballot(pl >= 0 && (pl >> 6) == logical);
    const int count = in == ~0ull ? 64 : __builtin_ctzll(~in);
    const int first = r;
    r += count;
    const uint64_t filled = wave_or(lane < count ? 1ull << (pl & 63) : 0ull);
    const auto slot_of = [&](int quad, int i) __attribute__((always_inline)) {
      if (values) return (quad & 15) * 4 + i;
      const int s = quad / VECS;
      return (s / kSlotStep * 4 + i) * kSlotStep + s % kSlotStep;
    };
    const auto vector_of = [&](int quad) __attribute__((always_inline)) { return values ? quad >> 4 : quad % VECS; };
    v4u x[QUADS][4];
#pragma unroll
    for (int u = 0; u < QUADS; ++u) {
      const int quad = u * kThreads + tid;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[u][i] = v4u{0, 0, 0, 0};
        if (quad >= kPageTokens / 4 * VECS) continue;
        const int s = slot_of(quad, i);
        if (filled >> s & 1) {
          const int row = first + __builtin_popcountll(filled & ((1ull << s) - 1));
          x[u][i] = __builtin_nontemporal_load(reinterpret_cast<const v4u *>(src + row * row_bytes + vector_of(quad) * 16));
        }
      }
    }
    if (page < 0) continue;
    const int held = min(max(len - logical * kPageTokens, 0), kPageTokens);
    const bool kept = (~filled & (held == 64 ? ~0ull : (1ull << held) - 1)) != 0;
    const int64_t at = static_cast<int64_t>(page) * n_kv_heads + h;
    float *scale_at = (values ? v_scale : k_scale) + at;
    uint8_t *out = (values ? v_pages : k_pages) + at * TILE;
    const float old = kept ? *scale_at : 0.f;
    // what is there beside a value that is written
    uint32_t there[QUADS][VE];
#pragma unroll
    for (int u = 0; u < QUADS; ++u) {
      const int quad = u * kThreads + tid;
      const uint32_t has = quad < kPageTokens / 4 * VECS ? static_cast<uint32_t>(filled >> (quad & 15) * 4) & 15u : 0u;
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        there[u][e] = 0;
        if (values && kept && has != 0 && has != 15)
          there[u][e] = *reinterpret_cast<uint32_t *>(out + (vector_of(quad) * VE + e) * kPageTokens + value_byte((quad & 15) * 4));
      }
    }
    // the rows' largest element (as bits: magnitudes order as whole numbers)
    uint32_t amax = 0;
#pragma unroll
    for (int u = 0; u < QUADS; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float f[VE];
        E::unpack(x[u][i], f);
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          const uint32_t b = __float_as_uint(f[e]) & 0x7FFFFFFFu;
          amax = max(amax, b < 0x7F800000u ? b : 0u);
        }
      }
    amax = static_cast<uint32_t>(wave_max_i(static_cast<int>(amax)));
    if (lane == 0) s_amax[turn][wave] = amax;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) amax = max(amax, s_amax[turn][w]);
    turn ^= 1;   // (the next page's maxima do not meet a wavefront that still reads these)
    const float scale = kept ? fmaxf(old, scale_for(amax)) : scale_for(amax);
    const float back = kept ? old / scale : 0.f;  // a power of two, at most 1
    const float inverse = 1.f / scale;

#pragma unroll
    for (int u = 0; u < QUADS; ++u) {
      const int quad = u * kThreads + tid;
      if (quad >= kPageTokens / 4 * VECS) continue;
      uint32_t w[4][VE / 4];   // bytes of the four slots
      uint32_t has = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        has |= static_cast<uint32_t>(filled >> slot_of(quad, i) & 1) << i;
        float f[VE];
        E::unpack(x[u][i], f);
#pragma unroll
        for (int e = 0; e < VE; ++e) f[e] = (__float_as_uint(f[e]) & 0x7F800000u) == 0x7F800000u ? __uint_as_float(0x7FC00000u) : f[e] * inverse;
#pragma unroll
        for (int e = 0; e < VE / 4; ++e) w[i][e] = pack_e4m3(f[4 * e], f[4 * e + 1], f[4 * e + 2], f[4 * e + 3]);
      }
      const int c = vector_of(quad) * VE;
      if (!values) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          typedef uint32_t Bytes __attribute__((ext_vector_type(VE / 4)));
          Bytes *to = reinterpret_cast<Bytes *>(out + slot_of(quad, i) * D + c);
          if (has >> i & 1) {
            Bytes b;
#pragma unroll
            for (int e = 0; e < VE / 4; ++e) b[e] = w[i][e];
            *to = b;
          } else if (!kept) {
            *to = Bytes(0);
          } else if (back != 1.f) {
            Bytes b = *to;
#pragma unroll
            for (int e = 0; e < VE / 4; ++e) b[e] = rescale_e4m3(b[e], back);
            *to = b;
          }
        }
      } else if (has != 0 || !kept || back != 1.f) {
        const uint32_t bytes = (has & 1 ? 0xFFu : 0u) | (has & 2 ? 0xFF00u : 0u) | (has & 4 ? 0xFF0000u : 0u) | (has & 8 ? 0xFF000000u : 0u);
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          uint32_t *to = reinterpret_cast<uint32_t *>(out + (c + e) * kPageTokens + value_byte((quad & 15) * 4));
          uint32_t beside = there[u][e];
          if (back != 1.f && kept && has != 15) beside = rescale_e4m3(has == 0 ? *to : beside, back);
          const int s = e % 4 * 8;
          const uint32_t fresh = (w[0][e / 4] >> s & 0xFF) | (w[1][e / 4] >> s & 0xFF) << 8 | (w[2][e / 4] >> s & 0xFF) << 16 |
                                 (w[3][e / 4] >> s & 0xFF) << 24;
          *to = (beside & ~bytes) | (fresh & bytes);
        }
      }
    }
    if (tid == 0) *scale_at = scale;
  }
}

// ---------------------------------------------------------------------------
// Pages onto pages: every workgroup moves kCopyBytes of one page's keys or values.  2000 pages of 8 heads of 128 (525 MB) 111 us, 0.95
// of a copy's rate; 32 pages 4.6 us.
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
  // Rows a workgroup looks at: a page's worth, or as few as make some 2048 workgroups of them.  Fewer are better where rows are dense (most
  // workgroups find no page of their own), more where many pages get a row each: 512 workgroups for 64 sequences of 64 rows take 15 us,
  // for 63 single rows and 2048 of a prompt 176; 2048 take 23 and 56.  The rows of one sequence alone are dense more often than
  // not: 1024 (2048 rows of a prompt 8.4 us with 1024, 14.9 with 2048; 512 rows of as many pages 38 and 34).
  const int64_t workgroups = t.n_seqs == 1 ? 1024 : 2048;
  const int64_t rows_per_block = std::max<int64_t>(
      {std::min<int64_t>(64, t.n_rows * d.n_kv_heads * 2 / workgroups), (t.n_rows + (int64_t(1) << 20) - 1) >> 20, 1});
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
