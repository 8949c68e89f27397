// Causal attention of rows over 8-bit pages.
//
// This file holds the dispatcher and the plain fp32 ALU kernel (contexts created with IFKV_FLAG_FORCE_GENERIC, cross-checking).  The
// matrix kernels live in attention_pages_matrix.hip.
#include <algorithm>

#include "attention_pages.h"

namespace ifkv {

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float e4m3_to_float(uint8_t b) { return __builtin_amdgcn_cvt_f32_fp8(b, 0); }

__device__ __forceinline__ float block_reduce_max(float v, float *red) {
  v = wave_max(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
}
__device__ __forceinline__ float block_reduce_sum(float v, float *red) {
  v = wave_sum(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return red[0] + red[1] + red[2] + red[3];
}

// One workgroup for each (row, query head).  256 tokens at a time: every thread forms one logit, the workgroup agrees on the
// running maximum and sum, then thread t adds to output column t % D over a share of the tokens.
template <typename Tag, int D>
__global__ __launch_bounds__(kThreads) void attend_pages_generic_kernel(PageTable t, int first_row, int n_rows, const uint8_t *__restrict__ k_pages,
                                                                        const uint8_t *__restrict__ v_pages,
                                                                        const float *__restrict__ k_scale, const float *__restrict__ v_scale,
                                                                        int n_pages, int n_q_heads, int n_kv_heads, float sm_scale,
                                                                        const void *__restrict__ q, int64_t q_stride, void *__restrict__ out,
                                                                        float *__restrict__ lse_out) {
  using E = Elem<Tag>;
  constexpr int PARTS = kThreads / D;
  __shared__ float s_q[D];
  __shared__ float s_p[kThreads];
  __shared__ int s_page[kThreads / kPageTokens];
  __shared__ float red[kThreads / 64];
  __shared__ float s_o[kThreads];
  const int tid = threadIdx.x, h = blockIdx.y, g = h / (n_q_heads / n_kv_heads);
  int lo, hi;
  const int s = static_cast<int>(blockIdx.x / n_rows);
  rows_of(t, s, lo, hi);
  const int i = first_row + static_cast<int>(blockIdx.x % n_rows);
  if (i >= hi - lo) return;
  const int r = lo + i;
  const int64_t row_head = static_cast<int64_t>(r) * n_q_heads + h;
  const int p = t.row_pos[r];
  const bool seen = p >= 0 && (p >> 6) < t.width;
  if (tid < D) s_q[tid] = seen ? E::load1(q, r * q_stride + h * D + tid) * sm_scale : 0.f;
  __syncthreads();
  const int c = tid % D, part = tid / D;
  float acc = 0.f, m_run = -INFINITY, l_run = 0.f;
  bool any = false;
  for (int64_t j0 = 0; seen && j0 <= p; j0 += kThreads) {
    const int64_t j = j0 + tid;
    int page = -1;
    if (j <= p) page = page_of(t, s, static_cast<int>(j >> 6), n_pages);
    const int64_t at = static_cast<int64_t>(page) * n_kv_heads + g;
    float logit = -INFINITY;
    if (page >= 0) {
      const uint8_t *k = k_pages + (at * kPageTokens + (j & 63)) * D;
      float dot = 0.f;
      for (int e = 0; e < D; ++e) dot = fmaf(s_q[e], e4m3_to_float(k[e]), dot);
      logit = dot * k_scale[at];
    }
    if ((tid & 63) == 0) s_page[tid >> 6] = page;
    any = __syncthreads_or(page >= 0) || any;
    const float m_new = fmaxf(m_run, block_reduce_max(logit, red));
    const float ref = m_new == -INFINITY ? 0.f : m_new;
    const float alpha = expf(m_run - ref);
    const float pj = page >= 0 ? expf(logit - ref) : 0.f;
    s_p[tid] = pj;
    l_run = l_run * alpha + block_reduce_sum(pj, red);  // its barriers publish s_p too
    m_run = m_new;
    acc *= alpha;
    const int nt = static_cast<int>(min<int64_t>(kThreads, p + 1 - j0));
    for (int jj = part; jj < nt; jj += PARTS) {
      if (s_page[jj >> 6] < 0) continue;
      const int64_t va = static_cast<int64_t>(s_page[jj >> 6]) * n_kv_heads + g;
      acc = fmaf(s_p[jj] * v_scale[va], e4m3_to_float(v_pages[(va * D + c) * kPageTokens + value_byte(jj & 63)]), acc);
    }
    __syncthreads();
  }
  s_o[tid] = acc;
  __syncthreads();
  if (tid < D) {
    float o = 0.f;
#pragma unroll
    for (int u = 0; u < PARTS; ++u) o += s_o[u * D + tid];
    E::store1(out, row_head * D + tid, any ? o / l_run : 0.f);
  }
  if (lse_out != nullptr && tid == 0) lse_out[row_head] = any ? m_run + logf(l_run) : -INFINITY;
}

template <typename Tag, int D>
hipError_t run_generic(ifkv_ctx *ctx, const ifkv_page_cache &pages, PageTable t, int max_rows, const void *q, int64_t q_stride, void *out,
                       float *lse_out) {
  const auto &d = ctx->desc;
  // a grid has fewer than 2^32 threads: so many rows of a sequence, and so many sequences, a launch
  constexpr int kMost = 1 << 23;
  const int rows = std::min(max_rows, kMost), step = kMost / rows;
  const int64_t e = static_cast<int64_t>(dtype_size(d.dtype));
  for (int s = 0; s < t.n_seqs; s += step)
    for (int r = 0; r < max_rows; r += rows) {
      const PageTable u = t.from(s, std::min(step, t.n_seqs - s));
      const int n = std::min(rows, max_rows - r);
      const int64_t skip = t.row_start != nullptr ? 0 : s;  // rows of the sequences before, where each has one
      hipLaunchKernelGGL((attend_pages_generic_kernel<Tag, D>), dim3(static_cast<unsigned>(u.n_seqs) * n, d.n_q_heads), dim3(kThreads), 0,
                         ctx->stream, u, r, n, static_cast<const uint8_t *>(pages.k),
                         static_cast<const uint8_t *>(pages.v), pages.k_scale, pages.v_scale, static_cast<int>(pages.n_pages), d.n_q_heads,
                         d.n_kv_heads, ctx->sm_scale, static_cast<const char *>(q) + skip * q_stride * e, q_stride,
                         static_cast<char *>(out) + skip * d.n_q_heads * D * e, lse_out != nullptr ? lse_out + skip * d.n_q_heads : nullptr);
    }
  return hipGetLastError();
}

}  // namespace

size_t attend_pages_scratch_bytes(const ifkv_ctx *ctx) {
  return ctx->desc.flags & IFKV_FLAG_FORCE_GENERIC ? 0 : attend_matrix_scratch_bytes(ctx);
}

hipError_t launch_attend_pages(ifkv_ctx *ctx, const ifkv_page_cache &pages, const PageTable &t, int32_t max_rows, const void *q,
                               int64_t q_stride, void *out, float *lse_out) {
  const auto &d = ctx->desc;
  if (!(d.flags & IFKV_FLAG_FORCE_GENERIC)) return launch_attend_matrix(ctx, pages, t, max_rows, q, q_stride, out, lse_out);
  if (d.dtype == IFKV_BF16) {
    if (d.head_dim == 128) return run_generic<BF16Tag, 128>(ctx, pages, t, max_rows, q, q_stride, out, lse_out);
    return run_generic<BF16Tag, 64>(ctx, pages, t, max_rows, q, q_stride, out, lse_out);
  }
  if (d.head_dim == 128) return run_generic<F32Tag, 128>(ctx, pages, t, max_rows, q, q_stride, out, lse_out);
  return run_generic<F32Tag, 64>(ctx, pages, t, max_rows, q, q_stride, out, lse_out);
}

}  // namespace ifkv
