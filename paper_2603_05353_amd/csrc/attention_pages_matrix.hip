// Attention over 8-bit pages on the matrix cores.
//
// Decoding reads every page once for a few query columns: memory bounds it, and what a kernel has to do is to keep requests in
// flight.  A wavefront takes whole pages, as many bytes as it likes to have under way, straight from memory into registers in
// the operand layout of the 16x16x32 bf16 instruction (no LDS, no barrier, no shuffle in the loop):
//   first product, S^T[token, column]: a lane's keys of a block of 16 tokens are d/4 bytes in a row of one token
//     (the order of the d elements along the reduction is free, queries follow it);
//   second product, O^T[d, column]: a lane's values are the 16 bytes in a row of one value row that ifkv.h's byte order makes
//     of the very tokens whose probabilities the lane holds.
// e4m3 numbers become bf16 exactly, two an instruction, with the page's scale multiplied in.
#include <algorithm>

#include "attention_pages.h"

namespace ifkv {

namespace {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;
constexpr float kLowest = -3.402823466e38f;
// Exponentials are taken against a reference that rises only where a logit exceeds it by more than 2^kSlack: sums stay below
// 2^(kSlack + 31), and most pages need no look at the other lanes' maxima.
constexpr float kSlack = 16.f;

template <typename Tag>
struct Precision;
template <>
struct Precision<BF16Tag> {
  static constexpr int kQ = 1, kP = 2;  // bf16 numbers that hold a query element and a probability
};
template <>
struct Precision<F32Tag> {
  static constexpr int kQ = 3, kP = 3;
};

// Partial results of one part: accumulators as the wavefront holds them, then reference and sum of every column.
template <int D, int NT>
struct Image {
  static constexpr int kRegs = NT * D / 16;       // f32x4 of a lane
  f32x4 o[kRegs][64];
  float ref[NT][16], sum[NT][16];
};

// DT blocks of 16 output rows of a column, from block dt0 on.
template <typename Tag, int D, int DT>
__device__ __forceinline__ void write_columns(void *out, float *lse_out, int64_t row_head, int dt0, int g, const f32x4 *o, int stride, float ref,
                                              float sum) {
  // a column without any token: zeros, and the logarithm of nothing
  const float inv = 1.f / sum;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) {
    f32x4 x = o[dt * stride];
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = ref == -INFINITY ? 0.f : x[e] * inv;
    const int64_t at = row_head * D + (dt0 + dt) * 16 + g * 4;
    if constexpr (Elem<Tag>::kBytes == 2) {
      typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
      *reinterpret_cast<bf16x4 *>(static_cast<__bf16 *>(out) + at) =
          bf16x4{static_cast<__bf16>(x[0]), static_cast<__bf16>(x[1]), static_cast<__bf16>(x[2]), static_cast<__bf16>(x[3])};
    } else {
      *reinterpret_cast<f32x4 *>(static_cast<float *>(out) + at) = x;
    }
  }
  if (lse_out != nullptr && g == 0) lse_out[row_head] = ref == -INFINITY ? -INFINITY : ref * kLn2 + logf(sum);
}

// ---------------------------------------------------------------------------
// A workgroup's four wavefronts take the pages of a part in turn, all for the same NT * 16 query columns, and join at the end.
// ---------------------------------------------------------------------------
template <typename Tag, int D, int NT>
__global__ __launch_bounds__(kAttendThreads, NT == 1 ? 2 : 1) void attend_pages_kernel(
    PageTable t, AttendPlan plan, int max_rows, const uint8_t *__restrict__ k_pages, const uint8_t *__restrict__ v_pages,
    const float *__restrict__ k_scale, const float *__restrict__ v_scale, int n_pages, int n_q_heads, int n_kv_heads, float logit_scale,
    const void *__restrict__ q, int64_t q_stride, void *__restrict__ out, float *__restrict__ lse_out, int2 *__restrict__ meta,
    Image<D, NT> *__restrict__ partials) {
  constexpr int QP = Precision<Tag>::kQ, PP = Precision<Tag>::kP;
  constexpr int KS = D / 32;       // steps of the first product
  constexpr int KV = D / 64;       // 16-byte key loads of a lane and block of 16 tokens
  constexpr int DT = D / 16;       // blocks of 16 output rows
  constexpr int TILE = kPageTokens * D;
  __shared__ union {
    AttendPlanMemory plan;
    Image<D, NT> image[2];
  } mem;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n = lane & 15, g = lane >> 4;
  const int h = blockIdx.y;
  AttendPart part;
  if (!find_part(t, plan, max_rows, blockIdx.x, h == 0, meta, mem.plan, part)) return;

  // this lane's column of every tile: its row and where it is in out; columns that see nothing get queries of zero, no
  // mask, and at the end zeros
  const int grp = plan.group;
  int pos[NT];
  int64_t row_head[NT];
  bool real[NT];   // a row of the sequence
  bf16x8 qf[NT][QP][KS];
  int lowest = INT32_MAX;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int c = part.block * plan.columns + nt * 16 + n;
    const int r = part.lo + c / grp;
    const int hq = h * grp + c % grp;
    real[nt] = r < part.hi;
    pos[nt] = real[nt] ? t.row_pos[r] : -1;
    row_head[nt] = static_cast<int64_t>(r) * n_q_heads + hq;
    const bool sees = pos[nt] >= 0 && (pos[nt] >> 6) < t.width;
    if (!sees) pos[nt] = INT32_MAX;
    lowest = min(lowest, pos[nt]);
    const char *src = static_cast<const char *>(q) + (r * q_stride + static_cast<int64_t>(hq) * D + g * (D / 4)) * Elem<Tag>::kBytes;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      if constexpr (QP == 1) {
        v4u w = {0, 0, 0, 0};
        if (sees) w = reinterpret_cast<const v4u *>(src)[ks];
        qf[nt][0][ks] = __builtin_bit_cast(bf16x8, w);
      } else {
        float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        if (sees) {
          *reinterpret_cast<f32x4 *>(x) = reinterpret_cast<const f32x4 *>(src)[2 * ks];
          *reinterpret_cast<f32x4 *>(x + 4) = reinterpret_cast<const f32x4 *>(src)[2 * ks + 1];
        }
        bf16x8 s[QP];
        split8<QP>(x, s);
#pragma unroll
        for (int p = 0; p < QP; ++p) {
          qf[nt][p][ks] = s[p];
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (p > 0 && !(fabsf(x[e]) < INFINITY)) qf[nt][p][ks][e] = static_cast<__bf16>(0.f);
        }
      }
    }
  }
  const int min_pos = wave_min_i(lowest);

  f32x4 o[DT][NT];
  float ref[NT], neg_ref[NT], sum[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    ref[nt] = -INFINITY;
    neg_ref[nt] = 0.f;
    sum[nt] = 0.f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[dt][nt] = f32x4{0, 0, 0, 0};
  }

  const int32_t *row_of_table = t.table + static_cast<int64_t>(part.seq) * t.width;
  // pages of this wavefront, 64 at a time: lane i knows the i-th
  for (int base = part.first + wave; base < part.last; base += 64 * kAttendWaves) {
    const int mine = base + lane * kAttendWaves;
    int entry = -1;
    if (mine < part.last) entry = row_of_table[mine];
    uint64_t todo = __ballot(entry >= 0 && entry < n_pages);
    if (todo == 0) continue;
    float ks_lane = 1.f, vs_lane = 1.f;
    if (entry >= 0 && entry < n_pages) {
      const int64_t at = static_cast<int64_t>(entry) * n_kv_heads + h;
      ks_lane = k_scale[at];
      vs_lane = v_scale[at];
    }
    v4u kb[4][KV], vb[DT];
    auto page_at = [&](int i) __attribute__((always_inline)) {
      return (static_cast<int64_t>(__builtin_amdgcn_readlane(entry, i)) * n_kv_heads + h) * TILE;
    };
    auto load_k = [&](int64_t at) __attribute__((always_inline)) {
      const uint8_t *src = k_pages + at + n * D + g * (D / 4);
#pragma unroll
      for (int rt = 0; rt < 4; ++rt)
#pragma unroll
        for (int u = 0; u < KV; ++u) kb[rt][u] = __builtin_nontemporal_load(reinterpret_cast<const v4u *>(src + rt * 16 * D + u * 16));
    };
    auto load_v = [&](int64_t at) __attribute__((always_inline)) {
      const uint8_t *src = v_pages + at + n * kPageTokens + g * 16;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) vb[dt] = __builtin_nontemporal_load(reinterpret_cast<const v4u *>(src + dt * 16 * kPageTokens));
    };
    int i = __builtin_ctzll(todo);
    {
      const int64_t at = page_at(i);
      load_k(at);
      load_v(at);
    }
    while (todo != 0) {
      todo &= todo - 1;
      const int next = todo != 0 ? __builtin_ctzll(todo) : i;   // (the last page is requested once more, from the cache)
      const int64_t next_at = page_at(next);
      const float ks_page = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ks_lane), i));
      const float vs_page = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(vs_lane), i));
      const int token0 = (base + i * kAttendWaves) * kPageTokens;

      f32x4 s[4][NT];
#pragma unroll
      for (int rt = 0; rt < 4; ++rt) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) s[rt][nt] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const v4u w = kb[rt][ks / 2];
          const bf16x8 a = ks % 2 == 0 ? widen(w.x, w.y, ks_page) : widen(w.z, w.w, ks_page);
#pragma unroll
          for (int p = QP - 1; p >= 0; --p)   // smallest first
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) s[rt][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, qf[nt][p][ks], s[rt][nt], 0, 0, 0);
        }
      }
      if (next != i) load_k(next_at);

      const bool masked = token0 + kPageTokens - 1 > min_pos;
      if (masked) {
#pragma unroll
        for (int rt = 0; rt < 4; ++rt)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (token0 + rt * 16 + g * 4 + e > pos[nt]) s[rt][nt][e] = -INFINITY;
      }
      bool rise = false;
      float top[NT];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float m = -INFINITY;
#pragma unroll
        for (int rt = 0; rt < 4; ++rt)
#pragma unroll
          for (int e = 0; e < 4; ++e) m = fmaxf(m, s[rt][nt][e]);
        top[nt] = m * logit_scale;
        rise = rise || ref[nt] == -INFINITY || top[nt] > ref[nt] + kSlack;
      }
      if (__ballot(rise) != 0) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float m = top[nt];
          m = fmaxf(m, __shfl_xor(m, 16, 64));
          m = fmaxf(m, __shfl_xor(m, 32, 64));
          const float old = ref[nt];
          if (token0 <= pos[nt]) ref[nt] = fmaxf(old, fmaxf(m, kLowest));
          neg_ref[nt] = ref[nt] == -INFINITY ? 0.f : -ref[nt];
          const float by = old == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(old - ref[nt]);
          sum[nt] *= by;
#pragma unroll
          for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[dt][nt][e] *= by;
        }
      }
      bf16x8 pf[2][NT][PP];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int st = 0; st < 2; ++st) {
          float p[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            p[e] = __builtin_amdgcn_exp2f(fmaf(s[2 * st + e / 4][nt][e % 4], logit_scale, neg_ref[nt]));
            sum[nt] += p[e];
          }
          split8<PP>(p, pf[st][nt]);
        }
      }
      if (masked) {
        // Values behind a column's token count nothing, NaN neither: NaN bytes become zero, and columns that do see one get it back.
        bool any = false;
        v4u spoiled[DT];
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t w = vb[dt][e];
            const uint32_t bad = (((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) >> 7;   // 1 in the bytes that are NaN
            any = any || bad != 0;
            spoiled[dt][e] = bad * 0x38u;                                                   // 1.0 in e4m3
            vb[dt][e] = w & ~(bad * 0xFFu);
          }
        }
        if (__ballot(any) != 0) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            bf16x8 seen[2];
#pragma unroll
            for (int st = 0; st < 2; ++st)
#pragma unroll
              for (int e = 0; e < 8; ++e)
                seen[st][e] = static_cast<__bf16>(token0 + (2 * st + e / 4) * 16 + g * 4 + e % 4 <= pos[nt] ? 1.f : 0.f);
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
              f32x4 count = {0, 0, 0, 0};
              count = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(spoiled[dt].x, spoiled[dt].y, 1.f), seen[0], count, 0, 0, 0);
              count = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(spoiled[dt].z, spoiled[dt].w, 1.f), seen[1], count, 0, 0, 0);
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (count[e] > 0.f) o[dt][nt][e] = __uint_as_float(0x7FC00000u);
            }
          }
        }
      }
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const bf16x8 a0 = widen(vb[dt].x, vb[dt].y, vs_page), a1 = widen(vb[dt].z, vb[dt].w, vs_page);
#pragma unroll
        for (int p = PP - 1; p >= 0; --p)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            o[dt][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a0, pf[0][nt][p], o[dt][nt], 0, 0, 0);
            o[dt][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a1, pf[1][nt][p], o[dt][nt], 0, 0, 0);
          }
      }
      if (next != i) load_v(next_at);
      i = next;
    }
  }

  // a column's tokens are spread over four lanes
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    sum[nt] += __shfl_xor(sum[nt], 16, 64);
    sum[nt] += __shfl_xor(sum[nt], 32, 64);
  }
  // wavefronts 2 and 3 into 0 and 1, then 1 into 0
#pragma unroll
  for (int half = 2; half >= 1; half >>= 1) {
    __syncthreads();   // (the plan's memory, or the images of the step before)
    if (wave >= half && wave < 2 * half) {
      Image<D, NT> &im = mem.image[wave - half];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) im.o[dt * NT + nt][lane] = o[dt][nt];
        if (g == 0) im.ref[nt][n] = ref[nt], im.sum[nt][n] = sum[nt];
      }
    }
    __syncthreads();
    if (wave < half) {
      const Image<D, NT> &im = mem.image[wave];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const float other = im.ref[nt][n], m = fmaxf(ref[nt], other);
        const float a = ref[nt] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ref[nt] - m);
        const float b = other == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(other - m);
        ref[nt] = m;
        sum[nt] = sum[nt] * a + im.sum[nt][n] * b;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          const f32x4 x = im.o[dt * NT + nt][lane];
#pragma unroll
          for (int e = 0; e < 4; ++e) o[dt][nt][e] = o[dt][nt][e] * a + x[e] * b;
        }
      }
    }
  }
  if (wave != 0) return;
  if (part.n_parts == 1) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
      if (real[nt]) write_columns<Tag, D, DT>(out, lse_out, row_head[nt], 0, g, &o[0][nt], NT, pos[nt] == INT32_MAX ? -INFINITY : ref[nt], sum[nt]);
    return;
  }
  Image<D, NT> &im = partials[static_cast<int64_t>(h) * 2 * plan.target_parts + part.slot];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) im.o[dt * NT + nt][lane] = o[dt][nt];
    if (g == 0) im.ref[nt][n] = pos[nt] == INT32_MAX ? -INFINITY : ref[nt], im.sum[nt][n] = sum[nt];
  }
}

// Joins the parts of an item: a workgroup for a quarter of the output rows of a tile of 16 columns.  Its wavefronts take the
// parts in turn, eight requests under way, and join.
constexpr int kMergeSplit = 4, kMergeBatch = 8;

template <typename Tag, int D, int NT>
__global__ __launch_bounds__(kAttendThreads) void attend_pages_merge_kernel(PageTable t, AttendPlan plan, int max_rows, int n_q_heads,
                                                                            const int2 *__restrict__ meta,
                                                                            const Image<D, NT> *__restrict__ partials,
                                                                            void *__restrict__ out, float *__restrict__ lse_out) {
  constexpr int DT = D / 16 / kMergeSplit;
  __shared__ f32x4 s_o[kAttendWaves - 1][DT][64];
  __shared__ float s_ref[kAttendWaves][16], s_sum[kAttendWaves][16];
  const int item = blockIdx.x / (NT * kMergeSplit), nt = blockIdx.x / kMergeSplit % NT, quarter = blockIdx.x % kMergeSplit;
  const int h = blockIdx.y;
  const int2 m = meta[item];
  if (m.y <= 1) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, g = lane >> 4;
  const Image<D, NT> *im = partials + static_cast<int64_t>(h) * 2 * plan.target_parts + m.x;
  float ref = -INFINITY, sum = 0.f;
  f32x4 o[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) o[dt] = f32x4{0, 0, 0, 0};
  for (int p0 = wave; p0 < m.y; p0 += kAttendWaves * kMergeBatch) {
    float refs[kMergeBatch], sums[kMergeBatch];
    f32x4 x[kMergeBatch][DT];
#pragma unroll
    for (int u = 0; u < kMergeBatch; ++u) {
      const int p = p0 + u * kAttendWaves;
      refs[u] = -INFINITY;
      sums[u] = 0.f;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) x[u][dt] = f32x4{0, 0, 0, 0};
      if (p < m.y) {
        refs[u] = im[p].ref[nt][n];
        sums[u] = im[p].sum[nt][n];
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) x[u][dt] = im[p].o[(quarter * DT + dt) * NT + nt][lane];
      }
    }
    float top = ref;
#pragma unroll
    for (int u = 0; u < kMergeBatch; ++u) top = fmaxf(top, refs[u]);
    const float a = ref == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ref - top);
    ref = top;
    sum *= a;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[dt][e] *= a;
#pragma unroll
    for (int u = 0; u < kMergeBatch; ++u) {
      const float b = refs[u] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(refs[u] - top);
      sum = fmaf(sums[u], b, sum);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[dt][e] = fmaf(x[u][dt][e], b, o[dt][e]);
    }
  }
  if (g == 0) s_ref[wave][n] = ref, s_sum[wave][n] = sum;
  if (wave > 0)
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) s_o[wave - 1][dt][lane] = o[dt];
  __syncthreads();
  if (wave > 0) return;
  float top = ref;
#pragma unroll
  for (int w = 1; w < kAttendWaves; ++w) top = fmaxf(top, s_ref[w][n]);
  const float a = ref == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ref - top);
  sum *= a;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[dt][e] *= a;
#pragma unroll
  for (int w = 1; w < kAttendWaves; ++w) {
    const float b = s_ref[w][n] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s_ref[w][n] - top);
    sum = fmaf(s_sum[w][n], b, sum);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      const f32x4 x = s_o[w - 1][dt][lane];
#pragma unroll
      for (int e = 0; e < 4; ++e) o[dt][e] = fmaf(x[e], b, o[dt][e]);
    }
  }
  int lo, hi;
  rows_of(t, item / plan.n_blocks, lo, hi);
  hi = min(hi, lo + max_rows);
  const int c = (item % plan.n_blocks) * plan.columns + nt * 16 + n;
  const int r = lo + c / plan.group;
  if (r < hi)
    write_columns<Tag, D, DT>(out, quarter == 0 ? lse_out : nullptr, static_cast<int64_t>(r) * n_q_heads + h * plan.group + c % plan.group,
                              quarter * DT, g, o, 1, top, sum);
}

// Workgroups that a launch is cut into, about: four times what the chip holds at two a CU, so that uneven parts even out.
constexpr int kTargetWorkgroups = 1024;
constexpr int kLeastPages = 8;                    // of a part: two for each wavefront
constexpr size_t kMetaBytes = kMaxItems * sizeof(int2);

template <typename Tag, int D, int NT>
size_t scratch_for(int n_kv_heads) {
  const int target = std::max(1, kTargetWorkgroups / NT / n_kv_heads);
  return kMetaBytes + static_cast<size_t>(2) * target * n_kv_heads * sizeof(Image<D, NT>);
}

template <typename Tag, int D, int NT>
hipError_t run(ifkv_ctx *ctx, const ifkv_page_cache &pages, const PageTable &t, int max_rows, const void *q, int64_t q_stride, void *out,
               float *lse_out) {
  const auto &d = ctx->desc;
  AttendPlan plan;
  plan.group = d.n_q_heads / d.n_kv_heads;
  plan.columns = NT * 16;
  plan.n_blocks = static_cast<int>((static_cast<int64_t>(max_rows) * plan.group + plan.columns - 1) / plan.columns);
  plan.least_pages = kLeastPages;
  const int64_t items = static_cast<int64_t>(t.n_seqs) * plan.n_blocks;
  const bool cut = t.width > kLeastPages && items <= kMaxItems && items * t.width < INT32_MAX;   // (pages are added up in 32 bits)
  plan.target_parts = cut ? std::max(1, kTargetWorkgroups / NT / d.n_kv_heads) : 0;
  int2 *meta = static_cast<int2 *>(ctx->page_partials);
  Image<D, NT> *partials = reinterpret_cast<Image<D, NT> *>(static_cast<char *>(ctx->page_partials) + kMetaBytes);
  // a grid has fewer than 2^32 threads: so many sequences a launch (all of them where items are cut)
  const int step = std::max(1, (1 << 23) / plan.n_blocks);
  for (int s = 0; s < t.n_seqs; s += step) {
    const PageTable u = t.from(s, std::min(step, t.n_seqs - s));
    const int64_t skip = t.row_start != nullptr ? 0 : s;  // rows of the sequences before, where each has one
    const int64_t n_items = static_cast<int64_t>(u.n_seqs) * plan.n_blocks;
    hipLaunchKernelGGL((attend_pages_kernel<Tag, D, NT>), dim3(static_cast<unsigned>(n_items + plan.target_parts), d.n_kv_heads),
                       dim3(kAttendThreads), 0, ctx->stream, u, plan, max_rows, static_cast<const uint8_t *>(pages.k),
                       static_cast<const uint8_t *>(pages.v), pages.k_scale, pages.v_scale, static_cast<int>(pages.n_pages), d.n_q_heads,
                       d.n_kv_heads, ctx->sm_scale * kLog2e, static_cast<const char *>(q) + skip * q_stride * Elem<Tag>::kBytes, q_stride,
                       static_cast<char *>(out) + skip * d.n_q_heads * D * Elem<Tag>::kBytes,
                       lse_out != nullptr ? lse_out + skip * d.n_q_heads : nullptr, meta, partials);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (!cut) return hipSuccess;
  hipLaunchKernelGGL((attend_pages_merge_kernel<Tag, D, NT>), dim3(static_cast<unsigned>(items * NT * kMergeSplit), d.n_kv_heads),
                     dim3(kAttendThreads), 0, ctx->stream, t,
                     plan, max_rows, d.n_q_heads, meta, partials, out, lse_out);
  return hipGetLastError();
}

template <typename Tag, int D>
hipError_t run_columns(ifkv_ctx *ctx, const ifkv_page_cache &pages, const PageTable &t, int max_rows, const void *q, int64_t q_stride,
                       void *out, float *lse_out) {
  const int64_t columns = static_cast<int64_t>(max_rows) * (ctx->desc.n_q_heads / ctx->desc.n_kv_heads);
  if (columns <= 16) return run<Tag, D, 1>(ctx, pages, t, max_rows, q, q_stride, out, lse_out);
  if (columns <= 32 || Precision<Tag>::kQ > 1) return run<Tag, D, 2>(ctx, pages, t, max_rows, q, q_stride, out, lse_out);
  if constexpr (Precision<Tag>::kQ == 1) return run<Tag, D, 4>(ctx, pages, t, max_rows, q, q_stride, out, lse_out);
}

}  // namespace

size_t attend_matrix_scratch_bytes(const ifkv_ctx *ctx) {
  const auto &d = ctx->desc;
  const bool wide = d.head_dim == 128;
  if (d.dtype == IFKV_F32) {
    return wide ? std::max(scratch_for<F32Tag, 128, 1>(d.n_kv_heads), scratch_for<F32Tag, 128, 2>(d.n_kv_heads))
                : std::max(scratch_for<F32Tag, 64, 1>(d.n_kv_heads), scratch_for<F32Tag, 64, 2>(d.n_kv_heads));
  }
  return wide ? std::max({scratch_for<BF16Tag, 128, 1>(d.n_kv_heads), scratch_for<BF16Tag, 128, 2>(d.n_kv_heads), scratch_for<BF16Tag, 128, 4>(d.n_kv_heads)})
              : std::max({scratch_for<BF16Tag, 64, 1>(d.n_kv_heads), scratch_for<BF16Tag, 64, 2>(d.n_kv_heads), scratch_for<BF16Tag, 64, 4>(d.n_kv_heads)});
}

hipError_t launch_attend_matrix(ifkv_ctx *ctx, const ifkv_page_cache &pages, const PageTable &t, int32_t max_rows, const void *q,
                                int64_t q_stride, void *out, float *lse_out) {
  const auto &d = ctx->desc;
  if (d.dtype == IFKV_BF16) {
    if (d.head_dim == 128) return run_columns<BF16Tag, 128>(ctx, pages, t, max_rows, q, q_stride, out, lse_out);
    return run_columns<BF16Tag, 64>(ctx, pages, t, max_rows, q, q_stride, out, lse_out);
  }
  if (d.head_dim == 128) return run_columns<F32Tag, 128>(ctx, pages, t, max_rows, q, q_stride, out, lse_out);
  return run_columns<F32Tag, 64>(ctx, pages, t, max_rows, q, q_stride, out, lse_out);
}

}  // namespace ifkv
