// Attention over 8-bit pages on the matrix cores.
//
// Decoding reads every page once for a few query columns: memory bounds it, and what a kernel has to do is to keep requests in
// flight.  Pages come into LDS by direct loads, in the order in which the lanes of the 16x16x32 bf16 instruction take their operands out
// again (no bank is asked twice, and nothing changes lanes):
//   first product, S^T[token, column]: a lane's keys of a block of 16 tokens are d/64 times 16 bytes in a row of one token
//     (the order of the d elements along the reduction is free, queries follow it);
//   second product, O^T[d, column]: a lane's values are the 16 bytes in a row of one value row that ifkv.h's byte order makes
//     of the very tokens whose probabilities the lane holds.
// e4m3 numbers become bf16 exactly, two an instruction, with the page's scale multiplied in.  (The e4m3 instruction with scales, queries as
// two e4m3 numbers, would need no conversion of keys, but its sums are off by up to 2^-15 of sum |q k|, bf16 ones by 2^-22.)
//
// Measured on one MI355X, a call with its join, where reading alone reaches 6.2 to 6.9 TB/s and a large bf16 product 1.2 PFLOP/s: 64
// sequences of 0.8K to 8K tokens, 32/8 heads of 128, 597 MB in 102 us (the kernel alone 6.2 TB/s); one of 130K tokens 49 to 51 us (266 MB);
// 35 columns of 12 sequences of up to 20K 47 to 50 us (195 MB); 512 rows over 32K 260 us (1.05 PFLOP/s); 300 tokens of one sequence 7.1 us, all
// of it latency: positions, table, scales and pages are each asked for with the answer to the one before.
#include <algorithm>

#include "attention_pages.h"
#include "lds_dma.h"

namespace ifkv {

namespace {

typedef uint32_t v2u __attribute__((ext_vector_type(2)));

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;
constexpr float kLowest = -3.402823466e38f;
// Exponentials are taken against a reference that rises only where a logit exceeds it by more than 2^kSlack: sums stay below
// 2^(kSlack + 31), and most pages need no look at the other lanes' maxima.
constexpr float kSlack = 16.f;

// bf16 numbers that hold a query element.
template <typename Tag>
constexpr int kQueryParts = 3;
template <>
constexpr int kQueryParts<BF16Tag> = 1;

// bf16 numbers that hold a probability in the second product, by tiles of 16 columns.  bf16 layers: two where memory bounds the call,
// up to 32 columns (32 columns of 12 sequences of up to 20K tokens 77 us, with one 75); one, like the result, where instructions do
// (35 columns 50 us, with two 56; 64 columns 98, with two 111).
template <typename Tag>
constexpr int weight_parts(int tiles) {
  return kQueryParts<Tag> > 1 ? 3 : tiles <= 2 ? 2 : 1;
}

// Partial results of a piece of an item: accumulators as the wavefronts hold them, then reference and sum of every column.
template <int D, int NT>
struct Image {
  f32x4 o[NT * D / 16][64];
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

// What a lane names of a page: bytes from the page's start (of its kv head) of the rt-th block of 16 tokens' u-th 16 bytes of keys,
// and of the dt-th block of 16 value rows.
template <int D>
__device__ __forceinline__ int key_offset(int lane, int rt, int u) {
  return (rt * 16 + (lane & 15)) * D + u * 64 + (lane >> 4) * 16;
}
__device__ __forceinline__ int value_offset(int lane, int dt) { return (dt * 16 + (lane & 15)) * kPageTokens + (lane >> 4) * 16; }

// NT * 16 query columns of a wavefront and what it has added up for them.  Lane l holds column l % 16 of every tile; the four
// lanes of a column share its reference, each has its own tokens' sum.
// FENCED: requests and products stay in the order in which they are written (where operands are not at hand for many at once).
template <typename Tag, int D, int NT, int PP, bool FENCED>
struct Columns {
  static constexpr int QP = kQueryParts<Tag>;
  static constexpr int KS = D / 32;       // steps of the first product
  static constexpr int KV = D / 64;       // 16-byte key loads of a lane and block of 16 tokens
  static constexpr int DT = D / 16;       // blocks of 16 output rows
  bf16x8 q[NT][QP][KS];
  f32x4 o[DT][NT];
  float ref[NT], neg_ref[NT], sum[NT];
  int pos[NT];          // INT32_MAX: sees nothing
  int64_t row_head[NT]; // -1: no row
  uint32_t nan_mark[NT]; // outputs that saw a value that is NaN beside tokens that they do not see
  int lowest, highest;  // positions of the wavefront's columns that see something (INT32_MAX and -1: none does)
  int n, g;

  // columns first_column .. of the sequence's
  __device__ __forceinline__ void start(const PageTable &t, const AttendItem &item, int first_column, int grp, int h, int n_q_heads,
                                        const void *queries, int64_t q_stride) {
    const int lane = threadIdx.x & 63;
    n = lane & 15;
    g = lane >> 4;
    lowest = INT32_MAX;
    highest = -1;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int c = first_column + nt * 16 + n;
      const int r = item.lo + c / grp;
      const int hq = h * grp + c % grp;
      const bool real = r < item.hi;
      pos[nt] = real ? t.row_pos[r] : -1;
      row_head[nt] = real ? static_cast<int64_t>(r) * n_q_heads + hq : -1;
      const bool sees = pos[nt] >= 0 && (pos[nt] >> 6) < t.width;
      if (sees) highest = max(highest, pos[nt]);
      if (!sees) pos[nt] = INT32_MAX;
      lowest = min(lowest, pos[nt]);
      const char *src = static_cast<const char *>(queries) + (r * q_stride + static_cast<int64_t>(hq) * D + g * 16) * Elem<Tag>::kBytes;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        constexpr int PER16 = 16 / Elem<Tag>::kVec;   // 16-byte vectors of 16 elements: steps 2 u and 2 u + 1 share those of key load u
        const int vec = ks / 2 * 4 * PER16 + ks % 2 * (PER16 / 2);
        if constexpr (QP == 1) {
          v4u w = {0, 0, 0, 0};
          if (sees) w = reinterpret_cast<const v4u *>(src)[vec];
          q[nt][0][ks] = __builtin_bit_cast(bf16x8, w);
        } else {
          float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
          if (sees) {
            *reinterpret_cast<f32x4 *>(x) = reinterpret_cast<const f32x4 *>(src)[vec];
            *reinterpret_cast<f32x4 *>(x + 4) = reinterpret_cast<const f32x4 *>(src)[vec + 1];
          }
          bf16x8 s[QP];
          split8<QP>(x, s);
#pragma unroll
          for (int p = 0; p < QP; ++p) {
            q[nt][p][ks] = s[p];
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (p > 0 && !(fabsf(x[e]) < INFINITY)) q[nt][p][ks][e] = static_cast<__bf16>(0.f);
          }
        }
      }
      ref[nt] = -INFINITY;
      neg_ref[nt] = 0.f;
      sum[nt] = 0.f;
      nan_mark[nt] = 0;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) o[dt][nt] = f32x4{0, 0, 0, 0};
    }
    lowest = __builtin_amdgcn_readfirstlane(wave_min_i(lowest));
    highest = __builtin_amdgcn_readfirstlane(wave_max_i(highest));
  }

  // keys.fetch(rt, i) requests, keys.open(., step) makes an operand, scaled, of what was fetched: kSteps steps each.  One block of
  // 16 tokens is requested while the one before is worked on.
  template <typename F>
  __device__ __forceinline__ void logits(F keys, f32x4 (&s)[4][NT]) {
    constexpr int N = KS / F::kSteps;
    typename F::Word next[N];
#pragma unroll
    for (int i = 0; i < N; ++i) next[i] = keys.fetch(0, i);
#pragma unroll
    for (int rt = 0; rt < 4; ++rt) {
      typename F::Word now[N];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        now[i] = next[i];
        if (rt < 3) next[i] = keys.fetch(rt + 1, i);
      }
      if (FENCED) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) s[rt][nt] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const bf16x8 a = keys.open(now[ks / F::kSteps], ks % F::kSteps);
#pragma unroll
        for (int p = QP - 1; p >= 0; --p)   // smallest first
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) s[rt][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, q[nt][p][ks], s[rt][nt], 0, 0, 0);
      }
      if (FENCED) __builtin_amdgcn_sched_barrier(0);
    }
  }

  __device__ __forceinline__ bool masked(int token0) const { return token0 + kPageTokens - 1 > lowest; }

  // masks a page's logits and sees to the references
  __device__ __forceinline__ void prepare(int token0, float logit_scale, f32x4 (&s)[4][NT]) {
    if (masked(token0)) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const int last = pos[nt] - token0 - g * 4;   // of the page's tokens, from the lane's first on
#pragma unroll
        for (int rt = 0; rt < 4; ++rt)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[rt][nt][e] = rt * 16 + e > last ? -INFINITY : s[rt][nt][e];
      }
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
  }

  // exponentials of half a page's logits, as the second product takes them
  __device__ __forceinline__ void weights(int half, float logit_scale, const f32x4 (&s)[4][NT], bf16x8 (&w)[NT][PP]) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float p[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] = __builtin_amdgcn_exp2f(fmaf(s[2 * half + e / 4][nt][e % 4], logit_scale, neg_ref[nt]));
      sum[nt] += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
      split8<PP>(p, w[nt]);
    }
  }

  // Values behind a column's token count nothing, NaN neither.  For pages that have such tokens, and NaN: ones(dt, half) is 1 where a
  // value is NaN; columns that see one are marked, and the caller takes those values for zero.
  template <typename F>
  __device__ __forceinline__ void mark_nan(int token0, F ones) {
#pragma unroll 1   // (a loop: a rare path must not take registers from the others)
    for (int dt = 0; dt < DT; ++dt) {
      const bf16x8 one[2] = {ones(dt, 0), ones(dt, 1)};
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const int last = pos[nt] - token0 - g * 4;
        f32x4 count = {0, 0, 0, 0};
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          bf16x8 seen;
#pragma unroll
          for (int e = 0; e < 8; ++e) seen[e] = static_cast<__bf16>((2 * half + e / 4) * 16 + e % 4 <= last ? 1.f : 0.f);
          count = __builtin_amdgcn_mfma_f32_16x16x32_bf16(one[half], seen, count, 0, 0, 0);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) nan_mark[nt] |= count[e] > 0.f ? 1u << (dt * 4 + e) : 0u;
      }
    }
  }

  // The second product, half a page after the other.
  // values.fetch(dt, half) requests, values.open makes the operand of a block of 16 output rows, scaled.  Four blocks are requested
  // while the four before are worked on, the second half's exponentials are formed while the first half's products run.
  template <typename F>
  __device__ __forceinline__ void add_values(F values, float logit_scale, const f32x4 (&s)[4][NT]) {
    constexpr int GROUPS = DT / 4;   // of a half
    bf16x8 w[2][NT][PP];
    typename F::Word next[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) next[i] = values.fetch(i, 0);
    if (FENCED) __builtin_amdgcn_sched_barrier(0);
    weights(0, logit_scale, s, w[0]);
#pragma unroll
    for (int j = 0; j < 2 * GROUPS; ++j) {
      const int half = j / GROUPS, dt0 = j % GROUPS * 4;
      typename F::Word now[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        now[i] = next[i];
        if (j + 1 < 2 * GROUPS) next[i] = values.fetch((j + 1) % GROUPS * 4 + i, (j + 1) / GROUPS);
      }
      if (FENCED) __builtin_amdgcn_sched_barrier(0);
      if (j == GROUPS - 1) weights(1, logit_scale, s, w[1]);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bf16x8 a = values.open(now[i]);
#pragma unroll
        for (int p = PP - 1; p >= 0; --p)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
            o[dt0 + i][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, w[half][nt][p], o[dt0 + i][nt], 0, 0, 0);
      }
      if (FENCED && j == GROUPS - 1) {   // after every product six of the exponentials' instructions
#pragma unroll
        for (int k = 0; k < 4 * NT * PP; ++k) {
          __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
          __builtin_amdgcn_sched_group_barrier(0x402, 6, 0);
        }
      }
      if (FENCED) __builtin_amdgcn_sched_barrier(0);
    }
  }

  // after the last page: a column's tokens are spread over four lanes; columns that see nothing had queries of zero and no mask
  __device__ __forceinline__ void complete() {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      if (pos[nt] == INT32_MAX) ref[nt] = -INFINITY;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (nan_mark[nt] >> (dt * 4 + e) & 1) o[dt][nt][e] = __uint_as_float(0x7FC00000u);
      sum[nt] += __shfl_xor(sum[nt], 16, 64);
      sum[nt] += __shfl_xor(sum[nt], 32, 64);
    }
  }

  // into an image of TILES tiles, as tiles from first on
  template <int TILES>
  __device__ __forceinline__ void save(Image<D, TILES> &im, int first) const {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) im.o[dt * TILES + first + nt][g * 16 + n] = o[dt][nt];
      if (g == 0) im.ref[first + nt][n] = ref[nt], im.sum[first + nt][n] = sum[nt];
    }
  }

  __device__ __forceinline__ void finish(void *out, float *lse_out) const {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
      if (row_head[nt] >= 0) write_columns<Tag, D, DT>(out, lse_out, row_head[nt], 0, g, &o[0][nt], NT, ref[nt], sum[nt]);
  }
};

// The e4m3 bytes of a word that are NaN, 1 in each.
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) { return (((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) >> 7; }
// The bf16 halves of a word whose exponent is all ones, 1 in each.
__device__ __forceinline__ uint32_t nan_halves(uint32_t w) { return (((w & 0x7F807F80u) + 0x00800080u) & 0x80008000u) >> 15; }

// Operands from e4m3 bytes in LDS, in the order of the lanes.
template <int KV>
struct NarrowKeys {
  static constexpr int kSteps = 2;
  typedef v4u Word;
  const v4u (*at)[64];
  int lane;
  float scale;
  __device__ __forceinline__ v4u fetch(int rt, int i) const { return at[rt * KV + i][lane]; }
  __device__ __forceinline__ bf16x8 open(const v4u &v, int step) const { return step == 0 ? widen(v.x, v.y, scale) : widen(v.z, v.w, scale); }
};
struct NarrowValues {
  typedef v2u Word;
  const v4u (*at)[64];
  int lane;
  float scale;
  __device__ __forceinline__ v2u fetch(int dt, int half) const { return reinterpret_cast<const v2u *>(&at[dt][lane])[half]; }
  __device__ __forceinline__ bf16x8 open(const v2u &v) const { return widen(v.x, v.y, scale); }
};
// Operands that are there.
template <int KV>
struct WideKeys {
  static constexpr int kSteps = 1;
  typedef v4u Word;
  const v4u (*at)[2][64];
  int lane;
  __device__ __forceinline__ v4u fetch(int rt, int i) const { return at[rt * KV + i / 2][i % 2][lane]; }
  __device__ __forceinline__ bf16x8 open(const v4u &v, int) const { return __builtin_bit_cast(bf16x8, v); }
};
struct WideValues {
  typedef v4u Word;
  const v4u (*at)[2][64];
  int lane;
  __device__ __forceinline__ v4u fetch(int dt, int half) const { return at[dt][half][lane]; }
  __device__ __forceinline__ bf16x8 open(const v4u &v) const { return __builtin_bit_cast(bf16x8, v); }
};

struct AttendArgs {
  PageTable t;
  AttendPlan plan;
  const uint8_t *k_pages, *v_pages;
  const float *k_scale, *v_scale;
  const void *q;
  void *out;
  float *lse_out;
  int *item_start;   // for the kernel that joins
  int64_t q_stride;
  int max_rows, n_pages, n_q_heads, n_kv_heads;
  float logit_scale;
};

// Goes through a unit's share: piece(item, kv head, first page, last page, slot) for every item that has pages in it.  slot:
// where partial results go, -1: the piece is the whole item.  A unit has two slots: the piece it begins with may be the rest
// of an item (or its middle), the one it ends with the beginning of one.
template <typename F>
__device__ __forceinline__ void each_piece(const AttendPlan &plan, int n_items, int n_kv_heads, const AttendPlanMemory &mem, uint32_t unit,
                                           F piece) {
  const auto scalar = [](uint32_t x) __attribute__((always_inline)) { return static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(x)); };
  const uint32_t total = scalar(mem.start[n_items]);
  if (total == 0) return;
  const Shares shares(plan, total * n_kv_heads);
  if (unit >= shares.units) return;
  uint32_t x = scalar(shares.edge(unit));
  const uint32_t end = scalar(shares.edge(unit + 1));
  uint32_t h = x / total, r = x - h * total;
  int item = 0;
  for (int half = kMaxItems / 2; half > 0; half >>= 1)   // the last item that begins at or before r
    if (item + half < n_items && static_cast<uint32_t>(mem.start[item + half]) <= r) item += half;
  item = scalar(item);
  while (x < end) {
    const uint32_t s = scalar(mem.start[item]), e = scalar(mem.start[item + 1]);
    if (s < e) {
      const uint32_t last = min(e, r + (end - x)), own = s + plan.start_pages, p = max(r, own);
      if (p < last)
        piece(item, static_cast<int>(h), static_cast<int>(p - own), static_cast<int>(last - own),
              p == own && last == e ? -1 : static_cast<int>(2 * unit + (p == own ? 1 : 0)));
      x += last - r;
      r = last;
    }
    if (r == e) ++item;
    if (r == total) r = 0, item = 0, ++h;
  }
}

// ---------------------------------------------------------------------------
// Up to 48 query columns a sequence: a workgroup's four wavefronts take the pages of a piece in turn and join at the end.  Each has
// room for the keys and the values of one page; direct loads fill it, the next page's keys as soon as this page's have been
// used, then its values, so half a page is always under way and no wavefront waits for another.
// ---------------------------------------------------------------------------
// wavefronts a SIMD that the registers leave
template <typename Tag, int D, int NT>
constexpr int kFewWaves = NT * kQueryParts<Tag> * D <= 256 || NT == 1 ? 2 : 1;

template <typename Tag, int D, int NT>
__global__ __launch_bounds__(kAttendThreads, (kFewWaves<Tag, D, NT>)) void attend_pages_kernel(AttendArgs a, Image<D, NT> *__restrict__ partials) {
  using Cols = Columns<Tag, D, NT, weight_parts<Tag>(NT), (NT > 1)>;
  constexpr int KV = Cols::KV, DT = Cols::DT, TILE = kPageTokens * D;
  constexpr int LOADS = TILE / 1024;   // of 1 KiB, for a page's keys or values
  __shared__ AttendPlanMemory plan_memory;
  __shared__ union {
    v4u tile[kAttendWaves][2][LOADS][64];   // keys and values of a page
    Image<D, NT> image[kAttendWaves];
  } mem;
  const PageTable &t = a.t;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int key_lane = key_offset<D>(lane, 0, 0), value_lane = value_offset(lane, 0);
  const v4u(*keys)[64] = mem.tile[wave][0];
  v4u(*values)[64] = mem.tile[wave][1];
  const uint32_t keys_at = lds_address(keys), values_at = lds_address(values);

  const auto piece = [&](int index, int h, int first, int last, int slot) __attribute__((always_inline)) {
    const AttendItem item(t, a.plan, a.max_rows, index);
    Cols c;
    c.start(t, item, item.block * a.plan.columns, a.plan.group, h, a.n_q_heads, a.q, a.q_stride);
    last = min(last, c.highest < 0 ? first : (c.highest >> 6) + 1);
    const int32_t *row_of_table = t.table + static_cast<int64_t>(item.seq) * t.width;
    // pages of this wavefront, 64 at a time: lane i knows the i-th
    for (int base = first + wave; base < last; base += 64 * kAttendWaves) {
      const int mine = base + lane * kAttendWaves;
      int entry = -1;
      if (mine < last) entry = row_of_table[mine];
      uint64_t todo = __ballot(entry >= 0 && entry < a.n_pages);
      if (todo == 0) continue;
      float ks_lane = 1.f, vs_lane = 1.f;
      if (entry >= 0 && entry < a.n_pages) {
        const int64_t at = static_cast<int64_t>(entry) * a.n_kv_heads + h;
        ks_lane = a.k_scale[at];
        vs_lane = a.v_scale[at];
      }
      auto page_at = [&](int i) __attribute__((always_inline)) {
        return (static_cast<int64_t>(__builtin_amdgcn_readlane(entry, i)) * a.n_kv_heads + h) * TILE;
      };
      const auto request_keys = [&](int64_t at) __attribute__((always_inline)) {
#pragma unroll
        for (int l = 0; l < LOADS; ++l) dma16_base_once(a.k_pages + at + l / KV * 16 * D + l % KV * 64, key_lane, keys_at + l * 1024);
      };
      const auto request_values = [&](int64_t at) __attribute__((always_inline)) {
#pragma unroll
        for (int l = 0; l < LOADS; ++l) dma16_base_once(a.v_pages + at + l * 16 * kPageTokens, value_lane, values_at + l * 1024);
      };
      int i = __builtin_ctzll(todo);
      wait_vmem<0>();   // (scales and queries: what follows counts its own requests)
      request_keys(page_at(i));
      request_values(page_at(i));
      while (true) {
        todo &= todo - 1;
        const bool more = todo != 0;
        const int next = more ? __builtin_ctzll(todo) : i;
        const int64_t next_at = page_at(next);
        const float ks_page = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ks_lane), i));
        const float vs_page = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(vs_lane), i));
        const int token0 = (base + i * kAttendWaves) * kPageTokens;
        wait_vmem<LOADS>();   // the keys are there, the values on their way
        f32x4 s[4][NT];
        c.logits(NarrowKeys<KV>{keys, lane, ks_page}, s);
        if (more) {
          wait_lds_reads();
          request_keys(next_at);
        }
        c.prepare(token0, a.logit_scale, s);
        if (more)
          wait_vmem<LOADS>();
        else
          wait_vmem<0>();
        if (c.masked(token0)) {
          uint32_t any = 0;
#pragma unroll 1
          for (int dt = 0; dt < DT; ++dt)
            for (int e = 0; e < 4; ++e) any |= nan_bytes(values[dt][lane][e]);
          if (__ballot(any != 0) != 0) {
            c.mark_nan(token0, [&](int dt, int half) __attribute__((always_inline)) {
              const v4u v = values[dt][lane];
              return widen(nan_bytes(v[2 * half]) * 0x38u, nan_bytes(v[2 * half + 1]) * 0x38u, 1.f);   // (0x38 is 1)
            });
#pragma unroll 1
            for (int dt = 0; dt < DT; ++dt) {
              v4u v = values[dt][lane];
              for (int e = 0; e < 4; ++e) v[e] &= ~(nan_bytes(v[e]) * 0xFFu);
              values[dt][lane] = v;
            }
          }
        }
        c.add_values(NarrowValues{values, lane, vs_page}, a.logit_scale, s);
        wait_lds_reads();
        if (!more) break;
        request_values(next_at);
        i = next;
      }
    }
    c.complete();
    // each wavefront joins a quarter of the output rows of all four
    __syncthreads();   // (the tiles have been read)
    c.save(mem.image[wave], 0);
    __syncthreads();
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      constexpr int MINE = DT / kAttendWaves;
      float by[kAttendWaves], ref = -INFINITY, sum = 0.f;
      f32x4 o[MINE];
#pragma unroll
      for (int w = 0; w < kAttendWaves; ++w) {
        by[w] = mem.image[w].ref[nt][c.n];
        ref = fmaxf(ref, by[w]);
      }
#pragma unroll
      for (int w = 0; w < kAttendWaves; ++w) {
        by[w] = by[w] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(by[w] - ref);
        sum = fmaf(mem.image[w].sum[nt][c.n], by[w], sum);
      }
#pragma unroll
      for (int i = 0; i < MINE; ++i) {
        const int at = (wave * MINE + i) * NT + nt;
        o[i] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < kAttendWaves; ++w) {
          const f32x4 x = mem.image[w].o[at][lane];
#pragma unroll
          for (int e = 0; e < 4; ++e) o[i][e] = fmaf(x[e], by[w], o[i][e]);
        }
        if (slot >= 0) partials[slot].o[at][lane] = o[i];
      }
      if (slot < 0) {
        if (c.row_head[nt] >= 0)
          write_columns<Tag, D, MINE>(a.out, wave == 0 ? a.lse_out : nullptr, c.row_head[nt], wave * MINE, c.g, o, 1, ref, sum);
      } else if (wave == 0 && c.g == 0) {
        partials[slot].ref[nt][c.n] = ref;
        partials[slot].sum[nt][c.n] = sum;
      }
    }
    __syncthreads();   // the images are given up
  };
  if (a.plan.units == 0) {
    piece(blockIdx.x, blockIdx.y, 0, INT32_MAX, -1);
    return;
  }
  add_up_items(t, a.plan, a.max_rows, blockIdx.x == 0, a.item_start, plan_memory);
  each_piece(a.plan, t.n_seqs * a.plan.n_blocks, a.n_kv_heads, plan_memory, blockIdx.x, piece);
}

// ---------------------------------------------------------------------------
// More columns (bf16 only): each of the four wavefronts has NT * 16 of its own and all of them go through the same pages.  A page's
// elements become bf16 once for all, a quarter by each wavefront, and lie in LDS in the order in which lanes take them for
// operands (no bank is asked twice); two pages have room, one that is worked on and one that is filled, with a barrier between them.
// ---------------------------------------------------------------------------
constexpr int kPageList = kAttendThreads;   // pages whose places are looked up together

template <typename Tag, int D, int NT>
__global__ __launch_bounds__(kAttendThreads, 2) void attend_pages_block_kernel(AttendArgs a, Image<D, 4 * NT> *__restrict__ partials) {
  using Cols = Columns<Tag, D, NT, weight_parts<Tag>(4 * NT), true>;
  constexpr int KV = Cols::KV, DT = Cols::DT, KS = Cols::KS, TILE = kPageTokens * D;
  constexpr int LOADS = 2 * TILE / 1024;              // of 1 KiB, a page: keys first
  constexpr int MINE = LOADS / kAttendWaves;          // of a wavefront
  __shared__ AttendPlanMemory plan_memory;
  __shared__ v4u s_page[2][LOADS][2][64];             // each 16 bytes of a page are two operands
  __shared__ int4 s_entry[kPageList];                 // page, its place in the sequence, scales
  __shared__ int s_count[kAttendWaves];
  const PageTable &t = a.t;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int offset[MINE];
#pragma unroll
  for (int u = 0; u < MINE; ++u) {
    const int l = wave * MINE + u;
    offset[u] = l < LOADS / 2 ? key_offset<D>(lane, l / KV, l % KV) : value_offset(lane, l - LOADS / 2);
  }
  const bool keys_mine = wave < kAttendWaves / 2;     // the first half of the loads are keys
  const uint8_t *pool = keys_mine ? a.k_pages : a.v_pages;

  const auto piece = [&](int index, int h, int first, int last, int slot) __attribute__((always_inline)) {
    const AttendItem item(t, a.plan, a.max_rows, index);
    Cols c;
    c.start(t, item, item.block * a.plan.columns + wave * NT * 16, a.plan.group, h, a.n_q_heads, a.q, a.q_stride);
    __syncthreads();   // (the piece before has been read)
    if (lane == 0) s_count[wave] = c.lowest;
    __syncthreads();
    const int block_lowest = min(min(s_count[0], s_count[1]), min(s_count[2], s_count[3]));
    const int32_t *row_of_table = t.table + static_cast<int64_t>(item.seq) * t.width;
    for (int base = first; base < last; base += kPageList) {
      __syncthreads();   // (the list before has been read)
      int entry = -1;
      if (base + tid < last && base + tid < t.width) entry = row_of_table[base + tid];
      const uint64_t there = __ballot(entry >= 0 && entry < a.n_pages);
      if (lane == 0) s_count[wave] = __builtin_popcountll(there);
      __syncthreads();
      int n_list = 0, at = __builtin_popcountll(there & ((1ull << lane) - 1));
#pragma unroll
      for (int w = 0; w < kAttendWaves; ++w) {
        if (w < wave) at += s_count[w];
        n_list += s_count[w];
      }
      if (entry >= 0 && entry < a.n_pages) {
        const int64_t s = static_cast<int64_t>(entry) * a.n_kv_heads + h;
        s_entry[at] = make_int4(entry, base + tid, __float_as_int(a.k_scale[s]), __float_as_int(a.v_scale[s]));
      }
      __syncthreads();
      if (n_list == 0) continue;
      v4u raw[MINE];   // this wavefront's quarter of the next page
      const auto load = [&](int p) __attribute__((always_inline)) {   // (behind the end: the last page once more)
        const int page = s_entry[min(p, n_list - 1)].x;
        const uint8_t *src = pool + (static_cast<int64_t>(page) * a.n_kv_heads + h) * TILE;
#pragma unroll
        for (int u = 0; u < MINE; ++u) raw[u] = *reinterpret_cast<const v4u *>(src + offset[u]);
      };
      const auto fill = [&](int p) __attribute__((always_inline)) {
        const int4 e = s_entry[min(p, n_list - 1)];
        const float scale = __int_as_float(keys_mine ? e.z : e.w);
#pragma unroll
        for (int u = 0; u < MINE; ++u) {
          v4u(*to)[64] = s_page[p & 1][wave * MINE + u];
          to[0][lane] = __builtin_bit_cast(v4u, widen(raw[u].x, raw[u].y, scale));
          to[1][lane] = __builtin_bit_cast(v4u, widen(raw[u].z, raw[u].w, scale));
        }
      };
      load(0);
      fill(0);
      load(1);
      for (int p = 0; p < n_list; ++p) {
        __syncthreads();   // page p is there, and nobody reads page p - 1 any more
        fill(p + 1);
        load(p + 2);
        asm volatile("" : : : "memory");   // (the requests go out here)
        const int token0 = __builtin_amdgcn_readfirstlane(s_entry[p].y) * kPageTokens;
        v4u(*page)[2][64] = s_page[p & 1];
        // every wavefront looks for NaN where any of them has tokens that it does not see: all find the same, and all have marked
        // their columns when the page is cleaned
        if (token0 + kPageTokens - 1 > block_lowest) {
          uint32_t any = 0;
#pragma unroll 1
          for (int l = LOADS; l < 2 * LOADS; ++l)
            for (int e = 0; e < 4; ++e) any |= nan_halves(page[l / 2][l % 2][lane][e]);
          if (__ballot(any != 0) != 0) {
            c.mark_nan(token0, [&](int dt, int half) __attribute__((always_inline)) {
              v4u v = page[LOADS / 2 + dt][half][lane];
              for (int e = 0; e < 4; ++e) v[e] = nan_halves(v[e]) * 0x3F80u;   // 1 in bf16
              return __builtin_bit_cast(bf16x8, v);
            });
            __syncthreads();
#pragma unroll 1
            for (int l = LOADS + wave; l < 2 * LOADS; l += kAttendWaves) {
              v4u v = page[l / 2][l % 2][lane];
              for (int e = 0; e < 4; ++e) v[e] &= ~(nan_halves(v[e]) * 0xFFFFu);
              page[l / 2][l % 2][lane] = v;
            }
            __syncthreads();
          }
        }
        if (token0 > c.highest) continue;
        f32x4 s[4][NT];
        // the two wavefronts of a SIMD: who is at products goes first, and of two the one that is further (280 -> 269 us at 512 rows
        // over 32K; with the exponentials between products 263)
        __builtin_amdgcn_s_setprio(1);
        c.logits(WideKeys<KV>{page, lane}, s);
        __builtin_amdgcn_s_setprio(0);
        c.prepare(token0, a.logit_scale, s);
        __builtin_amdgcn_s_setprio(2);
        c.add_values(WideValues{page + LOADS / 2, lane}, a.logit_scale, s);
        __builtin_amdgcn_s_setprio(0);
      }
    }
    c.complete();
    if (slot < 0)
      c.finish(a.out, a.lse_out);
    else
      c.save(partials[slot], wave * NT);
  };
  if (a.plan.units == 0) {
    const int lanes = item_lanes(a.plan, a.max_rows);
    const int n = __builtin_amdgcn_readfirstlane(item_pages(t, a.plan, a.max_rows, blockIdx.x, lane & (lanes - 1), lanes));
    if (n > 0) piece(blockIdx.x, blockIdx.y, 0, n, -1);
    return;
  }
  add_up_items(t, a.plan, a.max_rows, blockIdx.x == 0, a.item_start, plan_memory);
  each_piece(a.plan, t.n_seqs * a.plan.n_blocks, a.n_kv_heads, plan_memory, blockIdx.x, piece);
}

// Joins the pieces of an item: a workgroup for a quarter of the output rows of a tile of 16 columns.  Its wavefronts take the
// pieces in turn, eight requests under way, and join.  One wavefront where eight requests are about all pieces there are (64 sequences of up to
// 8K tokens, 512 items in 256 shares: 106.4 us a call, with four 108.1; 512 rows, 128 in 512: 264 and 268), four where there are more (one of
// 130K, 8 in 256: 51.5, with one 53.7).
constexpr int kMergeSplit = 4, kMergeBatch = 8;

template <typename Tag, int D, int NT, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void attend_pages_merge_kernel(PageTable t, AttendPlan plan, int max_rows, int n_q_heads,
                                                                        const int *__restrict__ item_start,
                                                                        const Image<D, NT> *__restrict__ partials, void *__restrict__ out,
                                                                        float *__restrict__ lse_out) {
  constexpr int DT = D / 16 / kMergeSplit;
  __shared__ f32x4 s_o[WAVES][DT][64];   // (the first one's is not used)
  __shared__ float s_ref[WAVES][16], s_sum[WAVES][16];
  const int item = blockIdx.x / (NT * kMergeSplit), nt = blockIdx.x / kMergeSplit % NT, quarter = blockIdx.x % kMergeSplit;
  const int h = blockIdx.y;
  const uint32_t s = item_start[item], e = item_start[item + 1], total = item_start[t.n_seqs * plan.n_blocks];
  if (s == e) return;
  const Shares shares(plan, total * gridDim.y);
  const uint32_t u0 = shares.unit_of(h * total + s + plan.start_pages), u1 = shares.unit_of(h * total + e - 1);
  const int pieces = static_cast<int>(u1 - u0) + 1;
  if (pieces == 1) return;   // the unit wrote the result
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, g = lane >> 4;
  const auto image = [&](int p) __attribute__((always_inline)) -> const Image<D, NT> & { return partials[2 * (u0 + p) + (p == 0 ? 1 : 0)]; };
  float ref = -INFINITY, sum = 0.f;
  f32x4 o[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) o[dt] = f32x4{0, 0, 0, 0};
  for (int p0 = wave; p0 < pieces; p0 += WAVES * kMergeBatch) {
    float refs[kMergeBatch], sums[kMergeBatch];
    f32x4 x[kMergeBatch][DT];
#pragma unroll
    for (int u = 0; u < kMergeBatch; ++u) {
      const int p = p0 + u * WAVES;
      refs[u] = -INFINITY;
      sums[u] = 0.f;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) x[u][dt] = f32x4{0, 0, 0, 0};
      if (p < pieces) {
        const Image<D, NT> &im = image(p);
        refs[u] = im.ref[nt][n];
        sums[u] = im.sum[nt][n];
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) x[u][dt] = im.o[(quarter * DT + dt) * NT + nt][lane];
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
  float top = ref;
  if constexpr (WAVES > 1) {
    if (g == 0) s_ref[wave][n] = ref, s_sum[wave][n] = sum;
    if (wave > 0)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) s_o[wave][dt][lane] = o[dt];
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int w = 1; w < WAVES; ++w) top = fmaxf(top, s_ref[w][n]);
    const float a = ref == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ref - top);
    sum *= a;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[dt][e] *= a;
#pragma unroll
    for (int w = 1; w < WAVES; ++w) {
      const float b = s_ref[w][n] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s_ref[w][n] - top);
      sum = fmaf(s_sum[w][n], b, sum);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const f32x4 x = s_o[w][dt][lane];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[dt][e] = fmaf(x[e], b, o[dt][e]);
      }
    }
  }
  const AttendItem rows(t, plan, max_rows, item);
  const int c = rows.block * plan.columns + nt * 16 + n;
  const int r = rows.lo + c / plan.group;
  if (r < rows.hi)
    write_columns<Tag, D, DT>(out, quarter == 0 ? lse_out : nullptr, static_cast<int64_t>(r) * n_q_heads + h * plan.group + c % plan.group,
                              quarter * DT, g, o, 1, top, sum);
}

constexpr size_t kTableBytes = (kMaxItems + 4) / 4 * 4 * sizeof(int);

// The longest sequences, in pages, whose items are taken whole by a workgroup each.  Without cuts there is nothing to plan and to
// join, 6 to 10 us less; what is lost is time at the end, when only the longest are left, and chips that are not full.  Whole / cut, us:
//   a workgroup for every CU or more, up to 48 columns: 24 pages (200 sequences) 68 / 79, 32 pages (32 sequences) 22.1 / 26.9, 47 pages
//     (32, 64 and 128 sequences) 28.6 / 29.9, 54.6 / 49.4, 99 / 88, 63 pages (64) 71 / 60;  blocks: 32 pages 53 / 64, 47 pages 35 / 45 and 69 / 72.6;
//   fewer: 16 pages (one sequence) 10.3 / 12.4, 32 pages 20 / 14;  blocks: 5 pages 12.3 / 15.8, 8 pages 15.3 / 15.9, 12 pages 19.0 / 16.0.
constexpr int kManyItems = 256;
constexpr int whole_pages(int tiles, bool many) { return many ? (tiles < 4 ? 40 : 64) : (tiles < 4 ? 20 : 8); }

// Workgroups of a launch that is cut: what the chip holds, so that all of them run at once and end together.  One a CU where every
// wavefront has its own pages (two a CU begin and join twice as often: one sequence of 130K tokens 54.8 instead of 51.5 us, 64 of up to
// 8K 111 instead of 102), two a CU for blocks that share pages (512 rows over 32K: 260 us, with one 354).
constexpr int kTeams = 256, kBlockTeams = 512;
constexpr int kLeastPages = kAttendWaves;   // of a unit: one for each wavefront
// What a workgroup that begins an item loses, in pages of those it reads meanwhile elsewhere: positions, queries, first pages, the
// join.  Without it shares that hold the ends of several items finish last: 64 sequences of up to 8K tokens 106 us, with 8 pages 102
// (16: 105); 20 columns of 64 123.6, with 12 116.6 (40: 124); 35 columns of 12 sequences 54.4, with 20 49 (40: 51); 36 columns of 64
// as blocks 140.8, with 6 130.5 (14: 135).
constexpr int start_pages(int tiles) { return tiles == 1 ? 8 : tiles == 2 ? 12 : tiles == 3 ? 20 : 6; }

template <typename Tag, int D, int TILES>
hipError_t run(ifkv_ctx *ctx, const ifkv_page_cache &pages, const PageTable &t, int max_rows, const void *q, int64_t q_stride, void *out,
               float *lse_out) {
  const auto &d = ctx->desc;
  AttendPlan plan;
  plan.group = d.n_q_heads / d.n_kv_heads;
  plan.columns = TILES * 16;
  plan.n_blocks = static_cast<int>((static_cast<int64_t>(max_rows) * plan.group + plan.columns - 1) / plan.columns);
  plan.least_pages = kLeastPages;
  plan.start_pages = start_pages(TILES);
  const int64_t items = static_cast<int64_t>(t.n_seqs) * plan.n_blocks;
  // (pages are added up in 32 bits)
  const bool cut = t.width > whole_pages(TILES, items * d.n_kv_heads >= kManyItems) && items <= kMaxItems &&
                   items * (t.width + int64_t(plan.start_pages)) < INT32_MAX / d.n_kv_heads;
  const int workgroups = TILES < 4 ? kTeams : kBlockTeams;
  plan.units = cut ? workgroups : 0;
  int *item_start = static_cast<int *>(ctx->page_partials);
  Image<D, TILES> *partials = reinterpret_cast<Image<D, TILES> *>(static_cast<char *>(ctx->page_partials) + kTableBytes);
  // a grid has fewer than 2^32 threads: so many sequences a launch (all of them where items are cut)
  const int step = std::max(1, (1 << 23) / plan.n_blocks);
  for (int s = 0; s < t.n_seqs; s += step) {
    const int64_t skip = t.row_start != nullptr ? 0 : s;  // rows of the sequences before, where each has one
    const AttendArgs a = {t.from(s, std::min(step, t.n_seqs - s)), plan, static_cast<const uint8_t *>(pages.k),
                          static_cast<const uint8_t *>(pages.v), pages.k_scale, pages.v_scale,
                          static_cast<const char *>(q) + skip * q_stride * Elem<Tag>::kBytes,
                          static_cast<char *>(out) + skip * d.n_q_heads * D * Elem<Tag>::kBytes,
                          lse_out != nullptr ? lse_out + skip * d.n_q_heads : nullptr, item_start, q_stride, max_rows,
                          static_cast<int>(pages.n_pages), d.n_q_heads, d.n_kv_heads, ctx->sm_scale * kLog2e};
    const dim3 block(kAttendThreads);
    const dim3 grid = cut ? dim3(workgroups) : dim3(static_cast<unsigned>(static_cast<int64_t>(a.t.n_seqs) * plan.n_blocks), d.n_kv_heads);
    if constexpr (TILES >= 4) {
      hipLaunchKernelGGL((attend_pages_block_kernel<Tag, D, TILES / 4>), grid, block, 0, ctx->stream, a, partials);
    } else {
      hipLaunchKernelGGL((attend_pages_kernel<Tag, D, TILES>), grid, block, 0, ctx->stream, a, partials);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (!cut) return hipSuccess;
  const dim3 grid(static_cast<unsigned>(items * TILES * kMergeSplit), d.n_kv_heads);
  if (workgroups <= kMergeBatch * items * d.n_kv_heads) {
    hipLaunchKernelGGL((attend_pages_merge_kernel<Tag, D, TILES, 1>), grid, dim3(64), 0, ctx->stream, t, plan, max_rows, d.n_q_heads, item_start,
                       partials, out, lse_out);
  } else {
    hipLaunchKernelGGL((attend_pages_merge_kernel<Tag, D, TILES, kAttendWaves>), grid, dim3(kAttendThreads), 0, ctx->stream, t, plan, max_rows,
                       d.n_q_heads, item_start, partials, out, lse_out);
  }
  return hipGetLastError();
}

constexpr int kShortPages = 4;

template <typename Tag, int D>
hipError_t run_columns(ifkv_ctx *ctx, const ifkv_page_cache &pages, const PageTable &t, int max_rows, const void *q, int64_t q_stride,
                       void *out, float *lse_out) {
  const int64_t columns = static_cast<int64_t>(max_rows) * (ctx->desc.n_q_heads / ctx->desc.n_kv_heads);
  // A wavefront with all columns converts a page's elements itself, alone and at its own pace; from four tiles on its registers do not
  // suffice, and blocks share the pages (12 sequences of up to 20K: 35 columns 50 us, as a block 57; 64 columns as a block 98).
  if (columns <= 16) return run<Tag, D, 1>(ctx, pages, t, max_rows, q, q_stride, out, lse_out);
  if (columns <= 32 || kQueryParts<Tag> > 1) return run<Tag, D, 2>(ctx, pages, t, max_rows, q, q_stride, out, lse_out);
  if constexpr (kQueryParts<Tag> == 1) {
    // 48 columns in a wavefront leave room for one workgroup a CU, blocks for two, and a block's wavefronts begin with a quarter as much each:
    // blocks where sequences are short, or where they are whole and more than the chip (35 columns of 2 sequences of 128 tokens 8.8 us,
    // otherwise 10.5; of 80 of 128 tokens 12.7 and 20.6, of 1200 32.5 and 37.0; of 12 of 512 14.7 and 13.5)
    const bool many = static_cast<int64_t>(t.n_seqs) * ctx->desc.n_kv_heads >= kManyItems;
    if (columns <= 48 && t.width > (many ? whole_pages(3, true) : kShortPages))
      return run<Tag, D, 3>(ctx, pages, t, max_rows, q, q_stride, out, lse_out);
    if (columns <= 64) return run<Tag, D, 4>(ctx, pages, t, max_rows, q, q_stride, out, lse_out);
    return run<Tag, D, 8>(ctx, pages, t, max_rows, q, q_stride, out, lse_out);
  }
}

}  // namespace

// Two slots for each unit of the largest launch that is cut.
size_t attend_matrix_scratch_bytes(const ifkv_ctx *ctx) {
  const bool wide = ctx->desc.head_dim == 128;
  if (ctx->desc.dtype == IFKV_BF16) return kTableBytes + 2 * kBlockTeams * (wide ? sizeof(Image<128, 8>) : sizeof(Image<64, 8>));
  return kTableBytes + 2 * kTeams * (wide ? sizeof(Image<128, 2>) : sizeof(Image<64, 2>));
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
