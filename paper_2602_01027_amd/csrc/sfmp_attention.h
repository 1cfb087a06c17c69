// Attention over the 8-bit paged cache: kernels and launches.  SINKS: the first tokens stay visible behind a window.
#pragma once
#include "sfmp_kv.h"
#include "sfmp_parts.h"

namespace sfmp {
namespace {

// Wavefronts of a workgroup: two per SIMD, or, where sums and operands take more than half of its registers, one.
template <int D, int NT>
constexpr int kWaves = D * NT >= 256 ? 4 : 8;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.69314718055994531f;
// Weights are rounded to fp16, which the matrix cores take them in (their sum is not), in units of 2^-14: they keep their 11 bits down to 2^-28 of the
// largest.  It adds up to a seventh to the error of an fp16 result (2.1e-4 of it in the 2-norm, with unrounded weights, 2.4e-4 at most in
// the cases measured) and none that shows to a bf16 one (1.7e-3).
constexpr float kWeightUnit = 16384.0f, kWeightBits = 14.0f;
// Sums are rescaled when a page's largest score (in units of ln 2) exceeds what they are relative to by more than this.
constexpr float kSlack = 16.0f;

struct AttentionArgs {
  KvView v;
  const uint16_t* Q;
  uint16_t* O;
  float* lse;       // or null
  int64_t q_stride, o_stride;
  int32_t q_heads, group, window, max_pages;
  float scale;
  bool bf16;
  int32_t sinks;    // (SINKS: at least 1, and a window)
};

// 8 codes -> 8 fp16 values, exactly.  INT8: a byte b under the bits 0x64 is the fp16 number 1024 + b.
template <int FMT>
__device__ __forceinline__ half8 operand_of(uint32_t lo, uint32_t hi) {
  union {
    half2_ h[4];
    uint32_t u[4];
    half8 v;
  } x;
  if constexpr (FMT == SFMP_KV_INT8) {
    x.u[0] = __builtin_amdgcn_perm(0x64646464u, lo, 0x04010400u);
    x.u[1] = __builtin_amdgcn_perm(0x64646464u, lo, 0x04030402u);
    x.u[2] = __builtin_amdgcn_perm(0x64646464u, hi, 0x04010400u);
    x.u[3] = __builtin_amdgcn_perm(0x64646464u, hi, 0x04030402u);
    const half2_ bias = {(_Float16)1152.0f, (_Float16)1152.0f};
#pragma unroll
    for (int i = 0; i < 4; ++i) x.h[i] -= bias;
  } else {
    x.h[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, false);
    x.h[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, true);
    x.h[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, false);
    x.h[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, true);
  }
  return x.v;
}

// What a wavefront has accumulated for 16 * NT query rows: lane l holds row l % 16 of every 16, of it the dims
// 16 dt + 4 (l / 16) + 0..3.
template <int D, int NT>
struct Partial {
  floatx4 o[NT][D / 16];
  float m[NT], l[NT];  // what the sums are relative to, in units of ln 2 (-infinity: no token yet), and the sum of 2^(score - m)
};

// The rows of a unit (one sequence, one key/value head, 16 * NT of its query rows).
template <int D, int NT>
struct Rows {
  half8 q[NT][D / 32];
  float factor[NT];  // score = factor * scale of K * product
  int at[NT];        // position of the row in the sequence
  int first, last;   // smallest and largest of them
};

// Query values as fp16, and what they have to be multiplied by.  bf16 rows are brought into the range of fp16 by a power of
// two (largest element in [2^10, 2^11)): elements down to 2^-25 of it stay exact, below the error is under 2^-35 of it.
// The lanes of a row are those that differ in the bits s1 and s2.
template <int N>
__device__ __forceinline__ float bring_to_fp16(const u32x4 (&raw)[N], half8 (&q)[N], bool bf16, int s1, int s2) {
  if (!bf16) {
#pragma unroll
    for (int s = 0; s < N; ++s) q[s] = __builtin_bit_cast(half8, raw[s]);
    return 1.0f;
  }
  uint32_t largest = 0;
#pragma unroll
  for (int s = 0; s < N; ++s)
#pragma unroll
    for (int j = 0; j < 4; ++j) largest = max(largest, max(raw[s][j] & 0x7FFFu, raw[s][j] >> 16 & 0x7FFFu));
  largest = max(largest, (uint32_t)__shfl_xor((int)largest, s1));
  largest = max(largest, (uint32_t)__shfl_xor((int)largest, s2));
  const int exponent = min(max((int)(largest >> 7), 11), 254);  // (biased; both powers of two stay normal)
  const float up = __uint_as_float((uint32_t)(127 + 127 + 10 - exponent) << 23);
#pragma unroll
  for (int s = 0; s < N; ++s)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      q[s][2 * j] = (_Float16)(__uint_as_float(raw[s][j] << 16) * up);
      q[s][2 * j + 1] = (_Float16)(__uint_as_float(raw[s][j] & 0xFFFF0000u) * up);
    }
  return __uint_as_float((uint32_t)(exponent - 10) << 23);
}

// Position of the row `token` of an entry, and the least and the largest one of the rows from .. to.
__device__ __forceinline__ int position_of(const KvEntry& e, int token) { return e.length - e.n + token; }
__device__ __forceinline__ int least_position(const KvEntry& e, int from, int) { return e.length - e.n + from; }
__device__ __forceinline__ int largest_position(const KvEntry& e, int, int to) { return e.length - e.n + to; }

template <int D, int NT, typename Entry>
__device__ __forceinline__ void load_rows(const AttentionArgs& a, const Entry& e, int head, int tile, Rows<D, NT>& r) {
  const int i16 = threadIdx.x & 15, g = (threadIdx.x & 63) >> 4;
  const int count = e.n * a.group;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int row = (tile * NT + nt) * 16 + i16;
    const int token = min(row, count - 1) / a.group, h = min(row, count - 1) - token * a.group;
    const uint16_t* const src = a.Q + (int64_t)(e.row0 + token) * a.q_stride + (int64_t)(head * a.group + h) * D;
    r.at[nt] = position_of(e, token);
    r.factor[nt] = a.scale * kLog2e;
    // step 2c + h of the matrix instructions takes the dims 64 c + 16 g + 8 h + 0..7 of lane group g, so that the
    // keys of two steps are 16 contiguous bytes
    u32x4 raw[D / 32];
#pragma unroll
    for (int s = 0; s < D / 32; ++s)
      raw[s] = *reinterpret_cast<const u32x4*>(src + 64 * (s / 2) + 16 * g + 8 * (s % 2));
    r.factor[nt] *= bring_to_fp16<D / 32>(raw, r.q[nt], a.bf16, 16, 32);
  }
  const int from = tile * NT * 16 / a.group, to = min((tile + 1) * NT * 16 - 1, count - 1) / a.group;
  r.first = least_position(e, from, to);
  r.last = largest_position(e, from, to);
}

// Pages of a sequence that any of the rows at [first, last] sees: the places begin .. end - 1 of a list of pages.  With SINKS the list holds
// the pages of the first tokens and then, `gap` pages further, those of the window; else all pages.
template <bool SINKS>
struct PageRange {
  int begin, end;
  __device__ __forceinline__ int page(int place) const { return place; }
};
template <>
struct PageRange<true> {
  int begin, end, edge, gap;
  __device__ __forceinline__ int page(int place) const { return place < edge ? place : place + gap; }
};
template <bool SINKS>
__device__ __forceinline__ PageRange<SINKS> no_pages() { return PageRange<SINKS>{}; }
template <bool SINKS>
__device__ __forceinline__ PageRange<SINKS> pages_seen(const AttentionArgs& a, int first, int last) {
  PageRange<SINKS> p;
  p.end = last < 0 ? 0 : last / kPage + 1;
  p.begin = a.window > 0 ? max(first - a.window + 1, 0) / kPage : 0;
  if constexpr (SINKS) {
    p.end = min(p.end, a.max_pages);
    p.edge = min((a.sinks - 1) / kPage + 1, p.end);
    p.gap = max(p.begin - p.edge, 0);
    p.begin = 0;
    p.end = max(p.end - p.gap, p.edge);
  } else {
    p.end = max(min(p.end, a.max_pages), p.begin);
  }
  return p;
}
// The places [from, to) of `all`, less the pages that rows which see `seen` do not (all of those are in `all`).
template <bool SINKS>
__device__ __forceinline__ PageRange<SINKS> common_pages(const PageRange<SINKS>& all, const PageRange<SINKS>& seen, int from, int to) {
  if constexpr (SINKS) {
    const int s0 = min(from, all.edge), s1 = max(min(min(to, all.edge), seen.edge), s0);
    const int w0 = max(max(from, all.edge) + all.gap, seen.edge + seen.gap), w1 = min(max(to, all.edge) + all.gap, seen.end + seen.gap);
    return PageRange<true>{s0, s1 + max(w1 - w0, 0), s1, w0 - s1};
  } else {
    return PageRange<false>{max(seen.begin, from), min(seen.end, to)};
  }
}

// The codes of one page and head in registers.
template <int D>
struct PageCodes {
  u32x4 k[D / 64][4];  // [64 dims][tile t]: key 16 (i / 4) + 4 t + i % 4 of lane i = l % 16, dims 64 c + 16 g + 0..15
  u32x4 v[D / 16];     // [16 dims]: dim 16 dt + i, tokens 16 g + 0..15
};
template <int D>
__device__ __forceinline__ void load_keys(const uint8_t* block, PageCodes<D>& c) {
  const int i16 = threadIdx.x & 15, g = (threadIdx.x & 63) >> 4;
  const uint8_t* const at = block + (16 * (i16 >> 2) + (i16 & 3)) * D + 16 * g;
#pragma unroll
  for (int x = 0; x < D / 64; ++x)
#pragma unroll
    for (int t = 0; t < 4; ++t) c.k[x][t] = *reinterpret_cast<const u32x4*>(at + 4 * t * D + 64 * x);
}
template <int D>
__device__ __forceinline__ void load_values(const uint8_t* block, PageCodes<D>& c) {
  const int i16 = threadIdx.x & 15, g = (threadIdx.x & 63) >> 4;
#pragma unroll
  for (int dt = 0; dt < D / 16; ++dt)
    c.v[dt] = *reinterpret_cast<const u32x4*>(block + kPage * D + (16 * dt + i16) * kPage + 16 * g);
}

// The places [begin, end) of the pages of a sequence, accumulated by one wavefront.
//
// The product of keys and queries comes out of the matrix instructions with lane (i, g) holding, for query row i, the
// keys 4 g + r of a tile of 16.  With the 16 rows of tile t being the keys 16 (i / 4) + 4 t + i % 4 of the page, these are
// the 16 consecutive keys 16 g .. 16 g + 15 over the four tiles: the very tokens that the lane reads of the transposed
// values with one load, and the place that the weights need as the other operand.  Nothing moves between lanes but the
// two steps of the maximum.
template <int D, int FMT, int NT, bool SINKS, typename Entry>
__device__ __forceinline__ void accumulate(const AttentionArgs& a, const Entry& e, int head, const PageRange<SINKS>& pages, int begin, int end,
                                           const Rows<D, NT>& r, Partial<D, NT>& p) {
  const int lane = threadIdx.x & 63, g = lane >> 4;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    p.m[nt] = -INFINITY;
    p.l[nt] = 0.0f;
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) p.o[nt][dt] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
  }
  if (begin >= end) return;
  // Numbers and scales of 64 pages at a time, one per lane
  int held_page = 0;
  float held_k = 0.0f, held_v = 0.0f;
  auto hold = [&](int place) {
    held_page = max(kv_page(a.v, e.slot, pages.page(min(place + lane, end - 1))), 0);
    const float* const s = kv_scale(a.v, held_page, head, 0);
    held_k = s[0];
    held_v = s[1];
  };
  hold(begin);
  const uint8_t* block = kv_block<D>(a.v, __builtin_amdgcn_readlane(held_page, 0), head, 0);
  PageCodes<D> c;
  load_keys<D>(block, c);
  load_values<D>(block, c);
  for (int place = begin; place < end; ++place) {
    const int at = (place - begin) % 64, page = pages.page(place);
    const float scale_k = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(held_k), at));
    const float scale_v = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(held_v), at));
    const bool more = place + 1 < end;
    if (more) {
      if (at == 63) hold(place + 1);
      block = kv_block<D>(a.v, __builtin_amdgcn_readlane(held_page, (at + 1) % 64), head, 0);
    }

    floatx4 s[NT][4];
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) s[nt][t] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int x = 0; x < D / 64; ++x)
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const half8 k = operand_of<FMT>(c.k[x][t][2 * h], c.k[x][t][2 * h + 1]);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
            s[nt][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, r.q[nt][2 * x + h], s[nt][t], 0, 0, 0);
        }
    if (more) load_keys<D>(block, c);  // (of the next page, while this one's values are used)

    const int token = page * kPage + 16 * g;  // of s[.][0][0]
    const bool masked = page * kPage + kPage - 1 > r.first || (a.window > 0 && page * kPage <= r.last - a.window);
    if (page * kPage + kPage > e.length) {
      // tokens that were never written: whatever the bytes are, they must not meet the weight 0 as a NaN
      int written = e.length - token;
      asm volatile("" : "+v"(written));
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const int left = written - 4 * w;
        const uint32_t keep = left >= 4 ? ~0u : left <= 0 ? 0u : (1u << (8 * left)) - 1;
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) c.v[dt][w] &= keep;
      }
    }

    // Weights of the page relative to its own largest one (in fp16, in units of 2^-14), the page relative to those before
    half8 w[NT][2];
    float scale[NT], now[NT], sum[NT], beta[NT];
    bool changed = false;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const float factor = scale_k * r.factor[nt];
      if (masked) {
        int to = r.at[nt] - token, from = a.window > 0 ? to - a.window : -1 - token;
        asm volatile("" : "+v"(to), "+v"(from));  // (or the compiler computes all of it for every page)
        if constexpr (SINKS) {
          int visible = a.sinks - token;
          asm volatile("" : "+v"(visible));
#pragma unroll
          for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int x = 0; x < 4; ++x)
              if (4 * t + x > to || (4 * t + x <= from && 4 * t + x >= visible)) s[nt][t][x] = -INFINITY;
        } else {
#pragma unroll
          for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int x = 0; x < 4; ++x)
              if (4 * t + x > to || 4 * t + x <= from) s[nt][t][x] = -INFINITY;
        }
      }
      float top = -INFINITY;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int x = 0; x < 4; ++x) top = fmaxf(top, s[nt][t][x]);
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const bool sees = top != -INFINITY;
      const float score = sees ? top * factor : -INFINITY, shift = kWeightBits - (sees ? score : 0.0f);
      now[nt] = score > p.m[nt] + kSlack ? score : p.m[nt];
      changed |= now[nt] != p.m[nt];
      float times = factor;
      if (__any(!(factor > 0.0f))) {  // a scale of K that is 0 or NaN: not to be multiplied with -infinity
        const float value = factor > 0.0f ? 1.0f : factor;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int x = 0; x < 4; ++x)
            if (!(factor > 0.0f) && s[nt][t][x] != -INFINITY) s[nt][t][x] = value;
        if (!(factor > 0.0f)) times = 1.0f;
      }
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int x = 0; x < 4; ++x) s[nt][t][x] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[nt][t][x], times, shift));
      sum[nt] = 0.0f;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          sum[nt] += s[nt][t][x];
          w[nt][t / 2][4 * (t % 2) + x] = (_Float16)s[nt][t][x];
        }
      beta[nt] = sees ? __builtin_amdgcn_exp2f(score - now[nt]) : 0.0f;
      scale[nt] = sees ? scale_v * (1.0f / kWeightUnit) * beta[nt] : 0.0f;  // (a scale that is NaN reaches the rows that see the page)
    }
    if (__any(changed)) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const float alpha = p.m[nt] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(p.m[nt] - now[nt]);
        p.m[nt] = now[nt];
        p.l[nt] *= alpha;
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) p.o[nt][dt] *= alpha;
      }
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) p.l[nt] = __builtin_fmaf(sum[nt], beta[nt], p.l[nt]);
    // The product of a page is taken by itself and added with the scale of V: sums of pages whose scales are far apart keep what an
    // fp32 sum keeps
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) {
      floatx4 page_o[NT];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) page_o[nt] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const half8 val = operand_of<FMT>(c.v[dt][2 * u], c.v[dt][2 * u + 1]);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) page_o[nt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(val, w[nt][u], page_o[nt], 0, 0, 0);
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int x = 0; x < 4; ++x) p.o[nt][dt][x] = __builtin_fmaf(page_o[nt][x], scale[nt], p.o[nt][dt][x]);
    }
    if (more) load_values<D>(block, c);
  }
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    p.l[nt] += __shfl_xor(p.l[nt], 16);
    p.l[nt] += __shfl_xor(p.l[nt], 32);
    p.l[nt] *= 1.0f / kWeightUnit;
  }
}

// Partial results in memory: as a wavefront holds them, a floatx4 per lane for every 16 rows and 16 dims, then m and l.
template <int D, int NT>
constexpr int kPartialVectors = NT * (D / 16) * 64;
template <int D, int NT>
constexpr int kPartialBytes = kPartialVectors<D, NT> * 16 + 2 * NT * 64 * 4;

template <int D, int NT>
__device__ __forceinline__ void store_partial(uint8_t* at, const Partial<D, NT>& p) {
  const int lane = threadIdx.x & 63;
  floatx4* const o = reinterpret_cast<floatx4*>(at);
  float* const ml = reinterpret_cast<float*>(at + kPartialVectors<D, NT> * 16);
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    ml[nt * 64 + lane] = p.m[nt];
    ml[(NT + nt) * 64 + lane] = p.l[nt];
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) o[(nt * (D / 16) + dt) * 64 + lane] = p.o[nt][dt];
  }
}

// Results of 16 rows, the dims 16 dt + 4 g + 0..3 of the lanes.
struct RowResult {
  bool there;
  uint16_t* dst;  // of the row's dims 4 g ...
  float inverse;
};
__device__ __forceinline__ RowResult row_result(const AttentionArgs& a, const KvEntry& e, int head, int row, int D, float m, float l,
                                                bool with_lse) {
  const int g = (threadIdx.x & 63) >> 4;
  RowResult r{row < e.n * a.group, nullptr, 0.0f};
  if (!r.there) return r;
  const int token = row / a.group, h = head * a.group + row - token * a.group;
  const bool empty = m == -INFINITY && l == 0.0f;  // (not where every score is a NaN)
  r.inverse = empty ? 0.0f : 1.0f / l;
  r.dst = a.O + (int64_t)(e.row0 + token) * a.o_stride + (int64_t)h * D + 4 * g;
  if (a.lse && with_lse && g == 0)
    a.lse[(int64_t)(e.row0 + token) * a.q_heads + h] = empty ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
  return r;
}
__device__ __forceinline__ void store_dims(const AttentionArgs& a, const RowResult& r, int dt, const floatx4& o) {
  u32x2 w;
#pragma unroll
  for (int x = 0; x < 2; ++x)
    w[x] = bits_of(o[2 * x] * r.inverse, a.bf16) | (uint32_t)bits_of(o[2 * x + 1] * r.inverse, a.bf16) << 16;
  *reinterpret_cast<u32x2*>(r.dst + 16 * dt) = w;
}
template <int D, int NT>
__device__ __forceinline__ void store_rows(const AttentionArgs& a, const KvEntry& e, int head, int tile, const Partial<D, NT>& p) {
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const RowResult r = row_result(a, e, head, (tile * NT + nt) * 16 + (threadIdx.x & 15), D, p.m[nt], p.l[nt], true);
    if (!r.there) continue;
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) store_dims(a, r, dt, p.o[nt][dt]);
  }
}

// 16 rows and 16 dims of the sum of partial results.
struct Slice {
  floatx4 o;
  float m, l;
};
// The slice of `count` partial results, `at(i)` their addresses.  A wavefront's work: adding up is spread over the wavefronts
// by slices.
template <int D, int NT, typename F>
__device__ __forceinline__ Slice add_partials(int count, int nt, int dt, F at) {
  const int lane = threadIdx.x & 63;
  auto ml = [&](int i) { return reinterpret_cast<const float*>(at(i) + kPartialVectors<D, NT> * 16) + nt * 64 + lane; };
  Slice s{floatx4{0.0f, 0.0f, 0.0f, 0.0f}, -INFINITY, 0.0f};
#pragma unroll 4
  for (int i = 0; i < count; ++i) s.m = fmaxf(s.m, *ml(i));
  const float base = s.m == -INFINITY ? 0.0f : s.m;
#pragma unroll 4
  for (int i = 0; i < count; ++i) {
    const float f = __builtin_amdgcn_exp2f(*ml(i) - base);
    s.l += ml(i)[NT * 64] * f;
    s.o += reinterpret_cast<const floatx4*>(at(i))[(nt * (D / 16) + dt) * 64 + lane] * f;
  }
  return s;
}
template <int D, int NT>
__device__ __forceinline__ void store_slice(const AttentionArgs& a, const KvEntry& e, int head, int tile, int nt, int dt, const Slice& s) {
  const RowResult r = row_result(a, e, head, (tile * NT + nt) * 16 + (threadIdx.x & 15), D, s.m, s.l, dt == 0);
  if (r.there) store_dims(a, r, dt, s.o);
}
template <int D, int NT>
__device__ __forceinline__ void store_partial_slice(uint8_t* at, int nt, int dt, const Slice& s) {
  const int lane = threadIdx.x & 63;
  reinterpret_cast<floatx4*>(at)[(nt * (D / 16) + dt) * 64 + lane] = s.o;
  if (dt == 0) {
    float* const ml = reinterpret_cast<float*>(at + kPartialVectors<D, NT> * 16);
    ml[nt * 64 + lane] = s.m;
    ml[(NT + nt) * 64 + lane] = s.l;
  }
}

// One workgroup per unit: its wavefronts take ranges of the pages and are joined in LDS.  One launch and the shortest chain of loads there
// is (length, page number, codes): 8 heads of 128 dims, 500 tokens 7.0 us (the smallest kernels here take 2.3).
template <int D, int FMT, int NT, bool SINKS>
__global__ __launch_bounds__((64 * kWaves<D, NT>)) void attend_unit_kernel(AttentionArgs a) {
  extern __shared__ __align__(16) uint8_t lds[];
  constexpr int WAVES = kWaves<D, NT>, BYTES = kPartialBytes<D, NT>;
  const int tile = blockIdx.x, head = blockIdx.y, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const KvEntry e = kv_entry(a.v, blockIdx.z);
  if (tile * NT * 16 >= e.n * a.group) return;
  Rows<D, NT> r;
  load_rows<D, NT>(a, e, head, tile, r);
  const PageRange<SINKS> all = e.slot < 0 ? no_pages<SINKS>() : pages_seen<SINKS>(a, r.first, r.last);
  const int each = (all.end - all.begin + WAVES - 1) / WAVES;
  const int begin = min(all.begin + wave * each, all.end), end = min(begin + each, all.end);
  Partial<D, NT> p;
  accumulate<D, FMT, NT, SINKS>(a, e, head, all, begin, end, r, p);
  store_partial<D, NT>(lds + wave * BYTES, p);
  __syncthreads();
  for (int slice = wave; slice < NT * D / 16; slice += WAVES) {
    const int nt = slice / (D / 16), dt = slice % (D / 16);
    store_slice<D, NT>(a, e, head, tile, nt, dt, add_partials<D, NT>(WAVES, nt, dt, [&](int i) { return lds + i * BYTES; }));
  }
}

// ---- the work cut into equal parts ---------------------------------------------------------------------------------
//
// All pages of all units in a row, by (batch entry, head, tile of rows, page): every workgroup takes `share` of them, every
// wavefront an equal part of that.  Each workgroup finds its part from the lengths of the batch (a prefix sum in LDS), so
// that neither the host nor another launch has to know them, and sequences of any lengths load every compute unit alike.
// A unit that lies inside one workgroup is finished there; one that is cut leaves a partial result per workgroup, which
// join_kernel adds up in order.

constexpr int kMostPlanned = 512;        // batch entries
constexpr int kMostPlannedPrompts = 256;  // (two workgroups share a compute unit's LDS)

template <int MOST>
struct Plan {
  int before[MOST + 1];  // pages of all units of the entries before
  int sums[16];
  // Of every wavefront: whether its part starts inside a unit (1: which ends in it, 2: which does not), and whether it ends
  // inside one that starts in it; then that unit, or, of the first wavefront, the one that it starts in
  struct {
    int left, right, entry, head, tile;
  } wave[9];
  KvEntry entry[MOST];
};

struct CutArgs {
  uint8_t* partials;   // [workgroup][2]: of a unit that began before the workgroup's part, of one that ends behind it
  KvEntry* entries;    // [batch]
  int32_t* before;     // [batch + 1]; what the first workgroup found
  int32_t workgroups, waves;
  int32_t least;       // pages of a wavefront
};

// Pages that the units of an entry read: all of them the same ones.
template <bool SINKS>
__device__ __forceinline__ PageRange<SINKS> pages_of_entry(const AttentionArgs& a, const KvEntry& e) {
  if (e.slot < 0 || e.n < 1) return no_pages<SINKS>();
  return pages_seen<SINKS>(a, e.length - e.n, e.length - 1);
}
__device__ __forceinline__ int tiles_of_entry(const AttentionArgs& a, const KvEntry& e, int rows) {
  return (e.n * a.group + rows - 1) / rows;
}

// Fills the plan; all threads of the workgroup.  Returns the pages of all units.
template <int THREADS, bool SINKS, int MOST>
__device__ int make_plan(const AttentionArgs& a, int rows, Plan<MOST>* plan) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int carry = 0;
  for (int base = 0; base < a.v.batch; base += THREADS) {
    const int b = base + threadIdx.x;
    int pages = 0;
    if (b < a.v.batch) {
      const KvEntry e = kv_entry(a.v, b);
      plan->entry[b] = e;
      const PageRange<SINKS> p = pages_of_entry<SINKS>(a, e);
      pages = (p.end - p.begin) * a.v.heads * tiles_of_entry(a, e, rows);
    }
    int up = pages;
#pragma unroll
    for (int s = 1; s < 64; s *= 2) {
      const int y = __shfl_up(up, s);
      if (lane >= s) up += y;
    }
    if (lane == 63) plan->sums[wave] = up;
    __syncthreads();
    int all = 0, ahead = carry;
    for (int w = 0; w < THREADS / 64; ++w) {
      if (w < wave) ahead += plan->sums[w];
      all += plan->sums[w];
    }
    if (b < a.v.batch) plan->before[b] = ahead + up - pages;
    carry += all;
    __syncthreads();
  }
  if (threadIdx.x == 0) plan->before[a.v.batch] = carry;
  __syncthreads();
  return carry;
}

// Pages of every workgroup and wavefront.
__device__ __forceinline__ Parts parts_of(const CutArgs& c, int total) { return Parts(total, c.workgroups, c.waves, c.least); }

// The batch entry that the page `at` of all belongs to: the last one that starts at or before it.
template <int MOST>
__device__ __forceinline__ int entry_of_page(const AttentionArgs& a, const Plan<MOST>& plan, int at) {
  const int lane = threadIdx.x & 63;
  int held = -1;
  for (int base = 0; base < a.v.batch; base += 64) {
    const uint64_t starts = __ballot(base + lane < a.v.batch && plan.before[min(base + lane, a.v.batch)] <= at);
    held += __popcll(starts);
    if (~starts) break;
  }
  return held;
}
// For the kernels that join partial results
template <int THREADS, int MOST>
__device__ __forceinline__ void keep_plan(const AttentionArgs& a, const CutArgs& c, const Plan<MOST>& plan) {
  if (blockIdx.x) return;
  for (int b = threadIdx.x; b <= a.v.batch; b += THREADS) {
    c.before[b] = plan.before[b];
    if (b < a.v.batch) c.entries[b] = plan.entry[b];
  }
}

// Bound by HBM: 131071 tokens of 8 heads of 128 dims (268 MB) 51.8 us, 5.2 TB/s with start and end (vector instructions issue in a quarter of
// that time, the matrix pipes are busy for 7 %); 64 sequences of 130 to 8190 tokens (261 MB, fp8) 56 us.  Requesting two pages ahead instead of
// one spilled registers and was slower.
template <int D, int FMT, int NT, bool SINKS>
__global__ __launch_bounds__((64 * kWaves<D, NT>)) void attend_cut_kernel(AttentionArgs a, CutArgs c) {
  extern __shared__ __align__(16) uint8_t lds[];
  constexpr int WAVES = kWaves<D, NT>, BYTES = kPartialBytes<D, NT>;
  Plan<kMostPlanned>& plan = *reinterpret_cast<Plan<kMostPlanned>*>(lds + 2 * WAVES * BYTES);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int total = make_plan<64 * WAVES, SINKS>(a, 16 * NT, &plan);
  const Part part = parts_of(c, total).part(blockIdx.x, wave);
  int at = part.begin;
  const int to = part.end;
  uint8_t* const partials = c.partials + (int64_t)blockIdx.x * 2 * BYTES;
  keep_plan<64 * WAVES>(a, c, plan);
  int left = 0, right = 0, held = 0, head = 0, tile = 0;
  while (at < to) {
    held = entry_of_page(a, plan, at);
    const KvEntry e = plan.entry[held];
    const PageRange<SINKS> pages = pages_of_entry<SINKS>(a, e);
    const int each = pages.end - pages.begin, tiles = tiles_of_entry(a, e, 16 * NT);
    const int unit = (at - plan.before[held]) / each, first = (at - plan.before[held]) - unit * each;
    const int count = min(each - first, to - at);
    head = unit / tiles, tile = unit - head * tiles;
    Rows<D, NT> r;
    load_rows<D, NT>(a, e, head, tile, r);
    Partial<D, NT> p;
    accumulate<D, FMT, NT, SINKS>(a, e, head, pages, pages.begin + first, pages.begin + first + count, r, p);
    at += count;
    const bool ends = first + count == each;
    if (first == 0 && ends) {
      store_rows<D, NT>(a, e, head, tile, p);
    } else {
      store_partial<D, NT>(lds + (2 * wave + (first == 0)) * BYTES, p);
      if (first == 0)
        right = 1;
      else
        left = ends ? 1 : 2;
      if (first == 0 || wave == 0) {  // (a part that starts inside a unit may end inside another: the first wavefront notes both)
        auto& mine = plan.wave[first == 0 ? wave : WAVES];
        mine.entry = held, mine.head = head, mine.tile = tile;
      }
    }
  }
  if (lane == 0) plan.wave[wave].left = left, plan.wave[wave].right = right;
  __syncthreads();
  // Every unit that is cut by the borders of wavefronts: from one that it starts in (or the workgroup's first) to one that it
  // ends in (or the last)
  const auto& flags = plan.wave[lane % WAVES];
  const uint32_t all = (1u << WAVES) - 1, ending = __ballot(flags.left == 1) & all, going = __ballot(flags.left == 2) & all;
  const uint32_t starting = __ballot(flags.right) & all;
  for (uint32_t todo = starting << 1 | ((ending | going) & 1); todo; todo &= todo - 1) {
    const int w = __builtin_ctz(todo) - 1;
    const bool from_before = w < 0;
    // wavefronts behind that continue the unit, until one that it ends in
    const int next = w + 1 + (from_before && !(ending & 1));
    const int run = __builtin_ctz(~(going >> next));
    const bool here = from_before && (ending & 1), ended = here || (next + run < WAVES && (ending >> (next + run) & 1));
    const int last = here ? 0 : next + run - 1 + ended;
    const uint8_t* const start = lds + (from_before ? 0 : 2 * w + 1) * BYTES;
    const int base = from_before ? 0 : w;
    const auto& of = plan.wave[from_before ? WAVES : w];
    for (int slice = wave; slice < NT * D / 16; slice += WAVES) {
      const int nt = slice / (D / 16), dt = slice % (D / 16);
      const Slice s = add_partials<D, NT>(last - base + 1, nt, dt, [&](int i) { return i ? lds + 2 * (base + i) * BYTES : start; });
      if (!from_before && ended)
        store_slice<D, NT>(a, plan.entry[of.entry], of.head, of.tile, nt, dt, s);
      else
        store_partial_slice<D, NT>(partials + (from_before ? 0 : BYTES), nt, dt, s);
    }
  }
}

// Adds up the partial results of the units that were cut by the borders of workgroups, and stores zeros for entries without
// pages.  Workgroup = (entry, head); PARTS = 1: wavefront w takes the dims 16 w + 0..15 and adds up its partial results one
// after the other.  PARTS = 8, where a unit is cut into many: a workgroup takes 32 dims, eight wavefronts share the
// partial results of 16 of them.  5.1 to 5.5 us (with one wavefront per 16 dims alone 10.4 for 131071 tokens).
template <int D, int NT, int PARTS, bool SINKS>
__global__ __launch_bounds__((PARTS == 1 ? 4 * D : 1024)) void join_kernel(AttentionArgs a, CutArgs c) {
  constexpr int BYTES = kPartialBytes<D, NT>;
  __shared__ __align__(16) floatx4 part_o[PARTS == 1 ? 1 : 16 * 64];
  __shared__ float part_m[PARTS == 1 ? 1 : 16 * 64], part_l[PARTS == 1 ? 1 : 16 * 64];
  const int b = blockIdx.x, head = blockIdx.y, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int dt = PARTS == 1 ? wave : blockIdx.z * 2 + wave / PARTS, part = PARTS == 1 ? 0 : wave % PARTS;
  const KvEntry e = c.entries[b];
  const int before = c.before[b];
  const Parts parts = parts_of(c, c.before[a.v.batch]);
  const PageRange<SINKS> pages = pages_of_entry<SINKS>(a, e);
  const int each = pages.end - pages.begin, tiles = tiles_of_entry(a, e, 16 * NT);
  for (int tile = 0; tile < tiles; ++tile) {
    const int start = before + (head * tiles + tile) * each;
    const int w0 = parts.workgroup_of(start), w1 = each > 0 ? parts.workgroup_of(start + each - 1) : w0;
    if (each > 0 && w0 == w1) continue;
    const int all = each > 0 ? w1 - w0 + 1 : 0, one = (all + PARTS - 1) / PARTS;
    const int from = min(part * one, all), count = min(one, all - from);
    auto at = [&](int i) { return c.partials + ((int64_t)(w0 + from + i) * 2 + (from + i == 0)) * BYTES; };
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      Slice s = add_partials<D, NT>(count, nt, dt, at);
      if constexpr (PARTS > 1) {
        __syncthreads();
        part_o[wave * 64 + lane] = s.o, part_m[wave * 64 + lane] = s.m, part_l[wave * 64 + lane] = s.l;
        __syncthreads();
        if (part) continue;
        for (int x = 1; x < PARTS; ++x) {
          const int y = (wave + x) * 64 + lane;
          const float top = fmaxf(s.m, part_m[y]), base = top == -INFINITY ? 0.0f : top;
          const float f1 = __builtin_amdgcn_exp2f(s.m - base), f2 = __builtin_amdgcn_exp2f(part_m[y] - base);
          s.m = top;
          s.l = s.l * f1 + part_l[y] * f2;
          s.o = s.o * f1 + part_o[y] * f2;
        }
      }
      store_slice<D, NT>(a, e, head, tile, nt, dt, s);
    }
  }
}

// ---- many rows -----------------------------------------------------------------------------------------------------
//
// Four wavefronts of 32 query rows each share the pages: every page is converted to fp16 once, into LDS, and read from there
// as matrix operands by all four.  While a page is multiplied, the next one is converted into another part of the LDS
// and the one after it is on its way from memory.  Two such groups in a workgroup take every other page of the same rows and
// are added up at the end: on every SIMD one wavefront multiplies while the other takes exponentials.  Keys and queries are
// multiplied as 32 x 32 x 16; with the bits 2 and 3 of a key's row exchanged the result is, lane by lane, the other operand of the product
// with the values.
//
// 2048 rows of 32 heads over themselves, 8 key heads of 128 dims: 55 us, 617 TFLOP/s of products that count (with one group 59 us; a large
// fp16 product of the library reaches 1110 here).  By the counters of a launch the matrix pipes are busy for 27 % of its cycles, vector instructions
// (conversion of pages, masks, exponentials, rescaling) issue for 41 %, the LDS is busy for 22 %: they overlap in part.

constexpr int kPromptRows = 128;  // of a workgroup
template <int D>
constexpr int kGroups = D == 256 ? 1 : 2;  // (256 dims: LDS for one)

template <int D>
struct PromptTile {
  static constexpr int KEY_PITCH = D * 2 + 16, VALUE_PITCH = kPage * 2 + 16;  // (rows of a column on different banks)
  __align__(16) uint8_t keys[kPage * KEY_PITCH];
  __align__(16) uint8_t values[D * VALUE_PITCH];
};

template <int D>
constexpr int kPromptPartialBytes = kPromptRows * (D + 2) * 4;  // floatx4 [4 wavefronts][D / 8][64], then m and l [128]

// Whole tiles: which (entry, tile, head) a workgroup is.  Tiles far down a prompt read the most pages: they come first, so that the
// short ones fill up what the long ones leave.  The heads of a tile are neighbours: on the XCDs in turn, each XCD's L2 holds
// the pages of its heads.
struct PromptUnit {
  int b, tile, head;
};
__device__ __forceinline__ PromptUnit prompt_unit(const AttentionArgs& a, int tiles, int x) {
  PromptUnit u;
  u.head = x % a.v.heads;
  x /= a.v.heads;
  u.b = x % a.v.batch;
  u.tile = tiles - 1 - x / a.v.batch;
  return u;
}

// What a lane of a prompt workgroup has accumulated: of row l % 32 of its wavefront the dims 32 x + 8 (r / 4) + 4 (l / 32) + r % 4.
typedef float floatx16 __attribute__((ext_vector_type(16)));
template <int D>
struct PromptSums {
  floatx16 o[D / 32];
  float m, l;
};

// The places [from, to) of the pages of an entry as far as the rows of a tile see them; all threads of the workgroup, the LDS free on entry and exit.  The sums are
// left with the first 256 threads.
template <int D, int FMT, int GROUPS, bool SINKS, typename Entry>
__device__ __forceinline__ void attend_tile(const AttentionArgs& a, const Entry& e, int kv_head, int tile_number, const PageRange<SINKS>& of_entry,
                                            int from, int to, PromptTile<D>* tiles, PromptSums<D>& sums) {
  constexpr int STEPS = D / 16, OT = D / 32, LOADS = D / 32;
  const int count = e.n * a.group;
  const int group = __builtin_amdgcn_readfirstlane(threadIdx.x >> 8), tid = threadIdx.x & 255;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = threadIdx.x & 63, i32 = lane & 31, h = lane >> 5;
  const int row0 = tile_number * kPromptRows, row = row0 + wave * 32 + i32;

  // Pages of the workgroup, and rows of the wavefront
  const int tile_from = row0 / a.group, tile_to = min(row0 + kPromptRows - 1, count - 1) / a.group;
  const int wave_from = min(row0 + wave * 32, count - 1) / a.group, wave_to = min(row0 + wave * 32 + 31, count - 1) / a.group;
  const PageRange<SINKS> seen = e.slot < 0 ? no_pages<SINKS>()
                                           : pages_seen<SINKS>(a, least_position(e, tile_from, tile_to), largest_position(e, tile_from, tile_to));
  const PageRange<SINKS> pages = common_pages<SINKS>(of_entry, seen, from, to);
  const int begin = pages.begin, end = pages.end;
  const int wave_first = least_position(e, wave_from, wave_to), wave_last = largest_position(e, wave_from, wave_to);
  const bool wave_used = row0 + wave * 32 < count;

  half8 q[STEPS];
  float row_factor = a.scale * kLog2e;
  const int at = position_of(e, min(row, count - 1) / a.group);
  {
    const int token = min(row, count - 1) / a.group, head = kv_head * a.group + min(row, count - 1) - token * a.group;
    const uint16_t* const src = a.Q + (int64_t)(e.row0 + token) * a.q_stride + (int64_t)head * D + 8 * h;
    u32x4 raw[STEPS];
#pragma unroll
    for (int s = 0; s < STEPS; ++s) raw[s] = *reinterpret_cast<const u32x4*>(src + 16 * s);
    row_factor *= bring_to_fp16<STEPS>(raw, q, a.bf16, 32, 32);
  }

  // 8 codes of the keys and of the values per thread and load, so that neighbours write 16 contiguous bytes each; keys go to the
  // row that has the bits 2 and 3 exchanged
  auto exchanged = [](int row) { return (row & ~12) | (row & 4) << 1 | (row & 8) >> 1; };
  u32x2 codes_k[LOADS], codes_v[LOADS];
  int held_page = 0;
  float held_k = 0.0f, held_v = 0.0f;
  auto hold = [&](int place) {
    held_page = max(kv_page(a.v, e.slot, pages.page(min(place + lane, end - 1))), 0);
    const float* const s = kv_scale(a.v, held_page, kv_head, 0);
    held_k = s[0];
    held_v = s[1];
  };
  auto request = [&](int place) {
    const uint8_t* const block = kv_block<D>(a.v, __builtin_amdgcn_readlane(held_page, (place - begin) % 64), kv_head, 0);
#pragma unroll
    for (int x = 0; x < LOADS; ++x) {
      codes_k[x] = *reinterpret_cast<const u32x2*>(block + x * 2048 + tid * 8);
      codes_v[x] = *reinterpret_cast<const u32x2*>(block + kPage * D + x * 2048 + tid * 8);
    }
  };
  auto convert = [&](int place, PromptTile<D>& tile) {
    const int page = pages.page(place);
    if (page * kPage + kPage > e.length) {  // tokens that were never written must not meet the weight 0 as a NaN
      int written = e.length - (page * kPage + tid * 8 % kPage);
      asm volatile("" : "+v"(written));
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        const int left = written - 4 * w;
        const uint32_t keep = left >= 4 ? ~0u : left <= 0 ? 0u : (1u << (8 * left)) - 1;
#pragma unroll
        for (int x = 0; x < LOADS; ++x) codes_v[x][w] &= keep;
      }
    }
#pragma unroll
    for (int x = 0; x < LOADS; ++x) {
      const int byte = x * 2048 + tid * 8;
      *reinterpret_cast<half8*>(tile.keys + exchanged(byte / D) * PromptTile<D>::KEY_PITCH + byte % D * 2) = operand_of<FMT>(codes_k[x][0], codes_k[x][1]);
      *reinterpret_cast<half8*>(tile.values + byte / kPage * PromptTile<D>::VALUE_PITCH + byte % kPage * 2) = operand_of<FMT>(codes_v[x][0], codes_v[x][1]);
    }
  };

  floatx16 (&o)[OT] = sums.o;
#pragma unroll
  for (int x = 0; x < OT; ++x)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[x][r] = 0.0f;
  float m = -INFINITY, l = 0.0f;
  float next_k = 0.0f, next_v = 0.0f;
  tiles += 2 * group;
  auto scales_of = [&](int place) {
    next_k = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(held_k), (place - begin) % 64));
    next_v = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(held_v), (place - begin) % 64));
  };
  if (begin < end) hold(begin);
  if (begin + group < end) {
    request(begin + group);
    scales_of(begin + group);
    convert(begin + group, tiles[0]);
    if (begin + group + GROUPS < end) request(begin + group + GROUPS);
  }
  __syncthreads();
  for (int step = 0; begin + step * GROUPS < end; ++step) {
    const int place = begin + group + step * GROUPS, page = pages.page(place);
    const PromptTile<D>& tile = tiles[step & 1];
    const float scale_k = next_k, scale_v = next_v;
    const bool skip = place >= end || !wave_used || page * kPage > wave_last ||
                      (a.window > 0 && page * kPage + kPage - 1 <= wave_first - a.window && !(SINKS && page * kPage < a.sinks));
    floatx16 s[2];
    if (!skip) {
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[kt][r] = 0.0f;
#pragma unroll
      for (int x = 0; x < STEPS; ++x)
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
          const half8 k = *reinterpret_cast<const half8*>(tile.keys + (32 * kt + i32) * PromptTile<D>::KEY_PITCH + (16 * x + 8 * h) * 2);
          s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k, q[x], s[kt], 0, 0, 0);
        }
    }
    if (place + GROUPS < end) {
      scales_of(place + GROUPS);
      convert(place + GROUPS, tiles[(step + 1) & 1]);
      const int ahead = place + 2 * GROUPS;
      if (ahead < end) {
        if ((ahead - begin) % 64 < GROUPS) hold(ahead - group);
        request(ahead);
      }
    }
    if (!skip) {
      const float factor = scale_k * row_factor;
      const bool masked = page * kPage + kPage - 1 > wave_first || (a.window > 0 && page * kPage <= wave_last - a.window);
      // s[kt][8 u + j] is the key 32 kt + 16 u + 8 h + j
      const int token = page * kPage + 8 * h;
      if (masked) {
        int to = at - token, from = a.window > 0 ? to - a.window : -1 - token;
        asm volatile("" : "+v"(to), "+v"(from));  // (or the compiler computes all of it for every page)
        if constexpr (SINKS) {
          int visible = a.sinks - token;
          asm volatile("" : "+v"(visible));
#pragma unroll
          for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              const int j = 32 * kt + 16 * (r / 8) + r % 8;
              if (j > to || (j <= from && j >= visible)) s[kt][r] = -INFINITY;
            }
        } else {
#pragma unroll
          for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              const int j = 32 * kt + 16 * (r / 8) + r % 8;
              if (j > to || j <= from) s[kt][r] = -INFINITY;
            }
        }
      }
      float top = -INFINITY;
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int r = 0; r < 16; ++r) top = fmaxf(top, s[kt][r]);
      top = fmaxf(top, __shfl_xor(top, 32));
      const bool sees = top != -INFINITY;
      const float score = sees ? top * factor : -INFINITY, shift = kWeightBits - (sees ? score : 0.0f);
      float times = factor;
      if (__any(!(factor > 0.0f))) {  // a scale of K that is 0 or NaN: not to be multiplied with -infinity
        const float value = factor > 0.0f ? 1.0f : factor;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (!(factor > 0.0f) && s[kt][r] != -INFINITY) s[kt][r] = value;
        if (!(factor > 0.0f)) times = 1.0f;
      }
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[kt][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kt][r], times, shift));
      // (the sums are kept relative to a score that the largest exceeds by no more than kSlack)
      const float now = score > m + kSlack ? score : m;
      if (__any(now != m)) {
        const float alpha = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - now);
        m = now;
        l *= alpha;
#pragma unroll
        for (int x = 0; x < OT; ++x) o[x] *= alpha;
      }
      const float beta = sees ? __builtin_amdgcn_exp2f(score - now) : 0.0f;
      const float scale = sees ? scale_v * (1.0f / kWeightUnit) * beta : 0.0f;  // (NaN: as above)
      half8 w[4];
      float sum = 0.0f;
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          sum += s[kt][r];
          w[2 * kt + r / 8][r % 8] = (_Float16)s[kt][r];
        }
      l = __builtin_fmaf(sum, beta, l);
      // (the product of a page by itself, as above)
#pragma unroll
      for (int x = 0; x < OT; ++x) {
        floatx16 page_o;
#pragma unroll
        for (int r = 0; r < 16; ++r) page_o[r] = 0.0f;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const half8 v = *reinterpret_cast<const half8*>(tile.values + (32 * x + i32) * PromptTile<D>::VALUE_PITCH + (16 * u + 8 * h) * 2);
          page_o = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, w[u], page_o, 0, 0, 0);
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) o[x][r] = __builtin_fmaf(page_o[r], scale, o[x][r]);
      }
    }
    __syncthreads();
  }
  l += __shfl_xor(l, 32);
  l *= 1.0f / kWeightUnit;
  if constexpr (GROUPS == 2) {
    floatx4* const other_o = reinterpret_cast<floatx4*>(tiles - 2 * group) + wave * (D / 8) * 64 + lane;
    float* const other_ml = reinterpret_cast<float*>(tiles - 2 * group) + kPromptRows * D + tid;
    if (group == 1) {
#pragma unroll
      for (int x = 0; x < OT; ++x)
#pragma unroll
        for (int q = 0; q < 4; ++q) other_o[(4 * x + q) * 64] = floatx4{o[x][4 * q], o[x][4 * q + 1], o[x][4 * q + 2], o[x][4 * q + 3]};
      other_ml[0] = m, other_ml[256] = l;
    }
    __syncthreads();
    if (group == 0) {
      const float m2 = other_ml[0], top = fmaxf(m, m2), base = top == -INFINITY ? 0.0f : top;
      const float f1 = __builtin_amdgcn_exp2f(m - base), f2 = __builtin_amdgcn_exp2f(m2 - base);
      m = top;
      l = l * f1 + other_ml[256] * f2;
#pragma unroll
      for (int x = 0; x < OT; ++x)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const floatx4 y = other_o[(4 * x + q) * 64];
#pragma unroll
          for (int j = 0; j < 4; ++j) o[x][4 * q + j] = o[x][4 * q + j] * f1 + y[j] * f2;
        }
    }
    __syncthreads();
  }
  sums.m = m;
  sums.l = l;
}

// A row of a tile, and where the dims 4 (l / 32) ... of it go.
__device__ __forceinline__ RowResult prompt_row(const AttentionArgs& a, const KvEntry& e, int kv_head, int tile, int D, float m, float l, bool with_lse) {
  const int lane = threadIdx.x & 63, h = lane >> 5, row = tile * kPromptRows + (threadIdx.x >> 6) * 32 + (lane & 31);
  RowResult r{row < e.n * a.group, nullptr, 0.0f};
  if (!r.there) return r;
  const int token = row / a.group, head = kv_head * a.group + row - token * a.group;
  const bool empty = m == -INFINITY && l == 0.0f;
  r.inverse = empty ? 0.0f : 1.0f / l;
  r.dst = a.O + (int64_t)(e.row0 + token) * a.o_stride + (int64_t)head * D + 4 * h;
  if (a.lse && with_lse && h == 0)
    a.lse[(int64_t)(e.row0 + token) * a.q_heads + head] = empty ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
  return r;
}
template <int D>
__device__ __forceinline__ void store_tile(const AttentionArgs& a, const KvEntry& e, int kv_head, int tile, const PromptSums<D>& s) {
  const RowResult r = prompt_row(a, e, kv_head, tile, D, s.m, s.l, true);
  if (!r.there) return;
#pragma unroll
  for (int x = 0; x < D / 32; ++x)
#pragma unroll
    for (int q = 0; q < 4; ++q)  // 8 dims and the two halves of them: in units of 16, as store_dims counts
      store_dims(a, RowResult{true, r.dst + 32 * x + 8 * q, r.inverse}, 0, floatx4{s.o[x][4 * q], s.o[x][4 * q + 1], s.o[x][4 * q + 2], s.o[x][4 * q + 3]});
}
template <int D>
__device__ __forceinline__ void store_tile_partial(uint8_t* to, const PromptSums<D>& s) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  floatx4* const po = reinterpret_cast<floatx4*>(to) + wave * (D / 8) * 64 + lane;
#pragma unroll
  for (int x = 0; x < D / 32; ++x)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      po[(4 * x + q) * 64] = floatx4{s.o[x][4 * q], s.o[x][4 * q + 1], s.o[x][4 * q + 2], s.o[x][4 * q + 3]};
  float* const ml = reinterpret_cast<float*>(to + kPromptRows * D * 4) + wave * 32 + (lane & 31);
  if (lane < 32) ml[0] = s.m, ml[kPromptRows] = s.l;
}

// One workgroup per tile.
template <int D, int FMT, bool SINKS>
__global__ __launch_bounds__((256 * kGroups<D>)) void attend_prompt_kernel(AttentionArgs a, int tiles) {
  extern __shared__ __align__(16) uint8_t lds[];
  const PromptUnit u = prompt_unit(a, tiles, blockIdx.x);
  const KvEntry e = kv_entry(a.v, u.b);
  if (u.tile * kPromptRows >= e.n * a.group) return;
  PromptSums<D> s;
  attend_tile<D, FMT, kGroups<D>, SINKS>(a, e, u.head, u.tile, pages_of_entry<SINKS>(a, e), 0, a.max_pages, reinterpret_cast<PromptTile<D>*>(lds), s);
  if (threadIdx.x < 256) store_tile<D>(a, e, u.head, u.tile, s);
}

// The work cut into equal parts, as above: few tiles with many pages each.  (All tiles of an entry count as many pages; a tile skips
// those behind its last row.)  6 chunks of 65 to 701 rows over 900 to 8001 tokens, 16 heads of 64 dims: 48 us, and 9 to join; one workgroup
// for each tile takes 97, as long as the longest.  One group of wavefronts: with two, 57.
template <int D, int FMT, bool SINKS>
__global__ __launch_bounds__(256, D == 256 ? 1 : 2) void attend_prompt_cut_kernel(AttentionArgs a, CutArgs c) {
  extern __shared__ __align__(16) uint8_t lds[];
  Plan<kMostPlannedPrompts>& plan = *reinterpret_cast<Plan<kMostPlannedPrompts>*>(lds + 2 * sizeof(PromptTile<D>));
  const int total = make_plan<256, SINKS>(a, kPromptRows, &plan);
  keep_plan<256>(a, c, plan);
  const Part part = parts_of(c, total).whole(blockIdx.x);
  int at = part.begin;
  const int to = part.end;
  uint8_t* const partials = c.partials + (int64_t)blockIdx.x * 2 * kPromptPartialBytes<D>;
  while (at < to) {
    const int held = entry_of_page(a, plan, at);
    const KvEntry e = plan.entry[held];
    const PageRange<SINKS> pages = pages_of_entry<SINKS>(a, e);
    const int each = pages.end - pages.begin, tiles = tiles_of_entry(a, e, kPromptRows);
    const int unit = (at - plan.before[held]) / each, first = (at - plan.before[held]) - unit * each;
    const int count = min(each - first, to - at), head = unit / tiles, tile = unit - head * tiles;
    PromptSums<D> s;
    attend_tile<D, FMT, 1, SINKS>(a, e, head, tile, pages, pages.begin + first, pages.begin + first + count, reinterpret_cast<PromptTile<D>*>(lds), s);
    at += count;
    if (first == 0 && count == each)
      store_tile<D>(a, e, head, tile, s);
    else
      store_tile_partial<D>(partials + (first == 0 ? kPromptPartialBytes<D> : 0), s);
  }
}

// Adds up the partial results of the tiles that were cut, and stores zeros for entries without pages.  Lanes as above; a workgroup
// takes 32 dims.
template <int D, bool SINKS>
__global__ __launch_bounds__(256) void join_prompt_kernel(AttentionArgs a, CutArgs c) {
  const int tile = blockIdx.x / (D / 32), x = blockIdx.x % (D / 32), head = blockIdx.y, b = blockIdx.z;
  const KvEntry e = c.entries[b];
  const int tiles = tiles_of_entry(a, e, kPromptRows);
  if (tile >= tiles) return;
  const Parts parts = parts_of(c, c.before[a.v.batch]);
  const PageRange<SINKS> pages = pages_of_entry<SINKS>(a, e);
  const int each = pages.end - pages.begin, start = c.before[b] + (head * tiles + tile) * each;
  const int w0 = parts.workgroup_of(start), w1 = each ? parts.workgroup_of(start + each - 1) : w0 - 1;
  if (w0 == w1) return;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  auto at = [&](int w) { return c.partials + ((int64_t)w * 2 + (w == w0)) * kPromptPartialBytes<D>; };
  auto ml = [&](int w) { return reinterpret_cast<const float*>(at(w) + kPromptRows * D * 4) + wave * 32 + (lane & 31); };
  float m = -INFINITY, l = 0.0f;
#pragma unroll 4
  for (int w = w0; w <= w1; ++w) m = fmaxf(m, *ml(w));
  const float base = m == -INFINITY ? 0.0f : m;
  floatx4 o[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) o[q] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 2
  for (int w = w0; w <= w1; ++w) {
    const float f = __builtin_amdgcn_exp2f(*ml(w) - base);
    l += ml(w)[kPromptRows] * f;
    const floatx4* const po = reinterpret_cast<const floatx4*>(at(w)) + wave * (D / 8) * 64 + lane;
#pragma unroll
    for (int q = 0; q < 4; ++q) o[q] += po[(4 * x + q) * 64] * f;
  }
  const RowResult r = prompt_row(a, e, head, tile, D, m, l, x == 0);
  if (!r.there) return;
#pragma unroll
  for (int q = 0; q < 4; ++q) store_dims(a, RowResult{true, r.dst + 32 * x + 8 * q, r.inverse}, 0, o[q]);
}

// ---- launches ------------------------------------------------------------------------------------------------------

template <int D, int FMT, int NT, bool SINKS>
int launch_units(const AttentionArgs& a, int max_rows, hipStream_t stream) {
  const void* const fn = (const void*)attend_unit_kernel<D, FMT, NT, SINKS>;
  if (int e = allow_full_lds(fn, "attend_unit_kernel")) return e;
  const int64_t tiles = ((int64_t)max_rows * a.group + 16 * NT - 1) / (16 * NT);
  constexpr int threads = 64 * kWaves<D, NT>, lds = kWaves<D, NT> * kPartialBytes<D, NT>;
  attend_unit_kernel<D, FMT, NT, SINKS><<<dim3((uint32_t)tiles, a.v.heads, a.v.batch), threads, lds, stream>>>(a);
  return kv_launched("attend_unit_kernel");
}

template <int D, int FMT, int NT, bool SINKS>
int launch_cut(const AttentionArgs& a, const CutArgs& c, hipStream_t stream) {
  const void* const fn = (const void*)attend_cut_kernel<D, FMT, NT, SINKS>;
  if (int e = allow_full_lds(fn, "attend_cut_kernel")) return e;
  constexpr int threads = 64 * kWaves<D, NT>, lds = 2 * kWaves<D, NT> * kPartialBytes<D, NT> + (int)sizeof(Plan<kMostPlanned>);
  static_assert(lds <= 160 * 1024, "LDS of a compute unit");
  attend_cut_kernel<D, FMT, NT, SINKS><<<c.workgroups, threads, lds, stream>>>(a, c);
  // (8 units of 65536 tokens 30.9 us against 36.0, 16 units 57.1 and 58.3, 32 the same, 64 of 16384 tokens 56.4 against 55.8)
  if ((int64_t)a.v.batch * a.v.heads * 8 <= c.workgroups)
    join_kernel<D, NT, 8, SINKS><<<dim3(a.v.batch, a.v.heads, D / 32), 1024, 0, stream>>>(a, c);
  else
    join_kernel<D, NT, 1, SINKS><<<dim3(a.v.batch, a.v.heads), 4 * D, 0, stream>>>(a, c);
  return kv_launched("attend_cut_kernel");
}

// How a call runs.
struct AttentionForm {
  int nt;          // tiles of 16 rows that a unit holds
  int workgroups;  // 0: one per unit
  int waves;       // of one
  bool may_cut;    // (with a window or without)
  int64_t cut_bytes;
  bool prompt;     // tiles of kPromptRows rows: then
  int tiles, units;
  int least;       // pages of a wavefront (of a prompt's workgroup)
  double time;     // us, as estimated; not of prompts
};

// With more rows of an entry and key/value head than these, attend_prompt_kernel (48 rows, 8 heads of 128 dims, us: one sequence of 512
// tokens 10.3 against 15.9, of 8192 25.8 and 31.8, 8 of 2048 28.7 and 29.1; 64 of 2048 100 and 91).
constexpr int kPromptFrom = 64;
constexpr int kMostCutTiles = 4;  // of an entry, in equal parts

int waves_of(int dim, int nt) { return dim * nt >= 256 ? 4 : 8; }

// Time (us) that equal parts take at least, and that a workgroup for each unit of p pages takes (choose_form).
double parts_start(int waves) { return waves == 8 ? 10.0 : 14.0; }
double time_of_units(int dim, int waves, int64_t units, int64_t p) {
  return 4.3 + (dim == 64 ? 1.25 : 2.7) * (double)((units + 255) / 256 * ((p + waves - 1) / waves));
}
// Partial results of the 256 workgroups, or of a prompt's parts.
int64_t cut_bytes_of(int dim, int nt) { return (int64_t)256 * 2 * (nt * (dim / 16) * 64 * 16 + 2 * nt * 64 * 4); }
int prompt_slots(int dim) { return dim == 256 ? 256 : 512; }
int64_t prompt_cut_bytes(int dim) { return (int64_t)prompt_slots(dim) * 2 * kPromptRows * (dim + 2) * 4; }
// (a page is converted once for all rows of a large tile: choose_form)
bool in_large_tiles(int dim, int64_t rows, int64_t units, int64_t all_pages) {
  return rows > kPromptFrom && (units > 256 || all_pages > (dim == 64 ? 64 : dim == 128 ? 16 : 32));
}

AttentionForm choose_form(int dim, int heads, int group, int batch, int all_rows, int max_rows, int max_tokens, int window, int sinks) {
  AttentionForm f{};
  const int64_t rows = (int64_t)max_rows * group, all_pages = ((int64_t)max_tokens + kPage - 1) / kPage;
  const int64_t seen = ((int64_t)window + max_rows) / kPage + 2 + ((int64_t)sinks + kPage - 1) / kPage, pages = window > 0 && seen < all_pages ? seen : all_pages;
  f.nt = dim < 256 && rows > 16 ? 2 : 1;
  const int64_t tiles = (rows + 16 * f.nt - 1) / (16 * f.nt), units = tiles * heads * batch;
  // Tiles of 128 rows for more than 64 (a page is converted once for all of them), but not where every small tile finds a compute
  // unit and reads few pages.  Small against large tiles, us: 68 rows, 8 heads of 128 dims, one sequence of 512 tokens 10.2 and 15.9,
  // of 1024 13.9 and 18.3, of 2048 23.6 and 20.8; 64 sequences of 512 tokens 56 and 34; 65 rows, 16 heads of 64 dims, 2048 tokens
  // 12.5 and 17.7; 100 rows, 4 heads of 256 dims, 2048 tokens 28.6 and 31.6, of 4096 49 and 36.
  if (in_large_tiles(dim, rows, units, all_pages)) {
    const int64_t most = (rows + kPromptRows - 1) / kPromptRows;
    f.prompt = true;
    f.tiles = (int)most;
    f.units = (int)(most * batch * heads);
    f.waves = 1;
    // Time (us) of a workgroup for each tile and of equal parts, fitted to 1 to 64 sequences of 512 to 32768 tokens, 64 to 2048 of
    // them new, of one length and of lengths down to an eighth.  The host knows the rows of all entries, and the longest alone: the
    // first form waits for it, the second reads what there is, and 0.6 of it is counted for each.  A tile ends at its last row, which
    // only helps the first form, and only where other tiles wait.
    const int slots = prompt_slots(dim);
    const double tiles_used = batch == 1 ? (double)most * heads : ((double)all_rows * group / kPromptRows + 0.5 * batch) * heads;
    const double whole_start = dim == 64 ? 6.5 : dim == 128 ? 9.0 : 9.5, whole_page = dim == 64 ? 0.78 : dim == 128 ? 1.09 : 3.9;
    const double cut_start = dim == 64 ? 10.0 : dim == 128 ? 14.0 : 18.0, cut_page = dim == 64 ? 1.9 : dim == 128 ? 2.7 : 4.0;
    // (least: more parts to join against fewer workgroups with work: 17 tiles of 2048 tokens 23.7 us with 4 pages, 26.6 with 8, of
    // 8192 tokens 40.8 and 35.3)
    f.least = all_pages <= 64 ? 4 : 8;
    auto cut_is_faster = [&](int64_t p) {
      const double each = (batch > 1 ? 0.6 : 1.0) * tiles_used * (double)p / slots;
      const double cut = cut_start + cut_page * (each > f.least ? each : f.least);
      const double whole = tiles_used > 256 ? whole_page * ((double)p - max_rows / (2.0 * kPage)) * (tiles_used / 256) : whole_page * (double)p;
      return cut < whole_start + whole;
    };
    f.may_cut = tiles_used < 512 && batch <= kMostPlannedPrompts && cut_is_faster(all_pages);
    if (f.may_cut && cut_is_faster(pages)) f.workgroups = slots;
    f.cut_bytes = prompt_cut_bytes(dim);
    return f;
  }
  f.least = 1;
  f.waves = waves_of(dim, f.nt);
  // Pages that a wavefront reads one after the other where each unit has a workgroup, and where the work is cut into equal parts.
  // Fitted to both forms over 1 to 200 sequences of 128 to 16384 tokens, of one length and of lengths down to a 16th: (4.3, 2.7),
  // (10, 5.0) us with 128 dims, int8.  The first form waits for its longest unit, the second reads what there is: the host knows
  // the longest sequence alone, and counts half of it for each.
  const double cut = (double)((units * pages + 256 * f.waves - 1) / (256 * f.waves)) * (batch > 1 ? 0.5 : 1.0);
  const double start = parts_start(f.waves), of_parts = start + (dim == 64 ? 2.9 : 5.0) * cut, of_units = time_of_units(dim, f.waves, units, pages);
  f.may_cut = batch <= kMostPlanned && tiles <= kMostCutTiles && time_of_units(dim, f.waves, units, all_pages) > start;
  f.cut_bytes = cut_bytes_of(dim, f.nt);
  if (f.may_cut && of_parts < of_units) f.workgroups = 256;
  f.time = f.workgroups ? of_parts : of_units;
  return f;
}

int64_t bytes_with_plan(int64_t cut_bytes) { return round_up_256(cut_bytes + kMostPlanned * (sizeof(KvEntry) + 4) + 4); }

// What a call needs: that of its form.
int64_t workspace_of_call(const AttentionForm& f) { return f.may_cut ? bytes_with_plan(f.cut_bytes) : 256; }

// What every call of no more entries, rows and tokens can do with: forms follow each other back and forth as a call grows, but each has its
// conditions, all of which grow with it, or hold up to a number of entries and of tiles.
int64_t workspace_up_to(int dim, int heads, int group, int batch, int max_rows, int max_tokens) {
  const int64_t rows = (int64_t)max_rows * group, all_pages = ((int64_t)max_tokens + kPage - 1) / kPage;
  const int64_t entries = batch < kMostPlanned ? batch : kMostPlanned;
  int64_t most = 256;
  for (int nt = 1; nt <= (dim < 256 && rows > 16 ? 2 : 1); ++nt) {
    const int64_t widest = dim < 256 && nt == 1 ? 1 : kMostCutTiles, all = (rows + 16 * nt - 1) / (16 * nt), tiles = all < widest ? all : widest;
    const int waves = waves_of(dim, nt);
    if (time_of_units(dim, waves, tiles * heads * entries, all_pages) > parts_start(waves)) {
      const int64_t bytes = bytes_with_plan(cut_bytes_of(dim, nt));
      most = bytes > most ? bytes : most;
    }
  }
  const int nt = dim < 256 ? 2 : 1;
  if (in_large_tiles(dim, rows, (rows + 16 * nt - 1) / (16 * nt) * heads * batch, all_pages)) {
    const int64_t bytes = bytes_with_plan(prompt_cut_bytes(dim));
    most = bytes > most ? bytes : most;
  }
  return most;
}

int check_sizes(const sfmp_kv_layout_t* layout, int32_t batch, int32_t rows, int32_t q_heads, int32_t max_rows, int32_t max_tokens) {
  if (int e = check_kv_layout(layout)) return e;
  if (batch < 0 || batch > 65535 || rows < 0 || rows > kMaxRows || max_rows < 0 || max_rows > rows || q_heads < 1 ||
      q_heads % layout->kv_heads || q_heads > 65536 || max_tokens < 1 || max_tokens > kMaxTablePages * kPage)
    return SFMP_ERR_SHAPE;
  const int64_t pages = ((int64_t)max_tokens + kPage - 1) / kPage;
  const int64_t unit_rows = (int64_t)max_rows * (q_heads / layout->kv_heads), tiles = (unit_rows + 15) / 16;
  if (unit_rows > kMaxRows || (tiles && pages > INT32_MAX / tiles) || (int64_t)batch * layout->kv_heads * pages * tiles > INT32_MAX) return SFMP_ERR_SHAPE;
  return SFMP_OK;
}

template <int D, int FMT, bool SINKS>
int launch_prompt(const AttentionArgs& a, const AttentionForm& f, const CutArgs& c, hipStream_t stream) {
  constexpr int threads = 256 * kGroups<D>, lds = 2 * kGroups<D> * (int)sizeof(PromptTile<D>);
  constexpr int cut_lds = 2 * (int)sizeof(PromptTile<D>) + (int)sizeof(Plan<kMostPlannedPrompts>);
  static_assert((D == 256 ? 1 : 2) * cut_lds <= 160 * 1024 && kPromptRows * D * 4 + 2048 <= lds, "LDS of a compute unit");
  if (f.workgroups) {
    if (int e = allow_full_lds((const void*)attend_prompt_cut_kernel<D, FMT, SINKS>, "attend_prompt_cut_kernel")) return e;
    attend_prompt_cut_kernel<D, FMT, SINKS><<<c.workgroups, 256, cut_lds, stream>>>(a, c);
    join_prompt_kernel<D, SINKS><<<dim3(f.tiles * (D / 32), a.v.heads, a.v.batch), 256, 0, stream>>>(a, c);
  } else {
    if (int e = allow_full_lds((const void*)attend_prompt_kernel<D, FMT, SINKS>, "attend_prompt_kernel")) return e;
    attend_prompt_kernel<D, FMT, SINKS><<<f.units, threads, lds, stream>>>(a, f.tiles);
  }
  return kv_launched("attend_prompt_kernel");
}

template <int D, int FMT, bool SINKS>
int launch_attention(const AttentionArgs& a, const AttentionForm& f, int max_rows, void* workspace, hipStream_t stream) {
  uint8_t* const entries = (uint8_t*)workspace + f.cut_bytes;
  const CutArgs c{(uint8_t*)workspace, (KvEntry*)entries, (int32_t*)(entries + kMostPlanned * sizeof(KvEntry)), f.workgroups, f.waves, f.least};
  if (f.prompt) return launch_prompt<D, FMT, SINKS>(a, f, c, stream);
  if constexpr (D < 256)
    if (f.nt == 2) return f.workgroups ? launch_cut<D, FMT, 2, SINKS>(a, c, stream) : launch_units<D, FMT, 2, SINKS>(a, max_rows, stream);
  return f.workgroups ? launch_cut<D, FMT, 1, SINKS>(a, c, stream) : launch_units<D, FMT, 1, SINKS>(a, max_rows, stream);
}


// Checks of a call behind those of make_kv_view and check_sizes; fills the rest of `a`.  (Nothing of it is used where there are no rows.)
int check_attention(const sfmp_kv_layout_t* layout, const sfmp_kv_tables_t* tables, const sfmp_kv_batch_t* batch, const void* Q_dev, int32_t q_heads,
                    int32_t dtype, int64_t q_stride, int32_t max_tokens, int32_t window, int32_t sinks, float scale, void* O_dev, int64_t o_stride,
                    float* lse_dev, AttentionArgs* a) {
  if (dtype != SFMP_TYPE_FP16 && dtype != SFMP_TYPE_BF16) return SFMP_ERR_LAYOUT;
  const int64_t width = (int64_t)q_heads * layout->head_dim;
  if (window < 0 || sinks < 0 || !(scale > 0.0f) || !(scale < INFINITY) || q_stride < width || o_stride < width || q_stride % 8 || o_stride % 8 ||
      q_stride > INT64_MAX / 8 / INT32_MAX || o_stride > INT64_MAX / 8 / INT32_MAX)
    return SFMP_ERR_SHAPE;
  if (batch->rows == 0 || batch->batch == 0) return SFMP_OK;
  if (!Q_dev || !O_dev) return SFMP_ERR_NULL;
  if (!kv_aligned(Q_dev, 16) || !kv_aligned(O_dev, 16) || !kv_aligned(lse_dev, 4)) return SFMP_ERR_ALIGN;
  a->Q = (const uint16_t*)Q_dev;
  a->O = (uint16_t*)O_dev;
  a->lse = lse_dev;
  a->q_stride = q_stride;
  a->o_stride = o_stride;
  a->q_heads = q_heads;
  a->group = q_heads / layout->kv_heads;
  // (a window longer than any sequence is none: positions less a window stay within 32 bits, also those of rows before the first token)
  a->window = window >= tables->table_pages * kPage ? 0 : window;
  a->sinks = sinks;
  a->max_pages = (max_tokens + kPage - 1) / kPage;
  a->scale = scale;
  a->bf16 = dtype == SFMP_TYPE_BF16;
  return SFMP_OK;
}

// A call (SINKS: sinks >= 1, 1 <= window < tokens of a table row).
template <bool SINKS>
int attend(const sfmp_kv_layout_t* layout, int32_t layer, const void* codes_dev, const float* scales_dev, const sfmp_kv_tables_t* tables,
           const sfmp_kv_batch_t* batch, const void* Q_dev, int32_t q_heads, int32_t dtype, int64_t q_stride, int32_t max_tokens,
           int32_t window, int32_t sinks, float scale, void* O_dev, int64_t o_stride, float* lse_dev, void* workspace_dev,
           int64_t workspace_bytes, void* hip_stream) {
  AttentionArgs a;
  if (int e = make_kv_view(layout, layer, codes_dev, scales_dev, tables, batch, &a.v)) return e;
  if (int e = check_sizes(layout, batch->batch, batch->rows, q_heads, batch->max_rows, max_tokens)) return e;
  if (int e = check_attention(layout, tables, batch, Q_dev, q_heads, dtype, q_stride, max_tokens, window, sinks, scale, O_dev, o_stride, lse_dev, &a)) return e;
  if (batch->rows == 0 || batch->batch == 0) return SFMP_OK;
  const AttentionForm f = batch->max_rows ? choose_form(layout->head_dim, layout->kv_heads, a.group, batch->batch, batch->rows, batch->max_rows,
                                                        max_tokens, window, SINKS ? sinks : 0)
                                          : AttentionForm{};
  if (!workspace_dev || !kv_aligned(workspace_dev, 256) || workspace_bytes < workspace_of_call(f)) return SFMP_ERR_WORKSPACE;
  if (batch->max_rows == 0) return SFMP_OK;
  auto with_dim = [&](auto fmt) {
    if (layout->head_dim == 64) return launch_attention<64, fmt(), SINKS>(a, f, batch->max_rows, workspace_dev, (hipStream_t)hip_stream);
    if (layout->head_dim == 128) return launch_attention<128, fmt(), SINKS>(a, f, batch->max_rows, workspace_dev, (hipStream_t)hip_stream);
    return launch_attention<256, fmt(), SINKS>(a, f, batch->max_rows, workspace_dev, (hipStream_t)hip_stream);
  };
  if (layout->format == SFMP_KV_INT8) return with_dim(std::integral_constant<int, SFMP_KV_INT8>{});
  return with_dim(std::integral_constant<int, SFMP_KV_FP8>{});
}

}  // namespace
}  // namespace sfmp
