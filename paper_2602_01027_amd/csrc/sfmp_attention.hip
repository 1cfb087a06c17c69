// Attention over the 8-bit paged cache.
#include "sfmp_kv.h"

namespace sfmp {
namespace {

// Wavefronts of a workgroup: two per SIMD, or, where sums and operands take more than half of its registers, one.
template <int D, int NT>
constexpr int kWaves = D * NT >= 256 ? 4 : 8;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.69314718055994531f;
// Weights are rounded to fp16 after multiplication by 2^14: a product with V then keeps its 11 bits down to 2^-28 of the largest.
constexpr float kWeightUnit = 16384.0f;
constexpr float kLeastReference = 7.8886090522101181e-31f;  // 2^-100

struct AttentionArgs {
  KvView v;
  const uint16_t* Q;
  uint16_t* O;
  float* lse;       // or null
  int64_t q_stride, o_stride;
  int32_t q_heads, group, window, max_pages;
  float scale;
  bool bf16;
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
  float m[NT], l[NT];  // running maximum of the scores (in units of ln 2) and sum of 2^(score - m)
};

// The rows of a unit (one sequence, one key/value head, 16 * NT of its query rows).
template <int D, int NT>
struct Rows {
  half8 q[NT][D / 32];
  float factor[NT];  // score = factor * scale of K * product
  int at[NT];        // position of the row in the sequence
  int first, last;   // smallest and largest of them
};

template <int D, int NT>
__device__ __forceinline__ void load_rows(const AttentionArgs& a, const KvEntry& e, int head, int tile, Rows<D, NT>& r) {
  const int i16 = threadIdx.x & 15, g = (threadIdx.x & 63) >> 4;
  const int count = e.n * a.group;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int row = (tile * NT + nt) * 16 + i16;
    const int token = min(row, count - 1) / a.group, h = min(row, count - 1) - token * a.group;
    const uint16_t* const src = a.Q + (int64_t)(e.row0 + token) * a.q_stride + (int64_t)(head * a.group + h) * D;
    r.at[nt] = e.length - e.n + token;
    r.factor[nt] = a.scale * kLog2e;
    // step 2c + h of the matrix instructions takes the dims 64 c + 16 g + 8 h + 0..7 of lane group g, so that the
    // keys of two steps are 16 contiguous bytes
    u32x4 raw[D / 32];
#pragma unroll
    for (int s = 0; s < D / 32; ++s)
      raw[s] = *reinterpret_cast<const u32x4*>(src + 64 * (s / 2) + 16 * g + 8 * (s % 2));
    if (!a.bf16) {
#pragma unroll
      for (int s = 0; s < D / 32; ++s) r.q[nt][s] = __builtin_bit_cast(half8, raw[s]);
    } else {
      // bf16 rows are brought into the range of fp16 by a power of two (largest element in [2^10, 2^11)): elements
      // down to 2^-25 of it stay exact, below the error is under 2^-35 of it
      uint32_t largest = 0;
#pragma unroll
      for (int s = 0; s < D / 32; ++s)
#pragma unroll
        for (int j = 0; j < 4; ++j) largest = max(largest, max(raw[s][j] & 0x7FFFu, raw[s][j] >> 16 & 0x7FFFu));
      largest = max(largest, (uint32_t)__shfl_xor((int)largest, 16));
      largest = max(largest, (uint32_t)__shfl_xor((int)largest, 32));
      const int exponent = min(max((int)(largest >> 7), 11), 254);  // (biased; both powers of two stay normal)
      const float up = __uint_as_float((uint32_t)(127 + 127 + 10 - exponent) << 23);
      r.factor[nt] *= __uint_as_float((uint32_t)(exponent - 10) << 23);
#pragma unroll
      for (int s = 0; s < D / 32; ++s)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          r.q[nt][s][2 * j] = (_Float16)(__uint_as_float(raw[s][j] << 16) * up);
          r.q[nt][s][2 * j + 1] = (_Float16)(__uint_as_float(raw[s][j] & 0xFFFF0000u) * up);
        }
    }
  }
  r.first = e.length - e.n + tile * NT * 16 / a.group;
  r.last = e.length - e.n + min((tile + 1) * NT * 16 - 1, count - 1) / a.group;
}

// Pages of a sequence that any of the rows at [first, last] sees.
struct PageRange {
  int begin, end;
};
__device__ __forceinline__ PageRange pages_seen(const AttentionArgs& a, int first, int last) {
  PageRange p;
  p.end = last < 0 ? 0 : last / kPage + 1;
  p.begin = a.window > 0 ? max(first - a.window + 1, 0) / kPage : 0;
  p.end = max(min(p.end, a.max_pages), p.begin);
  return p;
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

// Pages [begin, end) of a sequence, accumulated by one wavefront.
//
// The product of keys and queries comes out of the matrix instructions with lane (i, g) holding, for query row i, the
// keys 4 g + r of a tile of 16.  With the 16 rows of tile t being the keys 16 (i / 4) + 4 t + i % 4 of the page, these are
// the 16 consecutive keys 16 g .. 16 g + 15 over the four tiles: the very tokens that the lane reads of the transposed
// values with one load, and the place that the weights need as the other operand.  Nothing moves between lanes but the
// two steps of the maximum.
template <int D, int FMT, int NT>
__device__ __forceinline__ void accumulate(const AttentionArgs& a, const KvEntry& e, int head, int begin, int end,
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
  float reference = kLeastReference;  // largest scale of V so far: weights are multiplied by scale / reference
  // Numbers and scales of 64 pages at a time, one per lane
  int held_page = 0;
  float held_k = 0.0f, held_v = 0.0f;
  auto hold = [&](int page) {
    held_page = max(kv_page(a.v, e.slot, min(page + lane, end - 1)), 0);
    const float* const s = kv_scale(a.v, held_page, head, 0);
    held_k = s[0];
    held_v = s[1];
  };
  hold(begin);
  const uint8_t* block = kv_block<D>(a.v, __builtin_amdgcn_readlane(held_page, 0), head, 0);
  PageCodes<D> c;
  load_keys<D>(block, c);
  load_values<D>(block, c);
  for (int page = begin; page < end; ++page) {
    const int at = (page - begin) % 64;
    const float scale_k = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(held_k), at));
    const float scale_v = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(held_v), at));
    const bool more = page + 1 < end;
    if (more) {
      if (at == 63) hold(page + 1);
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
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const int left = e.length - (token + 4 * w);
        const uint32_t keep = left >= 4 ? ~0u : left <= 0 ? 0u : (1u << (8 * left)) - 1;
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) c.v[dt][w] &= keep;
      }
    }

    // running maximum and reference
    float factor[NT], now[NT];
    bool changed = scale_v > reference;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      factor[nt] = scale_k * r.factor[nt];
      float m = -INFINITY;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int x = 0; x < 4; ++x) s[nt][t][x] *= factor[nt];
      if (masked) {
        const int from = a.window > 0 ? r.at[nt] - a.window : -1;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const int j = token + 4 * t + x;
            if (j > r.at[nt] || j <= from) s[nt][t][x] = -INFINITY;
          }
      }
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int x = 0; x < 4; ++x) m = fmaxf(m, s[nt][t][x]);
      m = fmaxf(m, __shfl_xor(m, 16));
      m = fmaxf(m, __shfl_xor(m, 32));
      now[nt] = fmaxf(p.m[nt], m);
      changed |= now[nt] != p.m[nt];
    }
    if (__any(changed)) {
      float shrink = 1.0f;
      if (scale_v > reference) {
        shrink = reference / scale_v;
        reference = scale_v;
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const float alpha = now[nt] == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(p.m[nt] - now[nt]);
        p.m[nt] = now[nt];
        p.l[nt] *= alpha;
        const float both = alpha * shrink;
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) p.o[nt][dt] *= both;
      }
    }
    const float unit = scale_v * (kWeightUnit / reference);
    half8 w[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const float m = p.m[nt] == -INFINITY ? 0.0f : p.m[nt];
      float sum = 0.0f;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const float y = __builtin_amdgcn_exp2f(s[nt][t][x] - m);
          sum += y;
          w[nt][t / 2][4 * (t % 2) + x] = (_Float16)(y * unit);
          s[nt][t][x] = y;
        }
      if (masked && unit != unit) {  // a scale that is NaN reaches the rows that see the page, and no others
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int x = 0; x < 4; ++x)
            if (s[nt][t][x] == 0.0f) w[nt][t / 2][4 * (t % 2) + x] = (_Float16)0.0f;
      }
      p.l[nt] += sum;
    }
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int dt = 0; dt < D / 16; ++dt) {
        const half8 val = operand_of<FMT>(c.v[dt][2 * u], c.v[dt][2 * u + 1]);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
          p.o[nt][dt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(val, w[nt][u], p.o[nt][dt], 0, 0, 0);
      }
    if (more) load_values<D>(block, c);
  }
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    p.l[nt] += __shfl_xor(p.l[nt], 16);
    p.l[nt] += __shfl_xor(p.l[nt], 32);
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) p.o[nt][dt] *= reference * (1.0f / kWeightUnit);
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

template <int D, int NT>
__device__ __forceinline__ void merge_partial(const uint8_t* at, Partial<D, NT>& p) {
  const int lane = threadIdx.x & 63;
  const floatx4* const o = reinterpret_cast<const floatx4*>(at);
  const float* const ml = reinterpret_cast<const float*>(at + kPartialVectors<D, NT> * 16);
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const float m2 = ml[nt * 64 + lane], l2 = ml[(NT + nt) * 64 + lane];
    const float top = fmaxf(p.m[nt], m2), base = top == -INFINITY ? 0.0f : top;
    const float f1 = __builtin_amdgcn_exp2f(p.m[nt] - base), f2 = __builtin_amdgcn_exp2f(m2 - base);
    p.m[nt] = top;
    p.l[nt] = p.l[nt] * f1 + l2 * f2;
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) p.o[nt][dt] = p.o[nt][dt] * f1 + o[(nt * (D / 16) + dt) * 64 + lane] * f2;
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

// One workgroup per unit: its wavefronts take ranges of the pages and are joined in LDS.
template <int D, int FMT, int NT>
__global__ __launch_bounds__((64 * kWaves<D, NT>)) void attend_unit_kernel(AttentionArgs a) {
  extern __shared__ __align__(16) uint8_t lds[];
  constexpr int WAVES = kWaves<D, NT>, BYTES = kPartialBytes<D, NT>;
  const int tile = blockIdx.x, head = blockIdx.y, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const KvEntry e = kv_entry(a.v, blockIdx.z);
  if (tile * NT * 16 >= e.n * a.group) return;
  Rows<D, NT> r;
  load_rows<D, NT>(a, e, head, tile, r);
  const PageRange all = e.slot < 0 ? PageRange{0, 0} : pages_seen(a, r.first, r.last);
  const int each = (all.end - all.begin + WAVES - 1) / WAVES;
  const int begin = min(all.begin + wave * each, all.end), end = min(begin + each, all.end);
  Partial<D, NT> p;
  accumulate<D, FMT, NT>(a, e, head, begin, end, r, p);
  if (wave > 0) store_partial<D, NT>(lds + (wave - 1) * BYTES, p);
  __syncthreads();
  if (wave > 0) return;
#pragma unroll 1
  for (int at = 0; at < WAVES - 1; ++at) merge_partial<D, NT>(lds + at * BYTES, p);
  store_rows<D, NT>(a, e, head, tile, p);
}

// ---- the work cut into equal parts ---------------------------------------------------------------------------------
//
// All pages of all units in a row, by (batch entry, head, tile of rows, page): every workgroup takes `share` of them, every
// wavefront an equal part of that.  Each workgroup finds its part from the lengths of the batch (a prefix sum in LDS), so
// that neither the host nor another launch has to know them, and sequences of any lengths load every compute unit alike.
// A unit that lies inside one workgroup is finished there; one that is cut leaves a partial result per workgroup, which
// join_kernel adds up in order.

constexpr int kMostPlanned = 1024;  // batch entries

struct Plan {
  int before[kMostPlanned + 1];  // pages of all units of the entries before
  int sums[16];
  int left[8];  // of a wavefront whose part starts inside a unit: 1 if the unit ends in it, 2 if not
  KvEntry entry[kMostPlanned];
};

struct CutArgs {
  uint8_t* partials;  // [workgroup][2]: of a unit that began before the workgroup's part, of one that ends behind it
  int32_t workgroups, waves;
};

// Pages that the units of an entry read: all of them the same ones.
__device__ __forceinline__ PageRange pages_of_entry(const AttentionArgs& a, const KvEntry& e) {
  if (e.slot < 0 || e.n < 1) return PageRange{0, 0};
  return pages_seen(a, e.length - e.n, e.length - 1);
}
__device__ __forceinline__ int tiles_of_entry(const AttentionArgs& a, const KvEntry& e, int rows) {
  return (e.n * a.group + rows - 1) / rows;
}

// Fills the plan; all threads of the workgroup.  Returns the pages of all units.
template <int THREADS>
__device__ int make_plan(const AttentionArgs& a, int rows, Plan* plan) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int carry = 0;
  for (int base = 0; base < a.v.batch; base += THREADS) {
    const int b = base + threadIdx.x;
    int pages = 0;
    if (b < a.v.batch) {
      const KvEntry e = kv_entry(a.v, b);
      plan->entry[b] = e;
      const PageRange p = pages_of_entry(a, e);
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
struct Share {
  int of_wave, of_workgroup;
};
__device__ __forceinline__ Share share_of(const CutArgs& c, int total) {
  Share s;
  s.of_wave = max((total + c.workgroups * c.waves - 1) / (c.workgroups * c.waves), 1);
  s.of_workgroup = s.of_wave * c.waves;
  return s;
}

template <int D, int FMT, int NT>
__global__ __launch_bounds__((64 * kWaves<D, NT>)) void attend_cut_kernel(AttentionArgs a, CutArgs c) {
  extern __shared__ __align__(16) uint8_t lds[];
  constexpr int WAVES = kWaves<D, NT>, BYTES = kPartialBytes<D, NT>;
  Plan& plan = *reinterpret_cast<Plan*>(lds + (WAVES - 1) * BYTES);
  int* const left = plan.left;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int total = make_plan<64 * WAVES>(a, 16 * NT, &plan);
  const Share share = share_of(c, total);
  const int from = (int)min((int64_t)blockIdx.x * share.of_workgroup, (int64_t)total);
  int at = min(from + wave * share.of_wave, total);
  const int to = min(at + share.of_wave, total);
  uint8_t* const partials = c.partials + (int64_t)blockIdx.x * 2 * BYTES;
  int kind = 0;
  enum { kNone, kFromBefore, kFromHere };  // (of a unit that this wavefront has to complete)
  int open = kNone;
  Partial<D, NT> p;
  KvEntry e;
  int head = 0, tile = 0;
  while (at < to) {
    int lo = 0, hi = a.v.batch;  // the last entry that starts at or before `at`
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      (plan.before[mid] <= at ? lo : hi) = mid;
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    e = plan.entry[lo];
    const PageRange pages = pages_of_entry(a, e);
    const int each = pages.end - pages.begin, tiles = tiles_of_entry(a, e, 16 * NT);
    const int unit = (at - plan.before[lo]) / each, first = (at - plan.before[lo]) - unit * each;
    const int count = min(each - first, to - at);
    head = unit / tiles, tile = unit - head * tiles;
    Rows<D, NT> r;
    load_rows<D, NT>(a, e, head, tile, r);
    accumulate<D, FMT, NT>(a, e, head, pages.begin + first, pages.begin + first + count, r, p);
    at += count;
    const bool begins = first == 0, ends = first + count == each;
    if (begins && ends) {
      store_rows<D, NT>(a, e, head, tile, p);
    } else if (begins) {
      open = kFromHere;
    } else if (wave > 0) {
      store_partial<D, NT>(lds + (wave - 1) * BYTES, p);
      kind = ends ? 1 : 2;
    } else if (ends) {
      store_partial<D, NT>(partials, p);
    } else {
      open = kFromBefore;
    }
  }
  if ((threadIdx.x & 63) == 0) left[wave] = kind;
  __syncthreads();
  if (open == kNone) return;
  bool ended = false;
#pragma unroll 1
  for (int w = wave + 1; w < WAVES && !ended && left[w]; ++w) {
    merge_partial<D, NT>(lds + (w - 1) * BYTES, p);
    ended = left[w] == 1;
  }
  if (open == kFromBefore)
    store_partial<D, NT>(partials, p);
  else if (ended)
    store_rows<D, NT>(a, e, head, tile, p);
  else
    store_partial<D, NT>(partials + BYTES, p);
}

// One workgroup per head and batch entry: adds up the partial results of its units that were cut, and stores zeros for an
// entry without pages.  Wavefront w takes the dims 16 w + 0..15.
template <int D, int NT>
__global__ __launch_bounds__(4 * D) void join_kernel(AttentionArgs a, CutArgs c) {
  constexpr int BYTES = kPartialBytes<D, NT>;
  __shared__ Plan plan;
  const int total = make_plan<4 * D>(a, 16 * NT, &plan);
  const Share share = share_of(c, total);
  const int b = blockIdx.x, head = blockIdx.y, dt = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const KvEntry e = plan.entry[b];
  const PageRange pages = pages_of_entry(a, e);
  const int each = pages.end - pages.begin, tiles = tiles_of_entry(a, e, 16 * NT);
  for (int tile = 0; tile < tiles; ++tile) {
    const int start = plan.before[b] + (head * tiles + tile) * each;
    const int w0 = start / share.of_workgroup, w1 = (start + each - 1) / share.of_workgroup;
    if (each > 0 && w0 == w1) continue;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float m = -INFINITY, l = 0.0f;
      floatx4 o = {0.0f, 0.0f, 0.0f, 0.0f};
      if (each > 0) {
        auto ml_of = [&](int w) {
          return reinterpret_cast<const float*>(c.partials + ((int64_t)w * 2 + (w == w0)) * BYTES + kPartialVectors<D, NT> * 16) + nt * 64 + lane;
        };
        auto o_of = [&](int w) {
          return reinterpret_cast<const floatx4*>(c.partials + ((int64_t)w * 2 + (w == w0)) * BYTES) + (nt * (D / 16) + dt) * 64 + lane;
        };
#pragma unroll 8
        for (int w = w0; w <= w1; ++w) m = fmaxf(m, *ml_of(w));
        const float base = m == -INFINITY ? 0.0f : m;
#pragma unroll 8
        for (int w = w0; w <= w1; ++w) {
          const float f = __builtin_amdgcn_exp2f(*ml_of(w) - base);
          l += ml_of(w)[NT * 64] * f;
          o += *o_of(w) * f;
        }
      }
      const RowResult r = row_result(a, e, head, (tile * NT + nt) * 16 + (lane & 15), D, m, l, dt == 0);
      if (r.there) store_dims(a, r, dt, o);
    }
  }
}

// ---- launches ------------------------------------------------------------------------------------------------------

template <int D, int FMT, int NT>
int launch_units(const AttentionArgs& a, int max_rows, hipStream_t stream) {
  const void* const fn = (const void*)attend_unit_kernel<D, FMT, NT>;
  if (int e = allow_full_lds(fn, "attend_unit_kernel")) return e;
  const int64_t tiles = ((int64_t)max_rows * a.group + 16 * NT - 1) / (16 * NT);
  constexpr int threads = 64 * kWaves<D, NT>, lds = (kWaves<D, NT> - 1) * kPartialBytes<D, NT>;
  attend_unit_kernel<D, FMT, NT><<<dim3((uint32_t)tiles, a.v.heads, a.v.batch), threads, lds, stream>>>(a);
  return kv_launched("attend_unit_kernel");
}

template <int D, int FMT, int NT>
int launch_cut(const AttentionArgs& a, const CutArgs& c, hipStream_t stream) {
  const void* const fn = (const void*)attend_cut_kernel<D, FMT, NT>;
  if (int e = allow_full_lds(fn, "attend_cut_kernel")) return e;
  constexpr int threads = 64 * kWaves<D, NT>, lds = (kWaves<D, NT> - 1) * kPartialBytes<D, NT> + sizeof(Plan);
  attend_cut_kernel<D, FMT, NT><<<c.workgroups, threads, lds, stream>>>(a, c);
  join_kernel<D, NT><<<dim3(a.v.batch, a.v.heads), 4 * D, 0, stream>>>(a, c);
  return kv_launched("attend_cut_kernel");
}

// How a call runs.
struct AttentionForm {
  int nt;          // tiles of 16 rows that a unit holds
  int workgroups;  // 0: one per unit
  int waves;       // of one
  int64_t partial_bytes;
};

int waves_of(int dim, int nt) { return dim * nt >= 256 ? 4 : 8; }

AttentionForm choose_form(int dim, int heads, int group, int batch, int max_rows, int max_tokens) {
  AttentionForm f{};
  const int64_t rows = (int64_t)max_rows * group;
  f.nt = dim < 256 && rows > 16 ? 2 : 1;
  f.waves = waves_of(dim, f.nt);
  const int64_t tiles = (rows + 16 * f.nt - 1) / (16 * f.nt), units = tiles * heads * batch, pages = (max_tokens + kPage - 1) / kPage;
  const int64_t alone = (units + 255) / 256 * ((pages + f.waves - 1) / f.waves);
  const int64_t cut = (units * pages + 256 * f.waves - 1) / (256 * f.waves);
  if (batch <= kMostPlanned && tiles <= 4 && alone > cut + 8) {
    f.workgroups = 256;
    f.partial_bytes = (int64_t)f.workgroups * 2 * (f.nt * (dim / 16) * 64 * 16 + 2 * f.nt * 64 * 4);
  }
  return f;
}

template <int D, int FMT>
int launch_attention(const AttentionArgs& a, const AttentionForm& f, int max_rows, void* workspace, hipStream_t stream) {
  const CutArgs c{(uint8_t*)workspace, f.workgroups, f.waves};
  if constexpr (D < 256)
    if (f.nt == 2) return f.workgroups ? launch_cut<D, FMT, 2>(a, c, stream) : launch_units<D, FMT, 2>(a, max_rows, stream);
  return f.workgroups ? launch_cut<D, FMT, 1>(a, c, stream) : launch_units<D, FMT, 1>(a, max_rows, stream);
}

}  // namespace
}  // namespace sfmp

using namespace sfmp;

extern "C" int sfmp_kv_attention_workspace(const sfmp_kv_layout_t* layout, int32_t batch, int32_t rows, int32_t q_heads,
                                           int32_t max_rows, int32_t max_tokens, int64_t* bytes) {
  if (!bytes) return SFMP_ERR_NULL;
  if (int e = check_kv_layout(layout)) return e;
  if (batch < 0 || batch > 65535 || rows < 0 || rows > kMaxRows || max_rows < 0 || max_rows > rows || q_heads < 1 ||
      q_heads % layout->kv_heads || q_heads > 65536 || max_tokens < 1 || max_tokens > kMaxTablePages * kPage)
    return SFMP_ERR_SHAPE;
  const int64_t pages = ((int64_t)max_tokens + kPage - 1) / kPage;
  const int64_t tiles = ((int64_t)max_rows * (q_heads / layout->kv_heads) + 15) / 16;
  if ((tiles && pages > INT32_MAX / tiles) || (int64_t)batch * layout->kv_heads * pages * tiles > INT32_MAX) return SFMP_ERR_SHAPE;
  *bytes = 256;
  if (batch && max_rows) {
    const AttentionForm f = choose_form(layout->head_dim, layout->kv_heads, q_heads / layout->kv_heads, batch, max_rows, max_tokens);
    *bytes = round_up_256(f.partial_bytes + 1);
  }
  return SFMP_OK;
}

extern "C" int sfmp_kv_attention(const sfmp_kv_layout_t* layout, int32_t layer, const void* codes_dev,
                                 const float* scales_dev, const sfmp_kv_tables_t* tables, const sfmp_kv_batch_t* batch,
                                 const void* Q_dev, int32_t q_heads, int32_t dtype, int64_t q_stride, int32_t max_tokens,
                                 int32_t window, float scale, void* O_dev, int64_t o_stride, float* lse_dev,
                                 void* workspace_dev, int64_t workspace_bytes, void* hip_stream) {
  AttentionArgs a;
  if (int e = make_kv_view(layout, layer, codes_dev, scales_dev, tables, batch, &a.v)) return e;
  int64_t need = 0;
  if (int e = sfmp_kv_attention_workspace(layout, batch->batch, batch->rows, q_heads, batch->max_rows, max_tokens, &need)) return e;
  if (dtype != SFMP_TYPE_FP16 && dtype != SFMP_TYPE_BF16) return SFMP_ERR_LAYOUT;
  const int64_t width = (int64_t)q_heads * layout->head_dim;
  if (window < 0 || !(scale > 0.0f) || !(scale < INFINITY) || q_stride < width || o_stride < width || q_stride % 8 || o_stride % 8 ||
      q_stride > INT64_MAX / 8 / INT32_MAX || o_stride > INT64_MAX / 8 / INT32_MAX)
    return SFMP_ERR_SHAPE;
  if (batch->rows == 0 || batch->batch == 0) return SFMP_OK;
  if (!Q_dev || !O_dev) return SFMP_ERR_NULL;
  if (!kv_aligned(Q_dev, 16) || !kv_aligned(O_dev, 16) || !kv_aligned(lse_dev, 4)) return SFMP_ERR_ALIGN;
  if (!workspace_dev || !kv_aligned(workspace_dev, 256) || workspace_bytes < need) return SFMP_ERR_WORKSPACE;
  a.Q = (const uint16_t*)Q_dev;
  a.O = (uint16_t*)O_dev;
  a.lse = lse_dev;
  a.q_stride = q_stride;
  a.o_stride = o_stride;
  a.q_heads = q_heads;
  a.group = q_heads / layout->kv_heads;
  a.window = window;
  a.max_pages = (max_tokens + kPage - 1) / kPage;
  a.scale = scale;
  a.bf16 = dtype == SFMP_TYPE_BF16;
  const hipStream_t stream = (hipStream_t)hip_stream;
  if (batch->max_rows == 0) return SFMP_OK;
  const AttentionForm f = choose_form(layout->head_dim, layout->kv_heads, a.group, batch->batch, batch->max_rows, max_tokens);
  auto with_dim = [&](auto fmt) {
    if (layout->head_dim == 64) return launch_attention<64, fmt()>(a, f, batch->max_rows, workspace_dev, stream);
    if (layout->head_dim == 128) return launch_attention<128, fmt()>(a, f, batch->max_rows, workspace_dev, stream);
    return launch_attention<256, fmt()>(a, f, batch->max_rows, workspace_dev, stream);
  };
  if (layout->format == SFMP_KV_INT8) return with_dim(std::integral_constant<int, SFMP_KV_INT8>{});
  return with_dim(std::integral_constant<int, SFMP_KV_FP8>{});
}
