// Attention over the 8-bit paged cache.
#include "sfmp_kv.h"

namespace sfmp {
namespace {

constexpr int kWaves = 8;  // wavefronts of a workgroup
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
  float reference = kLeastReference;  // largest scale of V so far: weights are multiplied by scale / reference
  int held_page = 0;
  float held_k = 0.0f, held_v = 0.0f;
  for (int page = begin; page < end; ++page) {
    if ((page - begin) % 64 == 0) {  // the next 64 pages' numbers and scales, one per lane
      const int mine = min(page + lane, end - 1);
      held_page = max(kv_page(a.v, e.slot, mine), 0);
      const float* const s = kv_scale(a.v, held_page, head, 0);
      held_k = s[0];
      held_v = s[1];
    }
    const int at = (page - begin) % 64;
    const int id = __builtin_amdgcn_readlane(held_page, at);
    const float scale_k = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(held_k), at));
    const float scale_v = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(held_v), at));
    const uint8_t* const block = kv_block<D>(a.v, id, head, 0);
    PageCodes<D> c;
    load_keys<D>(block, c);
    load_values<D>(block, c);

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
        for (int x = 0; x < 4; ++x) {
          float z = s[nt][t][x] * factor[nt];
          if (masked) {
            const int j = token + 4 * t + x;
            if (j > r.at[nt] || (a.window > 0 && j <= r.at[nt] - a.window)) z = -INFINITY;
          }
          s[nt][t][x] = z;
          m = fmaxf(m, z);
        }
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
          // (a scale that is NaN reaches the rows that see the page, and no others)
          w[nt][t / 2][4 * (t % 2) + x] = (_Float16)(masked && y == 0.0f ? 0.0f : y * unit);
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
  }
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    p.l[nt] += __shfl_xor(p.l[nt], 16);
    p.l[nt] += __shfl_xor(p.l[nt], 32);
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) p.o[nt][dt] *= reference * (1.0f / kWeightUnit);
  }
}

template <int D, int NT>
__device__ __forceinline__ void merge(Partial<D, NT>& p, const floatx4* o, const float* m, const float* l) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const float m2 = m[nt * 64 + lane], l2 = l[nt * 64 + lane];
    const float top = fmaxf(p.m[nt], m2), base = top == -INFINITY ? 0.0f : top;
    const float f1 = __builtin_amdgcn_exp2f(p.m[nt] - base), f2 = __builtin_amdgcn_exp2f(m2 - base);
    p.m[nt] = top;
    p.l[nt] = p.l[nt] * f1 + l2 * f2;
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) p.o[nt][dt] = p.o[nt][dt] * f1 + o[(nt * (D / 16) + dt) * 64 + lane] * f2;
  }
}

// Results of the rows of a unit.
template <int D, int NT>
__device__ __forceinline__ void store_rows(const AttentionArgs& a, const KvEntry& e, int head, int tile, const Partial<D, NT>& p) {
  const int i16 = threadIdx.x & 15, g = (threadIdx.x & 63) >> 4;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int row = (tile * NT + nt) * 16 + i16;
    if (row >= e.n * a.group) continue;
    const int token = row / a.group, h = head * a.group + row - token * a.group;
    const bool empty = p.m[nt] == -INFINITY && p.l[nt] == 0.0f;  // (not where every score is a NaN)
    const float inverse = empty ? 0.0f : 1.0f / p.l[nt];
    uint16_t* const dst = a.O + (int64_t)(e.row0 + token) * a.o_stride + (int64_t)h * D + 4 * g;
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) {
      u32x2 w;
#pragma unroll
      for (int x = 0; x < 2; ++x)
        w[x] = bits_of(p.o[nt][dt][2 * x] * inverse, a.bf16) | (uint32_t)bits_of(p.o[nt][dt][2 * x + 1] * inverse, a.bf16) << 16;
      *reinterpret_cast<u32x2*>(dst + 16 * dt) = w;
    }
    if (a.lse && g == 0)
      a.lse[(int64_t)(e.row0 + token) * a.q_heads + h] = empty ? -INFINITY : (p.m[nt] + __builtin_amdgcn_logf(p.l[nt])) * kLn2;
  }
}

// One workgroup per unit: its wavefronts take ranges of the pages and are joined in LDS.
template <int D, int FMT, int NT>
__global__ __launch_bounds__(64 * kWaves) void attend_unit_kernel(AttentionArgs a) {
  extern __shared__ __align__(16) uint8_t lds[];
  constexpr int VALUES = NT * D / 16 * 64;  // floatx4 of a partial result
  floatx4* const o = reinterpret_cast<floatx4*>(lds);
  float* const ml = reinterpret_cast<float*>(lds + (kWaves - 1) * VALUES * 16);
  const int tile = blockIdx.x, head = blockIdx.y, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const KvEntry e = kv_entry(a.v, blockIdx.z);
  if (tile * NT * 16 >= e.n * a.group) return;
  Rows<D, NT> r;
  load_rows<D, NT>(a, e, head, tile, r);
  const PageRange all = e.slot < 0 ? PageRange{0, 0} : pages_seen(a, r.first, r.last);
  const int each = (all.end - all.begin + kWaves - 1) / kWaves;
  const int begin = min(all.begin + wave * each, all.end), end = min(begin + each, all.end);
  Partial<D, NT> p;
  accumulate<D, FMT, NT>(a, e, head, begin, end, r, p);
  if (wave > 0) {
    const int at = wave - 1;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      ml[(at * 2 * NT + nt) * 64 + lane] = p.m[nt];
      ml[(at * 2 * NT + NT + nt) * 64 + lane] = p.l[nt];
#pragma unroll
      for (int dt = 0; dt < D / 16; ++dt) o[at * VALUES + (nt * (D / 16) + dt) * 64 + lane] = p.o[nt][dt];
    }
  }
  __syncthreads();
  if (wave > 0) return;
  for (int at = 0; at < kWaves - 1; ++at)
    merge<D, NT>(p, o + at * VALUES, ml + at * 2 * NT * 64, ml + (at * 2 * NT + NT) * 64);
  store_rows<D, NT>(a, e, head, tile, p);
}

template <int D, int NT>
constexpr int unit_lds_bytes() { return (kWaves - 1) * (NT * D / 16 * 64 * 16 + 2 * NT * 64 * 4); }

template <int D, int FMT, int NT>
int launch_units(const AttentionArgs& a, int max_rows, hipStream_t stream) {
  const void* const fn = (const void*)attend_unit_kernel<D, FMT, NT>;
  if (int e = allow_full_lds(fn, "attend_unit_kernel")) return e;
  const int64_t tiles = ((int64_t)max_rows * a.group + 16 * NT - 1) / (16 * NT);
  attend_unit_kernel<D, FMT, NT><<<dim3((uint32_t)tiles, a.v.heads, a.v.batch), 64 * kWaves, unit_lds_bytes<D, NT>(), stream>>>(a);
  return kv_launched("attend_unit_kernel");
}

template <int D, int FMT>
int launch_attention(const AttentionArgs& a, int max_rows, hipStream_t stream) {
  if constexpr (D < 256)
    if ((int64_t)max_rows * a.group > 16) return launch_units<D, FMT, 2>(a, max_rows, stream);
  return launch_units<D, FMT, 1>(a, max_rows, stream);
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
  auto with_dim = [&](auto fmt) {
    if (layout->head_dim == 64) return launch_attention<64, fmt()>(a, batch->max_rows, stream);
    if (layout->head_dim == 128) return launch_attention<128, fmt()>(a, batch->max_rows, stream);
    return launch_attention<256, fmt()>(a, batch->max_rows, stream);
  };
  if (layout->format == SFMP_KV_INT8) return with_dim(std::integral_constant<int, SFMP_KV_INT8>{});
  return with_dim(std::integral_constant<int, SFMP_KV_FP8>{});
}
