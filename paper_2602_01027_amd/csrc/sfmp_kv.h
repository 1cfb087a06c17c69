// The 8-bit paged key/value cache as the kernels see it: argument checks, addresses, conversion of codes.  gfx950 only.
#pragma once
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "sfmp_device.h"
#include "sfmp_internal.h"

namespace sfmp {

constexpr int kPage = SFMP_KV_PAGE;
constexpr int kMaxTablePages = 1 << 20;  // (positions, rows and the pages of a call are added up in 32 bits)
constexpr int kMaxRows = 1 << 30;

// One layer of the cache and the rows of a call.
struct KvView {
  uint8_t* codes;       // of the layer: [pages][heads][2][64 * D]
  float* scales;        // of the layer: [pages][heads][2]
  const int32_t* table;
  const int32_t* lengths;
  const int32_t* slots;
  const int32_t* row_start;
  int32_t pages, heads, sequences, table_pages, batch, rows, max_rows;
};

inline bool kv_aligned(const void* p, uintptr_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

inline int check_kv_layout(const sfmp_kv_layout_t* L) {
  if (!L) return SFMP_ERR_NULL;
  sfmp_kv_layout_t want;
  if (int e = sfmp_kv_query(L->pages, L->kv_heads, L->head_dim, L->format, L->layers, &want)) return e;
  if (L->page_bytes != want.page_bytes || L->codes_bytes != want.codes_bytes || L->scales_bytes != want.scales_bytes)
    return SFMP_ERR_LAYOUT;
  return SFMP_OK;
}

inline int check_kv_tables(const sfmp_kv_tables_t* t, bool need_refs) {
  if (!t || !t->page_table_dev || !t->lengths_dev || (need_refs && !t->refs_dev)) return SFMP_ERR_NULL;
  if (t->sequences < 1 || t->table_pages < 1 || t->table_pages > kMaxTablePages) return SFMP_ERR_SHAPE;
  if (!kv_aligned(t->page_table_dev, 4) || !kv_aligned(t->lengths_dev, 4) || !kv_aligned(t->refs_dev, 4)) return SFMP_ERR_ALIGN;
  return SFMP_OK;
}

inline int check_kv_buffers(const void* codes, const void* scales) {
  if (!codes || !scales) return SFMP_ERR_NULL;
  return kv_aligned(codes, 16) && kv_aligned(scales, 8) ? SFMP_OK : SFMP_ERR_ALIGN;
}

// Checks of the calls that work on the rows of a batch; fills `view`.
inline int make_kv_view(const sfmp_kv_layout_t* L, int32_t layer, const void* codes, const float* scales,
                        const sfmp_kv_tables_t* t, const sfmp_kv_batch_t* b, KvView* view) {
  if (int e = check_kv_layout(L)) return e;
  if (int e = check_kv_tables(t, false)) return e;
  if (int e = check_kv_buffers(codes, scales)) return e;
  if (!b) return SFMP_ERR_NULL;
  if (layer < 0 || layer >= L->layers || b->batch < 0 || b->rows < 0 || b->max_rows < 0 || b->max_rows > b->rows || b->rows > kMaxRows ||
      (!b->row_start_dev && (b->rows != b->batch || (b->batch > 0 && b->max_rows != 1))) || (!b->slots_dev && b->batch > t->sequences))
    return SFMP_ERR_SHAPE;
  if (!kv_aligned(b->slots_dev, 4) || !kv_aligned(b->row_start_dev, 4)) return SFMP_ERR_ALIGN;
  *view = KvView{(uint8_t*)codes + (int64_t)layer * L->pages * L->page_bytes,
                 (float*)scales + (int64_t)layer * L->pages * L->kv_heads * 2, t->page_table_dev, t->lengths_dev,
                 b->slots_dev, b->row_start_dev, L->pages, L->kv_heads, t->sequences, t->table_pages, b->batch, b->rows, b->max_rows};
  return SFMP_OK;
}

inline int kv_launched(const char* what) {
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return SFMP_OK;
  note_hip_error(what, hipGetErrorString(e));
  return SFMP_ERR_HIP;
}

// ---- device ------------------------------------------------------------------------------------------------------

struct KvEntry {
  int32_t slot;     // -1: none (its length reads as 0)
  int32_t length;
  int32_t row0, n;  // its rows
};

__device__ __forceinline__ KvEntry kv_entry(const KvView& v, int b) {
  KvEntry e;
  e.slot = v.slots ? v.slots[b] : b;
  if ((uint32_t)e.slot >= (uint32_t)v.sequences) e.slot = -1;
  e.length = e.slot < 0 ? 0 : v.lengths[e.slot];
  e.length = min(max(e.length, 0), v.table_pages * kPage);
  if (v.row_start) {
    e.row0 = min(max(v.row_start[b], 0), v.rows);
    e.n = min(min(max(v.row_start[b + 1], e.row0), v.rows) - e.row0, v.max_rows);
  } else {
    e.row0 = b;
    e.n = 1;
  }
  return e;
}

// Number of the page in place `i` of a sequence's row (i inside the row); -1 if the table holds no page there.
__device__ __forceinline__ int32_t kv_page(const KvView& v, int slot, int i) {
  const int32_t id = v.table[(int64_t)slot * v.table_pages + i];
  return (uint32_t)id < (uint32_t)v.pages ? id : -1;
}

template <int D>
__device__ __forceinline__ uint8_t* kv_block(const KvView& v, int page, int head, int which) {
  return v.codes + (((int64_t)page * v.heads + head) * 2 + which) * (kPage * D);
}
__device__ __forceinline__ float* kv_scale(const KvView& v, int page, int head, int which) {
  return v.scales + ((int64_t)page * v.heads + head) * 2 + which;
}

template <int T>  // a SFMP_TYPE_
__device__ __forceinline__ float value_of(uint16_t bits) {
  if constexpr (T == SFMP_TYPE_BF16) return __uint_as_float((uint32_t)bits << 16);
  return (float)__builtin_bit_cast(_Float16, bits);
}
__device__ __forceinline__ float value_of(uint16_t bits, bool bf16) {
  return bf16 ? value_of<SFMP_TYPE_BF16>(bits) : value_of<SFMP_TYPE_FP16>(bits);
}
__device__ __forceinline__ uint16_t bits_of(float x, bool bf16) {
  if (!bf16) return __builtin_bit_cast(uint16_t, (_Float16)x);
  return __builtin_bit_cast(uint16_t, (__bf16)x);
}

// 4 codes -> 4 fp32 values (before the scale).  INT8: byte - 128.
template <int FMT>
__device__ __forceinline__ void decode4(uint32_t w, float (&x)[4]) {
  if constexpr (FMT == SFMP_KV_INT8) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = (float)((w >> (8 * i)) & 0xFFu) - 128.0f;
  } else {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
    x[0] = lo[0], x[1] = lo[1], x[2] = hi[0], x[3] = hi[1];
  }
}

// 4 fp32 values (divided by the scale) -> 4 codes, rounded to nearest even and limited to the largest code.
template <int FMT>
__device__ __forceinline__ uint32_t encode4(const float (&x)[4]) {
  if constexpr (FMT == SFMP_KV_INT8) {
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) w |= (uint32_t)((int)fminf(fmaxf(rintf(x[i]), -127.0f), 127.0f) + 128) << (8 * i);
    return w;
  } else {
    float y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = fminf(fmaxf(x[i], -448.0f), 448.0f);
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    return __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], lo, true);
  }
}
template <int FMT>
constexpr uint8_t kZeroCode = FMT == SFMP_KV_INT8 ? 128 : 0;

// Scale of a block from the bits of its largest magnitude (as unsigned numbers these are ordered finite < infinity < NaN).
template <int FMT>
__device__ __forceinline__ float scale_for(uint32_t largest_bits) {
  if (largest_bits >= 0x7F800000u) return __uint_as_float(0x7FC00000u);
  const float m = __uint_as_float(largest_bits);
  if (m < 7.8886090522101181e-31f) return 0.0f;  // 2^-100: below, 1 / scale and the scale itself near the ends of fp32
  if constexpr (FMT == SFMP_KV_INT8) return m / 127.0f;
  // 448 = 1.75 * 2^8
  const uint32_t exponent = (largest_bits >> 23) - 8 + ((largest_bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return __uint_as_float(exponent << 23);
}
__device__ __forceinline__ float inverse_scale(float s) { return s > 0.0f ? 1.0f / s : 0.0f; }

}  // namespace sfmp
