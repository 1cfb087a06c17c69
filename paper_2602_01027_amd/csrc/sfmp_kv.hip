// The 8-bit paged cache: quantising writes, read-back.
#include "sfmp_kv.h"

using namespace sfmp;

extern "C" int sfmp_kv_query(int32_t pages, int32_t kv_heads, int32_t head_dim, int32_t format, int32_t layers,
                             sfmp_kv_layout_t* out) {
  if (!out) return SFMP_ERR_NULL;
  if (pages < 1 || kv_heads < 1 || kv_heads > 1024 || layers < 1 || (head_dim != 64 && head_dim != 128 && head_dim != 256))
    return SFMP_ERR_SHAPE;
  if (format != SFMP_KV_INT8 && format != SFMP_KV_FP8) return SFMP_ERR_LAYOUT;
  const int64_t page_bytes = (int64_t)kv_heads * 2 * kPage * head_dim, all = (int64_t)pages * layers;
  if (all > INT64_MAX / page_bytes) return SFMP_ERR_SHAPE;
  *out = sfmp_kv_layout_t{pages, kv_heads, head_dim, format, layers, 0, page_bytes, all * page_bytes, all * kv_heads * 8};
  return SFMP_OK;
}

namespace {

// Quantises what a call writes into one (page, head, K or V).  Workgroup = 256 threads; thread = token tid / 4 of the page
// and every fourth run of 8 dims, so that four threads read 64 contiguous bytes of a row.  The values (codes of a page
// are transposed) go through LDS.
template <int D, int FMT>
__global__ __launch_bounds__(256) void append_kernel(KvView v, const uint16_t* K, const uint16_t* V, int64_t k_stride,
                                                     int64_t v_stride, bool bf16, int pages_per_entry) {
  constexpr int RUNS = D / 32, PITCH = kPage + 4;
  __shared__ uint32_t largest_of_wave[4];
  __shared__ __align__(16) uint8_t tile[D * PITCH];
  const int b = blockIdx.x / pages_per_entry, head = blockIdx.y, which = blockIdx.z;
  const KvEntry e = kv_entry(v, b);
  const int before = e.length - e.n, start = max(before, 0);  // (rows that would stand before token 0 are left out)
  const int place = start / kPage + blockIdx.x % pages_per_entry;
  if (e.n < 1 || place * kPage >= e.length) return;
  const int page = kv_page(v, e.slot, place);
  if (page < 0) return;
  const int first = max(start - place * kPage, 0), end = min(e.length - place * kPage, kPage);  // new tokens of the page

  const int token = threadIdx.x >> 2, quarter = threadIdx.x & 3;
  const bool fresh = token >= first && token < end;
  uint16_t raw[RUNS][8];
  uint32_t largest = 0;
  if (fresh) {
    const int64_t row = (int64_t)e.row0 + place * kPage + token - before;
    const uint16_t* src = (which ? V + row * v_stride : K + row * k_stride) + (int64_t)head * D;
#pragma unroll
    for (int i = 0; i < RUNS; ++i)
      *reinterpret_cast<u32x4*>(raw[i]) = *reinterpret_cast<const u32x4*>(src + 8 * (quarter + 4 * i));
#pragma unroll
    for (int i = 0; i < RUNS; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) largest = max(largest, __float_as_uint(value_of(raw[i][j], bf16)) & 0x7FFFFFFFu);
  }
#pragma unroll
  for (int s = 1; s < 64; s *= 2) largest = max(largest, (uint32_t)__shfl_xor((int)largest, s));
  if ((threadIdx.x & 63) == 0) largest_of_wave[threadIdx.x >> 6] = largest;
  float* const scale_at = kv_scale(v, page, head, which);
  const float held = first > 0 ? *scale_at : 0.0f;
  __syncthreads();
  largest = max(max(largest_of_wave[0], largest_of_wave[1]), max(largest_of_wave[2], largest_of_wave[3]));
  const float need = scale_for<FMT>(largest);
  // NaN in either stays
  const float scale = first == 0 || need != need ? need : need > held ? need : held;
  const bool grown = first > 0 && scale > held;
  const float kept = grown ? held / scale : 1.0f;
  const float inverse = inverse_scale(scale);
  if (threadIdx.x == 0 && (first == 0 || scale != held)) *scale_at = scale;

  uint8_t* const block = kv_block<D>(v, page, head, which);
  uint32_t codes[RUNS][2];
  if (fresh) {
#pragma unroll
    for (int i = 0; i < RUNS; ++i)
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        float x[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = inverse > 0.0f ? value_of(raw[i][4 * half + j], bf16) * inverse : 0.0f;
        codes[i][half] = encode4<FMT>(x);
      }
  } else {
#pragma unroll
    for (int i = 0; i < RUNS; ++i) codes[i][0] = codes[i][1] = kZeroCode<FMT> * 0x01010101u;
  }
  auto requantised = [&](uint32_t w) {
    float x[4];
    decode4<FMT>(w, x);
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] *= kept;
    return encode4<FMT>(x);
  };
  if (which == 0) {  // [token][dim]
#pragma unroll
    for (int i = 0; i < RUNS; ++i) {
      u32x2* const at = reinterpret_cast<u32x2*>(block + token * D + 8 * (quarter + 4 * i));
      if (fresh || first == 0) {
        *at = u32x2{codes[i][0], codes[i][1]};
      } else if (grown && token < first) {
        const u32x2 w = *at;
        *at = u32x2{requantised(w[0]), requantised(w[1])};
      }
    }
    return;
  }
  // [dim][token]: the codes are turned in LDS, then laid over what the page holds
#pragma unroll
  for (int i = 0; i < RUNS; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) tile[(8 * (quarter + 4 * i) + j) * PITCH + token] = codes[i][j >> 2] >> (8 * (j & 3));
  __syncthreads();
  for (int at = threadIdx.x * 4; at < D * kPage; at += 1024) {
    const int dim = at / kPage, t = at % kPage;  // 4 tokens of a dim
    const uint32_t w = *reinterpret_cast<const uint32_t*>(tile + dim * PITCH + t);
    if (first == 0) {
      *reinterpret_cast<uint32_t*>(block + at) = w;
    } else if (t + 4 > first ? t < end : grown) {
      uint32_t old = *reinterpret_cast<const uint32_t*>(block + at), fresh_bytes = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (t + j >= first && t + j < end) fresh_bytes |= 0xFFu << (8 * j);
      uint32_t mix = old;
      if (grown) {
        uint32_t earlier = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (t + j < first) earlier |= 0xFFu << (8 * j);
        mix = (requantised(old) & earlier) | (old & ~earlier);
      }
      *reinterpret_cast<uint32_t*>(block + at) = (w & fresh_bytes) | (mix & ~fresh_bytes);
    }
  }
}

// Reads back the part of a call that lies in one (page, head, K or V).  Thread = token tid / 4, as above; values of V are
// turned in LDS first.
template <int D, int FMT>
__global__ __launch_bounds__(256) void gather_kernel(KvView v, const int32_t* first_of, void* K, void* V, int64_t k_stride,
                                                     int64_t v_stride, int dtype, int pages_per_entry) {
  constexpr int RUNS = D / 32, PITCH = kPage + 4;
  __shared__ __align__(16) uint8_t tile[D * PITCH];
  const int b = blockIdx.x / pages_per_entry, head = blockIdx.y, which = blockIdx.z;
  const KvEntry e = kv_entry(v, b);
  const int start = max(first_of[b], 0);
  const int place = start / kPage + blockIdx.x % pages_per_entry;
  if (e.n < 1 || (int64_t)place * kPage >= (int64_t)start + e.n) return;
  const int token = threadIdx.x >> 2, quarter = threadIdx.x & 3;
  const int64_t at = (int64_t)place * kPage + token;
  const int page = e.slot >= 0 && (int64_t)place * kPage < e.length ? kv_page(v, e.slot, place) : -1;
  const float scale = page < 0 ? 0.0f : *kv_scale(v, page, head, which);
  uint32_t codes[RUNS][2];
  if (page >= 0) {
    const uint8_t* const block = kv_block<D>(v, page, head, which);
    if (which == 0) {
#pragma unroll
      for (int i = 0; i < RUNS; ++i) {
        const u32x2 w = *reinterpret_cast<const u32x2*>(block + token * D + 8 * (quarter + 4 * i));
        codes[i][0] = w[0], codes[i][1] = w[1];
      }
    } else {
      for (int x = threadIdx.x * 4; x < D * kPage; x += 1024)
        *reinterpret_cast<uint32_t*>(tile + x / kPage * PITCH + x % kPage) = *reinterpret_cast<const uint32_t*>(block + x);
      __syncthreads();
#pragma unroll
      for (int i = 0; i < RUNS; ++i)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          uint32_t w = 0;
#pragma unroll
          for (int j = 0; j < 4; ++j) w |= (uint32_t)tile[(8 * (quarter + 4 * i) + 4 * half + j) * PITCH + token] << (8 * j);
          codes[i][half] = w;
        }
    }
  }
  if (at < start || at >= (int64_t)start + e.n) return;
  const bool written = page >= 0 && at < e.length;
  const int64_t out = ((int64_t)e.row0 + at - start) * (which ? v_stride : k_stride) + (int64_t)head * D;
  void* const dst = which ? V : K;
#pragma unroll
  for (int i = 0; i < RUNS; ++i) {
    float x[8];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      float y[4];
      decode4<FMT>(codes[i][half], y);
#pragma unroll
      for (int j = 0; j < 4; ++j) x[4 * half + j] = written ? y[j] * scale : 0.0f;
    }
    const int64_t to = out + 8 * (quarter + 4 * i);
    if (dtype == SFMP_TYPE_FP32) {
      floatx4* const p = reinterpret_cast<floatx4*>((float*)dst + to);
      p[0] = floatx4{x[0], x[1], x[2], x[3]};
      p[1] = floatx4{x[4], x[5], x[6], x[7]};
    } else {
      u32x4 w;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        w[j] = bits_of(x[2 * j], dtype == SFMP_TYPE_BF16) | (uint32_t)bits_of(x[2 * j + 1], dtype == SFMP_TYPE_BF16) << 16;
      *reinterpret_cast<u32x4*>((uint16_t*)dst + to) = w;
    }
  }
}

template <typename F>
void for_kv_layout(const sfmp_kv_layout_t* L, F f) {
  auto with_format = [&](auto d) {
    if (L->format == SFMP_KV_INT8)
      f(d, std::integral_constant<int, SFMP_KV_INT8>{});
    else
      f(d, std::integral_constant<int, SFMP_KV_FP8>{});
  };
  if (L->head_dim == 64)
    with_format(std::integral_constant<int, 64>{});
  else if (L->head_dim == 128)
    with_format(std::integral_constant<int, 128>{});
  else
    with_format(std::integral_constant<int, 256>{});
}

int check_kv_rows(const void* p, int64_t stride, int64_t width, int size) {
  if (!p) return SFMP_ERR_NULL;
  if (stride < width || stride % 8 || stride > INT64_MAX / 8 / INT32_MAX) return SFMP_ERR_SHAPE;
  return kv_aligned(p, 16) && size ? SFMP_OK : SFMP_ERR_ALIGN;
}

}  // namespace

extern "C" int sfmp_kv_append(const sfmp_kv_layout_t* layout, int32_t layer, void* codes_dev, float* scales_dev,
                              const sfmp_kv_tables_t* tables, const sfmp_kv_batch_t* batch, const void* K_dev,
                              const void* V_dev, int32_t dtype, int64_t k_stride, int64_t v_stride, void* hip_stream) {
  KvView v;
  if (int e = make_kv_view(layout, layer, codes_dev, scales_dev, tables, batch, &v)) return e;
  if (dtype != SFMP_TYPE_FP16 && dtype != SFMP_TYPE_BF16) return SFMP_ERR_LAYOUT;
  if (v.rows == 0 || v.batch == 0) return SFMP_OK;
  const int64_t width = (int64_t)layout->kv_heads * layout->head_dim;
  if (int e = check_kv_rows(K_dev, k_stride, width, 2)) return e;
  if (int e = check_kv_rows(V_dev, v_stride, width, 2)) return e;
  const int64_t pages = ((int64_t)batch->max_rows + kPage - 2) / kPage + 1;
  if (pages * v.batch > INT32_MAX) return SFMP_ERR_SHAPE;
  const dim3 grid((uint32_t)(pages * v.batch), v.heads, 2);
  for_kv_layout(layout, [&](auto d, auto fmt) {
    append_kernel<d(), fmt()><<<grid, 256, 0, (hipStream_t)hip_stream>>>(v, (const uint16_t*)K_dev, (const uint16_t*)V_dev, k_stride,
                                                                         v_stride, dtype == SFMP_TYPE_BF16, (int)pages);
  });
  return kv_launched("append_kernel");
}

extern "C" int sfmp_kv_gather(const sfmp_kv_layout_t* layout, int32_t layer, const void* codes_dev,
                              const float* scales_dev, const sfmp_kv_tables_t* tables, const sfmp_kv_batch_t* batch,
                              const int32_t* first_dev, void* K_dev, void* V_dev, int32_t dtype, int64_t k_stride,
                              int64_t v_stride, void* hip_stream) {
  KvView v;
  if (int e = make_kv_view(layout, layer, codes_dev, scales_dev, tables, batch, &v)) return e;
  if (dtype != SFMP_TYPE_FP16 && dtype != SFMP_TYPE_BF16 && dtype != SFMP_TYPE_FP32) return SFMP_ERR_LAYOUT;
  if (v.rows == 0 || v.batch == 0) return SFMP_OK;
  if (!first_dev) return SFMP_ERR_NULL;
  if (!kv_aligned(first_dev, 4)) return SFMP_ERR_ALIGN;
  const int64_t width = (int64_t)layout->kv_heads * layout->head_dim;
  if (int e = check_kv_rows(K_dev, k_stride, width, 2)) return e;
  if (int e = check_kv_rows(V_dev, v_stride, width, 2)) return e;
  const int64_t pages = ((int64_t)batch->max_rows + kPage - 2) / kPage + 1;
  if (pages * v.batch > INT32_MAX) return SFMP_ERR_SHAPE;
  const dim3 grid((uint32_t)(pages * v.batch), v.heads, 2);
  for_kv_layout(layout, [&](auto d, auto fmt) {
    gather_kernel<d(), fmt()><<<grid, 256, 0, (hipStream_t)hip_stream>>>(v, first_dev, K_dev, V_dev, k_stride, v_stride, dtype,
                                                                         (int)pages);
  });
  return kv_launched("gather_kernel");
}
