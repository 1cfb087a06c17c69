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

// Rows and columns of 4 x 4 bytes exchanged: x[i] holds 4 tokens of dim i, then y[j] 4 dims of token j (and the other way).
__device__ __forceinline__ void turn4(const uint32_t (&x)[4], uint32_t (&y)[4]) {
  const uint32_t ab = __builtin_amdgcn_perm(x[1], x[0], 0x05010400u), cd = __builtin_amdgcn_perm(x[3], x[2], 0x05010400u);
  const uint32_t ef = __builtin_amdgcn_perm(x[1], x[0], 0x07030602u), gh = __builtin_amdgcn_perm(x[3], x[2], 0x07030602u);
  y[0] = __builtin_amdgcn_perm(cd, ab, 0x05040100u);
  y[1] = __builtin_amdgcn_perm(cd, ab, 0x07060302u);
  y[2] = __builtin_amdgcn_perm(gh, ef, 0x05040100u);
  y[3] = __builtin_amdgcn_perm(gh, ef, 0x07060302u);
}

// Who does what in a workgroup of D threads for the keys or the values of one (page, head): with keys a thread has 8 dims of
// every eighth token, so that a token is read and written by neighbours; with values 4 dims of 16 tokens, whose codes it
// turns in registers: values of a page lie as [dim][token].
template <int D>
struct PagePart {
  bool values;
  int dim;    // first
  int token;  // first
  __device__ __forceinline__ PagePart() {
    const int t = threadIdx.x;
    values = blockIdx.z;
    dim = values ? t % (D / 4) * 4 : t % (D / 8) * 8;
    token = values ? t / (D / 4) * 16 : t / (D / 8);
  }
  __device__ __forceinline__ int key_token(int i) const { return token + 8 * i; }  // i < 8
};

// Quantises what a call writes into one (page, head): s = max |x| / 127 (or the power of two that brings it under 448), codes rint(x / s).
// Tokens that the page held before keep their codes unless the scale grows: then they are read and rounded anew,
// rint(code s_old / s_new).  Bound by latency at a token per sequence (length, page number, rows, maximum over the workgroup, one after
// the other): 64 sequences, 8 heads of 128 dims 7.4 us, 2.1 MB of pages touched; a prompt of 2048 tokens 7.8 us, 12.6 MB.  One
// workgroup for each K and V of a (page, head), so that the maximum needs no second launch.
template <int D, int FMT>
__global__ __launch_bounds__(D) void append_kernel(KvView v, const uint16_t* K, const uint16_t* V, int64_t k_stride,
                                                       int64_t v_stride, bool bf16, int pages_per_entry) {
  __shared__ uint32_t largest_of_wave[D / 64];
  const int b = blockIdx.x / pages_per_entry, head = blockIdx.y;
  const KvEntry e = kv_entry(v, b);
  const int before = e.length - e.n, start = max(before, 0);  // (rows that would stand before token 0 are left out)
  const int place = start / kPage + blockIdx.x % pages_per_entry;
  if (e.n < 1 || place * kPage >= e.length) return;
  const int page = kv_page(v, e.slot, place);
  if (page < 0) return;
  const int first = max(start - place * kPage, 0), end = min(e.length - place * kPage, kPage);  // new tokens of the page
  const PagePart<D> part;
  float* const scale_at = kv_scale(v, page, head, part.values);
  const float held = first > 0 ? *scale_at : 0.0f;

  const int64_t row = (int64_t)e.row0 + place * kPage - before;  // of token 0 of the page
  uint32_t raw[32];  // keys: 8 times 8 dims; values: 16 times 4 dims
  uint32_t largest = 0;
  auto look = [&](uint32_t w) {
    largest = max(largest, max(__float_as_uint(value_of(w & 0xFFFFu, bf16)) & 0x7FFFFFFFu, __float_as_uint(value_of(w >> 16, bf16)) & 0x7FFFFFFFu));
  };
  if (!part.values) {
    const uint16_t* const src = K + row * k_stride + (int64_t)head * D + part.dim;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int token = part.key_token(i);
      u32x4 w = {0, 0, 0, 0};
      if (token >= first && token < end) w = *reinterpret_cast<const u32x4*>(src + token * k_stride);
#pragma unroll
      for (int j = 0; j < 4; ++j) raw[4 * i + j] = w[j];
    }
  } else {
    const uint16_t* const src = V + row * v_stride + (int64_t)head * D + part.dim;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const int token = part.token + j;
      u32x2 w = {0, 0};
      if (token >= first && token < end) w = *reinterpret_cast<const u32x2*>(src + token * v_stride);
      raw[2 * j] = w[0], raw[2 * j + 1] = w[1];
    }
  }
#pragma unroll
  for (int i = 0; i < 32; ++i) look(raw[i]);
#pragma unroll
  for (int s = 1; s < 64; s *= 2) largest = max(largest, (uint32_t)__shfl_xor((int)largest, s));
  if ((threadIdx.x & 63) == 0) largest_of_wave[threadIdx.x >> 6] = largest;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < D / 64; ++w) largest = max(largest, largest_of_wave[w]);
  const float need = scale_for<FMT>(largest);
  // NaN in either stays
  const float scale = first == 0 || need != need ? need : need > held ? need : held;
  const bool grown = first > 0 && scale > held;
  const float kept = grown ? held / scale : 1.0f;
  const float inverse = inverse_scale(scale);
  if (threadIdx.x == 0 && (first == 0 || scale != held)) *scale_at = scale;

  uint8_t* const block = kv_block<D>(v, page, head, part.values);
  auto encoded = [&](uint32_t a, uint32_t b) {  // 4 new values
    const float s = inverse > 0.0f ? inverse : 0.0f;
    float x[4] = {value_of(a & 0xFFFFu, bf16), value_of(a >> 16, bf16), value_of(b & 0xFFFFu, bf16), value_of(b >> 16, bf16)};
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = s > 0.0f ? x[j] * s : 0.0f;
    return encode4<FMT>(x);
  };
  auto requantised = [&](uint32_t w) {
    float x[4];
    decode4<FMT>(w, x);
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] *= kept;
    return encode4<FMT>(x);
  };
  if (!part.values) {  // [token][dim]
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int token = part.key_token(i);
      u32x2* const at = reinterpret_cast<u32x2*>(block + token * D + part.dim);
      if ((token >= first && token < end) || first == 0) {  // (codes of no value are those of zeros)
        *at = u32x2{encoded(raw[4 * i], raw[4 * i + 1]), encoded(raw[4 * i + 2], raw[4 * i + 3])};
      } else if (grown && token < first) {
        const u32x2 w = *at;
        *at = u32x2{requantised(w[0]), requantised(w[1])};
      }
    }
    return;
  }
  // [dim][token]
  const int from = part.token;
  if (from >= end && first > 0) return;
  if (from + 16 <= first && !grown) return;
  uint32_t turned[4][4];  // [dim][4 tokens each]
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    uint32_t x[4], y[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = encoded(raw[2 * (4 * q + j)], raw[2 * (4 * q + j) + 1]);
    turn4(x, y);
#pragma unroll
    for (int d = 0; d < 4; ++d) turned[d][q] = y[d];
  }
#pragma unroll
  for (int d = 0; d < 4; ++d) {
    uint8_t* const at = block + (part.dim + d) * kPage + from;
    u32x4 w = {turned[d][0], turned[d][1], turned[d][2], turned[d][3]};
    if (first > 0 && !grown && end - max(first, from) <= 2) {  // one or two tokens: what is there need not be read
      for (int token = max(first, from); token < min(end, from + 16); ++token) {
        const int j = token - from;
        const uint32_t word = j < 8 ? (j < 4 ? w[0] : w[1]) : (j < 12 ? w[2] : w[3]);
        at[j] = (uint8_t)(word >> (8 * (j & 3)));
      }
      continue;
    }
    if (first > 0 && (from < first || from + 16 > end)) {
      const u32x4 old = *reinterpret_cast<const u32x4*>(at);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        uint32_t fresh = 0, earlier = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int token = from + 4 * q + j;
          if (token >= first && token < end) fresh |= 0xFFu << (8 * j);
          if (token < first) earlier |= 0xFFu << (8 * j);
        }
        const uint32_t again = grown ? requantised(old[q]) : old[q];
        w[q] = (w[q] & fresh) | (again & earlier) | (old[q] & ~(fresh | earlier));
      }
    }
    *reinterpret_cast<u32x4*>(at) = w;
  }
}

// Reads back the part of a call that lies in one (page, head, K or V).  Workgroup = 256 threads; thread = token tid / 4 of the page
// and every fourth run of 8 dims, so that four threads write 64 contiguous bytes of a row; values are turned in LDS first.
// (Turned in registers, as they are written, 64 sequences' last pages took 11 us instead of 9.6.)  Bound by latency, too: 64 last pages
// 8.4 - 9.3 us, 2048 tokens of 8 heads of 128 dims 6.3 us for 12.6 MB.
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
  // (the table's entry is asked for before the length is known)
  const int listed = e.slot >= 0 && place < v.table_pages ? kv_page(v, e.slot, place) : -1;
  const int token = threadIdx.x >> 2, quarter = threadIdx.x & 3;
  const int64_t at = (int64_t)place * kPage + token;
  const int page = (int64_t)place * kPage < e.length ? listed : -1;
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
    append_kernel<d(), fmt()><<<grid, d(), 0, (hipStream_t)hip_stream>>>(v, (const uint16_t*)K_dev, (const uint16_t*)V_dev, k_stride,
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
