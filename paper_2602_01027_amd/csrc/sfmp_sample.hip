// Choice of the next token: temperature, top-k, top-p, min-p and one random number per row.
//
// Every filter keeps a prefix of the tokens ordered by (falling logit, rising number), and the token is where the running
// sum of weights passes a threshold.  So no sort is needed, only positions in that order: a histogram of counts and
// weights over 2048 bins of (l - m) / T finds the bin of a position, and the tokens of that one bin, a few hundred of a
// hundred thousand, are ranked against each other in LDS.  Weights are whole numbers (2^31 for the most probable token), so
// that their sums do not depend on the order in which workgroups and atomics add them.
#include <math.h>

#include "sfmp_device.h"
#include "sfmp_internal.h"

namespace sfmp {
namespace {

constexpr int kBins = 2048;
constexpr float kBinsPerUnit = 92.0f;  // weights are 0 below (l - m) / T = -32 ln 2 = -22.2
constexpr int kSliceThreads = 256;
constexpr int kPickThreads = 1024;
constexpr int kListed = 2048;          // tokens that are ranked in LDS

struct SampleArgs {
  const void* logits;
  int32_t rows, vocab, slices;
  int64_t stride;
  const float* temperature;
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  const float* uniform;
  int32_t* tokens;
  float* logprobs;
  float* slice_max;         // [rows][slices]
  unsigned long long* mass; // [rows][kBins]
  uint32_t* count;          // [rows][kBins]
};

template <int T>
__device__ __forceinline__ float logit_of(uint32_t bits) {
  float x;
  if constexpr (T == SFMP_TYPE_FP32)
    x = __uint_as_float(bits);
  else if constexpr (T == SFMP_TYPE_BF16)
    x = __uint_as_float(bits << 16);
  else
    x = (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
  return x != x ? -INFINITY : x;
}

// Calls f(number, logit) for the tokens [from, to) of a row; the threads take runs of 16 aligned bytes in turn.
template <int T, int THREADS, typename F>
__device__ __forceinline__ void for_each_logit(const void* row, int from, int to, F f) {
  constexpr int SIZE = T == SFMP_TYPE_FP32 ? 4 : 2, RUN = 16 / SIZE;
  const int lead = (int)((reinterpret_cast<uintptr_t>(row) & 15) / SIZE);  // elements between the aligned address and the row
  const uint8_t* const base = (const uint8_t*)row - lead * SIZE;
#pragma unroll 2
  for (int v = (from + lead) / RUN + threadIdx.x; v * RUN < to + lead; v += THREADS) {
    const int first = v * RUN - lead;
    if (first >= from && first + RUN <= to) {
      const u32x4 w = *reinterpret_cast<const u32x4*>(base + (int64_t)v * 16);
#pragma unroll
      for (int j = 0; j < RUN; ++j)
        f(first + j, logit_of<T>(SIZE == 4 ? w[j] : (j & 1) ? w[j / 2] >> 16 : w[j / 2] & 0xFFFFu));
    } else {
      for (int i = max(first, from); i < min(first + RUN, to); ++i)
        f(i, logit_of<T>(SIZE == 4 ? ((const uint32_t*)row)[i] : ((const uint16_t*)row)[i]));
    }
  }
}

__device__ __forceinline__ float max_of_wave(float x) {
#pragma unroll
  for (int s = 1; s < 64; s *= 2) x = fmaxf(x, __shfl_xor(x, s));
  return x;
}

// What the weights of a row are computed from.
struct Row {
  const void* logits;
  float m, inverse;
  __device__ __forceinline__ float y(float l) const {
    return l == m ? 0.0f : l == -INFINITY ? -INFINITY : (l - m) * inverse;
  }
  // (expf of a value far below is 0: the bins past the weights are not reached)
  static __device__ __forceinline__ uint32_t weight(float y) { return (uint32_t)rintf(expf(y) * 2147483648.0f); }
  static __device__ __forceinline__ int bin(float y) { return min((int)(-y * kBinsPerUnit), kBins - 1); }
};

template <int T>
__device__ __forceinline__ Row make_row(const SampleArgs& a, int r) {
  const int lane = threadIdx.x & 63;
  float m = -INFINITY;
  for (int s = lane; s < a.slices; s += 64) m = fmaxf(m, a.slice_max[(int64_t)r * a.slices + s]);
  const float t = a.temperature ? a.temperature[r] : 1.0f;
  return Row{(const uint8_t*)a.logits + r * a.stride * (T == SFMP_TYPE_FP32 ? 4 : 2), max_of_wave(m), 1.0f / fmaxf(t, 0.0f)};
}

__device__ __forceinline__ int slice_from(const SampleArgs& a, int s) { return (int)((int64_t)a.vocab * s / a.slices); }

// Largest logit of every slice; clears the histograms.
template <int T>
__global__ __launch_bounds__(kSliceThreads) void sample_max_kernel(SampleArgs a) {
  __shared__ float of_wave[kSliceThreads / 64];
  const int s = blockIdx.x, r = blockIdx.y;
  const void* const row = (const uint8_t*)a.logits + r * a.stride * (T == SFMP_TYPE_FP32 ? 4 : 2);
  float m = -INFINITY;
  for_each_logit<T, kSliceThreads>(row, slice_from(a, s), slice_from(a, s + 1), [&](int, float l) { m = fmaxf(m, l); });
  for (int i = s * kSliceThreads + threadIdx.x; i < kBins; i += a.slices * kSliceThreads) {
    a.mass[(int64_t)r * kBins + i] = 0;
    a.count[(int64_t)r * kBins + i] = 0;
  }
  m = max_of_wave(m);
  if ((threadIdx.x & 63) == 0) of_wave[threadIdx.x >> 6] = m;
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int i = 1; i < kSliceThreads / 64; ++i) m = fmaxf(m, of_wave[i]);
    a.slice_max[(int64_t)r * a.slices + s] = m;
  }
}

// Adds a slice to the histogram of its row.  A bin of a slice is one 64-bit word in LDS: its count above bit 46, its
// weight below (a slice has at most 2^15 tokens of at most 2^31).
constexpr int kCountBit = 46;
constexpr int kMostSlice = 1 << 15;
template <int T>
__global__ __launch_bounds__(kSliceThreads) void sample_bins_kernel(SampleArgs a) {
  __shared__ unsigned long long bins[kBins];
  const int s = blockIdx.x, r = blockIdx.y;
  for (int i = threadIdx.x; i < kBins; i += kSliceThreads) bins[i] = 0;
  const Row row = make_row<T>(a, r);
  __syncthreads();
  if (row.m == -INFINITY) return;
  for_each_logit<T, kSliceThreads>(row.logits, slice_from(a, s), slice_from(a, s + 1), [&](int, float l) {
    const float y = row.y(l);
    if (y > -23.0f) {
      const uint32_t w = Row::weight(y);
      if (w) atomicAdd(&bins[Row::bin(y)], (1ull << kCountBit) + w);
    }
  });
  __syncthreads();
  for (int i = threadIdx.x; i < kBins; i += kSliceThreads)
    if (const unsigned long long x = bins[i]) {
      atomicAdd(&a.mass[(int64_t)r * kBins + i], x & ((1ull << kCountBit) - 1));
      atomicAdd(&a.count[(int64_t)r * kBins + i], (uint32_t)(x >> kCountBit));
    }
}

// (Numbers in the order that logits have, falling: a smaller key is a more probable token.)
__device__ __forceinline__ uint32_t falling_key(float l) {
  const uint32_t u = __float_as_uint(l == 0.0f ? 0.0f : l);
  return u & 0x80000000u ? u : ~u & 0x7FFFFFFFu;
}

// A token found by position.
struct Place {
  unsigned long long before, through;  // running sum of weights up to it, and with it
  int token;
  float y;
};

// Everything that one workgroup shares while it places positions in a row.
struct PickShared {
  unsigned long long mass[kBins];  // prefix sums up to and with each bin
  uint32_t count[kBins];
  unsigned long long list_mass[kListed];
  uint64_t list_key[kListed];
  unsigned long long wave_mass[kPickThreads / 64];
  uint32_t wave_count[kPickThreads / 64];
  unsigned long long digit_mass[kBins];
  uint32_t digit_count[kBins];
  Place found;
  int listed, bin, digit;
  unsigned long long min_mass;
};

// Inclusive sums over kBins entries in place.
__device__ void prefix_sums(unsigned long long* mass, uint32_t* count, PickShared* sh) {
  const int i = threadIdx.x, lane = i & 63, wave = i >> 6;
  unsigned long long m1 = mass[2 * i], m2 = m1 + mass[2 * i + 1], m = m2;
  uint32_t c1 = count[2 * i], c2 = c1 + count[2 * i + 1], c = c2;
#pragma unroll
  for (int s = 1; s < 64; s *= 2) {
    const unsigned long long y = __shfl_up(m, s);
    const uint32_t z = __shfl_up(c, s);
    if (lane >= s) m += y, c += z;
  }
  if (lane == 63) sh->wave_mass[wave] = m, sh->wave_count[wave] = c;
  __syncthreads();
  unsigned long long mb = m - m2;
  uint32_t cb = c - c2;
  for (int w = 0; w < wave; ++w) mb += sh->wave_mass[w], cb += sh->wave_count[w];
  mass[2 * i] = mb + m1, mass[2 * i + 1] = mb + m2;
  count[2 * i] = cb + c1, count[2 * i + 1] = cb + c2;
  __syncthreads();
}

// What a position is sought by: the k-th token (from 1), the first whose running sum is at least `aim`, or the first whose
// running sum exceeds `passed`.
struct Sought {
  enum { kCount, kAtLeast, kAbove } by;
  uint32_t k;
  double aim;
  unsigned long long passed;
  __device__ __forceinline__ bool reached(uint32_t count, unsigned long long mass) const {
    return by == kCount ? count >= k : by == kAtLeast ? (double)mass >= aim : mass > passed;
  }
};

// Finds the token at a position; the histogram's prefix sums are in sh->mass and sh->count and reach it.
template <int T>
__device__ Place place_of(const SampleArgs& a, const Row& row, const Sought& sought, PickShared* sh) {
  const int i = threadIdx.x;
#pragma unroll
  for (int j = 2 * i; j <= 2 * i + 1; ++j)
    if (sought.reached(sh->count[j], sh->mass[j]) && (j == 0 || !sought.reached(sh->count[j - 1], sh->mass[j - 1])))
      sh->bin = j;
  __syncthreads();
  const int bin = sh->bin;
  unsigned long long mass_before = bin ? sh->mass[bin - 1] : 0;
  uint32_t count_before = bin ? sh->count[bin - 1] : 0;
  uint32_t members = sh->count[bin] - count_before;
  // Among the tokens of a crowded bin the position is narrowed by the digits of (logit, number), 11 bits at a time
  uint64_t prefix = 0;
  int shift = 64;
  auto member = [&](int token, float l, float y) {
    const uint64_t key = (uint64_t)falling_key(l) << 32 | (uint32_t)token;
    return y > -23.0f && Row::bin(y) == bin && (shift == 64 || (key >> shift) == prefix);
  };
  while (members > kListed) {
    for (int j = i; j < kBins; j += kPickThreads) sh->digit_mass[j] = 0, sh->digit_count[j] = 0;
    __syncthreads();
    const int next = max(shift - 11, 0);
    for_each_logit<T, kPickThreads>(row.logits, 0, a.vocab, [&](int token, float l) {
      const float y = row.y(l);
      if (!member(token, l, y)) return;
      const uint32_t w = Row::weight(y);
      if (!w) return;
      const uint64_t key = (uint64_t)falling_key(l) << 32 | (uint32_t)token;
      const int digit = (int)((key >> next) & ((1ull << (shift - next)) - 1));
      atomicAdd(&sh->digit_mass[digit], (unsigned long long)w);
      atomicAdd(&sh->digit_count[digit], 1u);
    });
    __syncthreads();
    prefix_sums(sh->digit_mass, sh->digit_count, sh);
#pragma unroll
    for (int j = 2 * i; j <= 2 * i + 1; ++j)
      if (sought.reached(count_before + sh->digit_count[j], mass_before + sh->digit_mass[j]) &&
          (j == 0 || !sought.reached(count_before + sh->digit_count[j - 1], mass_before + sh->digit_mass[j - 1])))
        sh->digit = j;
    __syncthreads();
    const int digit = sh->digit;
    members = sh->digit_count[digit] - (digit ? sh->digit_count[digit - 1] : 0);
    mass_before += digit ? sh->digit_mass[digit - 1] : 0;
    count_before += digit ? sh->digit_count[digit - 1] : 0;
    prefix = (shift == 64 ? 0 : prefix << (shift - next)) | (uint32_t)digit;
    shift = next;
    __syncthreads();
  }
  if (i == 0) sh->listed = 0;
  __syncthreads();
  for_each_logit<T, kPickThreads>(row.logits, 0, a.vocab, [&](int token, float l) {
    const float y = row.y(l);
    if (!member(token, l, y)) return;
    const uint32_t w = Row::weight(y);
    if (!w) return;
    const int at = atomicAdd(&sh->listed, 1);
    if (at < kListed) {
      sh->list_key[at] = (uint64_t)falling_key(l) << 32 | (uint32_t)token;
      sh->list_mass[at] = w;
    }
  });
  __syncthreads();
  const int listed = min(sh->listed, kListed);
  for (int j = i; j < listed; j += kPickThreads) {
    const uint64_t key = sh->list_key[j];
    unsigned long long before = mass_before;
    uint32_t rank = count_before;
    for (int x = 0; x < listed; ++x)
      if (sh->list_key[x] < key) before += sh->list_mass[x], ++rank;
    const unsigned long long through = before + sh->list_mass[j];
    if (sought.reached(rank + 1, through) && !((rank > 0) && sought.reached(rank, before))) {
      const uint32_t f = (uint32_t)(key >> 32), u = f & 0x80000000u ? f : ~f & 0x7FFFFFFFu;
      sh->found = Place{before, through, (int)(uint32_t)key, row.y(__uint_as_float(u))};
    }
  }
  __syncthreads();
  const Place p = sh->found;
  __syncthreads();
  return p;
}

// One workgroup per row: the kept weight, then the token.
template <int T>
__global__ __launch_bounds__(kPickThreads) void sample_pick_kernel(SampleArgs a) {
  extern __shared__ __align__(16) uint8_t lds[];
  PickShared* const sh = reinterpret_cast<PickShared*>(lds);
  const int r = blockIdx.x, i = threadIdx.x;
  const Row row = make_row<T>(a, r);
  if (row.m == -INFINITY) {
    if (i == 0) {
      a.tokens[r] = -1;
      if (a.logprobs) a.logprobs[r] = -INFINITY;
    }
    return;
  }
  for (int j = i; j < kBins; j += kPickThreads) {
    sh->mass[j] = a.mass[(int64_t)r * kBins + j];
    sh->count[j] = a.count[(int64_t)r * kBins + j];
  }
  if (i == 0) sh->min_mass = 0, sh->bin = sh->digit = 0, sh->found = Place{0, 0, 0, 0.0f};
  __syncthreads();
  prefix_sums(sh->mass, sh->count, sh);
  const unsigned long long total = sh->mass[kBins - 1];
  const uint32_t counted = sh->count[kBins - 1];  // tokens whose weight is not 0
  const bool greedy = a.temperature && a.temperature[r] <= 0.0f;
  const int top_k = greedy ? 1 : a.top_k ? a.top_k[r] : 0;
  const float top_p = a.top_p ? a.top_p[r] : 1.0f, min_p = a.min_p ? a.min_p[r] : 0.0f;
  unsigned long long kept = total;
  if (top_k > 0 && (uint32_t)top_k < counted)
    kept = place_of<T>(a, row, Sought{Sought::kCount, (uint32_t)top_k, 0.0, 0}, sh).through;
  const unsigned long long of_top_k = kept;
  if (top_p < 1.0f)
    kept = min(kept, place_of<T>(a, row, Sought{Sought::kAtLeast, 0, (double)top_p * (double)of_top_k, 0}, sh).through);
  if (min_p > 0.0f) {
    const float floor = logf(fminf(min_p, 1.0f));
    unsigned long long mine = 0;
    for_each_logit<T, kPickThreads>(row.logits, 0, a.vocab, [&](int, float l) {
      const float y = row.y(l);
      if (y >= floor && y > -23.0f) mine += Row::weight(y);
    });
#pragma unroll
    for (int s = 1; s < 64; s *= 2) mine += __shfl_xor(mine, s);
    if ((i & 63) == 0) atomicAdd(&sh->min_mass, mine);
    __syncthreads();
    kept = min(kept, sh->min_mass);
  }
  const unsigned long long passed = (unsigned long long)((double)a.uniform[r] * (double)kept);
  const Place p = place_of<T>(a, row, Sought{Sought::kAbove, 0, 0.0, min(passed, kept - 1)}, sh);
  if (i == 0) {
    a.tokens[r] = p.token;
    // (the most probable token weighs 2^31)
    if (a.logprobs) a.logprobs[r] = p.y - log1pf((float)(total - (1ull << 31)) * 4.65661287307739e-10f);
  }
}

int slices_of(int32_t rows, int32_t vocab) {
  // slices of 4096 tokens or more, two thousand workgroups at most; 2^15 tokens at most
  int64_t s = vocab / 4096;
  if (s * rows > 2048) s = 2048 / rows;
  const int64_t least = ((int64_t)vocab + kMostSlice - 1) / kMostSlice;
  if (s < least) s = least;
  return (int)s;
}

struct SampleWorkspace {
  int64_t max_at, mass_at, count_at, bytes;
};
SampleWorkspace sample_workspace(int32_t rows, int32_t vocab) {
  SampleWorkspace w;
  w.mass_at = 0;
  w.count_at = round_up_256((int64_t)rows * kBins * 8);
  w.max_at = w.count_at + round_up_256((int64_t)rows * kBins * 4);
  w.bytes = w.max_at + round_up_256((int64_t)rows * slices_of(rows ? rows : 1, vocab) * 4);
  if (w.bytes < 256) w.bytes = 256;
  return w;
}

template <int T>
int launch_sample(const SampleArgs& a, hipStream_t stream) {
  const dim3 grid(a.slices, a.rows);
  sample_max_kernel<T><<<grid, kSliceThreads, 0, stream>>>(a);
  sample_bins_kernel<T><<<grid, kSliceThreads, 0, stream>>>(a);
  const void* const pick = (const void*)sample_pick_kernel<T>;
  if (int e = allow_full_lds(pick, "sample_pick_kernel")) return e;
  sample_pick_kernel<T><<<a.rows, kPickThreads, sizeof(PickShared), stream>>>(a);
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return SFMP_OK;
  note_hip_error("sfmp_sample", hipGetErrorString(e));
  return SFMP_ERR_HIP;
}

}  // namespace
}  // namespace sfmp

using namespace sfmp;

extern "C" int sfmp_sample_workspace(int32_t rows, int32_t vocab, int64_t* bytes) {
  if (!bytes) return SFMP_ERR_NULL;
  if (rows < 0 || rows > 65535 || vocab < 1 || vocab > (1 << 24)) return SFMP_ERR_SHAPE;
  *bytes = sample_workspace(rows, vocab).bytes;
  return SFMP_OK;
}

extern "C" int sfmp_sample(const void* logits_dev, int32_t dtype, int32_t rows, int32_t vocab, int64_t stride,
                           const float* temperature_dev, const int32_t* top_k_dev, const float* top_p_dev,
                           const float* min_p_dev, const float* uniform_dev, int32_t* tokens_dev, float* logprobs_dev,
                           void* workspace_dev, int64_t workspace_bytes, void* hip_stream) {
  int64_t need = 0;
  if (int e = sfmp_sample_workspace(rows, vocab, &need)) return e;
  if (dtype != SFMP_TYPE_FP16 && dtype != SFMP_TYPE_BF16 && dtype != SFMP_TYPE_FP32) return SFMP_ERR_LAYOUT;
  if (stride < vocab || stride > INT64_MAX / 8 / 65536) return SFMP_ERR_SHAPE;
  if (rows == 0) return SFMP_OK;
  if (!logits_dev || !uniform_dev || !tokens_dev) return SFMP_ERR_NULL;
  auto off = [](const void* p, uintptr_t a) { return reinterpret_cast<uintptr_t>(p) % a != 0; };
  if (off(logits_dev, dtype == SFMP_TYPE_FP32 ? 4 : 2) || off(temperature_dev, 4) || off(top_k_dev, 4) || off(top_p_dev, 4) ||
      off(min_p_dev, 4) || off(uniform_dev, 4) || off(tokens_dev, 4) || off(logprobs_dev, 4))
    return SFMP_ERR_ALIGN;
  if (!workspace_dev || off(workspace_dev, 256) || workspace_bytes < need) return SFMP_ERR_WORKSPACE;
  const SampleWorkspace w = sample_workspace(rows, vocab);
  uint8_t* const at = (uint8_t*)workspace_dev;
  const SampleArgs a{logits_dev, rows, vocab, slices_of(rows, vocab), stride, temperature_dev, top_k_dev, top_p_dev, min_p_dev,
                     uniform_dev, tokens_dev, logprobs_dev, (float*)(at + w.max_at),
                     (unsigned long long*)(at + w.mass_at), (uint32_t*)(at + w.count_at)};
  const hipStream_t stream = (hipStream_t)hip_stream;
  if (dtype == SFMP_TYPE_FP16) return launch_sample<SFMP_TYPE_FP16>(a, stream);
  if (dtype == SFMP_TYPE_BF16) return launch_sample<SFMP_TYPE_BF16>(a, stream);
  return launch_sample<SFMP_TYPE_FP32>(a, stream);
}
