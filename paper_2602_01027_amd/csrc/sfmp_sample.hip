// Choice of the next token: temperature, top-k, top-p, min-p and one random number per row.
//
// Every filter keeps a prefix of the tokens ordered by (falling logit, rising number), and the token is where the running
// sum of weights passes a threshold.  So no sort of the row is needed, only a few positions in that order: a histogram of
// counts and weights over 4096 bins of (l - m) / T tells which bins the positions lie in, and the tokens of those bins, a few
// hundred of a hundred thousand, are collected and sorted in LDS, the gaps between the bins being known from the histogram.
// Weights are whole numbers (2^31 for the most probable token), so that their sums do not depend on the order in which
// workgroups and atomics add them.
//
// Few rows are cut into slices over many workgroups, which takes three launches (largest logit; histogram; collection) and
// a fourth for the choice.  Many rows have one workgroup each, which does all of it.
#include <float.h>
#include <math.h>

#include "sfmp_device.h"
#include "sfmp_internal.h"

namespace sfmp {
namespace {

constexpr int kBins = 4096;
constexpr float kBinsPerUnit = 184.0f;  // weights are 0 below (l - m) / T = -32 ln 2 = -22.2
constexpr float kLeast = -23.0f;
constexpr int kSliceThreads = 256;
constexpr int kPickThreads = 1024;
constexpr int kListed = 2048;           // most tokens that are sorted

struct Wanted;
struct Listed {
  uint64_t entry;                  // (key, token)
  unsigned long long mass_before;  // sums before its bin
  uint32_t count_before, none;
};

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
  Listed* list;             // [rows][kListed]
  Wanted* wanted;           // [rows]
  uint32_t* listed;         // [rows]
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
  return x;
}

typedef __attribute__((address_space(1))) u32x4 GlobalRun;

// Calls f(number, logit) for the tokens [from, to) of a row; the threads take runs of 16 aligned bytes in turn.
template <int T, int THREADS, int AHEAD = 4, typename F>
__device__ __forceinline__ void for_each_logit(const void* row, int from, int to, F f) {
  constexpr int SIZE = T == SFMP_TYPE_FP32 ? 4 : 2, RUN = 16 / SIZE;
  const int lead = (int)((reinterpret_cast<uintptr_t>(row) & 15) / SIZE);  // elements between the aligned address and the row
  const uint8_t* const base = (const uint8_t*)row - lead * SIZE;
  const int first = (from + lead + RUN - 1) / RUN, last = max((to + lead) / RUN, first);  // whole runs
  const GlobalRun* const runs = (const GlobalRun*)reinterpret_cast<uintptr_t>(base);
  // AHEAD runs at a time, as many more requested before
  u32x4 now[AHEAD], next[AHEAD];
  auto request = [&](u32x4 (&w)[AHEAD], int v) {
#pragma unroll
    for (int k = 0; k < AHEAD; ++k)
      if (v + k * THREADS < last) w[k] = runs[v + k * THREADS];
  };
  int v = first + threadIdx.x;
  request(now, v);
  for (; v < last; v += AHEAD * THREADS) {
    request(next, v + AHEAD * THREADS);
    int at = v;
    asm volatile("" : "+v"(at));  // (the numbers are made where they are used, not kept as RUN * AHEAD counters)
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      if (v + k * THREADS < last) {
#pragma unroll
        for (int j = 0; j < RUN; ++j) {
          const u32x4 w = now[k];
          f((at + k * THREADS) * RUN - lead + j, logit_of<T>(SIZE == 4 ? w[j] : (j & 1) ? w[j / 2] >> 16 : w[j / 2] & 0xFFFFu));
        }
      }
      now[k] = next[k];
    }
  }
  // before the first and behind the last
  const int head = min(first * RUN - lead, to), tail = max(last * RUN - lead, head);
  for (int side = 0; side < 2; ++side) {
    const int i = (side ? tail : from) + threadIdx.x;
    if (i < (side ? to : head)) f(i, logit_of<T>(SIZE == 4 ? ((const uint32_t*)row)[i] : ((const uint16_t*)row)[i]));
  }
}

__device__ __forceinline__ float max_of_wave(float x) {
#pragma unroll
  for (int s = 1; s < 64; s *= 2) x = fmaxf(x, __shfl_xor(x, s));
  return x;
}

// What a row is asked for.  Where an array is not given, another address is read in its place: without branches all five loads are
// under way together, from the kernel's start.
struct Asked {
  float temperature, top_p, min_p, uniform;
  int32_t top_k;
};
__device__ __forceinline__ Asked asked_of(const SampleArgs& a, int r) {
  const float* const any = a.uniform + r;
  const float t = *(a.temperature ? a.temperature + r : any), p = *(a.top_p ? a.top_p + r : any), q = *(a.min_p ? a.min_p + r : any);
  const int32_t k = *(a.top_k ? a.top_k + r : reinterpret_cast<const int32_t*>(any));
  return Asked{a.temperature ? t : 1.0f, a.top_p ? p : 1.0f, a.min_p ? q : 0.0f, *any, a.top_k ? k : 0};
}

// What the weights of a row are computed from.
struct Row {
  const void* logits;
  float m, inverse;
  bool plain;  // m and 1 / T are finite
  __device__ __forceinline__ Row(const void* p, float largest, float t) : logits(p) {
    // (the same for all lanes, which the compiler has to be told)
    m = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(largest)));
    inverse = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(1.0f / fmaxf(t, 0.0f))));
    plain = __builtin_amdgcn_readfirstlane(inverse < INFINITY && fabsf(m) < INFINITY);
  }
  // (l - m) / T; not above kLeast for a NaN
  template <bool PLAIN = false>
  __device__ __forceinline__ float y(float l) const {
    if (PLAIN) return (l - m) * inverse;
    return l == m ? 0.0f : l == -INFINITY ? -INFINITY : (l - m) * inverse;
  }
  static __device__ __forceinline__ uint32_t weight(float y) { return (uint32_t)rintf(expf(y) * 2147483648.0f); }
  static __device__ __forceinline__ int bin(float y) { return min((int)(-y * kBinsPerUnit), kBins - 1); }
};

template <int T>
__device__ __forceinline__ Row make_row(const SampleArgs& a, int r, float t) {
  const int lane = threadIdx.x & 63;
  float m = -INFINITY;
  for (int s = lane; s < a.slices; s += 64) m = fmaxf(m, a.slice_max[(int64_t)r * a.slices + s]);
  return Row((const uint8_t*)a.logits + r * a.stride * (T == SFMP_TYPE_FP32 ? 4 : 2), max_of_wave(m), t);
}

// (Numbers in the order that logits have, falling: a smaller key is a more probable token.)
__device__ __forceinline__ uint32_t falling_key(float l) {
  const uint32_t u = __float_as_uint(l == 0.0f ? 0.0f : l);
  return u & 0x80000000u ? u : ~u & 0x7FFFFFFFu;
}

__device__ __forceinline__ int slice_from(const SampleArgs& a, int s) { return (int)((int64_t)a.vocab * s / a.slices); }

// Largest logit of every slice; clears the histograms.  One row of 131072 fp16 tokens, 32 slices: 3.3 us, this and the next three bound by
// latency (a launch, a few dependent loads, a few barriers each; the logits are 0.26 MB).
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
  if (s == 0 && threadIdx.x == 0) a.listed[r] = 0;
  m = max_of_wave(m);
  if ((threadIdx.x & 63) == 0) of_wave[threadIdx.x >> 6] = m;
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int i = 1; i < kSliceThreads / 64; ++i) m = fmaxf(m, of_wave[i]);
    a.slice_max[(int64_t)r * a.slices + s] = m;
  }
}

// Adds a slice to the histogram of its row.  A bin of a slice is one 64-bit word in LDS: its count from bit 47 on, its
// weight below.  All of a slice may lie in one bin, with the largest weight each: 2^15 tokens of 2^31.  The same row: 6.3 us.
constexpr int kCountBit = 47;
constexpr int kMostSlice = 1 << 15;
static_assert((uint64_t)kMostSlice << 31 < 1ull << kCountBit && kMostSlice < 1 << (64 - kCountBit), "weight and count of a whole slice in one bin");
template <int T>
__global__ __launch_bounds__(kSliceThreads) void sample_bins_kernel(SampleArgs a) {
  __shared__ unsigned long long bins[kBins];
  const int s = blockIdx.x, r = blockIdx.y;
  for (int i = threadIdx.x; i < kBins; i += kSliceThreads) bins[i] = 0;
  const Row row = make_row<T>(a, r, a.temperature ? a.temperature[r] : 1.0f);
  __syncthreads();
  if (row.m == -INFINITY) return;
  auto add = [&](float y) {
    if (!(y > kLeast)) return;
    const uint32_t w = Row::weight(y);
    if (w) atomicAdd(&bins[Row::bin(y)], (1ull << kCountBit) + w);
  };
  const int from = slice_from(a, s), to = slice_from(a, s + 1);
  if (row.plain)
    for_each_logit<T, kSliceThreads>(row.logits, from, to, [&](int, float l) { add(row.template y<true>(l)); });
  else
    for_each_logit<T, kSliceThreads>(row.logits, from, to, [&](int, float l) { add(row.y(l)); });
  __syncthreads();
  for (int i = threadIdx.x; i < kBins; i += kSliceThreads)
    if (const unsigned long long x = bins[i]) {
      atomicAdd(&a.mass[(int64_t)r * kBins + i], x & ((1ull << kCountBit) - 1));
      atomicAdd(&a.count[(int64_t)r * kBins + i], (uint32_t)(x >> kCountBit));
    }
}

// What a workgroup that chooses, or collects for the choice, shares.
struct Mark {
  unsigned long long before, through;  // sums before a bin, and with it
  int bin;
};
struct PickShared {
  unsigned long long mass[kBins];      // of a row kernel: the histogram; then, for the wanted bins, what `base` says
  uint32_t count[kBins];
  uint64_t list[kListed];              // entries (key, token)
  unsigned long long wave_mass[kPickThreads / 64];
  uint32_t wave_count[kPickThreads / 64];
  Mark mark[6];
  unsigned long long through, min_mass, total;
  uint64_t found;
  float wave_max[kPickThreads / 64];
  uint32_t listed, counted;
};

// Sum over the threads before this one, and over all.
template <int THREADS>
__device__ __forceinline__ unsigned long long sum_before(unsigned long long x, PickShared* sh, unsigned long long* all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  unsigned long long up = x;
#pragma unroll
  for (int s = 1; s < 64; s *= 2) {
    const unsigned long long y = __shfl_up(up, s);
    if (lane >= s) up += y;
  }
  if (lane == 63) sh->wave_mass[wave] = up;
  __syncthreads();
  unsigned long long ahead = 0, sum = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) {
    const unsigned long long y = sh->wave_mass[w];
    if (w < wave) ahead += y;
    sum += y;
  }
  __syncthreads();
  *all = sum;
  return ahead + up - x;
}

// The filters of a row, and the bins that the end of each and the chosen token can lie in.
struct Wanted {
  int top_k;  // 0: all
  float top_p, floor, uniform;
  bool by_top_p, by_min_p;
  unsigned long long total, min_before;  // (before the bin of min-p's floor)
  int from[4];          // ranges of bins
  uint32_t span[4];     // bins of a range behind its first
  uint32_t tokens;      // in them
  __device__ __forceinline__ void range(int x, int first, int last) {
    from[x] = __builtin_amdgcn_readfirstlane(first);
    span[x] = __builtin_amdgcn_readfirstlane(last - first);
  }
  __device__ __forceinline__ bool has(int bin) const {
    bool y = false;
#pragma unroll
    for (int x = 0; x < 4; ++x) y |= (uint32_t)(bin - from[x]) <= span[x];
    return y;
  }
};
__device__ __forceinline__ Wanted filters_of(const Asked& x, uint32_t counted, unsigned long long total) {
  Wanted w;
  w.total = total;
  w.min_before = 0;
  w.uniform = x.uniform;
  w.top_k = x.temperature <= 0.0f ? 1 : x.top_k;
  if (w.top_k <= 0 || (uint32_t)w.top_k >= counted) w.top_k = 0;  // (counted: tokens whose weight is not 0)
  w.top_p = x.top_p;
  w.by_top_p = w.top_p < 1.0f;
  const float min_p = x.min_p;
  w.by_min_p = min_p > 0.0f;
  w.floor = w.by_min_p ? logf(fminf(min_p, 1.0f)) : -INFINITY;
  return w;
}

// The histogram in registers: every thread holds the bins EACH t .. EACH t + EACH - 1.
template <int THREADS>
struct Bins {
  static constexpr int EACH = kBins / THREADS;
  unsigned long long mass_before, mass[EACH];  // sums before the thread's bins, and with each
  uint32_t count_before, count[EACH];

  // mass and count hold the bins' own on entry
  __device__ __forceinline__ void add_up(PickShared* sh) {
    // (counts and weights of the threads in one go: a count below 2^24 under weights below 2^55 would not fit 64 bits)
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    unsigned long long m = 0;
    uint32_t c = 0;
#pragma unroll
    for (int j = 0; j < EACH; ++j) mass[j] = m += mass[j], count[j] = c += count[j];
    unsigned long long um = m;
    uint32_t uc = c;
#pragma unroll
    for (int s = 1; s < 64; s *= 2) {
      const unsigned long long y = __shfl_up(um, s);
      const uint32_t z = __shfl_up(uc, s);
      if (lane >= s) um += y, uc += z;
    }
    if (lane == 63) sh->wave_mass[wave] = um, sh->wave_count[wave] = uc;
    __syncthreads();
    mass_before = um - m, count_before = uc - c;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w)
      if (w < wave) mass_before += sh->wave_mass[w], count_before += sh->wave_count[w];
#pragma unroll
    for (int j = 0; j < EACH; ++j) mass[j] += mass_before, count[j] += count_before;
    if (threadIdx.x == THREADS - 1) sh->total = mass[EACH - 1], sh->counted = count[EACH - 1];
    __syncthreads();
  }
  // Marks the first bin whose running sums satisfy `reached`
  template <typename F>
  __device__ __forceinline__ void mark_first(F reached, Mark* mark) const {
    if (!reached(count[EACH - 1], mass[EACH - 1]) || (threadIdx.x > 0 && reached(count_before, mass_before))) return;
    bool done = false;
#pragma unroll
    for (int j = 0; j < EACH; ++j)
      if (!done && reached(count[j], mass[j])) {
        *mark = Mark{j ? mass[j - 1] : mass_before, mass[j], EACH * (int)threadIdx.x + j};
        done = true;
      }
  }
  __device__ __forceinline__ void mark_bin(int bin, Mark* mark) const {
#pragma unroll
    for (int j = 0; j < EACH; ++j)
      if (EACH * (int)threadIdx.x + j == bin) *mark = Mark{j ? mass[j - 1] : mass_before, mass[j], bin};
  }
};

// Which bins are wanted.  A position inside a bin leaves the weight kept by top-k uncertain by that bin, which may make two
// bins of one for the filters after it.  Leaves the sums before the wanted bins in sh->mass and sh->count.
template <int THREADS>
__device__ __forceinline__ Wanted find_wanted(const Asked& asked, const Bins<THREADS>& bins, PickShared* sh) {
  Wanted w = filters_of(asked, sh->counted, sh->total);
#pragma unroll
  for (int x = 0; x < 4; ++x) w.from[x] = 1 << 30, w.span[x] = 0;  // (none)
  const float u = w.uniform;
  unsigned long long least = w.total, most = w.total;  // both ends of the kept weight
  if (threadIdx.x == 0) sh->listed = 0;
  const int min_bin = w.floor > kLeast ? Row::bin(w.floor) : kBins - 1;
  if (w.by_min_p) bins.mark_bin(min_bin, &sh->mark[5]);
  if (w.top_k) {
    const uint32_t k = (uint32_t)w.top_k;
    bins.mark_first([&](uint32_t c, unsigned long long) { return c >= k; }, &sh->mark[0]);
    __syncthreads();
    const Mark x = sh->mark[0];
    w.range(0, x.bin, x.bin);
    least = x.before + 1, most = x.through;
  }
  if (w.by_top_p) {
    const double low = (double)w.top_p * (double)least, high = (double)w.top_p * (double)most;
    bins.mark_first([&](uint32_t, unsigned long long m) { return (double)m >= low; }, &sh->mark[1]);
    bins.mark_first([&](uint32_t, unsigned long long m) { return (double)m >= high; }, &sh->mark[2]);
    __syncthreads();
    const Mark x = sh->mark[1], y = sh->mark[2];
    w.range(1, x.bin, y.bin);
    least = min(least, x.before + 1), most = min(most, y.through);
  }
  if (w.by_min_p) {
    __syncthreads();
    const Mark x = sh->mark[5];
    w.range(2, min_bin, min_bin);
    w.min_before = x.before;
    least = min(least, max(x.before, 1ull)), most = min(most, x.through);
  }
  const unsigned long long low = min((unsigned long long)((double)u * (double)least), least - 1);
  const unsigned long long high = min((unsigned long long)((double)u * (double)most), most - 1);
  bins.mark_first([&](uint32_t, unsigned long long m) { return m > low; }, &sh->mark[3]);
  bins.mark_first([&](uint32_t, unsigned long long m) { return m > high; }, &sh->mark[4]);
  __syncthreads();
  w.range(3, sh->mark[3].bin, sh->mark[4].bin);
  uint32_t tokens = 0;
#pragma unroll
  for (int j = 0; j < Bins<THREADS>::EACH; ++j) {
    const int bin = Bins<THREADS>::EACH * threadIdx.x + j;
    if (w.has(bin)) {
      const uint32_t before = j ? bins.count[j - 1] : bins.count_before;
      tokens += bins.count[j] - before;
      sh->mass[bin] = j ? bins.mass[j - 1] : bins.mass_before;
      sh->count[bin] = before;
    }
  }
  if (tokens) atomicAdd(&sh->listed, tokens);
  __syncthreads();
  w.tokens = __builtin_amdgcn_readfirstlane(sh->listed);
  return w;
}

// The wanted bins as intervals of logits, with a margin for rounding: most tokens are told apart without their bin.  Where a bin's
// width in logits is no normal number (a temperature of infinity, or near the least one) or an interval passes the range of fp32, the
// bin alone decides.
struct Reach {
  float middle[4], half[4];
  __device__ __forceinline__ Reach(const Row& row, const Wanted& w) {
    const float unit = 1.0f / (kBinsPerUnit * row.inverse), margin = fabsf(row.m) * 2e-6f;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const bool none = w.from[x] >= kBins;
      const float high = row.m - (float)(w.from[x] - 1) * unit, low = row.m - (float)(w.from[x] + (int)w.span[x] + 2) * unit;
      float c = 0.5f * (high + low), h = 0.5001f * (high - low) + margin + fabsf(c) * 1e-6f;
      if (!row.plain || !(unit >= FLT_MIN && fabsf(c) < INFINITY && h < INFINITY)) c = 0.0f, h = INFINITY;
      if (none) h = -1.0f;
      middle[x] = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(c)));
      half[x] = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(h)));
    }
  }
  __device__ __forceinline__ bool may_hold(float l) const {
    bool y = false;
#pragma unroll
    for (int x = 0; x < 4; ++x) y |= fabsf(l - middle[x]) <= half[x];
    return y;
  }
};
__device__ __forceinline__ bool is_wanted(const Row& row, float l, const Reach& reach, const Wanted& w) {
  if (!reach.may_hold(l)) return false;
  const float y = row.y(l);
  return y > kLeast && w.has(Row::bin(y)) && Row::weight(y);
}
__device__ __forceinline__ uint64_t entry_of(int token, float l) { return (uint64_t)falling_key(l) << 32 | (uint32_t)token; }
__device__ __forceinline__ float logit_of_entry(uint64_t e) {
  const uint32_t f = (uint32_t)(e >> 32);
  return __uint_as_float(f & 0x80000000u ? f : ~f & 0x7FFFFFFFu);
}

// Sorts list[0, n) upwards, n a power of two from 64 to kListed, all entries different (but for the ~0 behind the last).
template <int THREADS>
__device__ __forceinline__ void sort_list(uint64_t* list, int n) {
  if (n <= 256) {
    // by rank: THREADS / n threads count the smaller ones of an entry
    const int shift = __builtin_ctz(THREADS) - __builtin_ctz(n), parts = 1 << shift;
    const int e = threadIdx.x >> shift, q = threadIdx.x & (parts - 1);
    const uint64_t x = list[e];
    int rank = 0;
#pragma unroll 4
    for (int j = q; j < n; j += parts) rank += list[j] < x || (j < e && list[j] == x);
    for (int s = 1; s < parts; s *= 2) rank += __shfl_xor(rank, s);
    __syncthreads();
    if (q == 0) list[rank] = x;
    __syncthreads();
    return;
  }
  // With strides up to 64 the elements of a wavefront's threads lie within 128 of its own: no barrier of the workgroup is needed
  // between those steps.
  for (int size = 2; size <= n; size *= 2)
    for (int stride = size / 2; stride > 0; stride /= 2) {
      for (int t = threadIdx.x; t < n / 2; t += THREADS) {
        const int i = 2 * t - (t & (stride - 1)), j = i + stride;
        const uint64_t x = list[i], y = list[j];
        if ((x > y) == ((i & size) == 0)) list[i] = y, list[j] = x;
      }
      if (stride > 64 || (stride == 1 && size >= 128))
        __syncthreads();
      else
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

// The choice, from the list of the tokens in the wanted bins (the first n of sh->list), the sums before these bins
// being in sh->mass and sh->count.
template <int THREADS>
__device__ __forceinline__ void choose_from_list(const Row& row, const Wanted& w, int n, PickShared* sh) {
  constexpr int EACH = kListed / THREADS;
  const int i = threadIdx.x;
  int size = 64;
  while (size < n) size *= 2;
  for (int j = n + i; j < size; j += THREADS) sh->list[j] = ~0ull;
  const int min_bin = w.from[2];
  if (i == 0) sh->min_mass = w.min_before, sh->found = 0;
  __syncthreads();
  sort_list<THREADS>(sh->list, size);
  // Thread i holds the entries EACH i ...: running sums over the list first
  float y[EACH];
  unsigned long long through[EACH];
  uint32_t weight[EACH];
  int bin[EACH];
  unsigned long long sum = 0;
#pragma unroll
  for (int x = 0; x < EACH; ++x) {
    const int j = EACH * i + x;
    weight[x] = 0, bin[x] = 0, y[x] = 0.0f;
    if (j < n) {
      y[x] = row.y(logit_of_entry(sh->list[j]));
      bin[x] = Row::bin(y[x]);
      weight[x] = Row::weight(y[x]);
    }
    sum += weight[x];
    through[x] = sum;
  }
  unsigned long long all;
  const unsigned long long before = sum_before<THREADS>(sum, sh, &all);
#pragma unroll
  for (int x = 0; x < EACH; ++x) through[x] += before;
  // ... then the first entry of each bin sets off its running sums against those of the row
#pragma unroll
  for (int x = 0; x < EACH; ++x) {
    const int j = EACH * i + x;
    if (j < n && (j == 0 || Row::bin(row.y(logit_of_entry(sh->list[j - 1]))) != bin[x])) {
      sh->mass[bin[x]] -= through[x] - weight[x];
      sh->count[bin[x]] -= (uint32_t)j;
    }
  }
  __syncthreads();
#pragma unroll
  for (int x = 0; x < EACH; ++x)
    if (weight[x]) through[x] += sh->mass[bin[x]];
  unsigned long long kept = w.total;
  if (w.top_k) {
#pragma unroll
    for (int x = 0; x < EACH; ++x)
      if (weight[x] && sh->count[bin[x]] + (uint32_t)(EACH * i + x + 1) == (uint32_t)w.top_k) sh->through = through[x];
    __syncthreads();
    kept = sh->through;
    __syncthreads();
  }
  if (w.by_top_p) {
    const double aim = (double)w.top_p * (double)kept;
#pragma unroll
    for (int x = 0; x < EACH; ++x) {
      const unsigned long long less = through[x] - weight[x];
      if (weight[x] && (double)through[x] >= aim && (less == 0 || (double)less < aim)) sh->through = through[x];
    }
    __syncthreads();
    kept = min(kept, sh->through);
    __syncthreads();
  }
  if (w.by_min_p) {
#pragma unroll
    for (int x = 0; x < EACH; ++x)
      if (weight[x] && bin[x] == min_bin && y[x] >= w.floor) atomicMax(&sh->min_mass, through[x]);
    __syncthreads();
    kept = min(kept, sh->min_mass);
  }
  const unsigned long long passed = min((unsigned long long)((double)w.uniform * (double)kept), kept - 1);
#pragma unroll
  for (int x = 0; x < EACH; ++x)
    if (weight[x] && through[x] > passed && through[x] - weight[x] <= passed) sh->found = sh->list[EACH * i + x];
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

// Finds the token at a position where the wanted bins are too crowded to be sorted (rows of nearly equal logits): its bin is
// narrowed by the digits of (logit, token), 12 bits at a time, until one token is left, each time over the whole row.
// Leaves the token's entry in sh->found, returns the running sum with it.  kPickThreads threads; sh->mass and sh->count
// are used for the digits.
template <int T>
__device__ __forceinline__ unsigned long long place_of(const SampleArgs& a, const Row& row, const Sought& sought, PickShared* sh) {
  constexpr int kDigitBits = 12;
  static_assert(kBins == 1 << kDigitBits, "digits are counted like bins");
  const int i = threadIdx.x;
  unsigned long long mass_before = 0;
  uint32_t count_before = 0;
  uint64_t prefix = 0;
  int bin = -1;
  for (int shift = 64 + kDigitBits; shift > 0;) {  // first the bins themselves, then the digits of one
    for (int j = i; j < kBins; j += kPickThreads) sh->mass[j] = 0, sh->count[j] = 0;
    __syncthreads();
    const int next = max(shift - kDigitBits, 0);
    for_each_logit<T, kPickThreads, 1>(row.logits, 0, a.vocab, [&](int token, float l) {
      const float y = row.y(l);
      if (!(y > kLeast)) return;
      const uint32_t w = Row::weight(y);
      if (!w) return;
      int digit = Row::bin(y);
      if (shift <= 64) {
        const uint64_t key = entry_of(token, l);
        if (digit != bin || (shift < 64 && (key >> shift) != prefix)) return;
        digit = (int)((key >> next) & ((1ull << (shift - next)) - 1));
      }
      atomicAdd(&sh->mass[digit], (unsigned long long)w);
      atomicAdd(&sh->count[digit], 1u);
    });
    __syncthreads();
    Bins<kPickThreads> sums;
#pragma unroll
    for (int j = 0; j < Bins<kPickThreads>::EACH; ++j) {
      sums.mass[j] = sh->mass[Bins<kPickThreads>::EACH * i + j];
      sums.count[j] = sh->count[Bins<kPickThreads>::EACH * i + j];
    }
    sums.add_up(sh);
    sums.mark_first([&](uint32_t c, unsigned long long m) { return sought.reached(count_before + c, mass_before + m); }, &sh->mark[0]);
    __syncthreads();
    const Mark x = sh->mark[0];
    if (x.bin / Bins<kPickThreads>::EACH == i) {
      uint32_t c = 0;
#pragma unroll
      for (int j = 0; j < Bins<kPickThreads>::EACH; ++j)
        if (x.bin % Bins<kPickThreads>::EACH == j) c = j ? sums.count[j - 1] : sums.count_before;
      sh->listed = c;
    }
    __syncthreads();
    mass_before += x.before;
    count_before += sh->listed;
    if (shift > 64)
      bin = x.bin;
    else
      prefix = (shift == 64 ? 0 : prefix << (shift - next)) | (uint32_t)x.bin;
    shift = next;
    __syncthreads();
  }
  if (i == 0) sh->found = prefix;
  __syncthreads();
  return mass_before + Row::weight(row.y(logit_of_entry(prefix)));
}

// (One place where the search stands in the code, and no call: a call's stack costs every launch of the kernel 7 us, whether a row is
// crowded or not.)
template <int T>
__device__ __forceinline__ void choose_crowded(const SampleArgs& a, const Row& row, const Wanted& w, PickShared* sh) {
  unsigned long long kept = w.total;
#pragma clang loop unroll(disable)
  for (int filter = 0; filter < 4; ++filter) {
    Sought sought{Sought::kCount, (uint32_t)w.top_k, 0.0, 0};
    if (filter == 0) {
      if (!w.top_k) continue;
    } else if (filter == 1) {
      if (!w.by_top_p) continue;
      sought.by = Sought::kAtLeast;
      sought.aim = (double)w.top_p * (double)kept;
    } else if (filter == 2) {
      if (!w.by_min_p) continue;
      if (threadIdx.x == 0) sh->min_mass = 0;
      __syncthreads();
      unsigned long long mine = 0;
      for_each_logit<T, kPickThreads, 1>(row.logits, 0, a.vocab, [&](int, float l) {
        const float y = row.y(l);
        if (y >= w.floor && y > kLeast) mine += Row::weight(y);
      });
#pragma unroll
      for (int s = 1; s < 64; s *= 2) mine += __shfl_xor(mine, s);
      if ((threadIdx.x & 63) == 0) atomicAdd(&sh->min_mass, mine);
      __syncthreads();
      kept = min(kept, sh->min_mass);
      continue;
    } else {
      sought.by = Sought::kAbove;
      sought.passed = min((unsigned long long)((double)w.uniform * (double)kept), kept - 1);
    }
    kept = min(kept, place_of<T>(a, row, sought, sh));
  }
}

__device__ __forceinline__ void store_choice(const SampleArgs& a, int r, const Row& row, const Wanted& w, const PickShared* sh) {
  if (threadIdx.x) return;
  const uint64_t found = sh->found;
  a.tokens[r] = (int32_t)(uint32_t)found;
  // (the most probable token weighs 2^31)
  if (a.logprobs)
    a.logprobs[r] = row.y(logit_of_entry(found)) - log1pf((float)(w.total - (1ull << 31)) * 4.65661287307739e-10f);
}
__device__ __forceinline__ void store_none(const SampleArgs& a, int r) {
  if (threadIdx.x) return;
  a.tokens[r] = -1;
  if (a.logprobs) a.logprobs[r] = -INFINITY;
}

// Slices: the tokens of the wanted bins into the row's list, with the sums before their bins; the workgroup of the first
// slice leaves what the choice needs to know beside.  Every workgroup adds up the row's histogram for itself (48 KiB from the L2, instead
// of a launch for it): 8.9 us.
template <int T>
__global__ __launch_bounds__(kSliceThreads) void sample_collect_kernel(SampleArgs a) {
  extern __shared__ __align__(16) uint8_t lds[];
  PickShared* const sh = reinterpret_cast<PickShared*>(lds);
  const int s = blockIdx.x, r = blockIdx.y;
  const Asked asked = asked_of(a, r);
  Bins<kSliceThreads> bins;
  {
    const int64_t at = (int64_t)r * kBins + Bins<kSliceThreads>::EACH * threadIdx.x;
#pragma unroll
    for (int j = 0; j < Bins<kSliceThreads>::EACH; ++j) bins.mass[j] = a.mass[at + j], bins.count[j] = a.count[at + j];
  }
  const Row row = make_row<T>(a, r, asked.temperature);
  if (row.m == -INFINITY) return;
  bins.add_up(sh);
  const Wanted w = find_wanted<kSliceThreads>(asked, bins, sh);
  if (s == 0 && threadIdx.x == 0) a.wanted[r] = w;
  if (w.tokens > kListed) return;
  const Reach reach(row, w);
  for_each_logit<T, kSliceThreads>(row.logits, slice_from(a, s), slice_from(a, s + 1), [&](int token, float l) {
    if (is_wanted(row, l, reach, w)) {
      const int bin = Row::bin(row.y(l));
      const uint32_t at = atomicAdd(&a.listed[r], 1u);
      if (at < kListed) a.list[(int64_t)r * kListed + at] = Listed{entry_of(token, l), sh->mass[bin], sh->count[bin], 0};
    }
  });
}

// One workgroup per row: the choice.  5.4 us: a chain of loads, a sort and some fifteen barriers.
template <int T>
__global__ __launch_bounds__(kPickThreads) void sample_pick_kernel(SampleArgs a) {
  extern __shared__ __align__(16) uint8_t lds[];
  PickShared* const sh = reinterpret_cast<PickShared*>(lds);
  const int r = blockIdx.x;
  const Listed* const list = a.list + (int64_t)r * kListed;
  const Listed mine = list[threadIdx.x];  // (requested before it is known how many there are)
  const Wanted w = a.wanted[r];
  const uint32_t listed = a.listed[r];
  const Row row = make_row<T>(a, r, a.temperature ? a.temperature[r] : 1.0f);
  if (row.m == -INFINITY) return store_none(a, r);
  if (w.tokens > kListed) {
    choose_crowded<T>(a, row, w, sh);
  } else {
    const int n = (int)min(w.tokens, listed);  // (as many as were collected: logits that another stream changes meanwhile leave fewer)
    for (int j = threadIdx.x; j < n; j += kPickThreads) {
      const Listed x = j < kPickThreads ? mine : list[j];
      sh->list[j] = x.entry;
      const int bin = Row::bin(row.y(logit_of_entry(x.entry)));
      sh->mass[bin] = x.mass_before;
      sh->count[bin] = x.count_before;
    }
    choose_from_list<kPickThreads>(row, w, n, sh);
  }
  store_choice(a, r, row, w, sh);
}

// One workgroup per row: everything.  256 rows of 100003 fp32 logits (102 MB) 62 us: about 20 us each for the maximum, which reads HBM, and for the histogram (some 20
// instructions and two LDS atomics per logit), 15 for collecting (the row comes out of a cache by then), the rest a chain of barriers:
// with 1000 tokens 13 us.  Vector instructions issue for half of a launch's cycles, the LDS is busy for 15 %, half of that conflicts.  Neither a shorter exponential nor one atomic for both sums made a difference; keeping a part of the row in
// registers between the passes was slower.
template <int T>
__global__ __launch_bounds__(kPickThreads) void sample_row_kernel(SampleArgs a) {
  extern __shared__ __align__(16) uint8_t lds[];
  PickShared* const sh = reinterpret_cast<PickShared*>(lds);
  const int r = blockIdx.x, i = threadIdx.x;
  const void* const logits = (const uint8_t*)a.logits + r * a.stride * (T == SFMP_TYPE_FP32 ? 4 : 2);
  const Asked asked = asked_of(a, r);
  for (int j = i; j < kBins; j += kPickThreads) sh->mass[j] = 0, sh->count[j] = 0;
  float m = -INFINITY;
  for_each_logit<T, kPickThreads>(logits, 0, a.vocab, [&](int, float l) { m = fmaxf(m, l); });
  m = max_of_wave(m);
  if ((i & 63) == 0) sh->wave_max[i >> 6] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kPickThreads / 64; ++w) m = fmaxf(m, sh->wave_max[w]);
  const Row row(logits, m, asked.temperature);
  if (row.m == -INFINITY) return store_none(a, r);
  auto add = [&](float y) {
    if (!(y > kLeast)) return;
    const uint32_t w = Row::weight(y);
    if (!w) return;
    atomicAdd(&sh->mass[Row::bin(y)], (unsigned long long)w);
    atomicAdd(&sh->count[Row::bin(y)], 1u);
  };
  if (row.plain)
    for_each_logit<T, kPickThreads>(logits, 0, a.vocab, [&](int, float l) { add(row.template y<true>(l)); });
  else
    for_each_logit<T, kPickThreads, 1>(logits, 0, a.vocab, [&](int, float l) { add(row.y(l)); });
  __syncthreads();
  Bins<kPickThreads> bins;
#pragma unroll
  for (int j = 0; j < Bins<kPickThreads>::EACH; ++j) {
    bins.mass[j] = sh->mass[Bins<kPickThreads>::EACH * i + j];
    bins.count[j] = sh->count[Bins<kPickThreads>::EACH * i + j];
  }
  bins.add_up(sh);
  const Wanted w = find_wanted<kPickThreads>(asked, bins, sh);
  if (w.tokens > kListed) {
    choose_crowded<T>(a, row, w, sh);
  } else {
    const Reach reach(row, w);
    __syncthreads();
    if (i == 0) sh->listed = 0;
    __syncthreads();
    for_each_logit<T, kPickThreads>(logits, 0, a.vocab, [&](int token, float l) {
      if (is_wanted(row, l, reach, w)) {
        const uint32_t at = atomicAdd(&sh->listed, 1u);
        if (at < kListed) sh->list[at] = entry_of(token, l);
      }
    });
    __syncthreads();
    choose_from_list<kPickThreads>(row, w, (int)min(w.tokens, sh->listed), sh);
  }
  store_choice(a, r, row, w, sh);
}

constexpr int kMostSlices = 512;
int slices_of(int32_t rows, int32_t vocab) {
  // slices of 4096 tokens or more, 512 workgroups at most (each adds a histogram of its own to the row's: 32 rows of 131072
  // tokens 36.7 us, with 1024 workgroups 47.5, with 256 39.9); 2^15 tokens at most
  int64_t s = vocab / 4096;
  if (s * rows > kMostSlices) s = kMostSlices / rows;
  const int64_t least = ((int64_t)vocab + kMostSlice - 1) / kMostSlice;
  if (s < least) s = least;
  return (int)s;
}

// One workgroup per row: its time grows with the vocabulary and hardly with the rows, that of four launches over slices with both.
// One row of 8000 tokens 14.7 us against 24.8, of 32000 19.0 and 23.4, of 131072 46.5 and 22.6; 32 rows of 50257 tokens
// 29.8 and 35.5, of 131072 52.6 and 37.4; 128 of them 67.7 and 72.8.
bool whole_rows(int32_t rows, int32_t vocab) { return rows >= 110 || (int64_t)vocab * (110 - rows) < 4200000; }

struct SampleWorkspace {
  int64_t max_at, mass_at, count_at, list_at, wanted_at, listed_at, bytes;
};
SampleWorkspace sample_workspace(int32_t rows, int64_t slices) {  // (of all rows)
  SampleWorkspace w{};
  w.bytes = 256;
  if (rows == 0) return w;
  w.count_at = round_up_256((int64_t)rows * kBins * 8);
  w.list_at = w.count_at + round_up_256((int64_t)rows * kBins * 4);
  w.wanted_at = w.list_at + round_up_256((int64_t)rows * kListed * sizeof(Listed));
  w.listed_at = w.wanted_at + round_up_256((int64_t)rows * sizeof(Wanted));
  w.max_at = w.listed_at + round_up_256((int64_t)rows * 4);
  w.bytes = w.max_at + round_up_256(slices * 4);
  return w;
}
// What a call needs
SampleWorkspace workspace_of_call(int32_t rows, int32_t vocab) {
  return whole_rows(rows, vocab) ? sample_workspace(0, 0) : sample_workspace(rows, (int64_t)rows * slices_of(rows, vocab));
}
// What every call of no more rows and tokens can do with: the most rows of such a vocabulary that are cut (whole_rows), and as many
// slices as calls up to there have.
int64_t workspace_up_to(int32_t rows, int32_t vocab) {
  int32_t cut = rows < 109 ? rows : 109;
  while (cut > 0 && whole_rows(cut, vocab)) --cut;
  const int64_t least = (int64_t)cut * (((int64_t)vocab + kMostSlice - 1) / kMostSlice);
  return sample_workspace(cut, least > kMostSlices ? least : kMostSlices).bytes;
}

template <int T>
int launch_sample(const SampleArgs& a, hipStream_t stream) {
  if (whole_rows(a.rows, a.vocab)) {
    if (int e = allow_full_lds((const void*)sample_row_kernel<T>, "sample_row_kernel")) return e;
    sample_row_kernel<T><<<a.rows, kPickThreads, sizeof(PickShared), stream>>>(a);
  } else {
    if (int e = allow_full_lds((const void*)sample_collect_kernel<T>, "sample_collect_kernel")) return e;
    if (int e = allow_full_lds((const void*)sample_pick_kernel<T>, "sample_pick_kernel")) return e;
    const dim3 grid(a.slices, a.rows);
    sample_max_kernel<T><<<grid, kSliceThreads, 0, stream>>>(a);
    sample_bins_kernel<T><<<grid, kSliceThreads, 0, stream>>>(a);
    sample_collect_kernel<T><<<grid, kSliceThreads, sizeof(PickShared), stream>>>(a);
    sample_pick_kernel<T><<<a.rows, kPickThreads, sizeof(PickShared), stream>>>(a);
  }
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return SFMP_OK;
  note_hip_error("sfmp_sample", hipGetErrorString(e));
  return SFMP_ERR_HIP;
}

int check_rows(int32_t rows, int32_t vocab) {
  return rows < 0 || rows > 65535 || vocab < 1 || vocab > (1 << 24) ? SFMP_ERR_SHAPE : SFMP_OK;
}

}  // namespace
}  // namespace sfmp

using namespace sfmp;

extern "C" int sfmp_sample_workspace(int32_t rows, int32_t vocab, int64_t* bytes) {
  if (!bytes) return SFMP_ERR_NULL;
  if (int e = check_rows(rows, vocab)) return e;
  *bytes = workspace_up_to(rows, vocab);
  return SFMP_OK;
}

extern "C" int sfmp_sample(const void* logits_dev, int32_t dtype, int32_t rows, int32_t vocab, int64_t stride,
                           const float* temperature_dev, const int32_t* top_k_dev, const float* top_p_dev,
                           const float* min_p_dev, const float* uniform_dev, int32_t* tokens_dev, float* logprobs_dev,
                           void* workspace_dev, int64_t workspace_bytes, void* hip_stream) {
  if (int e = check_rows(rows, vocab)) return e;
  if (dtype != SFMP_TYPE_FP16 && dtype != SFMP_TYPE_BF16 && dtype != SFMP_TYPE_FP32) return SFMP_ERR_LAYOUT;
  if (stride < vocab || stride > INT64_MAX / 8 / 65536) return SFMP_ERR_SHAPE;
  if (rows == 0) return SFMP_OK;
  if (!logits_dev || !uniform_dev || !tokens_dev) return SFMP_ERR_NULL;
  auto off = [](const void* p, uintptr_t a) { return reinterpret_cast<uintptr_t>(p) % a != 0; };
  if (off(logits_dev, dtype == SFMP_TYPE_FP32 ? 4 : 2) || off(temperature_dev, 4) || off(top_k_dev, 4) || off(top_p_dev, 4) ||
      off(min_p_dev, 4) || off(uniform_dev, 4) || off(tokens_dev, 4) || off(logprobs_dev, 4))
    return SFMP_ERR_ALIGN;
  const SampleWorkspace w = workspace_of_call(rows, vocab);
  if (!workspace_dev || off(workspace_dev, 256) || workspace_bytes < w.bytes) return SFMP_ERR_WORKSPACE;
  uint8_t* const at = (uint8_t*)workspace_dev;
  const SampleArgs a{logits_dev, rows, vocab, slices_of(rows, vocab), stride, temperature_dev, top_k_dev, top_p_dev, min_p_dev,
                     uniform_dev, tokens_dev, logprobs_dev, (float*)(at + w.max_at), (Listed*)(at + w.list_at), (Wanted*)(at + w.wanted_at),
                     (uint32_t*)(at + w.listed_at), (unsigned long long*)(at + w.mass_at), (uint32_t*)(at + w.count_at)};
  const hipStream_t stream = (hipStream_t)hip_stream;
  if (dtype == SFMP_TYPE_FP16) return launch_sample<SFMP_TYPE_FP16>(a, stream);
  if (dtype == SFMP_TYPE_BF16) return launch_sample<SFMP_TYPE_BF16>(a, stream);
  return launch_sample<SFMP_TYPE_FP32>(a, stream);
}
