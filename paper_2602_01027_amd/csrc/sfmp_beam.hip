// One step of a beam search: the best continuations of every request over its beams and the vocabulary.
//
// A continuation's value is score + (l - m) - ln sum exp(l - m) of its beam's row of logits.  Inside a row the order is that of the logits, so that a
// workgroup which holds a piece of a row in registers needs no more of it than its largest logits, as many as are wanted of the request, and its sum of
// exponentials: the row is read once.  A second launch, a workgroup per request, makes values of what the pieces of all beams have left and picks
// the best.
//
// Continuations of different beams can lie closer together than fp32 tells apart (scores of -50 in steps of 4e-6), so that values are fp64.  Of the
// sum, which fp32 exponentials make to some 2^-24 of each term, the listed terms - the largest ones, which are most of it where a beam is sure of its
// next token - are made again in fp64, and so are the additions of the runs that hold them, whose other terms fp32 would round to what stands beside
// them.  What is left is an error of 2^-24 of the other terms, with some factor: of rows without large terms no more is known than that.
#include <float.h>
#include <math.h>

#include "sfmp_device.h"
#include "sfmp_internal.h"

namespace sfmp {
namespace {

constexpr int kThreads = 512;        // of a piece
constexpr int kGroups = kThreads / 2;
constexpr int kMostBeams = 32, kMostChoices = 64;
constexpr int kMostListed = 8192;    // entries of the lists of a request

struct Piece {
  double sum;    // of exp(l - top)
  float top;     // its largest logit; -infinity: none
  int32_t unused;
};

struct BeamArgs {
  const void* logits;
  int64_t stride;
  int32_t requests, beams, vocab, choices, pieces, chunks_each;
  const float* scores;
  const float* weights;
  const int32_t* ended;
  int32_t end_token;
  float* next_scores;
  int32_t* parents;
  int32_t* tokens;
  uint32_t of_lists, of_pieces;   // x / (beams * pieces) and x / pieces as (x * of_...) >> 32, for x < 2^13
  Piece* piece;      // [rows][pieces]
  uint64_t* listed;  // [rows][pieces][choices], falling; 0: none
};

// Numbers in the order of the values (0 stays free: below all of them; -0 is 0)
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);
  return u ^ ((int32_t)u < 0 ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float logit_of_key(uint32_t key) {
  return __uint_as_float(key ^ ((int32_t)key < 0 ? 0x80000000u : 0xFFFFFFFFu));
}
__device__ __forceinline__ uint64_t key_of(double x) {
  const uint64_t u = (uint64_t)__double_as_longlong(x + 0.0);
  return u ^ ((int64_t)u < 0 ? ~0ull : 1ull << 63);
}

// NaN as -infinity, +infinity as the largest number
__device__ __forceinline__ float in_range(float x) { return x != x ? -INFINITY : fminf(x, FLT_MAX); }

template <int T>
__device__ __forceinline__ float logit_at(const u32x4& w, int j) {
  if constexpr (T == SFMP_TYPE_FP32) return __uint_as_float(w[j]);
  const uint32_t bits = j & 1 ? w[j / 2] >> 16 : w[j / 2] & 0xFFFFu;
  if constexpr (T == SFMP_TYPE_BF16) return __uint_as_float(bits << 16);
  return (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
}

// Terms of a sum in fp32, exp(l - base) but for a factor that all of them share, by one operation before the exponential: 2^(l k + c) with
// k = log2 e and c = -base k, each rounded to fp32.  l k is exact inside, so that the exponent is (l - base) k, off by its own rounding, and
// base k + c, some 2^-24 of base, which `factor` makes good.  Past kMostBase, where that is no small number: exp(l - base) from the difference.
constexpr float kLog2e = 1.44269502f, kMostBase = 4096.0f;
struct Terms {
  float base, c;
  __device__ __forceinline__ explicit Terms(float b) : base(b), c(-b * kLog2e) {}
  __device__ __forceinline__ bool far() const { return !(fabsf(base) < kMostBase); }
  __device__ __forceinline__ float operator()(float l) const { return __builtin_amdgcn_exp2f(__builtin_fmaf(l, kLog2e, c)); }
  __device__ __forceinline__ float of_any(float l) const {
    return __builtin_amdgcn_exp2f(far() ? (l - base) * kLog2e : __builtin_fmaf(l, kLog2e, c));
  }
  // (its logarithm: below 2^-11)
  __device__ __forceinline__ double log_factor() const { return far() ? 0.0 : -0.6931471805599453 * fma((double)base, (double)kLog2e, (double)c); }
  __device__ __forceinline__ double factor() const {
    const double x = log_factor();
    return 1.0 + x * (1.0 + x * (0.5 + x * (1.0 / 6.0)));
  }
};

// exp(d) for d <= 0 in fp64: 2^n times the series of r = d - n ln 2, |r| <= ln 2 / 2, whose first term left out is below 2^-47 (the library's
// function, with every argument's special cases, takes twice the registers).  Inside of loops every coefficient is made where it is used (INSIDE), or
// the compiler brings a register pair for each of them out; loads of them wait for one another.
constexpr int kTerms = 11;
template <bool INSIDE = false>
__device__ __forceinline__ double exp_of(double d) {
  constexpr double kInverseFactorials[kTerms] = {1.0 / 39916800.0, 1.0 / 3628800.0, 1.0 / 362880.0, 1.0 / 40320.0, 1.0 / 5040.0, 1.0 / 720.0,
                                                 1.0 / 120.0,      1.0 / 24.0,      1.0 / 6.0,      0.5,           1.0};
  d = fmax(d, -800.0);  // (0 there)
  const double n = rint(d * 1.4426950408889634);
  const double r = fma(n, -0.6931471805599453, d);
  double p = 0.0;
#pragma unroll
  for (int i = 0; i < kTerms; ++i) {
    double coefficient = kInverseFactorials[i];
    if constexpr (INSIDE) asm volatile("" : "+s"(coefficient));
    p = fma(p, r, coefficient);
  }
  p = fma(p, r, 1.0);
  return ldexp(p, (int)n);
}

// Maximum over a wavefront, in all lanes; without the LDS.
__device__ __forceinline__ uint32_t max_of_wave(uint32_t x) {
  auto step = [&](auto ctrl, auto rows) {
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, ctrl(), rows(), 0xF, false));
  };
  using std::integral_constant;
  constexpr integral_constant<int, 0xF> kAllRows{};
  step(integral_constant<int, 0x111>{}, kAllRows), step(integral_constant<int, 0x112>{}, kAllRows);  // from 1, 2, 4, 8 lanes before, in rows of 16
  step(integral_constant<int, 0x114>{}, kAllRows), step(integral_constant<int, 0x118>{}, kAllRows);
  step(integral_constant<int, 0x142>{}, integral_constant<int, 0xA>{});  // from the last lane of the row before
  step(integral_constant<int, 0x143>{}, integral_constant<int, 0xC>{});  // ... of the first two rows
  return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}
__device__ __forceinline__ uint64_t max_of_wave(uint64_t x) {
  const uint32_t high = max_of_wave((uint32_t)(x >> 32));
  return (uint64_t)high << 32 | max_of_wave((uint32_t)(x >> 32) == high ? (uint32_t)x : 0u);
}

// A threshold that at least k and no more than `most` of a workgroup's 256 keys reach (4 to a lane of a wavefront); where that many are equal,
// their value, which more reach.  `reach`: how many do.  0 if fewer than k keys are above 0.  From the largest key, less and less of whose bits
// from `bit` on, to the first that k keys reach, then bit by bit up again: the keys that matter agree with the largest in most of their bits.
template <typename Key>
__device__ __forceinline__ Key threshold_of(const Key (&key)[4], Key largest, int bit, int k, int most, int* reach) {
  auto count = [&](Key at) {
    int n = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) n += __popcll(__ballot(key[i] >= at));
    return n;
  };
  constexpr int BITS = (int)sizeof(Key) * 8;
  Key at = 0;
  *reach = kGroups;
  for (; bit < BITS; ++bit) {
    const Key next = largest >> bit << bit;
    const int n = next ? count(next) : 0;
    if (n < k) continue;
    at = next, *reach = n;
    break;
  }
  for (bit = min(bit, BITS) - 1; bit >= 0 && *reach > most; --bit) {
    const Key next = at | (Key)1 << bit;
    const int n = count(next);
    if (n < k) continue;
    at = next, *reach = n;
  }
  return at;
}

// A bound that at least `wanted` of different numbers in LDS reach, and no more than 64: bit by bit, from the first one in which `least`, which all of them
// reach, and `largest` differ.  `turns`: counters that take turns, the first of them 0.
template <int THREADS>
__device__ __forceinline__ uint64_t narrow(const uint64_t* list, int count, int wanted, uint64_t least, uint64_t largest, int* turns, int tid) {
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int bit = 63 - __builtin_clzll(least ^ largest | 1);
  uint64_t at = bit < 63 ? largest >> (bit + 1) << (bit + 1) : 0;
  for (int turn = 0; bit >= 0; --bit) {
    const uint64_t next = at | 1ull << bit;
    int n = 0;
    for (int base = wave * 64; base < count; base += THREADS) n += __popcll(__ballot(base + lane < count && list[base + lane] >= next));
    const int after = turn == 2 ? 0 : turn + 1;
    if (lane == 0 && n) atomicAdd(&turns[turn], n);
    if (tid == 0) turns[after] = 0;
    __syncthreads();
    const int all = turns[turn];
    turn = after;
    if (all < wanted) continue;
    at = next;
    if (all <= 64) break;
  }
  __syncthreads();
  return at;
}

// Ranks of `count` different numbers in LDS, falling; f(rank, number) for those below `wanted`.  Up to 64 are ranked by the first wavefront, a
// number per lane, some more by all threads (`ranks`: a counter for each); of many (a piece with logits for few threads: all of them are listed) those
// that a bound leaves.  32 rows of 50000 tokens, 64 choices, 848 numbers in the last pieces: 38 instead of 72 us (100 numbers, for a row of
// 131072: 38 so, 48 by a bound).
constexpr int kMostRanked = 256;
template <int THREADS, typename F>
__device__ __forceinline__ void rank_numbers(const uint64_t* list, int count, int wanted, uint64_t least, uint64_t largest, uint32_t* ranks, int* turns,
                                             int tid, F f) {
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  auto rank_few = [&](const uint64_t* few, int n) {
    if (wave) return;
    const uint64_t mine = lane < n ? few[lane] : 0;
    const int low = (int)(uint32_t)mine, high = (int)(uint32_t)(mine >> 32);
    int rank = 0;
    for (int j = 0; j < n; ++j)
      rank += ((uint64_t)(uint32_t)__builtin_amdgcn_readlane(high, j) << 32 | (uint32_t)__builtin_amdgcn_readlane(low, j)) > mine;
    if (lane < n && rank < wanted) f(rank, mine);
  };
  if (count <= 64) {
    rank_few(list, count);
    return;
  }
  if (count > kMostRanked) {
    const uint64_t bound = narrow<THREADS>(list, count, wanted, least, largest, turns, tid);
    uint64_t* const few = reinterpret_cast<uint64_t*>(ranks);
    if (tid == 0) turns[0] = 0;
    __syncthreads();
    for (int i = tid; i < count; i += THREADS)
      if (list[i] >= bound) few[atomicAdd(&turns[0], 1)] = list[i];
    __syncthreads();
    rank_few(few, turns[0]);
    return;
  }
  for (int i = tid; i < count; i += THREADS) ranks[i] = 0;
  __syncthreads();
  for (int base = 0; base < count; base += 64) {
    const uint64_t mine = base + lane < count ? list[base + lane] : ~0ull;
    uint32_t above = 0;
    for (int j = wave; j < count; j += THREADS / 64) above += list[j] > mine;
    if (base + lane < count && above) atomicAdd(&ranks[base + lane], above);
  }
  __syncthreads();
  for (int i = tid; i < count; i += THREADS)
    if ((int)ranks[i] < wanted) f((int)ranks[i], list[i]);
}

__device__ __forceinline__ double sum_of_wave(double x) {
#pragma unroll
  for (int s = 1; s < 64; s *= 2) x += __shfl_xor(x, s);
  return x;
}

// LDS of a piece, before the runs of the threads that are looked at, the list of numbers and their ranks
struct PieceLds {
  double sums[kThreads / 64];
  double scale, unused_scale;
  uint64_t carried[kMostChoices];
  uint32_t maxima[kGroups], firsts[kGroups];
  uint32_t bound, bound_not;    // numbers that are listed: those with larger keys, and of equal ones those with ~number >= bound_not
  uint32_t largest;
  int32_t threads, count, turns[3];
  uint8_t place[kThreads];      // of a thread's runs among those of the threads that are looked at
};
static_assert(sizeof(PieceLds) % 16 == 0, "runs of 16 bytes lie behind it");
// Pairs of threads that are looked at: those that `choices` need and, where others reach the bound too, some more.
constexpr int kMorePairs = 16;
__host__ __device__ constexpr int most_threads(int choices) { return 2 * (choices + kMorePairs); }
// Bytes of LDS: with each thread R runs and its number, and its logits and what it holds of the list as numbers.
__host__ __device__ constexpr int piece_lds(int choices, int R, int run) {
  return (int)sizeof(PieceLds) + most_threads(choices) * (R * 16 + 4) + (most_threads(choices) * R * run + kMostChoices) * 12;
}

// The largest logit of a thread (NaN are passed by).
template <int T, int R>
__device__ __forceinline__ float most_of(const u32x4 (&w)[R]) {
  if constexpr (T == SFMP_TYPE_FP16) {  // two at a time
    half2_ most = {(_Float16)-INFINITY, (_Float16)-INFINITY};
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t pair = w[r][j];  // (the cast of an element of a vector takes the first one)
        most = __builtin_elementwise_max(most, __builtin_bit_cast(half2_, pair));
      }
    return fmaxf((float)most[0], (float)most[1]);
  }
  // As whole numbers, positive floats are in their order: two at an operation, and none to quiet a NaN
  int32_t most = INT32_MIN;
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (T == SFMP_TYPE_BF16) most = max(most, (int32_t)(w[r][j] << 16));
      most = max(most, (int32_t)w[r][j]);  // (bf16: the lower half is more digits of the upper one, taken off below)
    }
  if constexpr (T == SFMP_TYPE_BF16) most &= 0xFFFF0000;
  if (most >= 0 && most <= 0x7F800000) return __uint_as_float((uint32_t)most);
  float x = -INFINITY;  // none is positive, or there is a NaN
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int j = 0; j < (T == SFMP_TYPE_FP32 ? 4 : 8); ++j) x = fmaxf(x, logit_at<T>(w[r], j));
  return x;
}

// What was made of w is made again from here on: its logits as fp32 take twice its registers, and what is kept of them keeps other workgroups out
// (118 registers and 2 workgroups of a compute unit; without it 64 and 4, 32 x 8 rows of 131072 bf16 logits in 35 instead of 39 us).
template <int R>
__device__ __forceinline__ void forget(u32x4 (&w)[R]) {
#pragma unroll
  for (int r = 0; r < R; ++r) asm volatile("" : "+v"(w[r]));
}

// The largest logits and the sum of exponentials of a piece of a row: chunks of R runs of 16 bytes per thread, in registers.
//
// Which logits are among the `choices` largest: a bound that between choices and choices + kMorePairs of the maxima of 256 pairs of threads reach is one
// that no fewer logits reach, and only the logits of those threads can (where more maxima than that are equal, those of the lowest numbers).  The
// threads leave their runs in LDS, where all threads look through them; what reaches the bound, a few more than are wanted, is ranked.  Chunks
// behind the first take the list along.
//
// Bound by vector instructions (they issue for 58 % of the cycles) and by the barriers of a chunk, of which one wavefront's search for the bound is the
// longest, with loads that wait behind them: as many wavefronts as fit share a compute unit (32, at 64 registers).  32 x 8 rows of 131072 bf16
// logits, 16 choices: 22 us, 3.0 TB/s.  The next chunk's loads in flight over this one's barriers cost a workgroup per compute unit and 2 us.
template <int T, int R>
__global__ __launch_bounds__(kThreads, 8) void beam_pieces_kernel(BeamArgs a) {
  constexpr int SIZE = T == SFMP_TYPE_FP32 ? 4 : 2, RUN = 16 / SIZE;
  extern __shared__ __align__(16) uint8_t lds[];
  PieceLds& shared = *reinterpret_cast<PieceLds*>(lds);
  const int threads_most = most_threads(a.choices);
  u32x4* const runs_of = reinterpret_cast<u32x4*>(lds + sizeof(PieceLds));           // [threads_most][R]
  uint64_t* const list = reinterpret_cast<uint64_t*>(runs_of + threads_most * R);    // [threads_most * R * RUN + kMostChoices]
  uint32_t* const ranks = reinterpret_cast<uint32_t*>(list + threads_most * R * RUN + kMostChoices);
  uint32_t* const owner = ranks + threads_most * R * RUN + kMostChoices;             // [threads_most]
  const int row = blockIdx.x / a.pieces, piece = blockIdx.x - row * a.pieces, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const uint8_t* const start = (const uint8_t*)a.logits + (int64_t)row * a.stride * SIZE;
  const int runs = (a.vocab + RUN - 1) / RUN;
  // (which thread has which logits must not depend on the row's alignment: rows of equal logits have equal sums)
  typedef u32x4 __attribute__((aligned(2))) Run;
  u32x4 w[R];
  auto load = [&](int first_run) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int i = (first_run + r * kThreads + tid) * RUN;
      constexpr uint32_t kNone = T == SFMP_TYPE_FP32 ? 0xFF800000u : T == SFMP_TYPE_BF16 ? 0xFF80FF80u : 0xFC00FC00u;  // -infinity
      w[r] = u32x4{kNone, kNone, kNone, kNone};
      if (i + RUN <= a.vocab) {
        w[r] = *reinterpret_cast<const Run*>(start + (int64_t)i * SIZE);
      } else if (i < a.vocab) {  // the row's end: its last 16 bytes, moved down, or element by element where it has no 16
        typedef unsigned __int128 Bits;
        const Bits none = (Bits)(((uint64_t)kNone << 32) | kNone) << 64 | (((uint64_t)kNone << 32) | kNone);
        Bits bits = none;
        if (a.vocab >= RUN) {
          const int over = (i + RUN - a.vocab) * SIZE * 8;
          const u32x4 x = *reinterpret_cast<const Run*>(start + (int64_t)(a.vocab - RUN) * SIZE);
          bits = __builtin_bit_cast(Bits, x) >> over | none << (128 - over);
        } else {
#pragma unroll 1
          for (int j = a.vocab - 1; j >= 0; --j)
            bits = bits << (SIZE * 8) | (SIZE == 4 ? ((const uint32_t*)start)[j] : (uint32_t)((const uint16_t*)start)[j]);
        }
        w[r] = __builtin_bit_cast(u32x4, bits);
      }
    }
  };
  // Logit number i of the threads that are looked at.
  auto left_logit = [&](int i) {
    uint32_t bits;
    if constexpr (SIZE == 4)
      bits = reinterpret_cast<const uint32_t*>(runs_of)[i];
    else
      bits = (uint32_t)reinterpret_cast<const uint16_t*>(runs_of)[i] << (i & 1 ? 16 : 0);
    return in_range(logit_at<T>(u32x4{bits, bits, bits, bits}, i & 1));
  };
  // What the sum of a chunk lacks of its runs with listed terms: these in fp64 instead of fp32, relative to what they were added with, and the other
  // terms as far as fp32 has rounded them to what stands beside them.  RUN threads for each listed term, a term of its run for each; of several
  // terms of a run those of the first one do it.  (32 x 8 rows of 131072, 16 choices: 31.6 us instead of 31.3; 34.0 with a thread for each term.)
  auto listed_again = [&](int first_run, float top) {
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));
    const int j = tid % RUN;
    const uint64_t x = shared.carried[tid / RUN];
    const int at = (int)~(uint32_t)x - first_run * RUN;
    if (!x || at < 0) return 0.0;  // (not of this chunk)
    const uint64_t least = max(shared.carried[a.choices - 1], (uint64_t)1);  // (of a list that is not full: all logits are listed)
    const int run = at / RUN;
    const float l = left_logit((shared.place[run % kThreads] * R + run / kThreads) * RUN + j);
    const Terms terms(top);
    const float term = terms.of_any(l);
    const bool again = l > -INFINITY && ((uint64_t)key_of(l) << 32 | ~(uint32_t)((first_run + run) * RUN + j)) >= least;
    const uint32_t all_again = (uint32_t)(__ballot(again) >> (tid & 63 & -RUN)) & ((1u << RUN) - 1);
    float part = 0.0f;  // (the same additions as before)
#pragma unroll
    for (int u = 0; u < RUN; ++u) part += __shfl(term, u, RUN);
    if (__builtin_ctz(all_again | 1u << RUN) != at % RUN) return 0.0;
    return (again ? exp_of<true>((double)l - (double)top - terms.log_factor()) : (double)term) - (j ? 0.0 : (double)part);
  };
  load(piece * a.chunks_each * (kThreads * R));  // (while the row's state is on its way)
  if ((a.ended && a.ended[row]) || !(a.scores[row] > -INFINITY)) return;  // (no logit of it counts)
  if (tid < kMostChoices) shared.carried[tid] = 0;
  float top = -INFINITY;
  double sum = 0.0;
  __syncthreads();
  for (int chunk = 0; chunk < a.chunks_each; ++chunk) {
    const int first_run = (piece * a.chunks_each + chunk) * (kThreads * R);
    if (first_run >= runs) break;
    if (chunk) load(first_run);
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));  // (or the compiler keeps what it makes of it, in registers, over all chunks)
    const int lane = tid & 63;
    const uint64_t held = tid < a.choices ? shared.carried[tid] : 0;
    const float most = in_range(most_of<T>(w));
    uint32_t my_key = most > -INFINITY ? key_of(most) : 0;
    const uint32_t pair_key = max(max(my_key, (uint32_t)(held >> 32)), (uint32_t)__shfl_xor((int)max(my_key, (uint32_t)(held >> 32)), 1));
    if ((tid & 1) == 0) shared.maxima[tid / 2] = pair_key;
    forget(w);
    __syncthreads();
    // the bound: one wavefront's work
    if (wave == 0) {
      uint32_t key[4], largest = 0;
      int reach;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        key[i] = shared.maxima[lane + 64 * i];
        largest = max(largest, key[i]);
      }
      largest = max_of_wave(largest);
      const uint32_t bound = threshold_of(key, largest, 20, a.choices, a.choices + kMorePairs, &reach);
      if (lane == 0) {
        shared.bound = bound, shared.bound_not = 0, shared.largest = largest;
        if (top > -INFINITY) {  // (of sums so far)
          const float base = logit_of_key(largest);
          shared.scale = exp_of<true>((double)top - (double)base) * Terms(top).factor() / Terms(base).factor();
        }
        // (more equal maxima than there is room for: marked)
        shared.count = 0, shared.turns[0] = 0, shared.threads = bound && reach > a.choices + kMorePairs ? -1 : 0;
      }
    }
    __syncthreads();
    auto same = [](uint32_t x) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)x); };  // (in all lanes)
    const uint32_t bound = same(shared.bound), largest = same(shared.largest);
    const bool crowded = (int32_t)same((uint32_t)shared.threads) < 0;
    if (largest == 0) {  // (no logit so far)
      __syncthreads();
      continue;
    }
    if (crowded) {
      uint32_t lowest = ~0u;
#pragma unroll
      for (int r = R - 1; r >= 0; --r) {
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = RUN - 1; j >= 0; --j) {
          const float x = in_range(logit_at<T>(w[r], j));
          if (x > -INFINITY && key_of(x) == bound) lowest = (first_run + r * kThreads + tid) * RUN + j;
        }
      }
      if ((uint32_t)(held >> 32) == bound) lowest = min(lowest, ~(uint32_t)held);
      lowest = min(lowest, (uint32_t)__shfl_xor((int)lowest, 1));
      if ((tid & 1) == 0) shared.firsts[tid / 2] = ~lowest;
      __syncthreads();
      if (wave == 0) {
        int more = 0, reach;
        uint32_t number[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t key = shared.maxima[lane + 64 * i];
          more += __popcll(__ballot(key > bound));
          number[i] = key == bound ? shared.firsts[lane + 64 * i] : 0;
        }
        const uint32_t bound_not = threshold_of(number, ~0u, 0, a.choices - more, a.choices - more, &reach);
        if (lane == 0) shared.bound_not = bound_not, shared.threads = 0;
      }
      __syncthreads();
    }
    const uint32_t bound_not = same(shared.bound_not);
    auto wanted = [&](uint32_t k, uint32_t not_number) { return k && (k > bound || (k == bound && not_number >= bound_not)); };
    // (in a crowd a thread of a pair whose maximum is the bound waits for its turn)
    bool looked_at = my_key && my_key >= bound;
    if (crowded && shared.maxima[tid / 2] == bound) looked_at &= shared.firsts[tid / 2] >= bound_not;
    if (looked_at) {
      const int at = atomicAdd(&shared.threads, 1);
      owner[at] = tid, shared.place[tid] = (uint8_t)at;
#pragma unroll
      for (int r = 0; r < R; ++r) runs_of[at * R + r] = w[r];
    }
    if (wanted((uint32_t)(held >> 32), (uint32_t)held)) list[atomicAdd(&shared.count, 1)] = held;
    forget(w);
    // the sum, relative to the largest logit so far; in fp32 for a run and in fp64 from there on
    if (top > -INFINITY) sum *= shared.scale;
    top = logit_of_key(largest);
    const Terms terms(top);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float part = 0.0f;
#pragma unroll
      for (int j = 0; j < RUN; ++j) part += terms(logit_at<T>(w[r], j));
      if (!(part <= 2.0f * RUN) || terms.far()) {  // a NaN or an infinity among them, or large numbers
        part = 0.0f;
#pragma unroll
        for (int j = 0; j < RUN; ++j) part += terms.of_any(in_range(logit_at<T>(w[r], j)));
      }
      sum += (double)part;
      __builtin_amdgcn_sched_barrier(0);  // (a run after the other: registers)
    }
    __syncthreads();
    const int numbers = shared.threads * (R * RUN);
    for (int i = tid; i < numbers; i += kThreads) {
      const int at = i / (R * RUN), r = i / RUN % R, j = i % RUN;
      const float x = left_logit(i);
      const uint32_t not_number = ~(uint32_t)((first_run + r * kThreads + (int)owner[at]) * RUN + j);
      if (x > -INFINITY && wanted(key_of(x), not_number)) list[atomicAdd(&shared.count, 1)] = (uint64_t)key_of(x) << 32 | not_number;
    }
    uint64_t none = 0;
    asm volatile("" : "+v"(none));  // (or two registers hold it over all chunks)
    if (tid < kMostChoices) shared.carried[tid] = none;  // (read at the chunk's start)
    __syncthreads();
    rank_numbers<kThreads>(list, shared.count, a.choices, (uint64_t)bound << 32, (uint64_t)largest << 32 | ~0u, ranks, shared.turns, tid,
                           [&](int rank, uint64_t x) { shared.carried[rank] = x; });
    __syncthreads();
    if (tid < a.choices * RUN) sum += listed_again(first_run, top);
  }
  sum = sum_of_wave(sum);
  if (lane == 0) shared.sums[wave] = sum;
  __syncthreads();
  if (wave == 0) {
    if (lane < a.choices) a.listed[((int64_t)row * a.pieces + piece) * a.choices + lane] = shared.carried[lane];
    if (lane == 0) {
      double all = 0.0;
      for (int i = 0; i < kThreads / 64; ++i) all += shared.sums[i];
      Piece p;
      p.sum = top > -INFINITY ? all * Terms(top).factor() : 0.0, p.top = top, p.unused = 0;
      a.piece[(int64_t)row * a.pieces + piece] = p;
    }
  }
}

// LDS of a request, before its entries
struct BestLds {
  uint64_t maxima[kGroups];
  uint32_t orders[kGroups];
  double tops[kMostBeams], scores[kMostBeams], weights[kMostBeams];
  int32_t states[kMostBeams];  // 0: of no more use, 1: goes on, 2: ended
  int32_t best[kMostChoices];
  uint64_t bound;
  uint32_t bound_order;
  int32_t count;
};

// Groups of threads whose entries may reach the bound, and these entries, at most.
constexpr int kMoreGroups = 16;
__host__ __device__ constexpr int most_found(int choices, int threads, int each) { return (choices + kMoreGroups) * (threads / kGroups) * each; }

// The best continuations of a request among the listed ones, EACH of them in the registers of a thread: a bound that between choices and choices + 16
// of the maxima of 256 groups of threads reach (of more equal ones the first ones), as above.  A chain of loads, an fp64 logarithm and the bound's search:
// 5.0 us for a request of 4 beams in 8 pieces each with 8 choices, 9.5 us for 32 requests of 8 beams in 8 pieces each with 16.
template <int THREADS, int EACH>
__global__ __launch_bounds__(THREADS) void beam_best_kernel(BeamArgs a) {
  constexpr int GROUP = THREADS / kGroups;  // threads
  extern __shared__ __align__(16) uint8_t lds[];
  BestLds& shared = *reinterpret_cast<BestLds*>(lds);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, request = blockIdx.x;
  const int lists = a.beams * a.pieces, all = lists * a.choices, most = most_found(a.choices, THREADS, EACH);
  uint64_t* const keys = reinterpret_cast<uint64_t*>(lds + sizeof(BestLds));
  double* const values = reinterpret_cast<double*>(keys + most);
  uint32_t* const order_keys = reinterpret_cast<uint32_t*>(values + most);
  // The i-th entry: of list i % lists its (i / lists)-th, so that the first ones of all lists fall to different threads
  uint64_t listed[EACH];
  int list_of[EACH];
#pragma unroll
  for (int x = 0; x < EACH; ++x) {
    const int i = tid + x * THREADS, rank = lists == 1 ? i : (int)__umulhi(i, a.of_lists);
    list_of[x] = i - rank * lists;
    listed[x] = i < all ? a.listed[((int64_t)request * lists + list_of[x]) * a.choices + rank] : 0;
    if (rank) list_of[x] |= 1 << 30;
  }
  // of every beam: score less the logarithm of the sum of exponentials, of which the largest logit is left aside
  for (int b = wave; b < a.beams; b += THREADS / 64) {
    const int64_t row = (int64_t)request * a.beams + b;
    Piece p = a.piece[row * a.pieces + min(lane, a.pieces - 1)];  // (of a row that does not go on, whatever lies there)
    const float score = a.scores[row];
    const int ended = a.ended ? a.ended[row] : 0;
    const float weight = a.weights ? a.weights[row] : 1.0f;
    double sum = 0.0;
    float top = -INFINITY;
    if (!ended && score > -INFINITY) {
      for (int i = lane; i < a.pieces; i += 64) {
        if (i >= 64) p = a.piece[row * a.pieces + i];
        if (p.top > top) sum *= exp_of((double)top - (double)p.top), top = p.top;
        if (p.top > -INFINITY) sum += p.sum * exp_of((double)p.top - (double)top);
      }
      float most_top = top;
#pragma unroll
      for (int s = 1; s < 64; s *= 2) most_top = fmaxf(most_top, __shfl_xor(most_top, s));
      sum = top > -INFINITY ? sum * exp_of((double)top - (double)most_top) : 0.0;
      sum = sum_of_wave(sum);
      top = most_top;
    }
    if (lane == 0) {
      shared.tops[b] = top;
      shared.scores[b] = ended ? (double)score : (double)score - log(sum);
      shared.weights[b] = weight;
      shared.states[b] = !(score > -INFINITY) ? 0 : ended ? 2 : top > -INFINITY ? 1 : 0;
    }
  }
  if (tid == 0) shared.count = 0;
  __syncthreads();
  uint64_t key[EACH], my_key = 0;
  uint32_t order[EACH], my_order = 0;  // (larger for those that come first)
  double value[EACH];
#pragma unroll
  for (int x = 0; x < EACH; ++x) {
    key[x] = 0, order[x] = 0, value[x] = 0.0;
    if (tid + x * THREADS < all) {
      const int which = list_of[x] & ~(1 << 30), b = a.pieces == 1 ? which : (int)__umulhi(which, a.of_pieces), state = shared.states[b];
      const bool first = list_of[x] == b * a.pieces;
      if (state == 2 ? first : state == 1 && listed[x]) {
        const uint32_t token = state == 2 ? (uint32_t)a.end_token : ~(uint32_t)listed[x];
        value[x] = shared.scores[b];
        if (state == 1) value[x] += (double)logit_of_key((uint32_t)(listed[x] >> 32)) - shared.tops[b];
        key[x] = key_of(value[x] * shared.weights[b]);
        order[x] = ~((uint32_t)b << 24 | token);
      }
    }
    if (key[x] > my_key || (key[x] == my_key && order[x] > my_order)) my_key = key[x], my_order = order[x];
  }
#pragma unroll
  for (int s = 1; s < GROUP; s *= 2) {
    const uint64_t k = __shfl_xor(my_key, s);
    const uint32_t o = (uint32_t)__shfl_xor((int)my_order, s);
    if (k > my_key || (k == my_key && o > my_order)) my_key = k, my_order = o;
  }
  if (tid % GROUP == 0) shared.maxima[tid / GROUP] = my_key, shared.orders[tid / GROUP] = my_order;
  __syncthreads();
  if (wave == 0) {
    uint64_t k[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) k[i] = shared.maxima[lane + 64 * i];
    int reach;
    const uint64_t largest = max_of_wave(max(max(k[0], k[1]), max(k[2], k[3])));
    const uint64_t bound = threshold_of(k, largest, 47, a.choices, a.choices + kMoreGroups, &reach);
    uint32_t bound_order = 0;
    if (bound && reach > a.choices + kMoreGroups) {  // equal ones: those that come first
      int more = 0;
      uint32_t o[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        more += __popcll(__ballot(k[i] > bound));
        o[i] = k[i] == bound ? shared.orders[lane + 64 * i] : 0;
      }
      bound_order = threshold_of(o, ~0u, 0, a.choices - more, a.choices - more, &reach);
    }
    if (lane == 0) shared.bound = bound, shared.bound_order = bound_order;
  }
  __syncthreads();
  const uint64_t bound = shared.bound;
  const uint32_t bound_order = shared.bound_order;
#pragma unroll
  for (int x = 0; x < EACH; ++x)
    if (key[x] && (key[x] > bound || (key[x] == bound && order[x] >= bound_order))) {
      const int at = atomicAdd(&shared.count, 1);
      keys[at] = key[x], order_keys[at] = order[x], values[at] = value[x];
    }
  __syncthreads();
  const int found = shared.count;
  if (found <= 64) {
    if (wave == 0) {
      const uint64_t k = lane < found ? keys[lane] : 0;
      const uint32_t o = lane < found ? order_keys[lane] : 0;
      int rank = 0;
      for (int j = 0; j < found; ++j) {
        const uint64_t kj = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(k >> 32), j) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)k, j);
        const uint32_t oj = (uint32_t)__builtin_amdgcn_readlane((int)o, j);
        rank += kj > k || (kj == k && oj > o);
      }
      if (lane < found && rank < a.choices) shared.best[rank] = lane;
    }
  } else {
    for (int i = tid; i < found; i += THREADS) {
      const uint64_t k = keys[i];
      const uint32_t o = order_keys[i];
      int above = 0;
#pragma unroll 4
      for (int j = 0; j < found; ++j) above += keys[j] > k || (keys[j] == k && order_keys[j] > o);
      if (above < a.choices) shared.best[above] = i;
    }
  }
  __syncthreads();
  if (tid < a.choices) {
    const int64_t to = (int64_t)request * a.choices + tid;
    const bool there = tid < found;
    const int at = there ? shared.best[tid] : 0;
    const uint32_t o = there ? ~order_keys[at] : 0;
    a.next_scores[to] = there ? (float)values[at] : -INFINITY;
    a.parents[to] = there ? (int)(request * a.beams + (o >> 24)) : -1;
    a.tokens[to] = there ? (int)(o & 0xFFFFFF) : -1;
  }
}

// How a call runs.  Chunks of 4 runs per thread have fewer barriers for their bytes (64 rows of 131072 16 us against 23), those of one run fill the GPU
// where there are few (4 rows of 32000 11.7 against 12.6).  Rows are cut into pieces up to some 2048 workgroups; 1024 or 4096 take the same.
struct BeamForm {
  int pieces, chunks_each;   // of a row
  int runs;                  // of 16 bytes per thread and chunk: 1 or 4
};
BeamForm choose_form(int size, int rows, int beams, int vocab, int choices) {
  BeamForm f;
  const int64_t small = (vocab + kThreads * 16 / size - 1) / (kThreads * 16 / size), large = (small + 3) / 4;
  f.runs = (int64_t)rows * large < 256 ? 1 : 4;
  const int64_t chunks = f.runs == 1 ? small : large;
  int64_t pieces = rows < 2048 ? 2048 / rows : 1;
  const int64_t most = kMostListed / (beams * choices);
  if (pieces > most) pieces = most;
  if (pieces > chunks) pieces = chunks;
  f.chunks_each = (int)((chunks + pieces - 1) / pieces);
  f.pieces = (int)((chunks + f.chunks_each - 1) / f.chunks_each);
  return f;
}
int64_t bytes_of(int64_t pieces, int choices) { return pieces * ((int64_t)sizeof(Piece) + 8 * choices); }

int check_sizes(int32_t requests, int32_t beams, int32_t vocab, int32_t choices) {
  return requests < 0 || beams < 1 || beams > kMostBeams || (int64_t)requests * beams > 65535 || vocab < 1 || vocab > 1 << 24 || choices < 1 ||
                 choices > kMostChoices
             ? SFMP_ERR_SHAPE
             : SFMP_OK;
}

template <int T, int R>
int launch_pieces(const BeamArgs& a, hipStream_t stream) {
  constexpr int RUN = T == SFMP_TYPE_FP32 ? 4 : 8;
  const int lds = piece_lds(a.choices, R, RUN);
  if (int e = allow_full_lds((const void*)beam_pieces_kernel<T, R>, "beam_pieces_kernel")) return e;
  beam_pieces_kernel<T, R><<<a.requests * a.beams * a.pieces, kThreads, lds, stream>>>(a);
  return SFMP_OK;
}
template <int T>
int launch_rows(const BeamArgs& a, const BeamForm& f, hipStream_t stream) {
  return f.runs == 1 ? launch_pieces<T, 1>(a, stream) : launch_pieces<T, 4>(a, stream);
}
template <int THREADS, int EACH>
int launch_best(const BeamArgs& a, hipStream_t stream) {
  const int lds = (int)sizeof(BestLds) + most_found(a.choices, THREADS, EACH) * 20;
  static_assert(THREADS * EACH <= kMostListed && sizeof(BestLds) + most_found(kMostChoices, THREADS, EACH) * 20 <= 160 * 1024, "LDS of a compute unit");
  if (int e = allow_full_lds((const void*)beam_best_kernel<THREADS, EACH>, "beam_best_kernel")) return e;
  beam_best_kernel<THREADS, EACH><<<a.requests, THREADS, lds, stream>>>(a);
  return SFMP_OK;
}
int launch_best_of(const BeamArgs& a, hipStream_t stream) {
  const int all = a.beams * a.pieces * a.choices;
  if (all <= 256) return launch_best<256, 1>(a, stream);
  if (all <= 1024) return launch_best<256, 4>(a, stream);
  if (all <= 4096) return launch_best<1024, 4>(a, stream);
  return launch_best<1024, 8>(a, stream);
}

bool aligned_to(const void* p, uintptr_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

}  // namespace
}  // namespace sfmp

using namespace sfmp;

extern "C" int sfmp_beam_select_workspace(int32_t requests, int32_t beams, int32_t vocab, int32_t choices, int64_t* bytes) {
  if (!bytes) return SFMP_ERR_NULL;
  if (int e = check_sizes(requests, beams, vocab, choices)) return e;
  // (of all types; pieces of a row fall as rows are added)
  const int64_t rows = (int64_t)requests * beams, chunks = (vocab + kThreads * 4 - 1) / (kThreads * 4);
  const int64_t few = rows * chunks, many = rows > 2048 ? rows : 2048;
  *bytes = round_up_256(bytes_of(few < many ? few : many, choices) + 1);
  return SFMP_OK;
}

extern "C" int sfmp_beam_select(const void* logits_dev, int32_t dtype, int32_t requests, int32_t beams, int32_t vocab, int64_t stride,
                                const float* scores_dev, const float* weights_dev, const int32_t* ended_dev, int32_t end_token, int32_t choices,
                                float* next_scores_dev, int32_t* parents_dev, int32_t* tokens_dev, void* workspace_dev, int64_t workspace_bytes,
                                void* hip_stream) {
  if (dtype != SFMP_TYPE_FP16 && dtype != SFMP_TYPE_BF16 && dtype != SFMP_TYPE_FP32) return SFMP_ERR_LAYOUT;
  if (int e = check_sizes(requests, beams, vocab, choices)) return e;
  if (stride < vocab || stride > INT64_MAX / 8 / 65536 || (ended_dev && (end_token < 0 || end_token >= vocab))) return SFMP_ERR_SHAPE;
  if (requests == 0) return SFMP_OK;
  if (!logits_dev || !scores_dev || !next_scores_dev || !parents_dev || !tokens_dev) return SFMP_ERR_NULL;
  const int size = dtype == SFMP_TYPE_FP32 ? 4 : 2;
  if (!aligned_to(logits_dev, size) || !aligned_to(scores_dev, 4) || !aligned_to(weights_dev, 4) || !aligned_to(ended_dev, 4) ||
      !aligned_to(next_scores_dev, 4) || !aligned_to(parents_dev, 4) || !aligned_to(tokens_dev, 4))
    return SFMP_ERR_ALIGN;
  const int rows = requests * beams;
  const BeamForm f = choose_form(size, rows, beams, vocab, choices);
  const int64_t pieces = (int64_t)rows * f.pieces;
  if (!workspace_dev || !aligned_to(workspace_dev, 256) || workspace_bytes < bytes_of(pieces, choices)) return SFMP_ERR_WORKSPACE;
  BeamArgs a{};
  a.logits = logits_dev, a.stride = stride;
  a.requests = requests, a.beams = beams, a.vocab = vocab, a.choices = choices, a.pieces = f.pieces, a.chunks_each = f.chunks_each;
  a.scores = scores_dev, a.weights = weights_dev, a.ended = ended_dev, a.end_token = end_token;
  a.next_scores = next_scores_dev, a.parents = parents_dev, a.tokens = tokens_dev;
  a.of_lists = (uint32_t)((1ull << 32) / (beams * f.pieces) + 1), a.of_pieces = (uint32_t)((1ull << 32) / f.pieces + 1);
  a.piece = (Piece*)workspace_dev;
  a.listed = (uint64_t*)(a.piece + pieces);
  const hipStream_t stream = (hipStream_t)hip_stream;
  const int e = dtype == SFMP_TYPE_FP32   ? launch_rows<SFMP_TYPE_FP32>(a, f, stream)
                : dtype == SFMP_TYPE_BF16 ? launch_rows<SFMP_TYPE_BF16>(a, f, stream)
                                          : launch_rows<SFMP_TYPE_FP16>(a, f, stream);
  if (e) return e;
  if (const int e2 = launch_best_of(a, stream)) return e2;
  const hipError_t error = hipGetLastError();
  if (error == hipSuccess) return SFMP_OK;
  note_hip_error("beam_pieces_kernel", hipGetErrorString(error));
  return SFMP_ERR_HIP;
}
