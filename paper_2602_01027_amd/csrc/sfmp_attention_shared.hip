// Attention of a batch whose sequences share their first pages, group by group: the shared pages are read once for the rows of
// the whole group.
//
// A row's softmax falls into that over the pages it shares and that over its sequence's own.  Of each part there are the largest score m, the
// sum l of 2^(score - m) and the sum o of 2^(score - m) V; both parts together have m = max(m1, m2), l = l1 2^(m1 - m) + l2 2^(m2 - m), o
// likewise.  So the rows of a group, which lie one behind the other, are one tall matrix over the shared pages, and every sequence goes on by
// itself behind them.  All of it is one row of (unit, page) steps, shared ones first, that is cut into parts as equal in time as the two kinds allow:
// a plan, made once for all layers of a step, says which workgroup starts where.  A launch does the parts, a second one adds up what they
// left, by rows.
#include "sfmp_attention.h"

namespace sfmp {
namespace {

constexpr int32_t kPlanMagic = 0x5348504C;
constexpr int kMostOwnRows = 64;     // rows of an entry and key head
constexpr int kPlanThreads = 1024, kShareThreads = 256;
// Rows and heads whose partial results four wavefronts add up: 2 sequences of 16000 tokens, 64 of them, 20.8 us a layer against 25.8 with one; 64 of
// 8000, 2048 of them, 41.1 against 38.7.
constexpr int kMostJoinedByAll = 512;
constexpr int kJoinAhead = 8;        // partial results that are asked for at a time
constexpr int kSlotsHeld = 1024;     // entries of a group whose slots are held in LDS
constexpr int kMostSlices = 64;      // workgroups that compare the tables of a group
constexpr int kPlanHeadBytes = 256;
constexpr int64_t kMostSteps = 1 << 29;  // of each kind: with the room behind units they have to fit 32 bits
constexpr int kMostParts = 2048;     // of shared pages, and of own ones: wavefronts of a launch

// Numbers that a plan and the calls that use it have to agree in.
struct PlanKey {
  int32_t magic, batch, rows, groups, heads, q_heads, dim, max_rows, max_tokens, window, sinks, pages, sequences, table_pages, with_slots, with_starts;
};
struct PlanHead {
  PlanKey key;
  int32_t usable;            // 0: more units than the workspace holds (group starts that do not ascend)
  int32_t group_workgroups;  // those that work on shared pages: the first ones
  int32_t of_group_part, of_own_part;   // steps of a part
};
// Rows of a group over the pages that its sequences share.
struct GroupPlan {
  int32_t slot;              // of a sequence that holds the pages
  int32_t common;            // pages that all rows of the group see in full (but for a window)
  int32_t row0, n;
  int32_t first, last;       // smallest and largest position
  int32_t each, tiles;       // places of the pages that the rows see, tiles of rows
  int32_t before, unit0;     // steps and units of the groups before
  int32_t whole;             // full pages of the shortest sequence
  int32_t unused[5];
};
// A sequence behind them.
struct EntryPlan {
  KvEntry entry;
  int32_t group;             // -1: none
  int32_t common;
  int32_t each, tiles, before, unit0;
  int32_t unused[6];
};
// Where a part starts: group or entry, its unit (head * tiles + tile), place of the page; its steps (0: none), and of the group or entry what the
// part needs, so that it does not have to wait for that as well.
struct PartStart {
  int32_t of, unit, first, left;
  int32_t common, each, tiles, unit0;
  int32_t slot, length, row0, n;   // (length: of an entry)
  int32_t from, to;                // (smallest and largest position: of a group)
  int32_t unused[2];
};
// What joins the results of a row, for the same reason: of its group and of its own pages the steps and units before, places of the pages
// (0: none), tiles, and its first row of products.
struct RowPlan {
  int32_t there;                   // 0: a row of no entry
  int32_t group_row, group_before, group_unit0;
  int32_t group_each, group_tiles, own_each, own_tiles;
  int32_t own_row, own_before, own_unit0, unused;
};
static_assert(sizeof(PlanKey) == 64 && sizeof(PlanHead) <= kPlanHeadBytes && sizeof(GroupPlan) == 64 && sizeof(EntryPlan) == 64 && sizeof(PartStart) == 64 &&
                  sizeof(RowPlan) == 48, "");

// How a call runs.
struct SharedForm {
  bool shared;               // else as sfmp_kv_attention
  int tile_rows;             // of a unit of shared pages: 16, 32 (a wavefront's) or kPromptRows (a workgroup's)
  int workgroups;
  int group_parts, own_parts;        // at most
  float least_of_steps, least_of_unit;   // steps of a part at least: the root of these times all steps and the longest unit's pages
  int own_least;                     // steps of a part
  int64_t group_units, own_units;    // at most
  float group_cost;                  // time of a step of shared pages, in that of an own one of a wavefront
};

struct SharedArgs {
  PlanHead* head;
  GroupPlan* groups;
  EntryPlan* entries;
  RowPlan* row_plans;        // [rows]
  int32_t* row_at;           // [rows] its position
  PartStart* group_starts;   // by workgroup, or by wavefront where a wavefront takes a part
  PartStart* own_starts;     // by wavefront
  PlanKey key;
  const int32_t* group_start;
  int32_t* prefix;           // or null
  int32_t* differs;          // [groups][slices] the first place that a workgroup found to differ
  int32_t slices;
  int32_t tile_rows, workgroups, own_least;
  float least_of_steps, least_of_unit;
  int64_t group_units, own_units;
  float group_cost;
  // partial results: o [slot][rows][dim], m and l [slot][rows][2].  The slot of a unit in a part is the sum of their numbers: from one
  // (part, unit) to the next in the row of steps, one of them or both go up by one.
  float* group_o;
  float* group_ml;
  float* own_o;
  float* own_ml;
};

// ---- the plan ------------------------------------------------------------------------------------------------------

// Pages of the list that are shared ones, and those that are not.
template <bool SINKS>
__device__ __forceinline__ PageRange<SINKS> pages_below(const PageRange<SINKS>& p, int common) {
  if constexpr (SINKS) {
    const int edge = min(p.edge, common), w0 = p.edge + p.gap, w1 = min(p.end + p.gap, common);
    return PageRange<true>{0, edge + max(w1 - w0, 0), edge, w0 - edge};
  } else {
    return PageRange<false>{p.begin, max(min(p.end, common), p.begin)};
  }
}
template <bool SINKS>
__device__ __forceinline__ PageRange<SINKS> pages_from(const PageRange<SINKS>& p, int common) {
  if constexpr (SINKS) {
    const int s0 = min(p.edge, common), w0 = max(p.edge + p.gap, common), w1 = p.end + p.gap;
    return PageRange<true>{s0, p.edge + max(w1 - w0, 0), p.edge, w0 - p.edge};
  } else {
    const int begin = max(p.begin, common);
    return PageRange<false>{begin, max(p.end, begin)};
  }
}
template <bool SINKS>
__device__ __forceinline__ PageRange<SINKS> pages_of_group(const AttentionArgs& a, const GroupPlan& g) {
  if (g.n < 1 || g.common < 1) return no_pages<SINKS>();
  return pages_below<SINKS>(pages_seen<SINKS>(a, g.first, g.last), g.common);
}
template <bool SINKS>
__device__ __forceinline__ PageRange<SINKS> own_pages(const AttentionArgs& a, const KvEntry& e, int common) {
  return pages_from<SINKS>(pages_of_entry<SINKS>(a, e), common);
}

// Least and largest values over the threads of a workgroup.
struct Extent {
  int whole, seen, first, last, end_row;
};

// What there is of a group, and where its sequences' rows of the page table differ first: gridDim.y workgroups per group take every gridDim.y-th run
// of 64 places.  The last ones take the entries that belong to no group.  Bound by chains of loads (group, slot, length, table): 3.8 us for 4
// sequences, 5.4 us for 64 over 33000 tokens (26 us with a workgroup per group).
__global__ __launch_bounds__(kShareThreads) void share_groups_kernel(AttentionArgs a, SharedArgs p) {
  __shared__ Extent all;
  __shared__ int differs;
  __shared__ int32_t slots[kSlotsHeld];
  const int g = blockIdx.x, tid = threadIdx.x, batch = a.v.batch, groups = p.key.groups;
  const bool none = g == groups, writes = blockIdx.y == 0;
  auto start_of = [&](int i) { return min(max(p.group_start[i], 0), batch); };
  // (none: the entries before the first group and behind the last)
  const int from = none ? 0 : start_of(g), to = none ? start_of(0) : max(start_of(g + 1), from);
  const int from2 = none ? start_of(groups) : to, to2 = none ? batch : to;
  if (tid == 0) all = Extent{kMaxTablePages, kMaxTablePages, INT32_MAX, INT32_MIN, 0}, differs = INT32_MAX;
  __syncthreads();
  if (p.entries)
    for (int i = (g * gridDim.y + blockIdx.y) * kShareThreads + tid; i < a.v.rows; i += gridDim.x * gridDim.y * kShareThreads) p.row_plans[i].there = 0;
  Extent mine{kMaxTablePages, kMaxTablePages, INT32_MAX, INT32_MIN, 0};
  for (int side = 0; side < 2; ++side) {
    const int begin = side ? max(from2, to) : from, end = side ? to2 : to;
    for (int b = begin + tid; b < end; b += kShareThreads) {
      const KvEntry e = kv_entry(a.v, b);
      if (b - begin < kSlotsHeld) slots[b - begin] = e.slot;
      mine.whole = min(mine.whole, e.length / kPage);
      if (e.n > 0) {
        mine.seen = min(mine.seen, max(e.length - e.n + 1, 0) / kPage);
        mine.first = min(mine.first, e.length - e.n), mine.last = max(mine.last, e.length - 1);
        mine.end_row = max(mine.end_row, e.row0 + e.n);
      }
      if (!writes || !p.entries) continue;
      for (int i = 0; i < e.n; ++i) p.row_at[e.row0 + i] = e.length - e.n + i;
      p.entries[b].entry = e;
      p.entries[b].group = none ? -1 : g;
    }
  }
  if (none) return;
  // (over the wavefront first: atomics of all lanes at one address take a turn for each)
#pragma unroll
  for (int s = 1; s < 64; s *= 2) {
    mine.whole = min(mine.whole, __shfl_xor(mine.whole, s)), mine.seen = min(mine.seen, __shfl_xor(mine.seen, s));
    mine.first = min(mine.first, __shfl_xor(mine.first, s)), mine.last = max(mine.last, __shfl_xor(mine.last, s));
    mine.end_row = max(mine.end_row, __shfl_xor(mine.end_row, s));
  }
  if (tid % 64 == 0) {
    atomicMin(&all.whole, mine.whole), atomicMin(&all.seen, mine.seen), atomicMin(&all.first, mine.first);
    atomicMax(&all.last, mine.last), atomicMax(&all.end_row, mine.end_row);
  }
  __syncthreads();
  const int32_t first_row = from < to ? kv_entry(a.v, from).row0 : 0;  // (asked for before the tables)
  const int most = from < to ? min(all.whole, a.v.table_pages) : 0;
  // (a sequence outside of the table has no page: then `most` is 0)
  auto id_of = [&](int slot, int place) { return a.v.table[(int64_t)slot * a.v.table_pages + place]; };
  constexpr int kRows = kShareThreads / 64, kAhead = 8;
  const int row = tid / 64, rows = to - from, near = min(rows, kSlotsHeld);
  int found = INT32_MAX;
  for (int place = blockIdx.y * 64 + tid % 64; place < most; place += gridDim.y * 64) {
    const int32_t id = id_of(slots[0], place);
    bool other = false;
    for (int b = row; b < near; b += kRows * kAhead) {
      int32_t x[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) x[u] = id_of(slots[min(b + u * kRows, near - 1)], place);
#pragma unroll
      for (int u = 0; u < kAhead; ++u) other |= x[u] != id;
    }
    for (int b = near + row; b < rows; b += kRows) other |= id_of(a.v.slots ? a.v.slots[from + b] : from + b, place) != id;
    if (other) {  // (the first of this thread's)
      found = place;
      break;
    }
  }
#pragma unroll
  for (int s = 1; s < 64; s *= 2) found = min(found, __shfl_xor(found, s));
  if (tid % 64 == 0 && found != INT32_MAX) atomicMin(&differs, found);
  __syncthreads();
  if (tid) return;
  if (!p.entries && gridDim.y == 1) {  // (all that is asked for)
    p.prefix[g] = min(most, differs) * kPage;
    return;
  }
  p.differs[g * p.slices + blockIdx.y] = differs;
  if (!writes) return;
  GroupPlan plan{};
  plan.row0 = plan.n = 0;
  if (from < to) {
    plan.slot = slots[0], plan.row0 = first_row;
    plan.n = (int)min((int64_t)max(all.end_row - first_row, 0), (int64_t)(to - from) * a.v.max_rows);
  }
  plan.first = all.first, plan.last = all.last;
  plan.whole = most, plan.common = to - from < 2 ? 0 : min(all.seen, a.max_pages);  // (as far as the tables agree)
  p.groups[g] = plan;
}

// Sums over the threads before this one, and over all of them (added to `all`).
struct Sums {
  int64_t group_steps, group_units, own_steps, own_units;
  __device__ __forceinline__ Sums& operator+=(const Sums& x) {
    group_steps += x.group_steps, group_units += x.group_units, own_steps += x.own_steps, own_units += x.own_units;
    return *this;
  }
};
__device__ __forceinline__ Sums scan_before(const Sums& x, Sums* sums, Sums* all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  Sums up = x;
#pragma unroll
  for (int s = 1; s < 64; s *= 2) {
    const Sums y{__shfl_up(up.group_steps, s), __shfl_up(up.group_units, s), __shfl_up(up.own_steps, s), __shfl_up(up.own_units, s)};
    if (lane >= s) up += y;
  }
  __syncthreads();
  if (lane == 63) sums[wave] = up;
  __syncthreads();
  Sums before = *all;
#pragma unroll 4  // (registers)
  for (int w = 0; w < kPlanThreads / 64; ++w) {
    const Sums y = sums[w];
    if (w < wave) before += y;
    *all += y;
  }
  before += up;
  return Sums{before.group_steps - x.group_steps, before.group_units - x.group_units, before.own_steps - x.own_steps, before.own_units - x.own_units};
}

// The row of steps and its parts: one workgroup, prefix sums over groups and entries, a binary search for each part.  What it finds of the first
// 1024 groups and entries it holds in LDS: it is bound by its chain of loads and barriers (11 us, whether 8 groups or 1), once for all layers.
template <bool SINKS>
__global__ __launch_bounds__(kPlanThreads) void share_parts_kernel(AttentionArgs a, SharedArgs p) {
  __shared__ Sums sums[kPlanThreads / 64];
  __shared__ int longest_of_all;
  __shared__ int32_t group_before[kPlanThreads], group_each[kPlanThreads], group_common[kPlanThreads];
  __shared__ int32_t group_tiles[kPlanThreads], group_unit0[kPlanThreads], group_row0[kPlanThreads], group_n[kPlanThreads];
  __shared__ int32_t own_before[kPlanThreads], own_each[kPlanThreads], own_common[kPlanThreads], own_tiles[kPlanThreads], own_unit0[kPlanThreads];
  __shared__ int32_t prefix[kPlanThreads];
  const int tid = threadIdx.x, lane = tid & 63, heads = a.v.heads, groups = p.key.groups;
  // (what is found is written at the end: a barrier behind a write waits for it.  Not where LDS does not hold it)
  const bool far = groups > kPlanThreads || a.v.batch > kPlanThreads;
  // (of the first entries: asked for before the groups)
  KvEntry near_entry{-1, 0, 0, 0};
  int near_group = -1;
  if (p.entries && tid < a.v.batch) near_entry = p.entries[tid].entry, near_group = p.entries[tid].group;
  // Where the tables of a group differ first: a wavefront per group, or a thread, where there are few numbers of each
  const bool alone = p.slices <= 4;
  for (int g = alone ? tid : tid >> 6; g < groups; g += alone ? kPlanThreads : kPlanThreads / 64) {
    GroupPlan plan = p.groups[g];
    int differs = INT32_MAX;
    for (int y = alone ? 0 : lane; y < p.slices; y += alone ? 1 : 64) differs = min(differs, p.differs[g * p.slices + y]);
    if (!alone)
#pragma unroll
      for (int s = 1; s < 64; s *= 2) differs = min(differs, __shfl_xor(differs, s));
    if (!alone && lane) continue;
    const int found = min(plan.whole, differs);
    if (far || !p.entries) {
      if (p.prefix) p.prefix[g] = found * kPage;
    } else {
      prefix[g] = found * kPage;
    }
    if (!p.entries) continue;
    plan.common = min(plan.common, found);
    const PageRange<SINKS> pages = pages_of_group<SINKS>(a, plan);
    plan.each = pages.end - pages.begin;
    plan.tiles = plan.each ? (plan.n * a.group + p.tile_rows - 1) >> __builtin_ctz(p.tile_rows) : 0;  // (below 2^31: choose_shared)
    if (far) p.groups[g].common = plan.common, p.groups[g].each = plan.each, p.groups[g].tiles = plan.tiles;
    if (g < kPlanThreads) group_common[g] = plan.common, group_each[g] = plan.each, group_tiles[g] = plan.tiles, group_row0[g] = plan.row0, group_n[g] = plan.n;
  }
  if (!p.entries) return;
  if (tid == 0) longest_of_all = 1;
  __syncthreads();
  Sums all{};
  int longest = 1, near_each = 0, near_tiles = 0, near_before = 0, near_unit0 = 0;
  for (int base = 0; base < max(groups, a.v.batch); base += kPlanThreads) {
    const int i = base + tid;
    Sums x{};
    if (i < groups) {
      const int each = base ? p.groups[i].each : group_each[i];
      x.group_units = (int64_t)(base ? p.groups[i].tiles : group_tiles[i]) * heads, x.group_steps = x.group_units * each;
      if (x.group_units) longest = max(longest, each);
    }
    if (i < a.v.batch) {
      KvEntry e = near_entry;
      int g = near_group;
      if (base) e = p.entries[i].entry, g = p.entries[i].group;
      const int common = g < 0 ? 0 : g < kPlanThreads ? group_common[g] : p.groups[g].common;
      const PageRange<SINKS> pages = own_pages<SINKS>(a, e, common);
      const int each = pages.end - pages.begin, tiles = each > 0 ? tiles_of_entry(a, e, 16) : 0;
      x.own_units = (int64_t)tiles * heads, x.own_steps = x.own_units * each;
      if (far) p.entries[i].common = common, p.entries[i].each = each, p.entries[i].tiles = tiles;
      if (base == 0) own_each[tid] = near_each = each, own_tiles[tid] = near_tiles = tiles, own_common[tid] = common;
    }
    const Sums before = scan_before(x, sums, &all);
    if (far && i < groups) p.groups[i].before = (int)before.group_steps, p.groups[i].unit0 = (int)before.group_units;
    if (far && i < a.v.batch) p.entries[i].before = (int)before.own_steps, p.entries[i].unit0 = (int)before.own_units;
    if (base) continue;
    group_before[tid] = (int)before.group_steps, group_unit0[tid] = (int)before.group_units;
    own_before[tid] = near_before = (int)before.own_steps, own_unit0[tid] = near_unit0 = (int)before.own_units;
  }
#pragma unroll
  for (int s = 1; s < 64; s *= 2) longest = max(longest, __shfl_xor(longest, s));
  if (lane == 0) atomicMax(&longest_of_all, longest);
  __syncthreads();
  longest = longest_of_all;
  const bool usable = all.group_units <= p.group_units && all.own_units <= p.own_units && all.group_steps <= kMostSteps && all.own_steps <= kMostSteps;
  const uint32_t group_steps = usable ? (uint32_t)all.group_steps : 0, own_steps = usable ? (uint32_t)all.own_steps : 0;
  // Workgroups for shared pages and for own ones, in the proportion of their times
  const bool wide = p.tile_rows == kPromptRows;
  const float group_time = (float)group_steps * p.group_cost, own_time = (float)own_steps;
  int group_workgroups = 0;
  if (group_steps) {
    group_workgroups = own_steps ? (int)((float)p.workgroups * group_time / (group_time + own_time) + 0.5f) : p.workgroups;
    group_workgroups = min(max(group_workgroups, 1), p.workgroups - (own_steps > 0));
  }
  const int group_parts = max(wide ? group_workgroups : 4 * group_workgroups, 1), own_parts = max(4 * (p.workgroups - group_workgroups), 1);
  // (parts of x steps: x steps after one another, what all parts leave to be written and read, and the longest unit's parts to be added up one after the
  // other; the least together at the root)
  const int least = max((int)(sqrtf((float)group_steps * p.least_of_steps + (float)longest * p.least_of_unit)), 1);
  // Parts that begin with a unit, each unit cut by itself, where there are parts enough for the units' last ones to be shorter: one that goes on in the next
  // unit loads rows anew and leaves two results (64 sequences behind 8192 tokens, 39.6 us a layer with parts of 7 of a unit's 128 pages, 33.7 with 8)
  const bool whole_units = groups <= 64 && all.group_units * 4 <= group_parts;
  const uint32_t inner_parts = whole_units ? group_parts - (uint32_t)all.group_units : group_parts;
  const int of_group = max((int)((group_steps + inner_parts - 1) / inner_parts), least);
  auto row_of_steps = [&](int each) { return whole_units ? (each + of_group - 1) / of_group * of_group : each; };
  uint32_t group_end = group_steps;
  if (whole_units) {  // (every wavefront for itself)
    const uint32_t steps = lane < groups ? (uint32_t)group_tiles[lane] * heads * row_of_steps(group_each[lane]) : 0;
    uint32_t up = steps;
#pragma unroll
    for (int s = 1; s < 64; s *= 2) {
      const uint32_t x = __shfl_up(up, s);
      if (lane >= s) up += x;
    }
    group_end = usable ? (uint32_t)__builtin_amdgcn_readlane((int)up, 63) : 0;
    if (tid < groups) {
      group_before[tid] = (int)(up - steps);
      if (far) p.groups[tid].before = (int)(up - steps);
    }
  }
  __syncthreads();
  const int of_own = max((int)((own_steps + own_parts - 1) / own_parts), p.own_least);
  for (int b = tid; b < a.v.batch; b += kPlanThreads) {
    KvEntry e = near_entry;
    int g = near_group;
    RowPlan r{};
    r.there = 1, r.own_each = near_each, r.own_tiles = near_tiles, r.own_before = near_before, r.own_unit0 = near_unit0;
    if (b >= kPlanThreads) {
      const EntryPlan own = p.entries[b];
      e = own.entry, g = own.group;
      r.own_each = own.each, r.own_tiles = own.tiles, r.own_before = own.before, r.own_unit0 = own.unit0;
    }
    int first_row = 0, rows = 0;
    if (g >= kPlanThreads) {
      const GroupPlan plan = p.groups[g];
      first_row = plan.row0, rows = plan.n;
      r.group_before = plan.before, r.group_unit0 = plan.unit0, r.group_each = plan.each, r.group_tiles = plan.tiles;
    } else if (g >= 0) {
      first_row = group_row0[g], rows = group_n[g];
      r.group_before = group_before[g], r.group_unit0 = group_unit0[g], r.group_each = group_each[g], r.group_tiles = group_tiles[g];
    }
    const int each_of_group = row_of_steps(r.group_each);
    for (int i = 0; i < e.n; ++i) {
      const int row = e.row0 + i - first_row;
      r.group_each = row >= 0 && row < rows ? each_of_group : 0;  // (with the room behind its last part)
      r.group_row = row * a.group, r.own_row = i * a.group;
      p.row_plans[e.row0 + i] = r;
    }
  }
  if (tid < 16) reinterpret_cast<int32_t*>(&p.head->key)[tid] = reinterpret_cast<const int32_t*>(&p.key)[tid];
  if (tid == 0) {
    p.head->usable = usable;
    p.head->group_workgroups = group_workgroups;
    p.head->of_group_part = of_group, p.head->of_own_part = of_own;
  }
  // The last of n groups or entries that starts at or before a step
  auto holder = [&](int at, int n, const int32_t* held, auto before_of) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      ((mid < kPlanThreads ? held[mid] : before_of(mid)) <= at ? lo : hi) = mid;
    }
    return lo;
  };
  for (int part = tid; part < (wide ? group_workgroups : 4 * group_workgroups); part += kPlanThreads) {
    if ((int64_t)part * of_group >= group_end) {
      p.group_starts[part].left = 0;
      continue;
    }
    const int at = part * of_group, g = holder(at, groups, group_before, [&](int i) { return p.groups[i].before; });
    GroupPlan plan = p.groups[g];
    if (g < kPlanThreads)
      plan.common = group_common[g], plan.each = group_each[g], plan.tiles = group_tiles[g], plan.before = group_before[g], plan.unit0 = group_unit0[g];
    const int each = max(row_of_steps(plan.each), 1), inside = at - plan.before, first = inside % each;
    p.group_starts[part] = PartStart{g,         inside / each, first,         whole_units ? min(of_group, plan.each - first) : min(of_group, (int)group_steps - at),
                                     plan.common, plan.each,   plan.tiles,    plan.unit0,
                                     plan.slot,   0,           plan.row0,     plan.n,
                                     plan.first,  plan.last};
  }
  for (int part = tid; part < 4 * (p.workgroups - group_workgroups); part += kPlanThreads) {
    PartStart& start = p.own_starts[4 * group_workgroups + part];
    if ((int64_t)part * of_own >= own_steps) {
      start.left = 0;
      continue;
    }
    const int at = part * of_own, b = holder(at, a.v.batch, own_before, [&](int i) { return p.entries[i].before; });
    EntryPlan plan = p.entries[b];
    if (b < kPlanThreads)
      plan.common = own_common[b], plan.each = own_each[b], plan.tiles = own_tiles[b], plan.before = own_before[b], plan.unit0 = own_unit0[b];
    const int each = max(plan.each, 1), inside = at - plan.before;
    start = PartStart{b,               inside / each,     inside % each,   min(of_own, (int)own_steps - at),
                      plan.common,     plan.each,         plan.tiles,      plan.unit0,
                      plan.entry.slot, plan.entry.length, plan.entry.row0, plan.entry.n};
  }
  if (far) return;
  if (tid < groups) {
    GroupPlan& plan = p.groups[tid];
    plan.common = group_common[tid], plan.each = group_each[tid], plan.tiles = group_tiles[tid];
    plan.before = group_before[tid], plan.unit0 = group_unit0[tid];
    if (p.prefix) p.prefix[tid] = prefix[tid];
  }
  if (tid < a.v.batch) {
    EntryPlan& plan = p.entries[tid];
    plan.common = own_common[tid], plan.each = near_each, plan.tiles = near_tiles, plan.before = near_before, plan.unit0 = near_unit0;
  }
}

// ---- attention -----------------------------------------------------------------------------------------------------

// The rows of a group as those of one entry.
struct GroupRows {
  int32_t slot, length, row0, n, first, last;
  const int32_t* at;
};
__device__ __forceinline__ int position_of(const GroupRows& e, int token) { return e.at[e.row0 + token]; }
__device__ __forceinline__ int least_position(const GroupRows& e, int, int) { return e.first; }
__device__ __forceinline__ int largest_position(const GroupRows& e, int, int) { return e.last; }

// Whether the plan is one for this call (the same in all lanes).
__device__ __forceinline__ bool plan_fits(const SharedArgs& p) {
  const int lane = threadIdx.x & 63;
  const bool other = lane < 16 && reinterpret_cast<const int32_t*>(p.head)[lane] != reinterpret_cast<const int32_t*>(&p.key)[lane];
  return !__any(other);
}

template <int D, int NT>
__device__ __forceinline__ void store_partial_rows(float* o, float* ml, int rows, const Partial<D, NT>& p) {
  const int i16 = threadIdx.x & 15, g = (threadIdx.x & 63) >> 4;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int row = 16 * nt + i16;
    if (row >= rows) continue;
    if (g == 0) ml[2 * row] = p.m[nt], ml[2 * row + 1] = p.l[nt];
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) *reinterpret_cast<floatx4*>(o + row * D + 16 * dt + 4 * g) = p.o[nt][dt];
  }
}

// NTP: tiles of 16 rows that a wavefront takes over shared pages; 0: a workgroup takes 128.
template <int D, int NTP>
constexpr int kWavesPerSimd = D == 256 || (D == 128 && NTP == 2) ? 1 : 2;

// The first workgroups take parts of shared pages, the others of own ones, in the proportion of their times.  A unit of shared pages is a tile of the
// group's rows and a key head: 16 or 32 rows of a wavefront by 16-row products, where a group has few, so that its bytes bound it, or 128 rows of
// a workgroup by 32-row products with the pages in LDS, as in prompts, where matrix instructions and the softmax
// between them do.  8 key heads of 128 dims: 64 sequences behind 32768 tokens (256 rows of a key head) 55 us, of which its products at the rate of a large
// one are 27; 8 groups of 8 sequences behind 1000 to 7000 tokens (32 rows of a key head) 24.7 us for 89 MB, 3.6 TB/s.
template <int D, int FMT, int NTP, bool SINKS>
__global__ __launch_bounds__(256, (kWavesPerSimd<D, NTP>)) void attend_shared_kernel(AttentionArgs a, SharedArgs p) {
  extern __shared__ __align__(16) uint8_t lds[];
  if (!plan_fits(p)) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int group_workgroups = p.head->group_workgroups, by_wave = blockIdx.x * 4 + wave, of_group = NTP ? by_wave : blockIdx.x;
  // (both kinds at once: a part waits for one load, not for two)
  const PartStart group_start = p.group_starts[of_group], own_start = p.own_starts[by_wave];
  asm volatile("" ::"s"(group_workgroups), "s"(group_start.left), "s"(own_start.left));
  if ((int)blockIdx.x < group_workgroups) {
    const int part = of_group;
    const PartStart& start = group_start;
    int left = start.left, g = start.of, unit = start.unit, first = start.first;
    GroupPlan plan{};
    plan.slot = start.slot, plan.common = start.common, plan.row0 = start.row0, plan.n = start.n, plan.first = start.from, plan.last = start.to;
    plan.each = start.each, plan.tiles = start.tiles, plan.unit0 = start.unit0;
    while (left > 0) {
      if (unit >= plan.tiles * a.v.heads) {  // the next group
        if (++g >= p.key.groups) break;
        plan = p.groups[g];
        unit = 0;
        continue;
      }
      const GroupRows e{plan.slot, plan.common * kPage, plan.row0, plan.n, plan.first, plan.last, p.row_at};
      const PageRange<SINKS> pages = pages_of_group<SINKS>(a, plan);
      const int head = unit / plan.tiles, tile = unit - head * plan.tiles, count = min(plan.each - first, left);
      const int64_t slot = (int64_t)part + plan.unit0 + unit;
      if constexpr (NTP > 0) {
        Rows<D, NTP> r;
        load_rows<D, NTP>(a, e, head, tile, r);
        Partial<D, NTP> sums;
        accumulate<D, FMT, NTP, SINKS>(a, e, head, pages, pages.begin + first, pages.begin + first + count, r, sums);
        store_partial_rows<D, NTP>(p.group_o + slot * (16 * NTP * D), p.group_ml + slot * (16 * NTP * 2), plan.n * a.group - tile * 16 * NTP, sums);
      } else {
        PromptSums<D> s;
        attend_tile<D, FMT, 1, SINKS>(a, e, head, tile, pages, pages.begin + first, pages.begin + first + count, reinterpret_cast<PromptTile<D>*>(lds), s);
        const int lane = threadIdx.x & 63, row = wave * 32 + (lane & 31), h = lane >> 5;
        if (row < plan.n * a.group - tile * kPromptRows) {
          float* const o = p.group_o + (slot * kPromptRows + row) * D + 4 * h;
#pragma unroll
          for (int x = 0; x < D / 32; ++x)
#pragma unroll
            for (int q = 0; q < 4; ++q)
              *reinterpret_cast<floatx4*>(o + 32 * x + 8 * q) = floatx4{s.o[x][4 * q], s.o[x][4 * q + 1], s.o[x][4 * q + 2], s.o[x][4 * q + 3]};
          float* const ml = p.group_ml + (slot * kPromptRows + row) * 2;
          if (h == 0) ml[0] = s.m, ml[1] = s.l;
        }
      }
      left -= count;
      first = 0;
      ++unit;
    }
    return;
  }
  const int part = by_wave - 4 * group_workgroups;
  const PartStart& start = own_start;
  int left = start.left, b = start.of, unit = start.unit, first = start.first;
  EntryPlan plan{};
  plan.entry = KvEntry{start.slot, start.length, start.row0, start.n};
  plan.common = start.common, plan.each = start.each, plan.tiles = start.tiles, plan.unit0 = start.unit0;
  while (left > 0) {
    if (unit >= plan.tiles * a.v.heads) {
      if (++b >= a.v.batch) break;
      plan = p.entries[b];
      unit = 0;
      continue;
    }
    const KvEntry e = plan.entry;
    const PageRange<SINKS> pages = own_pages<SINKS>(a, e, plan.common);
    const int head = unit / plan.tiles, tile = unit - head * plan.tiles, count = min(plan.each - first, left);
    const int64_t slot = (int64_t)part + plan.unit0 + unit;
    Rows<D, 1> r;
    load_rows<D, 1>(a, e, head, tile, r);
    Partial<D, 1> sums;
    accumulate<D, FMT, 1, SINKS>(a, e, head, pages, pages.begin + first, pages.begin + first + count, r, sums);
    store_partial_rows<D, 1>(p.own_o + slot * (16 * D), p.own_ml + slot * 32, e.n * a.group - tile * 16, sums);
    left -= count;
    first = 0;
    ++unit;
  }
}

// Adds up the partial results of a row and head: of the parts of its group's unit, then of its own one's.  J wavefronts share them (4 where there are few rows
// and heads, 1 for many).  Bound by its chain of loads (row, m and l, o; partial results are asked for 8 at a time): 5.9 us for 64 rows of 32 heads behind 1000 to
// 7000 tokens, 8.0 behind 32768.
template <int D, int J>
__global__ __launch_bounds__(256) void join_shared_kernel(AttentionArgs a, SharedArgs p) {
  constexpr int EACH = D / 64;
  typedef float Dims __attribute__((ext_vector_type(EACH)));
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), at = J == 4 ? blockIdx.x : blockIdx.x * 4 + wave;
  if (at >= a.v.rows * a.q_heads) return;
  const int row = at / a.q_heads, q_head = at - row * a.q_heads, head = q_head / a.group, h = q_head - head * a.group;
  const RowPlan plan = p.row_plans[row];  // (a place of the plan, whatever it holds)
  const int of_group_part = p.head->of_group_part, of_own_part = p.head->of_own_part, usable = p.head->usable;
  if (!plan_fits(p) || !usable || !plan.there) return;
  // parts [0, group_parts) and [group_parts, parts)
  int group_parts = 0, own_parts = 0;
  int64_t group_at = 0, own_at = 0;  // rows of the first partial results; those of the next parts lie a slot further each
  if (plan.group_each > 0) {
    const int i = plan.group_row + h, tile = i >> __builtin_ctz(p.tile_rows), unit = head * plan.group_tiles + tile;
    const int from = plan.group_before + unit * plan.group_each, w0 = from / of_group_part;
    group_parts = (from + plan.group_each - 1) / of_group_part - w0 + 1;
    group_at = ((int64_t)w0 + plan.group_unit0 + unit) * p.tile_rows + i - tile * p.tile_rows;
  }
  if (plan.own_each > 0) {
    const int i = plan.own_row + h, tile = i / 16, unit = head * plan.own_tiles + tile;
    const int from = plan.own_before + unit * plan.own_each, w0 = from / of_own_part;
    own_parts = (from + plan.own_each - 1) / of_own_part - w0 + 1;
    own_at = ((int64_t)w0 + plan.own_unit0 + unit) * 16 + i - tile * 16;
  }
  const int all = group_parts + own_parts, share = (all + J - 1) / J, first = J == 1 ? 0 : min(wave * share, all);
  const int parts = J == 1 ? all : min(share, all - first);  // (of this wavefront: from `first` on)
  auto ml_of = [&](int i) {
    i += first;
    return i < group_parts ? p.group_ml + 2 * (group_at + (int64_t)i * p.tile_rows) : p.own_ml + 2 * (own_at + (int64_t)(i - group_parts) * 16);
  };
  Dims x[kJoinAhead];
  auto ask = [&](int from) {
#pragma unroll
    for (int u = 0; u < kJoinAhead; ++u) {
      const int part = first + min(from + u, parts - 1);
      const float* const row_o =
          part < group_parts ? p.group_o + (group_at + (int64_t)part * p.tile_rows) * D : p.own_o + (own_at + (int64_t)(part - group_parts) * 16) * D;
      x[u] = reinterpret_cast<const Dims*>(row_o)[lane];
    }
  };
  if (parts > 0) ask(0);  // (while m and l are on their way)
  float m = -INFINITY;
  for (int i = lane; i < parts; i += 64) m = fmaxf(m, ml_of(i)[0]);
#pragma unroll
  for (int s = 1; s < 64; s *= 2) m = fmaxf(m, __shfl_xor(m, s));
  float base = m == -INFINITY ? 0.0f : m;
  Dims o = 0.0f;
  float l = 0.0f;
  for (int i0 = 0; i0 < parts; i0 += 64) {
    float f = 0.0f, li = 0.0f;
    if (i0 + lane < parts) {
      const float* const ml = ml_of(i0 + lane);
      f = __builtin_amdgcn_exp2f(ml[0] - base);
      li = ml[1] * f;
    }
#pragma unroll
    for (int s = 1; s < 64; s *= 2) li += __shfl_xor(li, s);
    l += li;
    const int count = min(parts - i0, 64);
    for (int i = 0; i < count; i += kJoinAhead) {
      if (i0 + i) ask(i0 + i);
#pragma unroll
      for (int u = 0; u < kJoinAhead; ++u) {
        const bool there = i + u < count;  // (the same in all lanes; what is asked for beyond is not used)
        const float fi = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), (i + u) & 63));
#pragma unroll
        for (int j = 0; j < EACH; ++j) o[j] = there ? __builtin_fmaf(x[u][j], fi, o[j]) : o[j];
      }
    }
  }
  if constexpr (J > 1) {
    __shared__ Dims wave_o[J][64];
    __shared__ float wave_m[J], wave_l[J];
    wave_o[wave][lane] = o;
    if (lane == 0) wave_m[wave] = m, wave_l[wave] = l;
    __syncthreads();
    if (wave) return;
    m = -INFINITY;
#pragma unroll
    for (int w = 0; w < J; ++w) m = fmaxf(m, wave_m[w]);
    base = m == -INFINITY ? 0.0f : m;
    o = 0.0f, l = 0.0f;
#pragma unroll
    for (int w = 0; w < J; ++w) {
      const float f = __builtin_amdgcn_exp2f(wave_m[w] - base);
      l += wave_l[w] * f;
#pragma unroll
      for (int j = 0; j < EACH; ++j) o[j] = __builtin_fmaf(wave_o[w][lane][j], f, o[j]);
    }
  }
  const bool empty = m == -INFINITY && l == 0.0f;  // (not where every score is a NaN)
  const float inverse = empty ? 0.0f : 1.0f / l;
  uint16_t* const dst = a.O + (int64_t)row * a.o_stride + (int64_t)q_head * D + lane * EACH;
  typedef uint16_t Bits __attribute__((ext_vector_type(EACH)));
  Bits bits;
#pragma unroll
  for (int j = 0; j < EACH; ++j) bits[j] = bits_of(o[j] * inverse, a.bf16);
  *reinterpret_cast<Bits*>(dst) = bits;
  if (a.lse && lane == 0) a.lse[at] = empty ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// ---- launches ------------------------------------------------------------------------------------------------------

// Time (us) that sharing takes at least: plan aside, two launches, a page of the group's rows and one of each sequence's own.
// Over 168 combinations of head layout, sequences and tokens (1 x 2 to 8 x 8 behind 300 to 5000) the rule costs 0.9 % against the faster way, at most
// 1.3 times.  8 heads of 128 dims: 16 sequences of 1000 tokens 12.2 us alone against 14.2 shared, 64 of 8000 102 against 33.
double least_time(int dim, int tile_rows, int64_t own_units) {
  const double start = tile_rows == kPromptRows ? (dim == 64 ? 13.0 : dim == 128 ? 16.0 : 27.0) : dim == 256 ? 13.5 : 11.5;
  return start + 0.012 * (double)own_units;
}

// Rows of a unit of shared pages: 32 of a wavefront while a key head has up to 64 (16 with 256 dims), else 128 of a workgroup.  16 sequences of
// 8000 tokens, 64 rows of 8 heads of 128 dims: 22.6 us a layer against 23.9; with 128 rows 27.7 against 31.9 there, but 48 against 43 for 32
// sequences of 500 to 4000 tokens behind 16384.  A step of 128 rows takes 2.2 to 3 times an own one of a wavefront (64 sequences behind 32768
// tokens: 73 us with 3, 79 with 4.5, 100 with 7).
SharedForm choose_shared(int dim, int heads, int group, int batch, int rows, int groups, int max_rows, int max_tokens, int window, int sinks) {
  SharedForm f{};
  const int64_t own_rows = (int64_t)max_rows * group, mean = groups ? ((int64_t)rows * group + groups - 1) / groups : 0;
  if (groups < 1 || groups >= batch || max_rows < 1 || own_rows > kMostOwnRows || (int64_t)rows * heads * group > INT32_MAX) return f;
  f.own_units = (int64_t)batch * ((own_rows + 15) / 16) * heads;
  f.tile_rows = dim == 256 ? (mean <= 64 ? 16 : kPromptRows) : mean <= 64 ? 32 : kPromptRows;
  // (what the host knows of how much is shared: no more than the pages of all but one sequence of each group.  The others are left to be read, which
  // takes a plan some 1.4 times as long.  2 to 96 sequences of 1000 to 8000 tokens in 1 group to as many as sequences but one, that share all but a page:
  // 1.4 % over the faster way, at most 1.33 times, and 5.8 % and 1.48 without this term (64 sequences of 3000 tokens in 63 groups 94 us a layer against 73,
  // 32 of 3000 in 24 36 against 26).  Where groups share nothing, which only the device finds out: 2.0 %, at most 1.27 times)
  const AttentionForm alone = choose_form(dim, heads, group, batch, rows, max_rows, max_tokens, window, window ? sinks : 0);
  const double beyond_start = alone.time - parts_start(alone.waves) - 3.0, left = 1.4 * groups / batch * (beyond_start > 0.0 ? beyond_start : 0.0);
  f.shared = alone.time - left > least_time(dim, f.tile_rows, f.own_units);
  if (!f.shared) return f;
  f.workgroups = dim == 256 || (dim == 128 && f.tile_rows == 32) ? 256 : 512;
  f.group_parts = f.tile_rows == kPromptRows ? f.workgroups : 4 * f.workgroups;
  f.own_parts = 4 * f.workgroups;
  // (us: a part leaves 8 bytes of a row and dimension at 4 TB/s, takes 0.09 to be added up by one wavefront, and for a step 1.5, 4
  // or 1.7; over 168 combinations 1.1 % less than the root of the longest unit's pages alone, 64 sequences behind 8192 tokens 34 against 38)
  const float step = f.tile_rows == kPromptRows ? (dim == 256 ? 4.0f : 1.5f) : 1.7f, rows_left = (float)(mean < f.tile_rows ? mean : f.tile_rows);
  f.least_of_steps = rows_left * (float)dim * 8.0f / 4e6f / step;
  f.least_of_unit = 0.09f / step / ((int64_t)rows * heads * group <= kMostJoinedByAll ? 4.0f : 1.0f);
  f.own_least = 1;
  f.group_units = ((int64_t)batch * own_rows / f.tile_rows + groups) * heads;
  f.group_cost = f.tile_rows == kPromptRows ? 3.0f : 1.0f;
  const int64_t units = f.group_units > f.own_units ? f.group_units : f.own_units;
  f.shared = units * ((max_tokens + kPage - 1) / kPage) <= kMostSteps;
  return f;
}

// Workgroups that compare the tables of a group: some thousand of all groups.
int slices_of(int groups, int table_pages) {
  const int want = (table_pages + 63) / 64, some = 1024 / (groups + 1);
  const int most = some < kMostSlices ? some : kMostSlices;
  return want < most ? want : most > 1 ? most : 1;
}

// Bytes of plan and workspace that a call needs.
int64_t plan_bytes(bool shared, int batch, int rows, int groups) {
  if (!shared) return kPlanHeadBytes;  // (not used)
  return kPlanHeadBytes + (int64_t)groups * sizeof(GroupPlan) + round_up_256((groups > 1024 ? groups : 1024) * (int64_t)4) +
         (int64_t)batch * sizeof(EntryPlan) + 2 * kMostParts * sizeof(PartStart) + round_up_256(rows * (int64_t)sizeof(RowPlan)) + round_up_256((int64_t)rows * 4);
}
int64_t shared_workspace(const SharedForm& f, int dim) {
  return ((f.group_parts + f.group_units) * f.tile_rows + (f.own_parts + f.own_units) * 16) * (dim + 2) * 4;
}
// ... and those that every call of no more entries, rows and groups can do with: the rows of partial results are the most with large tiles.
int64_t shared_workspace_up_to(int dim, int heads, int group, int batch, int groups, int max_rows) {
  if (batch < 2 || groups < 1 || max_rows < 1 || group > kMostOwnRows) return 0;
  const int64_t own_rows = (int64_t)max_rows * group < kMostOwnRows ? max_rows * group : kMostOwnRows;
  SharedForm f{};
  f.tile_rows = kPromptRows;
  f.group_parts = 512, f.own_parts = kMostParts;
  f.group_units = ((int64_t)batch * own_rows / kPromptRows + 1 + (groups < batch ? groups : batch - 1)) * heads;
  f.own_units = (int64_t)batch * ((own_rows + 15) / 16) * heads;
  return shared_workspace(f, dim);
}

SharedArgs shared_args(const SharedForm& f, const sfmp_kv_layout_t* layout, const sfmp_kv_tables_t* tables, const sfmp_kv_batch_t* batch,
                       const int32_t* group_start, int groups, int q_heads, int max_tokens, int window, int sinks, void* plan) {
  SharedArgs p{};
  uint8_t* at = (uint8_t*)plan;
  auto take = [&](int64_t bytes) { uint8_t* const x = at; at += bytes; return x; };
  p.slices = 1;
  if (f.shared) {
    p.head = (PlanHead*)take(kPlanHeadBytes);
    p.groups = (GroupPlan*)take((int64_t)groups * sizeof(GroupPlan));
    p.differs = (int32_t*)take(round_up_256((groups > 1024 ? groups : 1024) * (int64_t)4));
    p.slices = slices_of(groups, tables->table_pages);
    p.entries = (EntryPlan*)take((int64_t)batch->batch * sizeof(EntryPlan));
    p.group_starts = (PartStart*)take(kMostParts * sizeof(PartStart));
    p.own_starts = (PartStart*)take(kMostParts * sizeof(PartStart));
    p.row_plans = (RowPlan*)take(round_up_256(batch->rows * (int64_t)sizeof(RowPlan)));
    p.row_at = (int32_t*)take(round_up_256((int64_t)batch->rows * 4));
  }
  p.key = PlanKey{kPlanMagic, batch->batch, batch->rows, groups, layout->kv_heads, q_heads, layout->head_dim, batch->max_rows, max_tokens, window, sinks,
                  layout->pages, tables->sequences, tables->table_pages, batch->slots_dev != nullptr, batch->row_start_dev != nullptr};
  p.group_start = group_start;
  p.tile_rows = f.tile_rows, p.workgroups = f.workgroups, p.least_of_steps = f.least_of_steps, p.least_of_unit = f.least_of_unit, p.own_least = f.own_least;
  p.group_units = f.group_units, p.own_units = f.own_units, p.group_cost = f.group_cost;
  return p;
}

template <int D, int FMT, int NTP, bool SINKS>
int launch_shared(const AttentionArgs& a, const SharedArgs& p, hipStream_t stream) {
  constexpr int lds = NTP ? 0 : 2 * (int)sizeof(PromptTile<D>);
  static_assert(kWavesPerSimd<D, NTP> * lds <= 160 * 1024, "LDS of a compute unit");
  if (lds)
    if (int e = allow_full_lds((const void*)attend_shared_kernel<D, FMT, NTP, SINKS>, "attend_shared_kernel")) return e;
  attend_shared_kernel<D, FMT, NTP, SINKS><<<p.workgroups, 256, lds, stream>>>(a, p);
  const int64_t joins = (int64_t)a.v.rows * a.q_heads;  // (below 2^31: choose_shared)
  if (joins <= kMostJoinedByAll)
    join_shared_kernel<D, 4><<<(uint32_t)joins, 256, 0, stream>>>(a, p);
  else
    join_shared_kernel<D, 1><<<(uint32_t)((joins + 3) / 4), 256, 0, stream>>>(a, p);
  return kv_launched("attend_shared_kernel");
}

template <int D, int FMT, bool SINKS>
int launch_shared_rows(const AttentionArgs& a, const SharedArgs& p, hipStream_t stream) {
  if (p.tile_rows == kPromptRows) return launch_shared<D, FMT, 0, SINKS>(a, p, stream);
  return launch_shared<D, FMT, (D == 256 ? 1 : 2), SINKS>(a, p, stream);
}

template <bool SINKS>
int launch_shared_kind(int dim, int format, const AttentionArgs& a, const SharedArgs& p, hipStream_t stream) {
  if (format == SFMP_KV_INT8) {
    if (dim == 64) return launch_shared_rows<64, SFMP_KV_INT8, SINKS>(a, p, stream);
    if (dim == 128) return launch_shared_rows<128, SFMP_KV_INT8, SINKS>(a, p, stream);
    return launch_shared_rows<256, SFMP_KV_INT8, SINKS>(a, p, stream);
  }
  if (dim == 64) return launch_shared_rows<64, SFMP_KV_FP8, SINKS>(a, p, stream);
  if (dim == 128) return launch_shared_rows<128, SFMP_KV_FP8, SINKS>(a, p, stream);
  return launch_shared_rows<256, SFMP_KV_FP8, SINKS>(a, p, stream);
}

// What both calls take and check.
int check_shared(const sfmp_kv_layout_t* layout, const sfmp_kv_batch_t* batch, const int32_t* group_start, int32_t groups, int32_t q_heads,
                 int32_t max_tokens, int32_t window, int32_t sinks) {
  if (int e = check_sizes(layout, batch->batch, batch->rows, q_heads, batch->max_rows, max_tokens)) return e;
  if (groups < 0 || groups > 65535 || window < 0 || sinks < 0) return SFMP_ERR_SHAPE;
  if (groups && !group_start) return SFMP_ERR_NULL;
  if (!kv_aligned(group_start, 4)) return SFMP_ERR_ALIGN;
  return SFMP_OK;
}

int check_group_sizes(const sfmp_kv_layout_t* layout, int32_t batch, int32_t rows, int32_t groups, int32_t q_heads, int32_t max_rows, int32_t max_tokens) {
  if (int e = check_sizes(layout, batch, rows, q_heads, max_rows, max_tokens)) return e;
  return groups < 0 || groups > 65535 ? SFMP_ERR_SHAPE : SFMP_OK;
}

}  // namespace
}  // namespace sfmp

using namespace sfmp;

extern "C" int sfmp_kv_share_plan(const sfmp_kv_layout_t* layout, int32_t batch, int32_t rows, int32_t groups, int32_t q_heads, int32_t max_rows,
                                  int32_t max_tokens, int64_t* bytes) {
  if (!bytes) return SFMP_ERR_NULL;
  if (int e = check_group_sizes(layout, batch, rows, groups, q_heads, max_rows, max_tokens)) return e;
  *bytes = round_up_256(plan_bytes(batch > 1 && groups > 0, batch, rows, groups));
  return SFMP_OK;
}

extern "C" int sfmp_kv_attention_shared_workspace(const sfmp_kv_layout_t* layout, int32_t batch, int32_t rows, int32_t groups, int32_t q_heads,
                                                  int32_t max_rows, int32_t max_tokens, int64_t* bytes) {
  if (!bytes) return SFMP_ERR_NULL;
  if (int e = check_group_sizes(layout, batch, rows, groups, q_heads, max_rows, max_tokens)) return e;
  if (int e = sfmp_kv_attention_workspace(layout, batch, rows, q_heads, max_rows, max_tokens, bytes)) return e;
  const int64_t shared = round_up_256(shared_workspace_up_to(layout->head_dim, layout->kv_heads, q_heads / layout->kv_heads, batch, groups, max_rows));
  if (shared > *bytes) *bytes = shared;
  return SFMP_OK;
}

extern "C" int sfmp_kv_share(const sfmp_kv_layout_t* layout, const sfmp_kv_tables_t* tables, const sfmp_kv_batch_t* batch,
                             const int32_t* group_start_dev, int32_t groups, int32_t q_heads, int32_t max_tokens, int32_t window, int32_t sinks,
                             int32_t* prefix_dev, void* plan_dev, int64_t plan_bytes_given, void* hip_stream) {
  AttentionArgs a{};
  // (no pool is touched: any aligned address does for the check)
  if (int e = make_kv_view(layout, 0, (const void*)(uintptr_t)256, (const float*)(uintptr_t)256, tables, batch, &a.v)) return e;
  if (int e = check_shared(layout, batch, group_start_dev, groups, q_heads, max_tokens, window, sinks)) return e;
  if (!kv_aligned(prefix_dev, 4)) return SFMP_ERR_ALIGN;
  const SharedForm f = choose_shared(layout->head_dim, layout->kv_heads, q_heads / layout->kv_heads, batch->batch, batch->rows, groups, batch->max_rows,
                                     max_tokens, window, sinks);
  if (!plan_dev || !kv_aligned(plan_dev, 256) || plan_bytes_given < plan_bytes(f.shared, batch->batch, batch->rows, groups)) return SFMP_ERR_WORKSPACE;
  if (groups == 0 || (!f.shared && !prefix_dev)) return SFMP_OK;
  a.group = q_heads / layout->kv_heads;
  a.window = window >= tables->table_pages * kPage ? 0 : window;
  a.sinks = sinks;
  a.max_pages = (max_tokens + kPage - 1) / kPage;
  SharedArgs p = shared_args(f, layout, tables, batch, group_start_dev, groups, q_heads, max_tokens, window, sinks, plan_dev);
  p.prefix = prefix_dev;
  const hipStream_t stream = (hipStream_t)hip_stream;
  const bool sinks_seen = a.window && a.sinks;
  share_groups_kernel<<<dim3(groups + 1, p.slices), kShareThreads, 0, stream>>>(a, p);
  if (f.shared) (sinks_seen ? share_parts_kernel<true> : share_parts_kernel<false>)<<<1, kPlanThreads, 0, stream>>>(a, p);
  return kv_launched("share_groups_kernel");
}

extern "C" int sfmp_kv_attention_shared(const sfmp_kv_layout_t* layout, int32_t layer, const void* codes_dev, const float* scales_dev,
                                        const sfmp_kv_tables_t* tables, const sfmp_kv_batch_t* batch, const int32_t* group_start_dev, int32_t groups,
                                        const void* Q_dev, int32_t q_heads, int32_t dtype, int64_t q_stride, int32_t max_tokens, int32_t window,
                                        int32_t sinks, float scale, void* O_dev, int64_t o_stride, float* lse_dev, const void* plan_dev,
                                        int64_t plan_bytes_given, void* workspace_dev, int64_t workspace_bytes, void* hip_stream) {
  AttentionArgs a;
  if (int e = make_kv_view(layout, layer, codes_dev, scales_dev, tables, batch, &a.v)) return e;
  if (int e = check_shared(layout, batch, group_start_dev, groups, q_heads, max_tokens, window, sinks)) return e;
  const SharedForm f = choose_shared(layout->head_dim, layout->kv_heads, q_heads / layout->kv_heads, batch->batch, batch->rows, groups, batch->max_rows,
                                     max_tokens, window, sinks);
  if (!plan_dev || !kv_aligned(plan_dev, 256) || plan_bytes_given < plan_bytes(f.shared, batch->batch, batch->rows, groups)) return SFMP_ERR_WORKSPACE;
  if (!f.shared)
    return sfmp_kv_attention_sinks(layout, layer, codes_dev, scales_dev, tables, batch, Q_dev, q_heads, dtype, q_stride, max_tokens, window, sinks, scale,
                                   O_dev, o_stride, lse_dev, workspace_dev, workspace_bytes, hip_stream);
  if (int e = check_attention(layout, tables, batch, Q_dev, q_heads, dtype, q_stride, max_tokens, window, sinks, scale, O_dev, o_stride, lse_dev, &a)) return e;
  if (batch->rows == 0 || batch->batch == 0) return SFMP_OK;
  if (!workspace_dev || !kv_aligned(workspace_dev, 256) || workspace_bytes < shared_workspace(f, layout->head_dim)) return SFMP_ERR_WORKSPACE;
  SharedArgs p = shared_args(f, layout, tables, batch, group_start_dev, groups, q_heads, max_tokens, window, sinks, (void*)plan_dev);
  const int64_t group_rows = (f.group_parts + f.group_units) * f.tile_rows, own_rows = (f.own_parts + f.own_units) * 16;
  p.group_o = (float*)workspace_dev;
  p.own_o = p.group_o + group_rows * layout->head_dim;
  p.group_ml = p.own_o + own_rows * layout->head_dim;
  p.own_ml = p.group_ml + group_rows * 2;
  const hipStream_t stream = (hipStream_t)hip_stream;
  if (a.window && a.sinks) return launch_shared_kind<true>(layout->head_dim, layout->format, a, p, stream);
  return launch_shared_kind<false>(layout->head_dim, layout->format, a, p, stream);
}
