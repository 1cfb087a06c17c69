// Pages of the 8-bit cache: reserving (with copy on write), forking, freeing, compacting, reordering.
#include "sfmp_kv.h"

using namespace sfmp;

namespace {

constexpr int kThreads = 1024;  // of the kernels that one workgroup runs alone

// Workspace of the calls that hand out or move pages.
struct PagesWorkspace {
  int32_t* copies;     // [0]: pages to copy
  int32_t* source;     // [pages + SFMP_KV_MAX_BATCH] (a copied page may have several sources in turn, never more than it has holders)
  int32_t* target;
  int32_t* moved;      // [pages]: free pages that are handed out; or the new number of every page
};
int64_t ints_of(const sfmp_kv_layout_t* L) { return ((int64_t)L->pages + SFMP_KV_MAX_BATCH + 63) / 64 * 64; }
PagesWorkspace split(const sfmp_kv_layout_t* L, void* p) {
  int32_t* const at = (int32_t*)p;
  const int64_t n = ints_of(L);
  return PagesWorkspace{at, at + 64, at + 64 + n, at + 64 + 2 * n};
}

// Sum over the threads before this one, and over all of them (a workgroup of kThreads; `sums` holds 17 numbers).
__device__ __forceinline__ int scan_before(int x, int* sums, int* all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int up = x;
#pragma unroll
  for (int s = 1; s < 64; s *= 2) {
    const int y = __shfl_up(up, s);
    if (lane >= s) up += y;
  }
  __syncthreads();  // (the sums of an earlier call have been read)
  if (lane == 63) sums[wave] = up;
  __syncthreads();
  if (wave == 0) {
    int y = lane < kThreads / 64 ? sums[lane] : 0;
#pragma unroll
    for (int s = 1; s < kThreads / 64; s *= 2) {
      const int z = __shfl_up(y, s);
      if (lane >= s) y += z;
    }
    if (lane < kThreads / 64) sums[lane] = y;
  }
  __syncthreads();
  *all = sums[kThreads / 64 - 1];
  return up - x + (wave ? sums[wave - 1] : 0);
}

// One workgroup, thread i = sequence i of the call: pages wanted and free pages found are matched by prefix sums, so that the result is
// that of the calls one after the other.  Bound by a chain of loads (slot, length, table entry, refs) and some ten barriers: 16 forked
// sequences in a pool of 256 pages 6 us.  More workgroups would need another launch for the order, which costs as much.
__global__ __launch_bounds__(kThreads) void reserve_kernel(sfmp_kv_tables_t t, int32_t pages, const int32_t* slots,
                                                           const int32_t* counts, int32_t n, int32_t* status,
                                                           PagesWorkspace ws) {
  __shared__ int sums[17];
  __shared__ int shared_last[kThreads];  // the last page of a sequence, if partly filled and held by others too
  __shared__ int start[kThreads], place_of[kThreads], slot_of[kThreads];
  __shared__ int copies, bad;
  const int i = threadIdx.x;
  if (i == 0) copies = bad = 0;
  __syncthreads();
  int slot = 0, length = 0, add = 0, have = 0, more = 0, last = -1, holders = 0;
  if (i < n) {
    slot = slots[i];
    add = counts ? counts[i] : 1;
    if ((uint32_t)slot >= (uint32_t)t.sequences || add < 0 || add > t.table_pages * kPage) {
      bad = 1;
      slot = add = 0;
    } else {
      length = min(max(t.lengths_dev[slot], 0), t.table_pages * kPage);
      have = (length + kPage - 1) / kPage;
      const int need = (int)(((int64_t)length + add + kPage - 1) / kPage);
      more = need - have;
      if (need > t.table_pages) bad = 1;
      if (length % kPage && add > 0) {
        const int id = t.page_table_dev[(int64_t)slot * t.table_pages + have - 1];
        if ((uint32_t)id < (uint32_t)pages) {
          holders = t.refs_dev[id];
          if (holders > 1) last = id;
        }
      }
    }
  }
  shared_last[i] = last;
  __syncthreads();
  bool copy = false;
  if (last >= 0) {  // those before it in the call that hold the same page have left it by then
    int earlier = 0;
    for (int j = 0; j < i; ++j) earlier += shared_last[j] == last;
    copy = holders - earlier > 1;
  }
  int total = 0;
  const int mine = scan_before(more + copy, sums, &total);
  start[i] = mine;
  place_of[i] = have - copy;  // (the copy takes the place of the shared page)
  slot_of[i] = slot;
  __syncthreads();
  if (bad) {
    if (i == 0) *status = -1, *ws.copies = 0;
    return;
  }
  // the free pages of lowest number, as many as are wanted
  int found = 0;
  for (int base = 0; base < pages && found < total; base += 4 * kThreads) {
    const int at = base + 4 * i;
    bool free[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) free[j] = at + j < pages && t.refs_dev[at + j] <= 0;
    int all;
    int k = found + scan_before(free[0] + free[1] + free[2] + free[3], sums, &all);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (free[j]) {
        if (k < total) ws.moved[k] = at + j;
        ++k;
      }
    found += all;
  }
  if (found < total) {
    if (i == 0) *status = total - found, *ws.copies = 0;
    return;
  }
  __threadfence_block();
  __syncthreads();
  if (copy) {
    const int k = atomicAdd(&copies, 1);
    ws.source[k] = last;
    ws.target[k] = ws.moved[mine];
    atomicSub(&t.refs_dev[last], 1);
  }
  for (int k = i; k < total; k += kThreads) {
    int lo = 0, hi = n;  // the last sequence that starts at or before k
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      (start[mid] <= k ? lo : hi) = mid;
    }
    const int page = ws.moved[k];
    t.page_table_dev[(int64_t)slot_of[lo] * t.table_pages + place_of[lo] + (k - start[lo])] = page;
    t.refs_dev[page] = 1;
  }
  if (i < n) t.lengths_dev[slot] = length + add;
  __syncthreads();
  if (i == 0) *status = 0, *ws.copies = copies;
}

// One workgroup: which pages move where, refs renumbered (prefix sums over the live and the free pages; 1024 pages 4 us).
__global__ __launch_bounds__(kThreads) void compact_kernel(sfmp_kv_tables_t t, int32_t pages, int32_t* status,
                                                           PagesWorkspace ws) {
  __shared__ int sums[17];
  int live = 0;
  for (int at = threadIdx.x; at < pages; at += kThreads) live += t.refs_dev[at] > 0;
  int n_live;
  scan_before(live, sums, &n_live);
  int holes = 0, movers = 0;
  for (int base = 0; base < pages; base += kThreads) {
    const int at = base + threadIdx.x;
    const bool held = at < pages && t.refs_dev[at] > 0;
    const bool hole = at < n_live && !held, mover = at >= n_live && held;
    int all;
    // (both counts of a thread in one scan: at most kThreads of each)
    const int before = scan_before((int)hole | (int)mover << 16, sums, &all);
    if (hole) ws.target[holes + (before & 0xFFFF)] = at;
    if (mover) ws.source[movers + (before >> 16)] = at;
    if (at < pages) ws.moved[at] = at;
    holes += all & 0xFFFF;
    movers += all >> 16;
  }
  __threadfence_block();
  __syncthreads();
  for (int k = threadIdx.x; k < movers; k += kThreads) {
    const int from = ws.source[k], to = ws.target[k];
    ws.moved[from] = to;
    t.refs_dev[to] = t.refs_dev[from];
    t.refs_dev[from] = 0;
  }
  if (threadIdx.x == 0) *status = n_live, *ws.copies = movers;
}

// Copies pages source[k] -> target[k] of every layer, in pieces of 16 KiB; the workgroups from `copiers` on renumber the
// rows of the page table.  Bound by HBM: 257 MB read and written in 52.6 us, 4.9 TB/s, what a plain copy of 2 GiB reaches; 16 copied
// pages of 8 layers (34 MB, with the launch's start and end) 6 us.
__global__ __launch_bounds__(256) void move_pages_kernel(uint8_t* codes, float* scales, int64_t page_bytes, int32_t heads,
                                                         int32_t pages, int32_t layers, PagesWorkspace ws, int32_t copiers,
                                                         sfmp_kv_tables_t t) {
  if ((int)blockIdx.x >= copiers) {
    for (int s = blockIdx.x - copiers; s < t.sequences; s += gridDim.x - copiers) {
      const int held = (min(max(t.lengths_dev[s], 0), t.table_pages * kPage) + kPage - 1) / kPage;
      int32_t* const row = t.page_table_dev + (int64_t)s * t.table_pages;
      for (int j = threadIdx.x; j < held; j += 256) {
        const int id = row[j];
        if ((uint32_t)id < (uint32_t)pages) row[j] = ws.moved[id];
      }
    }
    return;
  }
  constexpr int kPiece = 16384;
  const int pieces = (int)((page_bytes + kPiece - 1) / kPiece);
  const int64_t items = (int64_t)*ws.copies * layers * pieces;
  for (int64_t item = blockIdx.x; item < items; item += copiers) {
    const int piece = (int)(item % pieces);
    const int64_t rest = item / pieces;
    const int k = (int)(rest / layers);
    const int64_t layer = rest % layers;
    const int64_t from = layer * pages + ws.source[k], to = layer * pages + ws.target[k];
    const int64_t at = (int64_t)piece * kPiece;
    const u32x4* const src = reinterpret_cast<const u32x4*>(codes + from * page_bytes + at);
    u32x4* const dst = reinterpret_cast<u32x4*>(codes + to * page_bytes + at);
    const int vectors = (int)(min((int64_t)kPiece, page_bytes - at) / 16);
    u32x4 x[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if ((int)threadIdx.x + 256 * j < vectors) x[j] = src[threadIdx.x + 256 * j];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if ((int)threadIdx.x + 256 * j < vectors) dst[threadIdx.x + 256 * j] = x[j];
    if (piece == 0)
      for (int j = threadIdx.x; j < 2 * heads; j += 256) scales[to * 2 * heads + j] = scales[from * 2 * heads + j];
  }
}

// One workgroup per child: its row of the table becomes its parent's, the holders of the pages are counted up (16 children of 16 pages
// 3.0 us: a launch and two dependent loads).
__global__ __launch_bounds__(256) void fork_kernel(sfmp_kv_tables_t t, int32_t pages, const int32_t* parents,
                                                   const int32_t* children) {
  const int parent = parents[blockIdx.x], child = children[blockIdx.x];
  if ((uint32_t)parent >= (uint32_t)t.sequences || (uint32_t)child >= (uint32_t)t.sequences || parent == child) return;
  const int length = min(max(t.lengths_dev[parent], 0), t.table_pages * kPage);
  for (int j = threadIdx.x; j < (length + kPage - 1) / kPage; j += 256) {
    const int id = t.page_table_dev[(int64_t)parent * t.table_pages + j];
    t.page_table_dev[(int64_t)child * t.table_pages + j] = id;
    if ((uint32_t)id < (uint32_t)pages) atomicAdd(&t.refs_dev[id], 1);
  }
  if (threadIdx.x == 0) t.lengths_dev[child] = length;
}

// One workgroup per sequence: pages behind what is kept lose a holder (16 sequences 2.6 us).
__global__ __launch_bounds__(256) void free_kernel(sfmp_kv_tables_t t, int32_t pages, const int32_t* slots,
                                                   const int32_t* keep) {
  const int slot = slots[blockIdx.x];
  if ((uint32_t)slot >= (uint32_t)t.sequences) return;
  const int length = min(max(t.lengths_dev[slot], 0), t.table_pages * kPage);
  const int kept = keep ? min(max(keep[blockIdx.x], 0), length) : 0;
  for (int j = (kept + kPage - 1) / kPage + threadIdx.x; j < (length + kPage - 1) / kPage; j += 256) {
    const int id = t.page_table_dev[(int64_t)slot * t.table_pages + j];
    if ((uint32_t)id < (uint32_t)pages) atomicSub(&t.refs_dev[id], 1);
  }
  __syncthreads();  // (every thread has read the length)
  if (threadIdx.x == 0) t.lengths_dev[slot] = kept;
}

// Sequences that become what their parents were.  Places of the page table do not depend on each other: a workgroup takes 2^bits of them for all
// sequences, through LDS, so that rows can be exchanged in place.  Holders change where a place gets another page; sums of whole numbers,
// the same in every order.  Lengths are read by all workgroups: they change here only where there is one (`last`), else in a launch of their own.
// Bound by its chain of loads (slot, length, place, holder): 4 sequences of 1024 tokens 2.3 us, 512 of 200 to 8190 6.6 and 1.4 us.
__global__ __launch_bounds__(kThreads) void reorder_kernel(sfmp_kv_tables_t t, int32_t pages, const int32_t* slots, const int32_t* parents, int32_t n,
                                                           int32_t bits, int32_t last) {
  extern __shared__ int32_t lds[];
  int32_t *const slot_of = lds, *const held_of = slot_of + kThreads, *const parent_of = held_of + kThreads;
  int32_t *const some = parent_of + kThreads, *const ids = some + 1;  // (whether a sequence has a page here); [n][2^bits]
  const int i = threadIdx.x, first = blockIdx.x << bits, all = n << bits;
  int length = 0, parent = -1;
  if (i == 0) *some = 0;
  __syncthreads();
  if (i < n) {
    int slot = slots[i];
    parent = parents[i];
    if ((uint32_t)slot >= (uint32_t)t.sequences) slot = -1;
    if ((uint32_t)parent >= (uint32_t)n) parent = -1;
    length = slot < 0 ? 0 : min(max(t.lengths_dev[slot], 0), t.table_pages * kPage);
    slot_of[i] = slot, held_of[i] = (length + kPage - 1) / kPage, parent_of[i] = parent;
  }
  if ((length + kPage - 1) / kPage > first) *some = 1;
  __syncthreads();
  if (*some) {
    auto place_of = [&](int x) { return first + (x & ((1 << bits) - 1)); };
#pragma unroll 4
    for (int x = i; x < all; x += kThreads) {
      const int y = x >> bits, place = place_of(x);
      if (place < held_of[y]) ids[x] = t.page_table_dev[(int64_t)slot_of[y] * t.table_pages + place];
    }
    __syncthreads();
#pragma unroll 4
    for (int x = i; x < all; x += kThreads) {
      const int y = x >> bits, place = place_of(x), from = parent_of[y];
      if (slot_of[y] < 0 || from == y) continue;
      const bool had = place < held_of[y], gets = from >= 0 && place < held_of[from];
      const int old = had ? ids[x] : -1, now = gets ? ids[(from << bits) + place - first] : -1;
      if (gets && !(had && old == now)) t.page_table_dev[(int64_t)slot_of[y] * t.table_pages + place] = now;
      if (old == now) continue;
      if ((uint32_t)old < (uint32_t)pages) atomicSub(&t.refs_dev[old], 1);
      if ((uint32_t)now < (uint32_t)pages) atomicAdd(&t.refs_dev[now], 1);
    }
  }
  if (!last) return;
  __syncthreads();
  held_of[i] = length;
  __syncthreads();
  if (i < n && slot_of[i] >= 0) t.lengths_dev[slot_of[i]] = parent >= 0 ? held_of[parent] : 0;
}
__global__ __launch_bounds__(kThreads) void reorder_lengths_kernel(sfmp_kv_tables_t t, const int32_t* slots, const int32_t* parents, int32_t n) {
  __shared__ int32_t length_of[kThreads];
  const int i = threadIdx.x, slot = i < n ? slots[i] : -1, parent = i < n ? parents[i] : -1;
  const bool there = (uint32_t)slot < (uint32_t)t.sequences;
  length_of[i] = there ? min(max(t.lengths_dev[slot], 0), t.table_pages * kPage) : 0;
  __syncthreads();
  if (there) t.lengths_dev[slot] = (uint32_t)parent < (uint32_t)n ? length_of[parent] : 0;
}

int check_pages_call(const sfmp_kv_layout_t* L, const sfmp_kv_tables_t* t) {
  if (int e = check_kv_layout(L)) return e;
  return check_kv_tables(t, true);
}

int check_pages_workspace(const sfmp_kv_layout_t* L, const void* workspace, int64_t bytes) {
  int64_t need = 0;
  if (int e = sfmp_kv_pages_workspace(L, &need)) return e;
  return workspace && kv_aligned(workspace, 256) && bytes >= need ? SFMP_OK : SFMP_ERR_WORKSPACE;
}

int launch_move(const sfmp_kv_layout_t* L, void* codes, float* scales, const sfmp_kv_tables_t* t, const PagesWorkspace& ws,
                int64_t most, bool renumber, void* stream) {
  const int64_t pieces = (L->page_bytes + 16383) / 16384 * L->layers * most;
  const int copiers = (int)(pieces < 2048 ? pieces : 2048);
  const int rows = renumber ? (t->sequences < 1024 ? t->sequences : 1024) : 0;
  move_pages_kernel<<<copiers + rows, 256, 0, (hipStream_t)stream>>>((uint8_t*)codes, scales, L->page_bytes, L->kv_heads,
                                                                     L->pages, L->layers, ws, copiers, *t);
  return kv_launched("move_pages_kernel");
}

}  // namespace

extern "C" int sfmp_kv_pages_workspace(const sfmp_kv_layout_t* layout, int64_t* bytes) {
  if (!bytes) return SFMP_ERR_NULL;
  if (int e = check_kv_layout(layout)) return e;
  *bytes = round_up_256((64 + 3 * ints_of(layout)) * 4);
  return SFMP_OK;
}

extern "C" int sfmp_kv_reserve(const sfmp_kv_layout_t* layout, void* codes_dev, float* scales_dev,
                               const sfmp_kv_tables_t* tables, const int32_t* slots_dev, const int32_t* counts_dev,
                               int32_t n, int32_t* status_dev, void* workspace_dev, int64_t workspace_bytes,
                               void* hip_stream) {
  if (int e = check_pages_call(layout, tables)) return e;
  if (int e = check_kv_buffers(codes_dev, scales_dev)) return e;
  if (n < 0 || n > SFMP_KV_MAX_BATCH) return SFMP_ERR_SHAPE;
  if (!status_dev || (n && !slots_dev)) return SFMP_ERR_NULL;
  if (!kv_aligned(slots_dev, 4) || !kv_aligned(counts_dev, 4) || !kv_aligned(status_dev, 4)) return SFMP_ERR_ALIGN;
  if (int e = check_pages_workspace(layout, workspace_dev, workspace_bytes)) return e;
  const PagesWorkspace ws = split(layout, workspace_dev);
  reserve_kernel<<<1, kThreads, 0, (hipStream_t)hip_stream>>>(*tables, layout->pages, slots_dev, counts_dev, n, status_dev, ws);
  if (int e = kv_launched("reserve_kernel")) return e;
  return n ? launch_move(layout, codes_dev, scales_dev, tables, ws, n, false, hip_stream) : SFMP_OK;
}

extern "C" int sfmp_kv_fork(const sfmp_kv_layout_t* layout, const sfmp_kv_tables_t* tables, const int32_t* parents_dev,
                            const int32_t* children_dev, int32_t n, void* hip_stream) {
  if (int e = check_pages_call(layout, tables)) return e;
  if (n < 0) return SFMP_ERR_SHAPE;
  if (n == 0) return SFMP_OK;
  if (!parents_dev || !children_dev) return SFMP_ERR_NULL;
  if (!kv_aligned(parents_dev, 4) || !kv_aligned(children_dev, 4)) return SFMP_ERR_ALIGN;
  fork_kernel<<<n, 256, 0, (hipStream_t)hip_stream>>>(*tables, layout->pages, parents_dev, children_dev);
  return kv_launched("fork_kernel");
}

extern "C" int sfmp_kv_free(const sfmp_kv_layout_t* layout, const sfmp_kv_tables_t* tables, const int32_t* slots_dev,
                            const int32_t* keep_dev, int32_t n, void* hip_stream) {
  if (int e = check_pages_call(layout, tables)) return e;
  if (n < 0) return SFMP_ERR_SHAPE;
  if (n == 0) return SFMP_OK;
  if (!slots_dev) return SFMP_ERR_NULL;
  if (!kv_aligned(slots_dev, 4) || !kv_aligned(keep_dev, 4)) return SFMP_ERR_ALIGN;
  free_kernel<<<n, 256, 0, (hipStream_t)hip_stream>>>(*tables, layout->pages, slots_dev, keep_dev);
  return kv_launched("free_kernel");
}

extern "C" int sfmp_kv_compact(const sfmp_kv_layout_t* layout, void* codes_dev, float* scales_dev,
                               const sfmp_kv_tables_t* tables, int32_t* status_dev, void* workspace_dev,
                               int64_t workspace_bytes, void* hip_stream) {
  if (int e = check_pages_call(layout, tables)) return e;
  if (int e = check_kv_buffers(codes_dev, scales_dev)) return e;
  if (!status_dev) return SFMP_ERR_NULL;
  if (!kv_aligned(status_dev, 4)) return SFMP_ERR_ALIGN;
  if (int e = check_pages_workspace(layout, workspace_dev, workspace_bytes)) return e;
  const PagesWorkspace ws = split(layout, workspace_dev);
  compact_kernel<<<1, kThreads, 0, (hipStream_t)hip_stream>>>(*tables, layout->pages, status_dev, ws);
  if (int e = kv_launched("compact_kernel")) return e;
  return launch_move(layout, codes_dev, scales_dev, tables, ws, (layout->pages + 1) / 2, true, hip_stream);
}

extern "C" int sfmp_kv_reorder(const sfmp_kv_layout_t* layout, const sfmp_kv_tables_t* tables, const int32_t* slots_dev,
                               const int32_t* parents_dev, int32_t n, void* hip_stream) {
  if (int e = check_pages_call(layout, tables)) return e;
  if (n < 0 || n > SFMP_KV_MAX_BATCH) return SFMP_ERR_SHAPE;
  if (n == 0) return SFMP_OK;
  if (!slots_dev || !parents_dev) return SFMP_ERR_NULL;
  if (!kv_aligned(slots_dev, 4) || !kv_aligned(parents_dev, 4)) return SFMP_ERR_ALIGN;
  const hipStream_t stream = (hipStream_t)hip_stream;
  int bits = 0;
  while (1 << bits < tables->table_pages) ++bits;
  // (one workgroup and no second launch, or 8 places to a workgroup)
  const bool one = (int64_t)n << bits <= 8192;
  if (!one) bits = 3;
  if (int e = allow_full_lds((const void*)reorder_kernel, "reorder_kernel")) return e;
  reorder_kernel<<<((tables->table_pages - 1) >> bits) + 1, kThreads, (3 * kThreads + 1 + (n << bits)) * 4, stream>>>(*tables, layout->pages, slots_dev,
                                                                                                                     parents_dev, n, bits, one);
  if (!one) reorder_lengths_kernel<<<1, kThreads, 0, stream>>>(*tables, slots_dev, parents_dev, n);
  return kv_launched("reorder_kernel");
}
