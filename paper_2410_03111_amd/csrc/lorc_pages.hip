// Bookkeeping of the paged cache on the device: giving out, sharing, releasing and renaming pages, and copying their contents.
// The state is the caller's block table (an id outside [0, n_pages) maps nothing) and one count per page of the entries that
// map it.  Everything here is integers: results do not depend on the order in which workgroups or atomics run, because pages
// are given out by rank (the k-th request takes the k-th lowest free page) and counts only ever see sums.
//
// What bounds these calls is the chain of launches and of trips to memory and, inside a plan, the instructions of the one compute unit
// that runs it; not the bytes (but for lorc_copy_pages).  So each call is a plan (one workgroup of 1024 threads that walks the counts of
// up to 16384 pages at a time and ranks by a sum over its waves) followed, where rows of the table change, by waves per row.  A plan in
// several workgroups would need another launch for every sum, 2 to 3 us each.
//
// Small calls (kSmallList entries of a table of kSmallRows rows, what a plan's LDS holds; kSmallTable table entries, which one workgroup
// changes in a step or two) keep what passes between threads in LDS and do the rows in the plan's launch.  Kernel times, small form /
// general form, of the same call: fork of 4 rows of 14 pages 6.0 / 7.5 us, 256 rows of 129 (rows in a launch of their own) 10.2 / 11.9 (looking at
// what the child's row mapped costs 0.3 and 0.7 more);
// compact a pool of 30 pages 6.8 / 13.8 us, of 9300 15.1 / 22.0; reserve 43 rows of 129 9.2 / 14.0.
#include <climits>

#include "lorc_device.h"
#include "lorc_kernels.h"

namespace lorc {

namespace {
constexpr int kPlanThreads = 1024, kPlanWaves = kPlanThreads / 64, kPerThread = 16, kStep = kPlanThreads * kPerThread;
constexpr int kSmallList = kPlanThreads, kSmallRows = 4096, kSmallTable = 8192;

__device__ __forceinline__ bool maps(int id, int n_pages) { return id >= 0 && id < n_pages; }
// Values that other waves of the workgroup wrote through atomics are read past the vector cache.
__device__ __forceinline__ int load_fresh(const int* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void store_fresh(int* p, int v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

__device__ __forceinline__ int wave_inclusive(int v) {
#pragma unroll
  for (int step = 1; step < 64; step <<= 1) {
    const int up = __shfl_up(v, step, 64);
    if ((int)(threadIdx.x & 63) >= step) v += up;
  }
  return v;
}

// Sum over the waves before this one of a wave's v; *total: over all of them.  `sums`: kPlanWaves words of LDS.
__device__ __forceinline__ int waves_exclusive(int v, int* sums, int* total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  __syncthreads();  // the words may still be read from the call before
  if (lane == 63) sums[w] = v;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int i = 0; i < kPlanWaves; ++i) {
    const int s = sums[i];
    before += i < w ? s : 0;
    all += s;
  }
  *total = all;
  return before;
}

// Exclusive prefix sum over the workgroup's threads; *total: the sum.
__device__ __forceinline__ int block_exclusive(int v, int* sums, int* total) {
  const int inc = wave_inclusive(v);
  return waves_exclusive(inc, sums, total) + inc - v;
}

__device__ __forceinline__ uint64_t lanes_below(int n) { return n <= 0 ? 0 : n >= 64 ? ~(uint64_t)0 : ((uint64_t)1 << n) - 1; }

// A pass over up to kStep pages: every wave walks `chunks` times 64 neighbours and keeps a bit for each page in scalar registers.  (Two other
// ways: a thread with sixteen neighbours of its own touches a cache line per lane with every load; sixteen chunks whatever the pool's
// size cost 5 us more, because what bounds a plan is its instructions: one compute unit runs them for all sixteen waves.)
struct Pages {
  uint64_t bits[kPerThread];
  int base, chunks;
  __device__ __forceinline__ int page(int u) const { return base + ((int)(threadIdx.x >> 6) * chunks + u) * 64 + (int)(threadIdx.x & 63); }
  __device__ __forceinline__ int first(int u) const { return base + (__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)) * chunks + u) * 64; }
};
__device__ __forceinline__ Pages pass_at(int base, int n_pages) {
  Pages f;
  const int chunks = (n_pages - base + kPlanThreads - 1) / kPlanThreads;
  f.base = base;
  f.chunks = chunks < kPerThread ? chunks : kPerThread;
  return f;
}
__device__ __forceinline__ Pages free_pages(const int* refs, int base, int n_pages) {
  Pages f = pass_at(base, n_pages);
  int v[kPerThread];
#pragma unroll
  for (int u = 0; u < kPerThread; ++u)
    if (u < f.chunks) v[u] = f.page(u) < n_pages ? refs[f.page(u)] : 1;
#pragma unroll
  for (int u = 0; u < kPerThread; ++u) f.bits[u] = u < f.chunks ? __ballot(v[u] <= 0) : 0;
  return f;
}
// The pages of a pass from `page` on are cleared.
__device__ __forceinline__ void keep_below(Pages& f, int page) {
#pragma unroll
  for (int u = 0; u < kPerThread; ++u)
    if (u < f.chunks) f.bits[u] &= lanes_below(page - f.first(u));
}
// emit(rank, page) for every page of the pass, ranks ascending from `seen`; returns how many there are.
template <typename F>
__device__ __forceinline__ int each_page(const Pages& f, int seen, int* sums, F emit) {
  int count = 0, total;
#pragma unroll
  for (int u = 0; u < kPerThread; ++u) count += __popcll(f.bits[u]);
  int rank = seen + waves_exclusive(count, sums, &total);
  const uint64_t lower = lanes_below(threadIdx.x & 63);
#pragma unroll
  for (int u = 0; u < kPerThread; ++u) {
    if (f.bits[u] == 0) continue;
    if (f.bits[u] >> (threadIdx.x & 63) & 1) emit(rank + __popcll(f.bits[u] & lower), f.page(u));
    rank += __popcll(f.bits[u]);
  }
  return total;
}

// emit(k, page) for the free pages of rank k < want, in ascending order; returns how many free pages there are among those walked
// (all of them where fewer than `want` exist).  first: the first pass, asked for early.
template <typename F>
__device__ __forceinline__ int each_free(const int* refs, int n_pages, const Pages& first, int want, int* sums, F emit) {
  int seen = 0;
  for (int base = 0; base < n_pages && seen < want; base += kStep)
    seen += each_page(base == 0 ? first : free_pages(refs, base, n_pages), seen, sums, [&](int k, int page) {
      if (k < want) emit(k, page);
    });
  return seen;
}
// Words that pass between the threads of a plan: in LDS, or in the workspace.
template <bool LDS>
__device__ __forceinline__ int get(const int* p) {
  if constexpr (LDS) return *p;
  return load_fresh(p);
}
template <bool LDS>
__device__ __forceinline__ void put(int* p, int v) {
  if constexpr (LDS) *p = v;
  else store_fresh(p, v);
}
// Meets the other waves; what any of them put is there to get afterwards.  (Nothing else passes between the threads of a plan, so
// that it needs no fence: one at device scope writes the caches back, 2 to 3 us each.)
__device__ __forceinline__ void plan_barrier() {
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();
}
}  // namespace

// ------------------------------------------------------------------------------------------------ copy
// One workgroup per 16 KiB piece of a page: 64 bytes per thread in flight.  Bound by memory: every byte is read and written once.
// 2100 pages of 64.5 KiB: 58 us, 4.7 TB/s read and written (a copy of 2 GiB on the same card: 4.8).
constexpr int kCopyBytes = 16 * 1024;
__global__ __launch_bounds__(256) void copy_pages_kernel(unsigned char* pool, size_t page_bytes, int n_pages, const int* __restrict__ src,
                                                         const int* __restrict__ dst, int pieces) {
  const int i = blockIdx.x / pieces, piece = blockIdx.x % pieces;
  const int from = __builtin_amdgcn_readfirstlane(src[i]), to = __builtin_amdgcn_readfirstlane(dst[i]);
  if (!maps(from, n_pages) || !maps(to, n_pages) || from == to) return;
  const size_t at = (size_t)piece * kCopyBytes;
  const int n16 = (int)((page_bytes - at < kCopyBytes ? page_bytes - at : kCopyBytes) >> 4);
  const u32x4* s = reinterpret_cast<const u32x4*>(pool + (size_t)from * page_bytes + at);
  u32x4* d = reinterpret_cast<u32x4*>(pool + (size_t)to * page_bytes + at);
  u32x4 v[4];
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int k = (int)threadIdx.x + 256 * u;
    if (k < n16) v[u] = s[k];
  }
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int k = (int)threadIdx.x + 256 * u;
    if (k < n16) d[k] = v[u];
  }
}

// ------------------------------------------------------------------------------------------------ fork
// One wave, or `waves` of them: the child's row, the counts of the pages that it shares, and of those that the row mapped before (behind a
// first entry that maps nothing).  The plan gave out its pages before any row is changed: what a row releases is free for the next call.
__device__ __forceinline__ void fork_row(const ForkParams& p, int parent, int child, int len, int fresh, int wave = 0, int waves = 1) {
  const int whole = len / kPage, *from = p.block_table + (size_t)parent * p.max_pages;
  int* to = p.block_table + (size_t)child * p.max_pages;
  for (int e = 64 * wave + (int)(threadIdx.x & 63); e < p.max_pages; e += 64 * waves) {
    int id = e < whole ? from[e] : e == whole ? fresh : -1;
    const int old = to[e];
    if (maps(old, p.n_pages)) atomicSub(p.page_refs + old, 1);
    if (!maps(id, p.n_pages)) id = -1;
    else if (e < whole) atomicAdd(p.page_refs + id, 1);
    else p.page_refs[id] = 1;
    to[e] = id;
  }
}

// owner: the lowest pair that names a row as its child; asks: the pairs that need a page, in order.  ROWS (with SMALL): the rows
// as well.
template <bool SMALL, bool ROWS>
__global__ __launch_bounds__(kPlanThreads) void fork_plan_kernel(ForkParams p) {
  __shared__ int sums[kPlanWaves], owner_lds[SMALL ? kSmallRows : 1], asks_lds[SMALL ? kSmallList : 1], fresh_lds[ROWS ? kSmallList : 1];
  int* owner = SMALL ? owner_lds : p.owner;
  int* asks = SMALL ? asks_lds : p.asks;
  const int tid = threadIdx.x;
  const Pages first_pass = free_pages(p.page_refs, 0, p.n_pages);
  for (int s = tid; s < p.n_seqs; s += kPlanThreads) put<SMALL>(owner + s, INT_MAX);
  const long most = (long)p.max_pages * kPage;
  auto named = [&](int i, int& parent, int& child, int& len) {
    parent = p.parents[i];
    child = p.children[i];
    len = p.lens[i];
    return parent >= 0 && parent < p.n_seqs && child >= 0 && child < p.n_seqs && parent != child && len >= 0 && len <= most;
  };
  plan_barrier();
  for (int i = tid; i < p.n; i += kPlanThreads) {
    int parent, child, len;
    if (named(i, parent, child, len)) atomicMin(owner + child, i);
  }
  plan_barrier();
  int asked = 0;
  for (int base = 0; base < p.n; base += kPlanThreads) {
    const int i = base + tid;
    int parent, child, len, tail = -1;
    bool ok = i < p.n && named(i, parent, child, len);
    ok = ok && get<SMALL>(owner + child) == i && get<SMALL>(owner + parent) == INT_MAX;
    if (ok) {
      const int head = p.block_table[(size_t)child * p.max_pages];
      if (len % kPage != 0) tail = p.block_table[(size_t)parent * p.max_pages + len / kPage];
      ok = !maps(head, p.n_pages);
    }
    const bool tails = ok && maps(tail, p.n_pages);
    int total;
    const int rank = asked + block_exclusive(tails ? 1 : 0, sums, &total);
    asked += total;
    if (tails) put<SMALL>(asks + rank, i);
    if (i < p.n) {
      p.status[i] = !ok ? LORC_PAGES_REFUSED : tails ? LORC_PAGES_SHORT : LORC_PAGES_OK;  // (short until a page is found below)
      p.copy_src[i] = tails ? tail : -1;
      p.copy_dst[i] = -1;
      if constexpr (ROWS) fresh_lds[i] = !ok ? -3 : tails ? -2 : -1;  // refused, short, no page of its own
    }
  }
  plan_barrier();
  const int found = each_free(p.page_refs, p.n_pages, first_pass, asked, sums, [&](int k, int page) {
    const int i = get<SMALL>(asks + k);
    p.copy_dst[i] = page;
    p.status[i] = LORC_PAGES_OK;
    if constexpr (ROWS) fresh_lds[i] = page;
  });
  for (int k = found + tid; k < asked; k += kPlanThreads) p.copy_src[get<SMALL>(asks + k)] = -1;
  if constexpr (ROWS) {
    plan_barrier();
    for (int i = tid >> 6; i < p.n; i += kPlanWaves)
      if (fresh_lds[i] >= -1) fork_row(p, p.parents[i], p.children[i], p.lens[i], fresh_lds[i]);
  }
}

__global__ __launch_bounds__(256) void fork_rows_kernel(ForkParams p, int waves) {
  const int at = blockIdx.x * 4 + (int)(threadIdx.x >> 6), i = at / waves;
  if (i >= p.n) return;
  const int status = p.status[i], parent = p.parents[i], child = p.children[i], len = p.lens[i], fresh = p.copy_dst[i];
  if (status == LORC_PAGES_OK) fork_row(p, parent, child, len, fresh, at % waves, waves);
}

// ------------------------------------------------------------------------------------------------ free
// `waves` waves per row.  An entry is claimed by an exchange, so that a row named twice is released once.
__global__ __launch_bounds__(256) void free_rows_kernel(int* block_table, int n_seqs, int max_pages, int* page_refs, int n_pages,
                                                        const int* __restrict__ seqs, int n, int waves) {
  const int at = blockIdx.x * 4 + (int)(threadIdx.x >> 6), lane = threadIdx.x & 63, i = at / waves;
  if (i >= n) return;
  const int s = seqs[i];
  if (s < 0 || s >= n_seqs) return;
  int* row = block_table + (size_t)s * max_pages;
  for (int e = 64 * (at % waves) + lane; e < max_pages; e += 64 * waves) {
    const int id = atomicExch(row + e, -1);
    if (maps(id, n_pages)) atomicSub(page_refs + id, 1);
  }
}

// ------------------------------------------------------------------------------------------------ compact
// U pages are in use: the k-th lowest free page (below U) takes the contents of the k-th highest used one (at U or above).  RENAME: the
// table as well.
template <bool RENAME>
__global__ __launch_bounds__(kPlanThreads) void compact_plan_kernel(CompactParams p) {
  __shared__ int sums[kPlanWaves];
  const int tid = threadIdx.x;
  int n_free = 0;
  for (int base = 0; base < p.n_pages; base += kStep) n_free += each_page(free_pages(p.page_refs, base, p.n_pages), 0, sums, [](int, int) {});
  const int used = p.n_pages - n_free;
  int holes = 0;  // free pages below `used`: as many as used pages from there on
  for (int base = 0; base < used; base += kStep) {
    Pages f = free_pages(p.page_refs, base, p.n_pages);
    keep_below(f, used);
    holes += each_page(f, holes, sums, [&](int k, int page) {
      if (k < p.max_moves) store_fresh(p.move_dst + k, page);
    });
  }
  const int moves = holes < p.max_moves ? holes : p.max_moves;
  for (int k = moves + tid; k < p.max_moves; k += kPlanThreads) p.move_src[k] = p.move_dst[k] = -1;
  for (int id = tid; id < p.n_pages; id += kPlanThreads) store_fresh(p.page_map + id, id);
  int walked = 0;  // used pages from `used` on
  for (int base = used / kStep * kStep; base < p.n_pages; base += kStep) {
    Pages f = free_pages(p.page_refs, base, p.n_pages), below = f;
#pragma unroll
    for (int u = 0; u < kPerThread; ++u) f.bits[u] = below.bits[u] = u < f.chunks ? ~f.bits[u] : 0;
    keep_below(f, p.n_pages);
    keep_below(below, used);
#pragma unroll
    for (int u = 0; u < kPerThread; ++u) f.bits[u] &= ~below.bits[u];
    walked += each_page(f, walked, sums, [&](int k, int page) {
      if (holes - 1 - k < moves) store_fresh(p.move_src + holes - 1 - k, page);  // rank from the top
    });
  }
  plan_barrier();
  for (int k = tid; k < moves; k += kPlanThreads) {
    const int from = load_fresh(p.move_src + k), to = load_fresh(p.move_dst + k);
    p.page_refs[to] = p.page_refs[from];
    p.page_refs[from] = 0;
    store_fresh(p.page_map + from, to);
  }
  if constexpr (RENAME) {
    plan_barrier();
    for (int e = tid; e < p.n_seqs * p.max_pages; e += kPlanThreads) {
      const int id = p.block_table[e];
      if (!maps(id, p.n_pages)) continue;
      const int to = load_fresh(p.page_map + id);
      if (to != id) p.block_table[e] = to;
    }
  }
}

// The same for pools of up to kStep pages: one pass, whose counts stay in registers; moves and the map pass through LDS.
template <bool RENAME>
__global__ __launch_bounds__(kPlanThreads) void compact_small_kernel(CompactParams p) {
  __shared__ int sums[kPlanWaves];
  __shared__ uint16_t dst_of[kStep / 2], new_id[RENAME ? kStep : 1];  // ids below kStep; half of them at most move
  const int tid = threadIdx.x, lane = tid & 63;
  int refs[kPerThread];
  Pages hole = pass_at(0, p.n_pages), top = hole;
#pragma unroll
  for (int u = 0; u < kPerThread; ++u)
    if (u < top.chunks) refs[u] = top.page(u) < p.n_pages ? p.page_refs[top.page(u)] : 0;
  int count = 0, used, tops;
#pragma unroll
  for (int u = 0; u < kPerThread; ++u) {
    top.bits[u] = u < top.chunks ? __ballot(refs[u] > 0) : 0;
    hole.bits[u] = u < top.chunks ? ~top.bits[u] : 0;
    count += __popcll(top.bits[u]);
  }
  waves_exclusive(count, sums, &used);
  keep_below(hole, used);
  const int holes = each_page(hole, 0, sums, [&](int k, int page) {
    if (k < p.max_moves) {
      dst_of[k] = (uint16_t)page;
      p.move_dst[k] = page;
    }
  });
  const int moves = holes < p.max_moves ? holes : p.max_moves;
  for (int i = moves + tid; i < p.max_moves; i += kPlanThreads) p.move_src[i] = p.move_dst[i] = -1;
  Pages below = top;
  keep_below(below, used);
  count = 0;
#pragma unroll
  for (int u = 0; u < kPerThread; ++u) {
    top.bits[u] &= ~below.bits[u];
    count += __popcll(top.bits[u]);
  }
  const uint64_t lower = lanes_below(lane);
  int k = holes - 1 - waves_exclusive(count, sums, &tops);  // rank from the top  (the barrier also covers dst_of)
#pragma unroll
  for (int u = 0; u < kPerThread; ++u) {
    if (u >= top.chunks) continue;
    const int page = top.page(u);
    int to = page;
    if (top.bits[u] != 0) {
      const int mine = k - __popcll(top.bits[u] & lower);
      if ((top.bits[u] >> lane & 1) && mine < moves) {
        to = dst_of[mine];
        p.move_src[mine] = page;
        p.page_refs[to] = refs[u];
        p.page_refs[page] = 0;
      }
      k -= __popcll(top.bits[u]);
    }
    if (page < p.n_pages) p.page_map[page] = to;
    if constexpr (RENAME) new_id[page] = (uint16_t)to;
  }
  if constexpr (RENAME) {
    __syncthreads();
    for (int e = tid; e < p.n_seqs * p.max_pages; e += kPlanThreads) {
      const int id = p.block_table[e];
      if (!maps(id, p.n_pages)) continue;
      const int to = new_id[id];
      if (to != id) p.block_table[e] = to;
    }
  }
}

__global__ __launch_bounds__(256) void rename_pages_kernel(int* block_table, size_t entries, const int* __restrict__ page_map, int n_pages) {
  const size_t e = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (e >= entries) return;
  const int id = block_table[e];
  if (!maps(id, n_pages)) return;
  const int to = page_map[id];
  if (to != id) block_table[e] = to;
}

// ------------------------------------------------------------------------------------------------ reserve
constexpr int kRowDepth = 5;  // loads in flight per lane: 80 entries of a row

// Sixteen lanes: the row's unmapped entries below n_e take the pages of rank `rank` and on.  (Every lane of a wave calls it.)
__device__ __forceinline__ void reserve_row(const ReserveParams& p, int s, int n_e, int rank, const int* pages) {
  const int lane = threadIdx.x & 63, l16 = lane & 15;
  int* row = p.block_table + (size_t)s * p.max_pages;
  for (int e0 = 0; __any(e0 < n_e); e0 += 16 * kRowDepth) {
    int id[kRowDepth];
#pragma unroll
    for (int u = 0; u < kRowDepth; ++u) id[u] = e0 + 16 * u + l16 < n_e ? row[e0 + 16 * u + l16] : 0;
#pragma unroll
    for (int u = 0; u < kRowDepth; ++u) {
      const bool missing = e0 + 16 * u + l16 < n_e && !maps(id[u], p.n_pages);
      const uint32_t who = (uint32_t)(__ballot(missing) >> (lane & 48)) & 0xffffu;
      if (missing) {
        const int page = pages[rank + __popc(who & ((1u << l16) - 1u))];
        row[e0 + 16 * u + l16] = page;
        p.page_refs[page] = 1;
      }
      rank += __popc(who);
    }
  }
}

// owner: the first place in the list that names a row; first: rank of the first new page, of a place in the list (SMALL) or of a row;
// pages: the free pages by rank.  SMALL: the rows as well.
template <bool SMALL>
__global__ __launch_bounds__(kPlanThreads) void reserve_plan_kernel(ReserveParams p) {
  __shared__ int sums[kPlanWaves], owner_lds[SMALL ? kSmallRows : 1], first_lds[SMALL ? kSmallList : 1], pages_lds[SMALL ? kSmallTable : 1];
  int* owner = SMALL ? owner_lds : p.owner;
  int* pages = SMALL ? pages_lds : p.pages;
  const int tid = threadIdx.x;
  const Pages first_pass = free_pages(p.page_refs, 0, p.n_pages);
  for (int s = tid; s < p.n_seqs; s += kPlanThreads) put<SMALL>(owner + s, INT_MAX);
  const long most = (long)p.max_pages * kPage;
  auto named = [&](int i, int& s, int& len) {
    s = p.seqs[i];
    len = p.lens[i];
    return s >= 0 && s < p.n_seqs && len >= 0 && len <= most;
  };
  auto first_of = [&](int i, int s) { return SMALL ? first_lds + i : p.first + s; };
  plan_barrier();
  for (int i = tid; i < p.n; i += kPlanThreads) {
    int s, len;
    if (named(i, s, len)) atomicMin(owner + s, i);
  }
  plan_barrier();
  for (int i = tid >> 4; i < p.n; i += kPlanThreads / 16) {  // how many entries of the row map nothing yet: sixteen lanes per row
    int s, len;
    const bool mine = named(i, s, len) && get<SMALL>(owner + s) == i;
    const int n_e = mine ? (len + kPage - 1) / kPage : 0;
    const int* row = p.block_table + (size_t)(mine ? s : 0) * p.max_pages;
    int missing = 0;
    for (int e0 = tid & 15; e0 < n_e; e0 += 16 * kRowDepth) {
      int id[kRowDepth];
#pragma unroll
      for (int u = 0; u < kRowDepth; ++u) id[u] = e0 + 16 * u < n_e ? row[e0 + 16 * u] : 0;  // (0 is a page)
#pragma unroll
      for (int u = 0; u < kRowDepth; ++u) missing += maps(id[u], p.n_pages) ? 0 : 1;
    }
#pragma unroll
    for (int step = 1; step < 16; step <<= 1) missing += __shfl_xor(missing, step, 16);
    if (mine && (tid & 15) == 0) put<SMALL>(first_of(i, s), missing);
  }
  plan_barrier();
  int asked = 0;
  for (int base = 0; base < p.n; base += kPlanThreads) {
    const int i = base + tid;
    int s, len;
    const bool ok = i < p.n && named(i, s, len) && get<SMALL>(owner + s) == i;
    const int missing = ok ? get<SMALL>(first_of(i, s)) : 0;
    int total;
    const int rank = asked + block_exclusive(missing, sums, &total);
    asked += total;
    if (ok) put<SMALL>(first_of(i, s), rank);
    if (i < p.n) p.status[i] = !ok ? LORC_PAGES_REFUSED : missing;  // (the count, until it is known whether they are there)
  }
  plan_barrier();
  const int found = each_free(p.page_refs, p.n_pages, first_pass, asked, sums, [&](int k, int page) { pages[k] = page; });
  for (int i = tid; i < p.n; i += kPlanThreads) {
    int s, len;
    const bool ok = named(i, s, len) && get<SMALL>(owner + s) == i;
    if (!ok) {
      if constexpr (SMALL) first_lds[i] = -1;
      continue;
    }
    const int missing = p.status[i], rank = get<SMALL>(first_of(i, s));
    const bool served = missing == 0 || rank + missing <= found;
    p.status[i] = served ? LORC_PAGES_OK : LORC_PAGES_SHORT;
    if constexpr (SMALL) first_lds[i] = served && missing > 0 ? rank : -1;
  }
  if constexpr (SMALL) {
    plan_barrier();
    for (int i0 = 0; i0 < p.n; i0 += kPlanThreads / 16) {
      const int i = i0 + (tid >> 4), rank = i < p.n ? first_lds[i] : -1;
      reserve_row(p, rank >= 0 ? p.seqs[i] : 0, rank >= 0 ? (p.lens[i] + kPage - 1) / kPage : 0, rank, pages);
    }
  }
}

// Sixteen lanes per place in the list (a large call's `first` is the row's).
__global__ __launch_bounds__(256) void reserve_rows_kernel(ReserveParams p) {
  const int i = blockIdx.x * 16 + (int)(threadIdx.x >> 4);
  const bool served = i < p.n && p.status[i] == LORC_PAGES_OK;
  const int s = served ? p.seqs[i] : 0;
  reserve_row(p, s, served ? (p.lens[i] + kPage - 1) / kPage : 0, served ? p.first[s] : 0, p.pages);
}

// ------------------------------------------------------------------------------------------------ host
int launch_copy_pages(void* pool, size_t page_bytes, int n_pages, const int32_t* src, const int32_t* dst, int count, hipStream_t s) {
  const size_t pieces = (page_bytes + kCopyBytes - 1) / kCopyBytes;
  return launch_parts(count, (int)(launch_blocks(256) / pieces), [&](int first, int n) {
    return launch_kernel(copy_pages_kernel, dim3((uint32_t)(pieces * n)), dim3(256), 0, s, static_cast<unsigned char*>(pool), page_bytes, n_pages,
                         src + first, dst + first, (int)pieces);
  });
}

// Waves of a row, 64 entries each: a wave that walks a row waits for memory at every step (256 forks of rows of 129 entries: 4.9 -> 3.8 us).
static int waves_per_row(int n, int max_pages) {
  const int want = (max_pages + 63) / 64, most = (1 << 30) / n;
  return want < most ? want : most;
}

int launch_fork(const ForkParams& p, hipStream_t s) {
  const bool small = p.n <= kSmallList && p.n_seqs <= kSmallRows, rows = small && (long)p.n * p.max_pages <= kSmallTable;
  if (int rc = launch_kernel(rows ? fork_plan_kernel<true, true> : small ? fork_plan_kernel<true, false> : fork_plan_kernel<false, false>, dim3(1),
                             dim3(kPlanThreads), 0, s, p))
    return rc;
  if (rows) return LORC_OK;
  const int waves = waves_per_row(p.n, p.max_pages);
  return launch_parts(p.n, 4 * launch_blocks(256) / waves, [&](int first, int n) {
    ForkParams part = p;
    part.parents += first;
    part.children += first;
    part.lens += first;
    part.status += first;
    part.copy_dst += first;
    part.n = n;
    return launch_kernel(fork_rows_kernel, dim3((n * waves + 3) / 4), dim3(256), 0, s, part, waves);
  });
}

int launch_free(int32_t* block_table, int n_seqs, int max_pages, int32_t* page_refs, int n_pages, const int32_t* seqs, int n, hipStream_t s) {
  const int waves = waves_per_row(n, max_pages);
  return launch_parts(n, 4 * launch_blocks(256) / waves, [&](int first, int here) {
    return launch_kernel(free_rows_kernel, dim3((here * waves + 3) / 4), dim3(256), 0, s, block_table, n_seqs, max_pages, page_refs, n_pages, seqs + first,
                         here, waves);
  });
}

int launch_compact(const CompactParams& p, hipStream_t s) {
  const size_t entries = (size_t)p.n_seqs * p.max_pages;
  const bool rename = entries <= kSmallTable, small = p.n_pages <= kStep;
  if (int rc = launch_kernel(small ? (rename ? compact_small_kernel<true> : compact_small_kernel<false>)
                                   : rename ? compact_plan_kernel<true> : compact_plan_kernel<false>, dim3(1), dim3(kPlanThreads), 0, s, p))
    return rc;
  if (rename) return LORC_OK;
  return launch_kernel(rename_pages_kernel, dim3((uint32_t)((entries + 255) / 256)), dim3(256), 0, s, p.block_table, entries, p.page_map, p.n_pages);
}

int launch_reserve(const ReserveParams& p, hipStream_t s) {
  // (first is kept by place in the list only where the rows are done in the same launch)
  const bool rows = p.n <= kSmallList && p.n_seqs <= kSmallRows && (long)p.n * p.max_pages <= kSmallTable;
  if (int rc = launch_kernel(rows ? reserve_plan_kernel<true> : reserve_plan_kernel<false>, dim3(1), dim3(kPlanThreads), 0, s, p))
    return rc;
  if (rows) return LORC_OK;
  return launch_parts(p.n, 16 * launch_blocks(256), [&](int first, int n) {
    ReserveParams part = p;
    part.seqs += first;
    part.lens += first;
    part.status += first;
    part.n = n;
    return launch_kernel(reserve_rows_kernel, dim3((n + 15) / 16), dim3(256), 0, s, part);
  });
}

}  // namespace lorc
