// Bookkeeping of the paged cache on the device: giving out, sharing, releasing and renaming pages, and copying their contents.
// The state is the caller's block table (an id outside [0, n_pages) maps nothing) and one count per page of the entries that
// map it.  Everything here is integers: results do not depend on the order in which workgroups or atomics run, because pages
// are given out by rank (the k-th request takes the k-th lowest free page) and counts only ever see sums.
//
// What bounds these calls is the chain of launches and of trips to memory, not the bytes: so each is a plan (one workgroup of
// 1024 threads that walks the counts 16 to a thread and ranks by a scan over the workgroup) followed, where rows of the table
// change, by one wave per row.  A plan in several workgroups would need another launch for every scan, 2 to 3 us each, which is
// what one workgroup takes for the counts of 16384 pages.  Small calls (kSmallList entries of a table of kSmallRows rows, kSmallTable
// table entries to change) keep what passes between threads in LDS and do the rows in the plan's launch.
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

// Exclusive prefix sum over the workgroup's threads; *total: the sum.  `sums`: kPlanWaves words of LDS.
__device__ __forceinline__ int block_exclusive(int v, int* sums, int* total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int inc = wave_inclusive(v);
  __syncthreads();  // the words may still be read from the call before
  if (lane == 63) sums[w] = inc;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int i = 0; i < kPlanWaves; ++i) {
    const int s = sums[i];
    before += i < w ? s : 0;
    all += s;
  }
  *total = all;
  return before + inc - v;
}

// The counts of up to 16 consecutive pages from `first` on, as a mask of those that are free (bit set) and how many are there.
__device__ __forceinline__ uint32_t free_mask(const int* refs, int first, int n_pages) {
  uint32_t mask = 0;
  if (first + kPerThread <= n_pages && (reinterpret_cast<uintptr_t>(refs) & 15) == 0) {
#pragma unroll
    for (int u = 0; u < kPerThread / 4; ++u) {
      const int4 v = *reinterpret_cast<const int4*>(refs + first + 4 * u);
      mask |= (v.x <= 0 ? 1u : 0u) << (4 * u) | (v.y <= 0 ? 2u : 0u) << (4 * u) | (v.z <= 0 ? 4u : 0u) << (4 * u) | (v.w <= 0 ? 8u : 0u) << (4 * u);
    }
  } else {
    for (int u = 0; u < kPerThread; ++u)
      if (first + u < n_pages && refs[first + u] <= 0) mask |= 1u << u;
  }
  return mask;
}

// emit(k, page) for the free pages of rank k < want, in ascending order; returns how many free pages there are among those walked
// (all of them where fewer than `want` exist).  first_mask: free_mask of the thread's first 16 pages, asked for early.
template <typename F>
__device__ __forceinline__ int each_free(const int* refs, int n_pages, uint32_t first_mask, int want, int* sums, F emit) {
  int seen = 0;
  for (int base = 0; base < n_pages && seen < want; base += kStep) {
    const int first = base + (int)threadIdx.x * kPerThread;
    uint32_t mask = base == 0 ? first_mask : first < n_pages ? free_mask(refs, first, n_pages) : 0u;
    int total;
    int rank = seen + block_exclusive(__popc(mask), sums, &total);
    while (mask != 0 && rank < want) {
      emit(rank++, first + __ffs(mask) - 1);
      mask &= mask - 1;
    }
    seen += total;
  }
  return seen;
}
__device__ __forceinline__ uint32_t first_free_mask(const int* refs, int n_pages) {
  const int first = (int)threadIdx.x * kPerThread;
  return first < n_pages ? free_mask(refs, first, n_pages) : 0u;
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
// One wave: the child's row, and the counts of the pages that it shares.
__device__ __forceinline__ void fork_row(const ForkParams& p, int parent, int child, int len, int fresh) {
  const int whole = len / kPage, *from = p.block_table + (size_t)parent * p.max_pages;
  int* to = p.block_table + (size_t)child * p.max_pages;
  for (int e = threadIdx.x & 63; e < p.max_pages; e += 64) {
    int id = e < whole ? from[e] : e == whole ? fresh : -1;
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
  const uint32_t first_mask = first_free_mask(p.page_refs, p.n_pages);
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
  const int found = each_free(p.page_refs, p.n_pages, first_mask, asked, sums, [&](int k, int page) {
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

__global__ __launch_bounds__(256) void fork_rows_kernel(ForkParams p) {
  const int i = blockIdx.x * 4 + (int)(threadIdx.x >> 6);
  if (i >= p.n || p.status[i] != LORC_PAGES_OK) return;
  fork_row(p, p.parents[i], p.children[i], p.lens[i], p.copy_dst[i]);
}

// ------------------------------------------------------------------------------------------------ free
// One wave per row.  An entry is claimed by an exchange, so that a row named twice is released once.
__global__ __launch_bounds__(256) void free_rows_kernel(int* block_table, int n_seqs, int max_pages, int* page_refs, int n_pages,
                                                        const int* __restrict__ seqs, int n) {
  const int i = blockIdx.x * 4 + (int)(threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (i >= n) return;
  const int s = seqs[i];
  if (s < 0 || s >= n_seqs) return;
  int* row = block_table + (size_t)s * max_pages;
  for (int e = lane; e < max_pages; e += 64) {
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
  const uint32_t first_mask = first_free_mask(p.page_refs, p.n_pages);
  auto mask_of = [&](int base) {
    const int first = base + tid * kPerThread;
    return base == 0 ? first_mask : first < p.n_pages ? free_mask(p.page_refs, first, p.n_pages) : 0u;
  };
  int n_free = 0;
  for (int base = 0; base < p.n_pages; base += kStep) {
    int total;
    block_exclusive(__popc(mask_of(base)), sums, &total);
    n_free += total;
  }
  const int used = p.n_pages - n_free;
  int holes = 0;  // free pages below `used`: as many as used pages from there on
  for (int base = 0; base < used; base += kStep) {
    const int first = base + tid * kPerThread, n_here = used - first;
    uint32_t mask = mask_of(base);
    if (n_here < kPerThread) mask &= n_here <= 0 ? 0u : (1u << n_here) - 1u;
    int total;
    int rank = holes + block_exclusive(__popc(mask), sums, &total);
    for (uint32_t m = mask; m != 0; m &= m - 1, ++rank)
      if (rank < p.max_moves) store_fresh(p.move_dst + rank, first + __ffs(m) - 1);
    holes += total;
  }
  const int moves = holes < p.max_moves ? holes : p.max_moves;
  for (int k = moves + tid; k < p.max_moves; k += kPlanThreads) p.move_src[k] = p.move_dst[k] = -1;
  for (int id = tid; id < p.n_pages; id += kPlanThreads) store_fresh(p.page_map + id, id);
  int rest = holes;  // used pages not yet walked
  for (int base = used / kStep * kStep; base < p.n_pages; base += kStep) {
    const int first = base + tid * kPerThread;
    int n_here = p.n_pages - first, skip = used - first;  // pages [skip, n_here) of the thread's count
    n_here = n_here < 0 ? 0 : (n_here > kPerThread ? kPerThread : n_here);
    skip = skip < 0 ? 0 : (skip > n_here ? n_here : skip);
    const uint32_t mask = ~mask_of(base) & ((1u << n_here) - 1u) & ~((1u << skip) - 1u);
    int total;
    int k = rest - 1 - block_exclusive(__popc(mask), sums, &total);  // rank from the top
    for (uint32_t m = mask; m != 0; m &= m - 1, --k)
      if (k < moves) store_fresh(p.move_src + k, first + __ffs(m) - 1);
    rest -= total;
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

__global__ __launch_bounds__(256) void rename_pages_kernel(int* block_table, size_t entries, const int* __restrict__ page_map, int n_pages) {
  const size_t e = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (e >= entries) return;
  const int id = block_table[e];
  if (!maps(id, n_pages)) return;
  const int to = page_map[id];
  if (to != id) block_table[e] = to;
}

// ------------------------------------------------------------------------------------------------ reserve
// Sixteen lanes: the row's unmapped entries below n_e take the pages of rank `rank` and on.  (Every lane of a wave calls it.)
__device__ __forceinline__ void reserve_row(const ReserveParams& p, int s, int n_e, int rank, const int* pages) {
  const int lane = threadIdx.x & 63, l16 = lane & 15;
  int* row = p.block_table + (size_t)s * p.max_pages;
  for (int e0 = 0; __any(e0 < n_e); e0 += 64) {
    int id[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) id[u] = e0 + 16 * u + l16 < n_e ? row[e0 + 16 * u + l16] : 0;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
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
  const uint32_t first_mask = first_free_mask(p.page_refs, p.n_pages);
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
#pragma unroll 4
    for (int e = tid & 15; e < n_e; e += 16) missing += maps(row[e], p.n_pages) ? 0 : 1;
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
  const int found = each_free(p.page_refs, p.n_pages, first_mask, asked, sums, [&](int k, int page) { pages[k] = page; });
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
  if (pieces * (size_t)count > 0x7fffffffu) return LORC_EINVAL;
  return launch_kernel(copy_pages_kernel, dim3((uint32_t)(pieces * count)), dim3(256), 0, s, static_cast<unsigned char*>(pool), page_bytes,
                       n_pages, src, dst, (int)pieces);
}

int launch_fork(const ForkParams& p, hipStream_t s) {
  const bool small = p.n <= kSmallList && p.n_seqs <= kSmallRows, rows = small && (long)p.n * p.max_pages <= kSmallTable;
  if (int rc = launch_kernel(rows ? fork_plan_kernel<true, true> : small ? fork_plan_kernel<true, false> : fork_plan_kernel<false, false>, dim3(1),
                             dim3(kPlanThreads), 0, s, p))
    return rc;
  return rows ? LORC_OK : launch_kernel(fork_rows_kernel, dim3((p.n + 3) / 4), dim3(256), 0, s, p);
}

int launch_free(int32_t* block_table, int n_seqs, int max_pages, int32_t* page_refs, int n_pages, const int32_t* seqs, int n, hipStream_t s) {
  return launch_kernel(free_rows_kernel, dim3((n + 3) / 4), dim3(256), 0, s, block_table, n_seqs, max_pages, page_refs, n_pages, seqs, n);
}

int launch_compact(const CompactParams& p, hipStream_t s) {
  const size_t entries = (size_t)p.n_seqs * p.max_pages;
  const bool rename = entries <= kSmallTable;
  if (int rc = launch_kernel(rename ? compact_plan_kernel<true> : compact_plan_kernel<false>, dim3(1), dim3(kPlanThreads), 0, s, p)) return rc;
  if (rename) return LORC_OK;
  return launch_kernel(rename_pages_kernel, dim3((uint32_t)((entries + 255) / 256)), dim3(256), 0, s, p.block_table, entries, p.page_map, p.n_pages);
}

int launch_reserve(const ReserveParams& p, hipStream_t s) {
  // (first is kept by place in the list only where the rows are done in the same launch)
  const bool rows = p.n <= kSmallList && p.n_seqs <= kSmallRows && (long)p.n * p.max_pages <= kSmallTable;
  if (int rc = launch_kernel(rows ? reserve_plan_kernel<true> : reserve_plan_kernel<false>, dim3(1), dim3(kPlanThreads), 0, s, p))
    return rc;
  return rows ? LORC_OK : launch_kernel(reserve_rows_kernel, dim3((p.n + 15) / 16), dim3(256), 0, s, p);
}

}  // namespace lorc
