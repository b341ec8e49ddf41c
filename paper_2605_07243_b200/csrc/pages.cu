// Pages of a cache shared between sequences: fork, reserve (copy on write), release, compact, and the copies of
// their contents.
//
// The bookkeeping is integers on the device, so that a step of branching needs no round trip to the host.  It is bound by
// latency: a few thousand integers and a chain of dependent steps (claim, check, count, rank, apply).  fork,
// release and reserve run as ONE CTA, whose barriers separate the steps: splitting them over launches costs
// more than the work.  compact walks every table and runs as one cluster of 8 CTAs for the same reason.
// Results do not depend on the order in which threads run: counts and minima are the only atomics, and every
// rank comes from a prefix sum in list or page order.
// The copies are bound by memory (every byte read and written once): a grid of a few CTAs per SM over
// (pair, layer, array, 16 KB piece), 64 bytes in flight per thread.
#include <cooperative_groups.h>

#include "common.cuh"

namespace sb {

namespace cgp = cooperative_groups;

constexpr int PG_THREADS = 1024;
constexpr int PG_WARPS = PG_THREADS / 32;
constexpr int PG_CLUSTER = 8;

// Exclusive prefix sum of one int per thread over the CTA; *total = the sum.  s: PG_WARPS + 1 ints.
__device__ inline int block_exclusive(int v, int* s, int* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int inc = v;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int t = __shfl_up_sync(0xffffffffu, inc, d);
    if (lane >= d) inc += t;
  }
  if (lane == 31) s[warp] = inc;
  __syncthreads();
  if (warp == 0) {
    const int w = lane < PG_WARPS ? s[lane] : 0;
    int winc = w;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int t = __shfl_up_sync(0xffffffffu, winc, d);
      if (lane >= d) winc += t;
    }
    s[lane] = winc - w;
    if (lane == 31) s[PG_WARPS] = winc;
  }
  __syncthreads();
  const int r = s[warp] + inc - v;
  *total = s[PG_WARPS];
  __syncthreads();
  return r;
}

__device__ inline int pages_for(int positions, int page_size) {  // positions >= 0; no overflow near INT_MAX
  return positions / page_size + (positions % page_size != 0 ? 1 : 0);
}

// claim[slot] = the first list entry that names it.  Contains barriers.
__device__ inline void claim_slots(int* claim, const sb_page_pool& pool, const int* slots, int n) {
  for (int i = threadIdx.x; i < pool.n_slots; i += PG_THREADS) claim[i] = 0x7fffffff;
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += PG_THREADS) {
    const int s = slots[i];
    if (s >= 0 && s < pool.n_slots) atomicMin(&claim[s], i);
  }
  __syncthreads();
}

// True when the pages [first, last) of a slot are inside the pool and have holders.  One warp.
__device__ inline bool pages_sound(const sb_page_pool& pool, int slot, int first, int last) {
  bool bad = false;
  for (int p = first + (threadIdx.x & 31); p < last; p += 32) {
    const int page = pool.page_table[(long long)slot * pool.max_pages + p];
    bad |= page < 0 || page >= pool.num_pages || pool.refs[page] < 1;
  }
  return !__any_sync(0xffffffffu, bad);
}

__global__ void __launch_bounds__(PG_THREADS) pages_release_kernel(const sb_page_pool pool, int n,
                                                                   const int* __restrict__ slots,
                                                                   const int* __restrict__ keep_len, int* ws, int* status) {
  pdl_wait();
  pdl_release();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int* claim = ws;
  claim_slots(claim, pool, slots, n);
  for (int i = warp; i < n; i += PG_WARPS) {
    const int s = slots[i], keep = keep_len[i];
    int err = 0;
    if (s < 0 || s >= pool.n_slots || claim[s] != i) {
      err = SB_ERR_INVALID_ARG;
    } else {
      const int held = pool.held[s];
      if (keep < 0 || held < 0 || held > pool.max_pages) err = SB_ERR_BOUNDS;
      else if (pages_for(keep, pool.page_size) > held) err = SB_ERR_BOUNDS;
      else if (!pages_sound(pool, s, pages_for(keep, pool.page_size), held)) err = SB_ERR_BOUNDS;
    }
    if (lane == 0) status[i] = err;
  }
  __syncthreads();  // every entry is judged on the state before the call
  for (int i = warp; i < n; i += PG_WARPS) {
    if (status[i]) continue;
    const int s = slots[i], first = pages_for(keep_len[i], pool.page_size), held = pool.held[s];
    int* row = pool.page_table + (long long)s * pool.max_pages;
    for (int p = first + lane; p < held; p += 32) {
      atomicSub(&pool.refs[row[p]], 1);
      row[p] = -1;
    }
    __syncwarp();
    if (lane == 0) pool.held[s] = first;
  }
}

__global__ void __launch_bounds__(PG_THREADS) pages_fork_kernel(const sb_page_pool pool, int n, const int* __restrict__ src,
                                                                const int* __restrict__ dst, const int* __restrict__ len,
                                                                int* ws, int* status) {
  pdl_wait();
  pdl_release();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int* claim = ws;
  claim_slots(claim, pool, dst, n);
  for (int i = warp; i < n; i += PG_WARPS) {
    const int s = src[i], d = dst[i], l = len[i];
    int err = 0;
    if (d < 0 || d >= pool.n_slots || claim[d] != i || s < 0 || s >= pool.n_slots || s == d) {
      err = SB_ERR_INVALID_ARG;
    } else {
      const int held = pool.held[s];
      if (l < 0 || held < 0 || held > pool.max_pages || pool.held[d] != 0) err = SB_ERR_BOUNDS;
      else if (pages_for(l, pool.page_size) > held) err = SB_ERR_BOUNDS;
      else if (!pages_sound(pool, s, 0, pages_for(l, pool.page_size))) err = SB_ERR_BOUNDS;
    }
    if (lane == 0) status[i] = err;
  }
  __syncthreads();
  // A destination held nothing when it was judged, so no entry reads a row that another one writes.
  for (int i = warp; i < n; i += PG_WARPS) {
    if (status[i]) continue;
    const int need = pages_for(len[i], pool.page_size);
    const int* from = pool.page_table + (long long)src[i] * pool.max_pages;
    int* to = pool.page_table + (long long)dst[i] * pool.max_pages;
    for (int p = lane; p < need; p += 32) {
      const int page = from[p];
      to[p] = page;
      atomicAdd(&pool.refs[page], 1);
    }
    if (lane == 0) pool.held[dst[i]] = need;
  }
}

// The logical pages [first, last) that hold positions [keep, upto) of a slot: none for an empty range, wherever it lies.
struct PageRange {
  int first, last;
  __device__ PageRange(int keep, int upto, int page_size)
      : first(keep / page_size), last(upto > keep ? pages_for(upto, page_size) : first) {}
};

struct ReserveWs {
  int *claim, *count, *first_of, *free_ids, *want, *copies;
  __device__ ReserveWs(int* ws, const sb_page_pool& pool, int n) {
    claim = ws;
    count = claim + pool.n_slots;
    first_of = count + pool.num_pages;
    free_ids = first_of + pool.num_pages;
    want = free_ids + pool.num_pages;
    copies = want + n;
  }
};

__global__ void __launch_bounds__(PG_THREADS) pages_reserve_kernel(const sb_page_pool pool, int n,
                                                                   const int* __restrict__ slots,
                                                                   const int* __restrict__ keep_len,
                                                                   const int* __restrict__ new_len, int* copy_src,
                                                                   int* copy_dst, int* n_copies, int* wsp, int* status) {
  __shared__ int s_scan[PG_WARPS + 1];
  pdl_wait();
  pdl_release();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, ps = pool.page_size;
  ReserveWs ws(wsp, pool, n);
  __shared__ unsigned long long s_wants;
  if (tid == 0) s_wants = 0;
  for (int i = tid; i < pool.num_pages; i += PG_THREADS) {
    ws.count[i] = 0;
    ws.first_of[i] = 0x7fffffff;
  }
  claim_slots(ws.claim, pool, slots, n);
  // judge every entry; count, for every page that will be written, its holders in this call and the first of them
  for (int i = warp; i < n; i += PG_WARPS) {
    const int s = slots[i], keep = keep_len[i], upto = new_len[i];
    int err = 0;
    if (s < 0 || s >= pool.n_slots || ws.claim[s] != i) {
      err = SB_ERR_INVALID_ARG;
    } else {
      const int held = pool.held[s];
      if (keep < 0 || upto < keep || held < 0 || held > pool.max_pages) err = SB_ERR_BOUNDS;
      else if (pages_for(upto, ps) > pool.max_pages || pages_for(keep, ps) > held) err = SB_ERR_BOUNDS;
      else {
        const PageRange r(keep, upto, ps);
        const int last = min(held, r.last);
        if (!pages_sound(pool, s, r.first, last)) err = SB_ERR_BOUNDS;
        else
          for (int p = r.first + lane; p < last; p += 32) {
            const int page = pool.page_table[(long long)s * pool.max_pages + p];
            atomicAdd(&ws.count[page], 1);
            atomicMin(&ws.first_of[page], i);
          }
      }
    }
    if (lane == 0) status[i] = err;
  }
  __syncthreads();
  // A shared page is replaced, except for the first holder when all holders are in the call.
  auto replaced = [&](int page, int i) {
    const int r = pool.refs[page];
    return r > 1 && !(ws.count[page] == r && ws.first_of[page] == i);
  };
  for (int i = warp; i < n; i += PG_WARPS) {
    int wants = 0, copies = 0;
    if (status[i] == 0) {
      const int s = slots[i], keep = keep_len[i], held = pool.held[s];
      const PageRange r(keep, new_len[i], ps);
      const int last = min(held, r.last);
      const int* row = pool.page_table + (long long)s * pool.max_pages;
      for (int p0 = r.first; p0 < last; p0 += 32) {
        const int p = p0 + lane;
        const bool rep = p < last && replaced(row[p], i);
        wants += __popc(__ballot_sync(0xffffffffu, rep));
        copies += __popc(__ballot_sync(0xffffffffu, rep && (long long)p * ps < keep));
      }
      wants += max(0, r.last - max(held, r.first));
    }
    if (lane == 0) {
      ws.want[i] = wants;
      ws.copies[i] = copies;
      atomicAdd(&s_wants, (unsigned long long)wants);
    }
  }
  __syncthreads();
  // ranks in list order; what the pool cannot hold at all is refused below, without sums that might leave 32 bits
  const bool too_many = s_wants > (unsigned long long)pool.num_pages;
  int wants_total = too_many ? 1 : 0, copies_total = 0;
  for (int i0 = 0; i0 < n; i0 += PG_THREADS) {
    const int i = i0 + tid;
    int t;
    const int w = i < n ? ws.want[i] : 0;
    const int wx = block_exclusive(too_many ? 0 : w, s_scan, &t);
    if (i < n) ws.want[i] = wants_total + wx;
    wants_total += t;
    const int c = i < n ? ws.copies[i] : 0;
    const int cx = block_exclusive(c, s_scan, &t);
    if (i < n) ws.copies[i] = copies_total + cx;
    copies_total += t;
    // an entry that asked for nothing is served whatever the pool holds: keep that in the sign of its rank
    if (i < n && w == 0) ws.want[i] = -1;
  }
  // the lowest free pages, ascending
  int found = 0;
  for (int p0 = 0; p0 < pool.num_pages && found < wants_total && !too_many; p0 += PG_THREADS) {
    const int p = p0 + tid;
    const int is_free = p < pool.num_pages && pool.refs[p] == 0 ? 1 : 0;
    int t;
    const int at = found + block_exclusive(is_free, s_scan, &t);
    if (is_free) ws.free_ids[at] = p;
    found += t;
  }
  __syncthreads();
  if (found < wants_total) {
    for (int i = tid; i < n; i += PG_THREADS) {
      if (status[i] == 0 && ws.want[i] >= 0) status[i] = SB_ERR_NO_PAGES;
      copy_src[i] = -1;
      copy_dst[i] = -1;
    }
    if (tid == 0) *n_copies = 0;
    return;
  }
  for (int i = copies_total + tid; i < n; i += PG_THREADS) {
    copy_src[i] = -1;
    copy_dst[i] = -1;
  }
  if (tid == 0) *n_copies = copies_total;
  // Every decision reads refs as they were: all are taken before any is changed.  A warp's first 32 pages
  // (keep and new length within 32 pages of each other: nearly always all of them) are decided here, ...
  for (int i0 = 0; i0 < n; i0 += PG_WARPS) {
    const int i = i0 + warp;
    const bool on = i < n && status[i] == 0 && ws.want[i] >= 0;
    if (on) {
      const int s = slots[i], keep = keep_len[i], held = pool.held[s];
      const PageRange r(keep, new_len[i], ps);
      const int last = r.last;
      int* row = pool.page_table + (long long)s * pool.max_pages;
      int rank = ws.want[i];
      for (int p0 = r.first; p0 < last; p0 += 32) {
        const int p = p0 + lane;
        // ... and each replacement is noted in the table as -2 - fresh until every warp has decided
        const bool have = p < min(held, last);
        const int page = have ? row[p] : -1;
        const bool rep = have && replaced(page, i);
        const bool want = rep || (p >= held && p < last);
        const unsigned m = __ballot_sync(0xffffffffu, want);
        if (want) {
          const int fresh = ws.free_ids[rank + __popc(m & ((1u << lane) - 1u))];
          if (rep && (long long)p * ps < keep) {
            copy_src[ws.copies[i]] = page;
            copy_dst[ws.copies[i]] = fresh;
          }
          row[p] = -2 - fresh;
          if (rep) ws.first_of[fresh] = page;  // a free page has no holder: its entry is unused
          else ws.first_of[fresh] = -1;
        }
        rank += __popc(m);
      }
    }
  }
  __syncthreads();
  for (int i = warp; i < n; i += PG_WARPS) {
    if (status[i] || ws.want[i] < 0) continue;
    const int s = slots[i];
    const PageRange r(keep_len[i], new_len[i], ps);
    const int last = r.last;
    int* row = pool.page_table + (long long)s * pool.max_pages;
    for (int p = r.first + lane; p < last; p += 32) {
      const int noted = row[p];
      if (noted <= -2) {
        const int fresh = -2 - noted, old = ws.first_of[fresh];
        row[p] = fresh;
        pool.refs[fresh] = 1;
        if (old >= 0) atomicSub(&pool.refs[old], 1);
      }
    }
    __syncwarp();
    if (lane == 0 && last > pool.held[s]) pool.held[s] = last;
  }
}

// Workspace of compact: [0] damage flag, [1 + c] used pages, [9 + c] moving pages, [17 + c] holes of CTA c's
// range; from 64: target page of every page that moves, from 64 + num_pages: the holes.
__global__ void __launch_bounds__(PG_THREADS) __cluster_dims__(PG_CLUSTER, 1, 1)
    pages_compact_kernel(const sb_page_pool pool, int* copy_src, int* copy_dst, int max_copies, int* n_copies, int* n_used,
                         int* ws, int* status) {
  __shared__ int s_scan[PG_WARPS + 1];
  cgp::cluster_group cluster = cgp::this_cluster();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, c = (int)cluster.block_rank();
  const int chunk = ceil_div(pool.num_pages, PG_CLUSTER);
  const int p_lo = min(pool.num_pages, c * chunk), p_hi = min(pool.num_pages, p_lo + chunk);
  volatile int* vws = ws;
  int* target = ws + 64;
  int* holes = target + pool.num_pages;
  pdl_wait();
  pdl_release();
  int mine = 0;
  for (int p = p_lo + tid; p < p_hi; p += PG_THREADS) mine += pool.refs[p] != 0 ? 1 : 0;
  int t;
  block_exclusive(mine, s_scan, &t);
  if (tid == 0) vws[1 + c] = t;
  if (c == 0 && tid == 0) vws[0] = 0;
  cluster.sync();
  int used = 0;
  for (int k = 0; k < PG_CLUSTER; ++k) used += vws[1 + k];
  // tables are checked while the pages are counted
  bool bad = false;
  for (int s = c * PG_WARPS + warp; s < pool.n_slots; s += PG_CLUSTER * PG_WARPS) {
    const int held = pool.held[s];
    if (held < 0 || held > pool.max_pages) bad = true;
    else if (!pages_sound(pool, s, 0, held)) bad = true;
  }
  if (bad && lane == 0) atomicOr(&ws[0], 1);
  int moving = 0, free_low = 0;
  for (int p = p_lo + tid; p < p_hi; p += PG_THREADS) {
    const bool u = pool.refs[p] != 0;
    moving += u && p >= used ? 1 : 0;
    free_low += !u && p < used ? 1 : 0;
  }
  int t2;
  block_exclusive(moving, s_scan, &t);
  block_exclusive(free_low, s_scan, &t2);
  if (tid == 0) {
    vws[9 + c] = t;
    vws[17 + c] = t2;
  }
  cluster.sync();
  const bool damaged = vws[0] != 0;
  int move_base = 0, hole_base = 0, moves = 0;
  for (int k = 0; k < PG_CLUSTER; ++k) {
    moves += vws[9 + k];
    move_base += k < c ? vws[9 + k] : 0;
    hole_base += k < c ? vws[17 + k] : 0;
  }
  if (damaged) moves = 0;
  // holes in ascending order; the moving pages' ranks go to `target` until the holes are known
  for (int p0 = p_lo; p0 < p_hi; p0 += PG_THREADS) {
    const int p = p0 + tid;
    const bool u = p < p_hi && pool.refs[p] != 0;
    const int is_move = u && p >= used ? 1 : 0, is_hole = p < p_hi && !u && p < used ? 1 : 0;
    const int mr = move_base + block_exclusive(is_move, s_scan, &t);
    move_base += t;
    const int hr = hole_base + block_exclusive(is_hole, s_scan, &t);
    hole_base += t;
    if (is_move) target[p] = mr;
    if (is_hole) holes[hr] = p;
  }
  cluster.sync();
  if (!damaged) {
    for (int p = max(p_lo, used) + tid; p < p_hi; p += PG_THREADS) {
      const int r = pool.refs[p];
      if (r == 0) continue;
      const int k = target[p], to = holes[k];
      target[p] = to;
      pool.refs[to] = r;  // a hole below `used`: nobody else touches its entry
      pool.refs[p] = 0;
      copy_src[k] = p;
      copy_dst[k] = to;
    }
  }
  for (int i = moves + c * PG_THREADS + tid; i < max_copies; i += PG_CLUSTER * PG_THREADS) {
    copy_src[i] = -1;
    copy_dst[i] = -1;
  }
  if (c == 0 && tid == 0) {
    *n_copies = moves;
    if (n_used) *n_used = used;
    status[0] = damaged ? (int)SB_ERR_BOUNDS : 0;
  }
  cluster.sync();
  if (damaged) return;
  for (int s = c * PG_WARPS + warp; s < pool.n_slots; s += PG_CLUSTER * PG_WARPS) {
    const int held = pool.held[s];
    int* row = pool.page_table + (long long)s * pool.max_pages;
    for (int p = lane; p < held; p += 32) {
      const int page = row[p];
      if (page >= used) row[p] = target[page];
    }
  }
}

// ---- contents -----------------------------------------------------------------------------------------------------

constexpr int PC_THREADS = 256;
constexpr int PC_PIECE = 16 * 1024;  // bytes per work item: 4 x 16 bytes per thread

struct PageArrays {
  sb_page_array a[SB_MAX_PAGE_ARRAYS];
  int piece_end[SB_MAX_PAGE_ARRAYS];  // pieces of arrays 0..i of one page
  int n;
};

__global__ void __launch_bounds__(PC_THREADS) pages_copy_kernel(const PageArrays arr, int n_layers, int num_pages,
                                                                const int* __restrict__ copy_src,
                                                                const int* __restrict__ copy_dst,
                                                                const int* __restrict__ n_copies, int max_copies) {
  pdl_wait();
  pdl_release();
  const int pairs = min(max(*n_copies, 0), max_copies);
  const int pieces = arr.piece_end[arr.n - 1];
  const long long items = (long long)pairs * n_layers * pieces;
  for (long long it = blockIdx.x; it < items; it += gridDim.x) {
    const long long page_it = it / pieces;
    int piece = (int)(it - page_it * pieces);
    const int layer = (int)(page_it / pairs), pair = (int)(page_it - (long long)layer * pairs);
    const int s = copy_src[pair], d = copy_dst[pair];
    if (s < 0 || s >= num_pages || d < 0 || d >= num_pages) continue;
    int k = 0;
    while (piece >= arr.piece_end[k]) ++k;
    if (k > 0) piece -= arr.piece_end[k - 1];
    const sb_page_array a = arr.a[k];
    char* base = static_cast<char*>(a.base) + layer * a.layer_stride;
    const long long at = (long long)piece * PC_PIECE;
    const int bytes = (int)min((long long)PC_PIECE, a.page_bytes - at);
    const char* from = base + s * a.page_bytes + at;
    char* to = base + d * a.page_bytes + at;
    const bool wide = ((reinterpret_cast<uintptr_t>(from) | reinterpret_cast<uintptr_t>(to) | (uintptr_t)bytes) & 15) == 0;
    if (wide) {
      uint4 v[PC_PIECE / 16 / PC_THREADS];
#pragma unroll
      for (int i = 0; i < PC_PIECE / 16 / PC_THREADS; ++i) {
        const int off = (i * PC_THREADS + threadIdx.x) * 16;
        if (off < bytes) v[i] = __ldcs(reinterpret_cast<const uint4*>(from + off));
      }
#pragma unroll
      for (int i = 0; i < PC_PIECE / 16 / PC_THREADS; ++i) {
        const int off = (i * PC_THREADS + threadIdx.x) * 16;
        if (off < bytes) __stcs(reinterpret_cast<uint4*>(to + off), v[i]);
      }
    } else {
      for (int off = threadIdx.x * 4; off < bytes; off += PC_THREADS * 4)
        *reinterpret_cast<uint32_t*>(to + off) = *reinterpret_cast<const uint32_t*>(from + off);
    }
  }
}

static sb_status check_pool(const sb_page_pool* pool) {
  if (!pool || pool->num_pages < 1 || pool->n_slots < 1 || pool->max_pages < 1 || !pool->page_table || !pool->held || !pool->refs)
    return SB_ERR_INVALID_ARG;
  if (pool->page_size < 16 || (pool->page_size & (pool->page_size - 1))) return SB_ERR_UNSUPPORTED;
  return SB_OK;
}

static sb_status check_pool_ws(const sb_page_pool* pool, int n, const void* ws, size_t bytes) {
  if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255) || bytes < sb_pages_workspace_bytes(pool, n)) return SB_ERR_WORKSPACE;
  return SB_OK;
}

}  // namespace sb

extern "C" size_t sb_pages_workspace_bytes(const sb_page_pool* pool, int32_t n) {
  if (sb::check_pool(pool) != SB_OK || n < 0) return 0;
  const size_t ints = (size_t)pool->n_slots + 3 * (size_t)pool->num_pages + 2 * (size_t)n + 64;
  return (ints * 4 + 255) & ~(size_t)255;
}

extern "C" sb_status sb_pages_fork(const sb_page_pool* pool, int32_t n, const int32_t* src, const int32_t* dst,
                                   const int32_t* len, void* workspace, size_t workspace_bytes, int32_t* status,
                                   void* stream) {
  sb::TraceRange trace_range("sb_pages_fork");
  using namespace sb;
  sb_status st = check_pool(pool);
  if (st != SB_OK) return st;
  if (n < 0 || (n > 0 && (!src || !dst || !len || !status))) return SB_ERR_INVALID_ARG;
  if ((st = check_pool_ws(pool, n, workspace, workspace_bytes)) != SB_OK) return st;
  if (n == 0) return SB_OK;
  return launch_dependent(pages_fork_kernel, dim3(1), dim3(PG_THREADS), static_cast<cudaStream_t>(stream), *pool, n, src, dst,
                          len, static_cast<int*>(workspace), status);
}

extern "C" sb_status sb_pages_reserve(const sb_page_pool* pool, int32_t n, const int32_t* slots, const int32_t* keep_len,
                                      const int32_t* new_len, int32_t* copy_src, int32_t* copy_dst, int32_t* n_copies,
                                      void* workspace, size_t workspace_bytes, int32_t* status, void* stream) {
  sb::TraceRange trace_range("sb_pages_reserve");
  using namespace sb;
  sb_status st = check_pool(pool);
  if (st != SB_OK) return st;
  if (n < 0 || !n_copies || (n > 0 && (!slots || !keep_len || !new_len || !copy_src || !copy_dst || !status)))
    return SB_ERR_INVALID_ARG;
  if ((st = check_pool_ws(pool, n, workspace, workspace_bytes)) != SB_OK) return st;
  return launch_dependent(pages_reserve_kernel, dim3(1), dim3(PG_THREADS), static_cast<cudaStream_t>(stream), *pool, n, slots,
                          keep_len, new_len, copy_src, copy_dst, n_copies, static_cast<int*>(workspace), status);
}

extern "C" sb_status sb_pages_release(const sb_page_pool* pool, int32_t n, const int32_t* slots, const int32_t* keep_len,
                                      void* workspace, size_t workspace_bytes, int32_t* status, void* stream) {
  sb::TraceRange trace_range("sb_pages_release");
  using namespace sb;
  sb_status st = check_pool(pool);
  if (st != SB_OK) return st;
  if (n < 0 || (n > 0 && (!slots || !keep_len || !status))) return SB_ERR_INVALID_ARG;
  if ((st = check_pool_ws(pool, n, workspace, workspace_bytes)) != SB_OK) return st;
  if (n == 0) return SB_OK;
  return launch_dependent(pages_release_kernel, dim3(1), dim3(PG_THREADS), static_cast<cudaStream_t>(stream), *pool, n, slots,
                          keep_len, static_cast<int*>(workspace), status);
}

extern "C" sb_status sb_pages_compact(const sb_page_pool* pool, int32_t* copy_src, int32_t* copy_dst, int32_t max_copies,
                                      int32_t* n_copies, int32_t* n_used, void* workspace, size_t workspace_bytes,
                                      int32_t* status, void* stream) {
  sb::TraceRange trace_range("sb_pages_compact");
  using namespace sb;
  sb_status st = check_pool(pool);
  if (st != SB_OK) return st;
  if (max_copies < pool->num_pages / 2 || !n_copies || !status || (max_copies > 0 && (!copy_src || !copy_dst)))
    return SB_ERR_INVALID_ARG;
  if ((st = check_pool_ws(pool, 0, workspace, workspace_bytes)) != SB_OK) return st;
  return launch_dependent(pages_compact_kernel, dim3(PG_CLUSTER), dim3(PG_THREADS), static_cast<cudaStream_t>(stream), *pool,
                          copy_src, copy_dst, max_copies, n_copies, n_used, static_cast<int*>(workspace), status);
}

extern "C" sb_status sb_pages_copy(const sb_page_array* arrays, int32_t n_arrays, int32_t n_layers, int32_t num_pages,
                                   const int32_t* copy_src, const int32_t* copy_dst, const int32_t* n_copies,
                                   int32_t max_copies, void* stream) {
  sb::TraceRange trace_range("sb_pages_copy");
  using namespace sb;
  if (!arrays || n_arrays < 1 || n_layers < 1 || num_pages < 1 || max_copies < 0 || !n_copies ||
      (max_copies > 0 && (!copy_src || !copy_dst)))
    return SB_ERR_INVALID_ARG;
  if (n_arrays > SB_MAX_PAGE_ARRAYS) return SB_ERR_UNSUPPORTED;
  PageArrays arr;
  arr.n = n_arrays;
  long long pieces = 0;
  for (int i = 0; i < n_arrays; ++i) {
    const sb_page_array& a = arrays[i];
    if (!a.base || a.page_bytes < 4 || a.page_bytes % 4 != 0 || a.layer_stride < 0 || a.layer_stride % 4 != 0 ||
        (reinterpret_cast<uintptr_t>(a.base) & 3))
      return SB_ERR_INVALID_ARG;
    if (n_layers > 1 && a.layer_stride / num_pages < a.page_bytes) return SB_ERR_INVALID_ARG;  // layers would overlap
    arr.a[i] = a;
    pieces += (a.page_bytes + PC_PIECE - 1) / PC_PIECE;
    if (pieces > (1 << 30)) return SB_ERR_UNSUPPORTED;
    arr.piece_end[i] = (int)pieces;
  }
  if (max_copies == 0) return SB_OK;
  // four CTAs per SM when the list could be long enough to fill them
  const long long most = (long long)max_copies * n_layers * pieces;
  const int fill = 4 * device_sms(), grid = (int)(most < fill ? most : fill);
  return launch_dependent(pages_copy_kernel, dim3(grid), dim3(PC_THREADS), static_cast<cudaStream_t>(stream), arr, n_layers,
                          num_pages, copy_src, copy_dst, n_copies, max_copies);
}
