// Pages of the cache that several sequences may hold: copying, forking, handing out and taking back, freeing behind a window,
// moving together.  refs[p] counts the places of the block table that hold page p; 0: the page is free.  Everything is decided on
// the device (the host knows neither lengths nor pages), so a serving step can be captured into a graph with these calls in it.
//
// Bookkeeping is one cluster of up to eight blocks a call, which meets between the phases that read and those that write: what
// a call decides is decided from the state before it, and free pages are ranked by prefix sums over the pages, lowest first, so
// results are the same from run to run.  Bound: latency, of three to five trips to L2 with a cluster barrier behind each.  Books that
// the threads of one block can keep in registers are read once instead.  Pages that move are listed in the workspace, and a second
// launch copies them in all layers: bound by HBM (100 MB read and written in 32 us, at the rate of a plain copy), past the other
// numbers in L2.
#include <algorithm>

#include "kvp_cache8.h"
#include "kvp_host.h"
#include "kvp_sm100.cuh"

namespace kvp {
namespace {

constexpr int BOOK_THREADS = 1024, BOOK_WARPS = BOOK_THREADS / 32, BOOK_BLOCKS = 8;
constexpr int MOST_ROWS = 1 << 14;         // rows of the block table: 12 bytes of shared memory each
constexpr int COPY_THREADS = 256, COPY_FLY = 4, COPIES_AN_SM = 8;
constexpr int COPY_CHUNK = COPY_THREADS * COPY_FLY * 16;   // bytes that a block has in flight
constexpr int MANY_POOLS = 64, FEW_POOLS = 8;              // owners of a launch: 2 KB of parameters, or 256 bytes

struct Book {
  int32_t* refs;            // [n_pages]
  int32_t* table;           // [B, max_pages]
  int32_t* lengths;         // [B]
  int B, page_size, max_pages, n_pages;
  __device__ __forceinline__ int places(int length) const { return min(max(0, length / page_size + (length % page_size > 0)), max_pages); }
  __device__ __forceinline__ bool is_page(int page) const { return unsigned(page) < unsigned(n_pages); }
  __device__ __forceinline__ int32_t& at(int row, int place) const { return table[size_t(row) * max_pages + place]; }
};

// The workspace: a list of pages to be copied, and what a call keeps between its phases.
struct BookSpace {
  int32_t* n_copies;        // [1]
  int32_t* counts;          // [3][BOOK_BLOCKS]
  int32_t *src, *dst;       // [max(n_pages, B)]
  int32_t* rows;            // [2][B]
  int32_t* places;          // fork: [B, max_pages], compact: [n_pages]
};
size_t align256(size_t x) { return (x + 255) & ~size_t(255); }
size_t list_entries(const kvp_decode_desc* d) { return std::max(d->n_pages, d->B); }
size_t book_bytes(const kvp_decode_desc* d) {
  return 256 + 2 * align256(list_entries(d) * 4) + align256(size_t(2) * d->B * 4) +
         align256(std::max(size_t(d->B) * d->max_pages, size_t(d->n_pages)) * 4);
}
BookSpace book_space(const kvp_decode_desc* d, void* ws) {
  uint8_t* p = static_cast<uint8_t*>(ws);
  BookSpace s;
  s.n_copies = reinterpret_cast<int32_t*>(p);
  s.counts = s.n_copies + 4;
  s.src = reinterpret_cast<int32_t*>(p += 256);
  s.dst = reinterpret_cast<int32_t*>(p += align256(list_entries(d) * 4));
  s.rows = reinterpret_cast<int32_t*>(p += align256(list_entries(d) * 4));
  s.places = reinterpret_cast<int32_t*>(p += align256(size_t(2) * d->B * 4));
  return s;
}
static_assert(16 + 3 * BOOK_BLOCKS * 4 <= 256, "the counts share the first 256 bytes of the workspace");

// Sum over the threads of the block before this one; total: of all.
__device__ __forceinline__ unsigned long long block_scan(unsigned long long v, unsigned long long* s_warp, unsigned long long& total) {
  const int warp = threadIdx.x >> 5, lane = lane_id();
  unsigned long long sum = v;
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const unsigned long long o = __shfl_up_sync(0xffffffffu, sum, d);
    if (lane >= d) sum += o;
  }
  __syncthreads();                      // (the last call's sums have been read)
  if (lane == 31) s_warp[warp] = sum;
  __syncthreads();
  unsigned long long w = s_warp[lane];
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const unsigned long long o = __shfl_up_sync(0xffffffffu, w, d);
    if (lane >= d) w += o;
  }
  total = __shfl_sync(0xffffffffu, w, 31);
  const unsigned long long before = __shfl_sync(0xffffffffu, w, (warp + 31) & 31);
  return (warp > 0 ? before : 0) + sum - v;
}
static_assert(BOOK_WARPS == 32, "a lane a warp");

// The pages of this block of the cluster, in whole rounds of the block's threads.
struct Slice {
  int begin, end;
  __device__ __forceinline__ explicit Slice(int n_pages) {
    const int blocks = int(cluster_nctarank()), each = ((n_pages + blocks - 1) / blocks + BOOK_THREADS - 1) / BOOK_THREADS * BOOK_THREADS;
    begin = int(min((long long)n_pages, (long long)each * cluster_ctarank()));
    end = int(min((long long)n_pages, (long long)begin + each));
  }
};
// counts[i] of the blocks before this one, and of all
__device__ __forceinline__ int sum_blocks(const int32_t* counts, int& total) {
  int before = 0;
  total = 0;
  for (int i = 0; i < int(cluster_nctarank()); ++i) {
    const int n = __ldcg(counts + i);
    before += i < int(cluster_ctarank()) ? n : 0;
    total += n;
  }
  return before;
}
template <typename F>
__device__ __forceinline__ int count_pages(const Slice& s, F f, unsigned long long* s_warp) {
  unsigned long long n = 0, total;
  for (int p = s.begin + int(threadIdx.x); p < s.end; p += BOOK_THREADS) n += f(p) ? 1 : 0;
  block_scan(n, s_warp, total);
  return int(total);
}

// ---------------------------------------------------------------------------------------------
// fork: row b goes on from what row parent[b] was
// ---------------------------------------------------------------------------------------------
// Rows' new places wait in the workspace until every row's old ones have been read.  A warp has 32 places of a row.
__global__ void __launch_bounds__(BOOK_THREADS, 1) fork_kernel(const __grid_constant__ Book p, const __grid_constant__ BookSpace ws, const int32_t* parent) {
  grid_dep_launch();
  grid_dep_wait();
  const int lane = lane_id();
  const uint32_t per_row = (p.max_pages + 31) / 32;
  const int first = int(cluster_ctarank()) * BOOK_WARPS + int(threadIdx.x >> 5), warps = int(cluster_nctarank()) * BOOK_WARPS;
  for (int phase = 0; phase < 2; ++phase) {
    for (uint32_t w = first; w < uint32_t(p.B) * per_row; w += warps) {
      const int row = int(w / per_row), place = int(w % per_row) * 32 + lane;
      const int from = parent[row];
      if (from == row || from < -1 || from >= p.B) continue;
      if (phase == 0) {
        const int length = from < 0 ? 0 : p.lengths[from];
        const int had = p.places(p.lengths[row]), have = p.places(length);
        if (place == 0) ws.rows[row] = length;
        if (place >= max(had, have)) continue;
        const int before = place < had ? p.at(row, place) : -1, after = place < have ? p.at(from, place) : -1;
        ws.places[size_t(row) * p.max_pages + place] = after;
        if (before == after) continue;
        if (p.is_page(before)) atomicSub(p.refs + before, 1);
        if (p.is_page(after)) atomicAdd(p.refs + after, 1);
      } else {
        // (lengths change behind the next meeting, so both sides still see the old one here)
        const int had = p.places(p.lengths[row]), have = p.places(__ldcg(ws.rows + row));
        if (place < max(had, have)) p.at(row, place) = __ldcg(ws.places + size_t(row) * p.max_pages + place);
      }
    }
    cluster_sync_all();
  }
  for (int row = int(cluster_ctarank()) * BOOK_THREADS + int(threadIdx.x); row < p.B; row += int(cluster_nctarank()) * BOOK_THREADS) {
    const int from = parent[row];
    if (from != row && from >= -1 && from < p.B) p.lengths[row] = __ldcg(ws.rows + row);
  }
}

// ---------------------------------------------------------------------------------------------
// resize: rows grow (a page that is shared is copied first) and shrink
// ---------------------------------------------------------------------------------------------
constexpr int STAYS = -1, GAP = -2;   // of a row, in the place of the page that it grows in: it does not grow in one; it grows in a place without
                                      // one (freed behind a window before the row shrank into it), and gets one there
struct Resized {            // one row, from the state before the call
  int had, have;            // places
  int end;                  // page that the row grows in, or one of the above
};
__device__ __forceinline__ int grows_in(const Book& p, int row, int length, int longer, int had) {
  if (longer <= length || length <= 0 || length % p.page_size == 0 || had <= 0) return STAYS;
  const int page = p.at(row, had - 1);
  return p.is_page(page) ? page : GAP;
}
__device__ __forceinline__ Resized resized(const Book& p, const int32_t* to, int row) {
  const int length = p.lengths[row], longer = to[row];
  Resized r;
  r.had = p.places(length);
  r.have = p.places(longer);
  r.end = grows_in(p, row, length, longer, r.had);
  return r;
}
__global__ void __launch_bounds__(BOOK_THREADS, 1) resize_kernel(const __grid_constant__ Book p, const __grid_constant__ BookSpace ws, const int32_t* to, int32_t* lacking) {
  extern __shared__ unsigned long long s_begin[];        // [B + 1] first new page of each row in 40 bits, above them the copies before it
  int* const s_end = reinterpret_cast<int*>(s_begin + p.B + 1);
  __shared__ unsigned long long s_warp[32];
  __shared__ int s_bad;
  constexpr int COPY_BIT = 40;
  grid_dep_launch();
  grid_dep_wait();
  const int rank = int(cluster_ctarank()), blocks = int(cluster_nctarank()), tid = int(threadIdx.x);
  // 1. what each row needs, and the free pages of each block's slice
  if (tid == 0) s_bad = 0;
  __syncthreads();
  bool bad = false;
  for (int row = tid; row < p.B; row += BOOK_THREADS) {
    s_end[row] = resized(p, to, row).end;
    bad |= to[row] < 0 || to[row] > (long long)p.max_pages * p.page_size;
  }
  if (bad) s_bad = 1;
  __syncthreads();
  for (int row = rank * BOOK_THREADS + tid; row < p.B; row += blocks * BOOK_THREADS) {
    const Resized r = resized(p, to, row);
    bool copies = false;
    if (r.end >= 0) {
      const int held = p.refs[r.end];
      if (held > 1) {                    // (all rows one after the other: 17 us where 300 share a page and grow, 59 where 1024 do, 1.0 ms where 16384 do)
        int growing = 0, lowest = row;
        for (int other = p.B - 1; other >= 0; --other)
          if (s_end[other] == r.end) {
            ++growing;
            lowest = other;
          }
        copies = growing != held || lowest != row;
      }
    }
    ws.rows[row] = max(0, r.have - r.had) + (r.end == GAP);
    ws.rows[p.B + row] = copies;
  }
  const Slice slice(p.n_pages);
  const int free_here = count_pages(slice, [&](int page) { return p.refs[page] == 0; }, s_warp);
  if (tid == 0) ws.counts[rank] = free_here;
  cluster_sync_all();
  // 2. whether there is room
  unsigned long long sum = 0;
  for (int row0 = 0; row0 < p.B; row0 += BOOK_THREADS) {
    const int row = row0 + tid;
    const unsigned long long copies = row < p.B ? __ldcg(ws.rows + p.B + row) : 0, more = row < p.B ? __ldcg(ws.rows + row) : 0;
    unsigned long long total;
    const unsigned long long before = block_scan((copies << COPY_BIT) + copies + more, s_warp, total);
    if (row < p.B) s_begin[row] = sum + before;
    sum += total;
  }
  if (tid == 0) s_begin[p.B] = sum;
  constexpr unsigned long long PAGES = (1ull << COPY_BIT) - 1;
  const long long need = (long long)(sum & PAGES);
  int n_free;
  long long rank_of = sum_blocks(ws.counts, n_free);
  const int short_of = s_bad ? -1 : int(max(0ll, min(0x7fffffffll, need - n_free)));
  if (rank == 0 && tid == 0) {
    *lacking = short_of;
    *ws.n_copies = short_of != 0 ? 0 : int(sum >> COPY_BIT);
  }
  if (short_of != 0) return;             // (the same in all blocks)
  __syncthreads();
  // 3. free pages to the rows, in order
  for (int page0 = slice.begin; page0 < slice.end && rank_of < need; page0 += BOOK_THREADS) {
    const int page = page0 + tid;
    const bool free = page < slice.end && p.refs[page] == 0;
    unsigned long long total;
    const long long k = rank_of + (long long)block_scan(free ? 1 : 0, s_warp, total);
    rank_of += (long long)total;
    if (!free || k >= need) continue;
    int lo = 0, hi = p.B - 1;            // last row that begins at or before k
    while (lo < hi) {
      const int mid = (lo + hi + 1) / 2;
      if ((long long)(s_begin[mid] & PAGES) <= k) lo = mid; else hi = mid - 1;
    }
    const int i = int(k - (long long)(s_begin[lo] & PAGES)), copies = int((s_begin[lo + 1] >> COPY_BIT) - (s_begin[lo] >> COPY_BIT));
    const int from = p.places(p.lengths[lo]) - copies - (s_end[lo] == GAP);       // place of its first
    if (i < copies) {
      const int at = int(s_begin[lo] >> COPY_BIT);
      ws.src[at] = s_end[lo];
      ws.dst[at] = page;
    }
    p.at(lo, from + i) = page;
    p.refs[page] = 1;
  }
  cluster_sync_all();
  // 4. what the rows give up
  for (int row = rank * BOOK_WARPS + (tid >> 5); row < p.B; row += blocks * BOOK_WARPS) {
    const int lane = lane_id(), had = p.places(p.lengths[row]), have = p.places(to[row]);
    if (lane == 0 && (s_begin[row + 1] >> COPY_BIT) != (s_begin[row] >> COPY_BIT)) atomicSub(p.refs + s_end[row], 1);
    for (int place = have + lane; place < had; place += 32) {
      const int page = p.at(row, place);
      if (p.is_page(page)) atomicSub(p.refs + page, 1);
      p.at(row, place) = -1;
    }
    __syncwarp();
    if (lane == 0) p.lengths[row] = to[row];
  }
}

// ---------------------------------------------------------------------------------------------
// the same for small books: one block, whose threads keep what they have read
// ---------------------------------------------------------------------------------------------
// Every number is read once, as many as the threads have at a time, and what is decided stays in registers and shared memory: one chain
// of loads instead of one for each phase (32 rows of 25 places, two resizes with what they copy, from a graph: 16.4 -> 10.8 us; 64 rows of
// 24, a fork and two resizes 57 -> 49).
constexpr int FEW_PAGES = 8, FEW_PLACES = 4;      // of a thread: pages, and places of the table
__global__ void __launch_bounds__(BOOK_THREADS, 1) fork_few_kernel(const __grid_constant__ Book p, const int32_t* parent) {
  grid_dep_launch();
  grid_dep_wait();
  const int lane = lane_id(), per_row = (p.max_pages + 31) / 32, items = p.B * per_row;
  int row[FEW_PLACES], place[FEW_PLACES], from[FEW_PLACES], length[FEW_PLACES], had[FEW_PLACES], have[FEW_PLACES], before[FEW_PLACES], after[FEW_PLACES];
#pragma unroll
  for (int u = 0; u < FEW_PLACES; ++u) {
    const int w = u * BOOK_WARPS + int(threadIdx.x >> 5);
    row[u] = w < items ? w / per_row : -1;
    place[u] = w % per_row * 32 + lane;
    from[u] = row[u] >= 0 ? parent[row[u]] : 0;
    if (from[u] == row[u] || from[u] < -1 || from[u] >= p.B) row[u] = -1;
  }
#pragma unroll
  for (int u = 0; u < FEW_PLACES; ++u) {
    length[u] = row[u] >= 0 && from[u] >= 0 ? p.lengths[from[u]] : 0;
    had[u] = row[u] >= 0 ? p.places(p.lengths[row[u]]) : 0;
    have[u] = p.places(length[u]);
  }
#pragma unroll
  for (int u = 0; u < FEW_PLACES; ++u) {
    before[u] = place[u] < had[u] ? p.at(row[u], place[u]) : -1;
    after[u] = place[u] < have[u] ? p.at(from[u], place[u]) : -1;
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < FEW_PLACES; ++u) {
    if (row[u] < 0) continue;
    if (place[u] == 0) p.lengths[row[u]] = length[u];
    if (place[u] < max(had[u], have[u])) p.at(row[u], place[u]) = after[u];
    if (before[u] == after[u]) continue;
    if (p.is_page(before[u])) atomicSub(p.refs + before[u], 1);
    if (p.is_page(after[u])) atomicAdd(p.refs + after[u], 1);
  }
}
__global__ void __launch_bounds__(BOOK_THREADS, 1) resize_few_kernel(const __grid_constant__ Book p, const __grid_constant__ BookSpace ws, const int32_t* to, int32_t* lacking) {
  __shared__ int s_need[BOOK_THREADS + 1], s_copies[BOOK_THREADS + 1], s_had[BOOK_THREADS], s_have[BOOK_THREADS];   // first new page and copy of each row
  __shared__ __align__(16) int s_end[BOOK_THREADS];
  __shared__ unsigned long long s_warp[32];
  grid_dep_launch();
  grid_dep_wait();
  const int tid = int(threadIdx.x), each = (p.n_pages + BOOK_THREADS - 1) / BOOK_THREADS, lane = lane_id();
  uint32_t free = 0;                     // of the thread's pages, tid * each + u
#pragma unroll
  for (int u = 0; u < FEW_PAGES; ++u)
    if (u < each && tid * each + u < p.n_pages && p.refs[tid * each + u] == 0) free |= 1u << u;
  const bool is_row = tid < p.B;
  const int length = is_row ? p.lengths[tid] : 0, longer = is_row ? to[tid] : 0, had = p.places(length), have = p.places(longer);
  const int end = is_row ? grows_in(p, tid, length, longer, had) : STAYS;
  const int held = end >= 0 ? p.refs[end] : 0;
  s_had[tid] = had;
  s_have[tid] = have;
  s_end[tid] = end;
  const bool bad = __syncthreads_or(longer < 0 || longer > (long long)p.max_pages * p.page_size) != 0;
  bool copies = false;
  if (held > 1) {
    int growing = 0, lowest = tid;
    for (int i = (p.B - 1) / 4; i >= 0; --i) {
      const int4 of = reinterpret_cast<const int4*>(s_end)[i];
      growing += (of.x == end) + (of.y == end) + (of.z == end) + (of.w == end);
      lowest = min(lowest, of.x == end ? 4 * i : of.y == end ? 4 * i + 1 : of.z == end ? 4 * i + 2 : of.w == end ? 4 * i + 3 : lowest);
    }
    copies = growing != held || lowest != tid;
  }
  // new pages, copies and free pages ahead of the thread's, 20 bits each (none is above FEW_PAGES * BOOK_THREADS)
  const unsigned long long mine = (unsigned long long)(max(0, have - had) + copies + (end == GAP)) | (unsigned long long)copies << 20 | (unsigned long long)__popc(free) << 40;
  unsigned long long total;
  const unsigned long long ahead = block_scan(mine, s_warp, total);
  constexpr uint32_t LOW = (1u << 20) - 1;
  const int need = int(total & LOW), n_free = int(total >> 40);
  s_need[tid] = int(ahead & LOW);
  s_copies[tid] = int(ahead >> 20 & LOW);
  if (tid == 0) {
    s_need[BOOK_THREADS] = need;
    s_copies[BOOK_THREADS] = int(total >> 20 & LOW);
  }
  const int short_of = bad ? -1 : max(0, need - n_free);
  if (tid == 0) {
    *lacking = short_of;
    *ws.n_copies = short_of != 0 ? 0 : int(total >> 20 & LOW);
  }
  if (short_of != 0) return;             // (the same in all threads)
  __syncthreads();
  for (int k = int(ahead >> 40); free != 0 && k < need; free &= free - 1, ++k) {
    const int page = tid * each + __ffs(free) - 1;
    int lo = 0, hi = p.B - 1;            // last row that begins at or before k
    while (lo < hi) {
      const int mid = (lo + hi + 1) / 2;
      if (s_need[mid] <= k) lo = mid; else hi = mid - 1;
    }
    const int i = k - s_need[lo], its_copies = s_copies[lo + 1] - s_copies[lo];
    if (i < its_copies) {
      ws.src[s_copies[lo]] = s_end[lo];
      ws.dst[s_copies[lo]] = page;
    }
    p.at(lo, s_had[lo] - its_copies - (s_end[lo] == GAP) + i) = page;
    p.refs[page] = 1;
  }
  if (copies) atomicSub(p.refs + end, 1);
  if (is_row) p.lengths[tid] = longer;
  // (what a row gives up is at other places and of other pages than what the others get)
  for (int row = tid >> 5; row < p.B; row += BOOK_WARPS)
    for (int place = s_have[row] + lane; place < s_had[row]; place += 32) {
      const int page = p.at(row, place);
      if (p.is_page(page)) atomicSub(p.refs + page, 1);
      p.at(row, place) = -1;
    }
}
__global__ void __launch_bounds__(BOOK_THREADS, 1) compact_few_kernel(const __grid_constant__ Book p, const __grid_constant__ BookSpace ws, int32_t* used_out) {
  __shared__ uint16_t s_hole[FEW_PAGES * BOOK_THREADS / 2], s_to[FEW_PAGES * BOOK_THREADS];    // holes by rank; new numbers of the pages that move
  __shared__ unsigned long long s_warp[32];
  __shared__ int s_below;
  grid_dep_launch();
  grid_dep_wait();
  const int tid = int(threadIdx.x), each = (p.n_pages + BOOK_THREADS - 1) / BOOK_THREADS, lane = lane_id();
  const int per_row = (p.max_pages + 31) / 32, items = p.B * per_row;
  int refs[FEW_PAGES], named[FEW_PLACES];
#pragma unroll
  for (int u = 0; u < FEW_PAGES; ++u) refs[u] = u < each && tid * each + u < p.n_pages ? p.refs[tid * each + u] : 0;
#pragma unroll
  for (int u = 0; u < FEW_PLACES; ++u) {
    const int w = u * BOOK_WARPS + (tid >> 5), row = w / per_row, place = w % per_row * 32 + lane;
    named[u] = w < items && place < p.places(p.lengths[row]) ? p.at(row, place) : -1;
  }
  int mine = 0;
#pragma unroll
  for (int u = 0; u < FEW_PAGES; ++u) mine += refs[u] != 0;
  unsigned long long total;
  const int ahead = int(block_scan(mine, s_warp, total)), used = int(total);
  // Holes are the free pages below `used`, movers the used ones at or above it: as many.  A page's rank among either follows from
  // the number of used pages below it.
  if (tid == 0 && used == p.n_pages) s_below = used;
  for (int u = 0, before = ahead; u < each; ++u) {
    const int page = tid * each + u;
    if (page >= p.n_pages) break;
    int r = 0;
#pragma unroll
    for (int k = 0; k < FEW_PAGES; ++k) r = k == u ? refs[k] : r;
    if (page == used) s_below = before;
    if (page < used && r == 0) s_hole[page - before] = uint16_t(page);
    if (page >= used) s_to[page] = 0xffff;
    before += r != 0;
  }
  __syncthreads();
  const int below = s_below;             // used pages below `used`
  if (tid == 0) {
    *used_out = used;
    *ws.n_copies = used - below;
  }
  if (used == below) return;             // (the same in all threads)
  for (int u = 0, before = ahead; u < each; ++u) {
    const int page = tid * each + u;
    if (page >= p.n_pages) break;
    int r = 0;
#pragma unroll
    for (int k = 0; k < FEW_PAGES; ++k) r = k == u ? refs[k] : r;
    if (page >= used && r != 0) {
      const int rank = before - below, to = s_hole[rank];
      s_to[page] = uint16_t(to);
      ws.src[rank] = page;
      ws.dst[rank] = to;
      p.refs[to] = r;
      p.refs[page] = 0;
    }
    before += r != 0;
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < FEW_PLACES; ++u) {
    if (named[u] < used || named[u] >= p.n_pages || s_to[named[u]] == 0xffff) continue;
    const int w = u * BOOK_WARPS + (tid >> 5);
    p.at(w / per_row, w % per_row * 32 + lane) = s_to[named[u]];
  }
}
static_assert(FEW_PAGES * BOOK_THREADS < 0xffff && FEW_PLACES * BOOK_WARPS <= BOOK_THREADS, "numbers of pages in 16 bits; a thread a row");

// ---------------------------------------------------------------------------------------------
// trim: places that no later token sees
// ---------------------------------------------------------------------------------------------
constexpr int TRIM_THREADS = 256;
__global__ void __launch_bounds__(TRIM_THREADS) trim_kernel(const __grid_constant__ Book p, int window, int sinks) {
  grid_dep_launch();
  grid_dep_wait();
  const int row = blockIdx.x, length = p.lengths[row];
  // the next token, at position length, sees positions above length - window
  const int keep = min(p.places(length), max(0, (length - window + 1)) / p.page_size), first = sinks / p.page_size + (sinks % p.page_size > 0);
  for (int place = first + int(threadIdx.x); place < keep; place += TRIM_THREADS) {
    const int page = p.at(row, place);
    if (!p.is_page(page)) continue;
    atomicSub(p.refs + page, 1);
    p.at(row, place) = -1;
  }
}

// ---------------------------------------------------------------------------------------------
// compact: used pages from the end of the pool into the free ones at its front
// ---------------------------------------------------------------------------------------------
__global__ void __launch_bounds__(BOOK_THREADS, 1) compact_kernel(const __grid_constant__ Book p, const __grid_constant__ BookSpace ws, int32_t* used_out) {
  __shared__ unsigned long long s_warp[32];
  grid_dep_launch();
  grid_dep_wait();
  const int rank = int(cluster_ctarank()), blocks = int(cluster_nctarank()), tid = int(threadIdx.x);
  const Slice slice(p.n_pages);
  const int used_here = count_pages(slice, [&](int page) { return p.refs[page] != 0; }, s_warp);
  if (tid == 0) ws.counts[rank] = used_here;
  cluster_sync_all();
  int used;
  const int used_before = sum_blocks(ws.counts, used);
  // Holes are the free pages below `used`, movers the used ones at or above it: as many.  A page's rank among either follows from
  // the number of used pages below it.
  const int holes_here = count_pages(slice, [&](int page) { return page < used && p.refs[page] == 0; }, s_warp);
  if (tid == 0) ws.counts[BOOK_BLOCKS + rank] = holes_here;
  cluster_sync_all();
  int holes;
  sum_blocks(ws.counts + BOOK_BLOCKS, holes);
  long long seen = used_before;
  for (int page0 = slice.begin; page0 < slice.end; page0 += BOOK_THREADS) {
    const int page = page0 + tid;
    const bool is_used = page < slice.end && p.refs[page] != 0;
    unsigned long long total;
    const long long before = seen + (long long)block_scan(is_used ? 1 : 0, s_warp, total);   // used pages below this one
    seen += (long long)total;
    if (page >= slice.end) continue;
    if (page < used && !is_used) ws.dst[page - before] = page;
    if (page >= used && is_used) ws.src[before - (used - holes)] = page;
  }
  cluster_sync_all();
  for (int i = rank * BOOK_THREADS + tid; i < holes; i += blocks * BOOK_THREADS) {
    const int from = __ldcg(ws.src + i), to = __ldcg(ws.dst + i);
    ws.places[from] = to;
    p.refs[to] = p.refs[from];
    p.refs[from] = 0;
  }
  if (rank == 0 && tid == 0) {
    *used_out = used;
    *ws.n_copies = holes;
  }
  cluster_sync_all();
  if (holes == 0) return;
  const int lane = lane_id();
  const uint32_t per_row = (p.max_pages + 31) / 32;
  for (uint32_t w = rank * BOOK_WARPS + (tid >> 5); w < uint32_t(p.B) * per_row; w += blocks * BOOK_WARPS) {
    const int row = int(w / per_row), place = int(w % per_row) * 32 + lane;
    if (place >= p.places(p.lengths[row])) continue;
    const int page = p.at(row, place);
    if (page < used || page >= p.n_pages) continue;
    const int to = __ldcg(ws.places + page);
    if (unsigned(to) < unsigned(used)) p.at(row, place) = to;
  }
}

// ---------------------------------------------------------------------------------------------
// copying
// ---------------------------------------------------------------------------------------------
struct Pools {
  uint8_t *k, *v, *k_scale, *v_scale;      // scales: null in a bf16 cache
};
struct CopySizes {
  const int32_t *src, *dst;
  const int32_t* n_device;                 // entries of the list, or null: n
  int n, n_pages, n_pools;
  uint32_t page_bytes, scale_bytes;        // of K or V
};
template <int NP>
struct CopyParams : CopySizes {
  Pools at[NP];
};
// A block takes pieces of 16 KB, all layers' K and V of an entry behind one another; scales go with the first piece of a page.
template <int NP>
__global__ void __launch_bounds__(COPY_THREADS) copy_pages_kernel(const __grid_constant__ CopyParams<NP> p) {
  grid_dep_launch();
  grid_dep_wait();
  const int n = p.n_device != nullptr ? __ldcg(p.n_device) : p.n;
  const uint32_t pieces = (p.page_bytes + COPY_CHUNK - 1) / COPY_CHUNK, per_entry = pieces * 2 * p.n_pools;
  for (long long w = blockIdx.x; w < (long long)n * per_entry; w += gridDim.x) {
    const int entry = int(w / per_entry);
    const uint32_t in = uint32_t(w % per_entry), which = in / pieces, piece = in % pieces;
    const int from = __ldcg(p.src + entry), to = __ldcg(p.dst + entry);
    if (from == to || unsigned(from) >= unsigned(p.n_pages) || unsigned(to) >= unsigned(p.n_pages)) continue;
    const Pools& at = p.at[which >> 1];
    uint8_t* const pool = which & 1 ? at.v : at.k;
    const uint8_t* const src = pool + size_t(from) * p.page_bytes;
    uint8_t* const dst = pool + size_t(to) * p.page_bytes;
    uint4 held[COPY_FLY];
#pragma unroll
    for (int u = 0; u < COPY_FLY; ++u) {
      const uint32_t off = piece * COPY_CHUNK + (u * COPY_THREADS + threadIdx.x) * 16;
      if (off < p.page_bytes) held[u] = __ldcs(reinterpret_cast<const uint4*>(src + off));
    }
#pragma unroll
    for (int u = 0; u < COPY_FLY; ++u) {
      const uint32_t off = piece * COPY_CHUNK + (u * COPY_THREADS + threadIdx.x) * 16;
      if (off < p.page_bytes) __stcs(reinterpret_cast<uint4*>(dst + off), held[u]);
    }
    uint8_t* const scales = which & 1 ? at.v_scale : at.k_scale;
    if (piece == 0 && scales != nullptr)
      for (uint32_t i = threadIdx.x; i < p.scale_bytes; i += COPY_THREADS) scales[size_t(to) * p.scale_bytes + i] = scales[size_t(from) * p.scale_bytes + i];
  }
}

template <int NP>
cudaError_t launch_copy(const CopyParams<MANY_POOLS>& all, long long most, cudaStream_t stream) {
  CopyParams<NP> p;
  static_cast<CopySizes&>(p) = all;
  std::copy(all.at, all.at + all.n_pools, p.at);
  const long long blocks = most * ((all.page_bytes + COPY_CHUNK - 1) / COPY_CHUNK) * 2 * all.n_pools;
  return launch_kernel(copy_pages_kernel<NP>, unsigned(std::min(blocks, (long long)COPIES_AN_SM * sm_count())), COPY_THREADS, 0, stream, 1, p);
}
// most: entries of the list at most (n_device holds their number), or all of them
int copy_pages(const kvp_decode_desc* d, const int32_t* donor, const int32_t* src, const int32_t* dst, const int32_t* n_device, int most, void* const* k_cache,
               void* const* v_cache, uint8_t* const* k_scale, uint8_t* const* v_scale, cudaStream_t stream) {
  CopyParams<MANY_POOLS> p;
  p.src = src;
  p.dst = dst;
  p.n_device = n_device;
  p.n = most;
  p.n_pages = d->n_pages;
  p.n_pools = 0;
  p.page_bytes = uint32_t(d->Hkv) * d->page_size * d->dh * (k_scale != nullptr ? 1 : 2);
  p.scale_bytes = uint32_t(d->Hkv) * (d->page_size / CACHE_BLOCK);
  for (int l = 0; l <= d->L; ++l) {
    if (l < d->L && donor[l] == l) {
      const bool scaled = k_scale != nullptr;
      p.at[p.n_pools++] = Pools{static_cast<uint8_t*>(k_cache[l]), static_cast<uint8_t*>(v_cache[l]), scaled ? k_scale[l] : nullptr, scaled ? v_scale[l] : nullptr};
    }
    if (p.n_pools == MANY_POOLS || (l == d->L && p.n_pools > 0)) {
      const cudaError_t e = p.n_pools <= FEW_POOLS ? launch_copy<FEW_POOLS>(p, most, stream) : launch_copy<MANY_POOLS>(p, most, stream);
      if (e != cudaSuccess) return KVP_ERR_CUDA;
      p.n_pools = 0;
    }
  }
  return KVP_OK;
}

// ---------------------------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------------------------
// Sizes that all of these calls go by; Hq, dtype and num_splits are not read.
int check_book(const kvp_decode_desc* d) {
  if (d == nullptr) return KVP_ERR_INVALID_ARG;
  if (d->L < 1 || d->B < 1 || d->Hkv < 1 || d->max_pages < 1 || d->n_pages < 1) return KVP_ERR_INVALID_ARG;
  if ((d->dh != 64 && d->dh != 128) || d->page_size < CACHE_BLOCK || d->page_size % CACHE_BLOCK != 0 || (long long)d->max_pages * d->page_size > 0x7fffffffLL ||
      (long long)d->Hkv * d->page_size * d->dh > (1 << 30) || d->B > MOST_ROWS || (long long)d->B * ((d->max_pages + 31) / 32) > 0x7fffffffLL || d->n_pages > 0x7fffffff - BOOK_BLOCKS * BOOK_THREADS)
    return KVP_ERR_UNSUPPORTED;
  return KVP_OK;
}
int check_pools(const kvp_decode_desc* d, const int32_t* donor, void* const* k_cache, void* const* v_cache, uint8_t* const* k_scale, uint8_t* const* v_scale) {
  if (donor == nullptr || k_cache == nullptr || v_cache == nullptr || (k_scale == nullptr) != (v_scale == nullptr)) return KVP_ERR_INVALID_ARG;
  for (int l = 0; l < d->L; ++l)
    if (donor[l] < 0 || donor[l] > l || donor[donor[l]] != donor[l]) return KVP_ERR_BAD_DONOR;
  for (int l = 0; l < d->L; ++l) {
    if (donor[l] != l) continue;
    if (k_cache[l] == nullptr || v_cache[l] == nullptr || (k_scale != nullptr && (k_scale[l] == nullptr || v_scale[l] == nullptr))) return KVP_ERR_INVALID_ARG;
    if (!aligned16(k_cache[l]) || !aligned16(v_cache[l])) return KVP_ERR_UNSUPPORTED;
  }
  return KVP_OK;
}
int check_space(const kvp_decode_desc* d, const void* ws, size_t ws_bytes) {
  if (ws == nullptr || ws_bytes < book_bytes(d)) return KVP_ERR_WORKSPACE;
  return aligned16(ws) ? KVP_OK : KVP_ERR_UNSUPPORTED;
}
Book book_of(const kvp_decode_desc* d, int32_t* refs, int32_t* table, int32_t* lengths) {
  return Book{refs, table, lengths, d->B, d->page_size, d->max_pages, d->n_pages};
}
// Blocks of the cluster: one where its threads have no more than a few places and pages each.
int book_blocks(const kvp_decode_desc* d) {
  const long long work = (long long)d->B * d->max_pages + d->n_pages;
  return work <= 8 * BOOK_THREADS ? 1 : BOOK_BLOCKS;
}
// Rows, pages and places that one block's threads can keep
bool few(const kvp_decode_desc* d) {
  return d->n_pages <= FEW_PAGES * BOOK_THREADS && (long long)d->B * ((d->max_pages + 31) / 32) <= FEW_PLACES * BOOK_WARPS;
}

}  // namespace
}  // namespace kvp

using namespace kvp;

extern "C" {

size_t kvp_pages_workspace_bytes(const kvp_decode_desc* d) { return check_book(d) == KVP_OK ? book_bytes(d) : 0; }

int kvp_pages_copy(const kvp_decode_desc* d, const int32_t* donor, int32_t n, const int32_t* src, const int32_t* dst, void* const* k_cache, void* const* v_cache,
                   uint8_t* const* k_scale, uint8_t* const* v_scale, kvp_stream_t stream) {
  int rc = check_book(d);
  if (rc != KVP_OK) return rc;
  if (n < 0 || (n > 0 && (src == nullptr || dst == nullptr))) return KVP_ERR_INVALID_ARG;
  rc = check_pools(d, donor, k_cache, v_cache, k_scale, v_scale);
  if (rc != KVP_OK || n == 0) return rc;
  return copy_pages(d, donor, src, dst, nullptr, n, k_cache, v_cache, k_scale, v_scale, reinterpret_cast<cudaStream_t>(stream));
}

int kvp_pages_fork(const kvp_decode_desc* d, const int32_t* parent, int32_t* refs, int32_t* block_table, int32_t* lengths, void* ws, size_t ws_bytes,
                   kvp_stream_t stream) {
  int rc = check_book(d);
  if (rc != KVP_OK) return rc;
  if (parent == nullptr || refs == nullptr || block_table == nullptr || lengths == nullptr) return KVP_ERR_INVALID_ARG;
  rc = check_space(d, ws, ws_bytes);
  if (rc != KVP_OK) return rc;
  const int blocks = book_blocks(d);
  const Book book = book_of(d, refs, block_table, lengths);
  const cudaError_t e = few(d) ? launch_kernel(fork_few_kernel, 1, BOOK_THREADS, 0, reinterpret_cast<cudaStream_t>(stream), 1, book, parent)
                               : launch_kernel(fork_kernel, blocks, BOOK_THREADS, 0, reinterpret_cast<cudaStream_t>(stream), blocks, book, book_space(d, ws), parent);
  return e == cudaSuccess ? KVP_OK : KVP_ERR_CUDA;
}

int kvp_pages_resize(const kvp_decode_desc* d, const int32_t* donor, const int32_t* new_lengths, int32_t* refs, int32_t* block_table, int32_t* lengths,
                     int32_t* lacking, void* ws, size_t ws_bytes, void* const* k_cache, void* const* v_cache, uint8_t* const* k_scale, uint8_t* const* v_scale,
                     kvp_stream_t stream_) {
  int rc = check_book(d);
  if (rc != KVP_OK) return rc;
  if (new_lengths == nullptr || refs == nullptr || block_table == nullptr || lengths == nullptr || lacking == nullptr) return KVP_ERR_INVALID_ARG;
  rc = check_pools(d, donor, k_cache, v_cache, k_scale, v_scale);
  if (rc != KVP_OK) return rc;
  rc = check_space(d, ws, ws_bytes);
  if (rc != KVP_OK) return rc;
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
  const BookSpace space = book_space(d, ws);
  const int blocks = book_blocks(d), smem = (d->B + 1) * 8 + d->B * 4;
  if (allow_smem<resize_kernel>((MOST_ROWS + 1) * 8 + MOST_ROWS * 4) != cudaSuccess) return KVP_ERR_CUDA;
  const Book book = book_of(d, refs, block_table, lengths);
  const cudaError_t e = few(d) ? launch_kernel(resize_few_kernel, 1, BOOK_THREADS, 0, stream, 1, book, space, new_lengths, lacking)
                               : launch_kernel(resize_kernel, blocks, BOOK_THREADS, smem, stream, blocks, book, space, new_lengths, lacking);
  if (e != cudaSuccess) return KVP_ERR_CUDA;
  return copy_pages(d, donor, space.src, space.dst, space.n_copies, d->B, k_cache, v_cache, k_scale, v_scale, stream);
}

int kvp_pages_trim(const kvp_decode_desc* d, int32_t window, int32_t sinks, int32_t* refs, int32_t* block_table, const int32_t* lengths, kvp_stream_t stream) {
  const int rc = check_book(d);
  if (rc != KVP_OK) return rc;
  if (window < 1 || sinks < 0 || refs == nullptr || block_table == nullptr || lengths == nullptr) return KVP_ERR_INVALID_ARG;
  const cudaError_t e = launch_kernel(trim_kernel, d->B, TRIM_THREADS, 0, reinterpret_cast<cudaStream_t>(stream), 1,
                                      book_of(d, refs, block_table, const_cast<int32_t*>(lengths)), window, sinks);
  return e == cudaSuccess ? KVP_OK : KVP_ERR_CUDA;
}

int kvp_pages_compact(const kvp_decode_desc* d, const int32_t* donor, int32_t* refs, int32_t* block_table, const int32_t* lengths, int32_t* used, void* ws,
                      size_t ws_bytes, void* const* k_cache, void* const* v_cache, uint8_t* const* k_scale, uint8_t* const* v_scale, kvp_stream_t stream_) {
  int rc = check_book(d);
  if (rc != KVP_OK) return rc;
  if (refs == nullptr || block_table == nullptr || lengths == nullptr || used == nullptr) return KVP_ERR_INVALID_ARG;
  rc = check_pools(d, donor, k_cache, v_cache, k_scale, v_scale);
  if (rc != KVP_OK) return rc;
  rc = check_space(d, ws, ws_bytes);
  if (rc != KVP_OK) return rc;
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
  const BookSpace space = book_space(d, ws);
  const int blocks = book_blocks(d);
  const Book book = book_of(d, refs, block_table, const_cast<int32_t*>(lengths));
  const cudaError_t e = few(d) ? launch_kernel(compact_few_kernel, 1, BOOK_THREADS, 0, stream, 1, book, space, used)
                               : launch_kernel(compact_kernel, blocks, BOOK_THREADS, 0, stream, blocks, book, space, used);
  if (e != cudaSuccess) return KVP_ERR_CUDA;
  return copy_pages(d, donor, space.src, space.dst, space.n_copies, d->n_pages, k_cache, v_cache, k_scale, v_scale, stream);
}

}  // extern "C"
