// Pages of a growing cache: room for new rows, sequences that go on from others, and pages moved together.
//
// A page is free if no table entry names it (refs[page] == 0).  New pages are the lowest free ones in ascending order, dealt to
// the requests in the order (layer, sequence, head, page), so the outcome depends on nothing but the inputs.  The kernels:
//   0. where sequences change places: pages_stage_kernel (in place) sets all arrays aside, pages_refs_kernel (into other arrays)
//      copies refs, ahead of step 1, which adjusts them.  Staging goes by the width of the tables, whatever the lengths (8
//      sequences x 32 layers x 8 heads, 13 pages at most each: tables 14 pages wide 14 us for the whole fork, 8192 wide 50).
//   1. pages_carry_kernel   (`to` is another set of arrays, or sequences change places) tables, lens and refs of `to` from those
//      of `from`, counts of shared pages adjusted.  Grid over the table, bound by its bytes.
//   2. pages_deal_kernel / pages_pair_kernel   one cluster of 8 CTAs, because every page's place depends on all pages below it:
//      each warp counts its consecutive share of refs, the sums meet in the CTA and, through distributed shared memory, in the
//      cluster, and a second look at the share gives each free page its rank.  Bound by the latency of those steps; refs come from
//      the L2 in 16-byte loads.  (A scan of the CTA for every 4096 pages, or shares of threads, whose entries of the lists lie in
//      sectors of their own: 45 us for 290000 pages, 27 this way, both with a cold L2.)
//   3. pages_copy_kernel / pages_move_kernel   rows of part-filled pages to their copies, or whole pages downwards together with the
//      tables that name them.  Bound by memory.
// All or nothing: step 2 knows whether there is room before it changes anything; where step 1 has already written in place
// (a fork), step 3 puts the staged tables back.
#pragma once

#include <cooperative_groups.h>

#include "pkv_common.cuh"

namespace pkv {

constexpr int kPgThreads = 1024;           // of a CTA of the cluster
constexpr int kPgCluster = 8;
constexpr int kPgCarryThreads = 256;
constexpr int kPgCopyThreads = 128;

// Tables, lens and refs of one side.
struct PageArrays {
  int32_t* tables;
  int32_t* lens;
  int32_t* refs;
};

struct PagesParams {
  PageArrays from, to;                     // from: the staged copy where the call works in place and sequences change
  PageArrays home;                         // from's own arrays (step 3 puts them back if there was no room)
  PageArrays staged;                       // room for a copy of them in the workspace
  void* k_pool;
  void* v_pool;
  int32_t* pos_pool;                       // or null
  const int32_t* parents;                  // [to_batch], or null: everyone its own
  const int32_t* add;                      // [layers][..], or null
  int64_t add_stride;
  int32_t* granted;                        // [layers][to_batch], or null
  int32_t* used;                           // compaction, or null
  int32_t layers, from_batch, to_batch, num_kv_heads, max_pages, page_size, num_pages;
  int32_t in_place;
  int32_t row_pieces;                      // 16-byte pieces of a row
  uint32_t* status;
  int32_t* state;                          // [0] 1 if the call was met, [1] number of page moves
  int32_t* list;                           // [num_pages] dealt pages; compaction: free pages to move into
  int32_t* second;                         // [num_pages] compaction: pages that move
  int32_t* place;                          // [num_pages] compaction: new place of every page from the border on
};

__device__ __forceinline__ int32_t pg_clamped(int32_t rows, const PagesParams& p) {
  const int64_t most = static_cast<int64_t>(p.max_pages) * p.page_size;
  return static_cast<int32_t>(min(static_cast<int64_t>(max(rows, 0)), most));
}
__device__ __forceinline__ int pg_pages(const PagesParams& p, int rows) { return rows / p.page_size + (rows % p.page_size ? 1 : 0); }

// What sequence c of `to` becomes in a layer.
struct PgChild {
  int parent;                              // -1: empty
  bool first;                              // its parent's first child
  int32_t rows, full, part;                // of the parent: rows, full pages, rows of the last page if it is not full
  int32_t keeps;                           // pages whose entries it takes over
  uint32_t rows_new;                       // (below 2^30 + 2^31)
  int pages;
};
__device__ __forceinline__ int pg_parent(const PagesParams& p, int c) {
  if (!p.parents) return c;
  const int par = p.parents[c];
  return par < 0 || par >= p.from_batch ? -1 : par;
}
__device__ __forceinline__ PgChild pg_child(const PagesParams& p, int l, int c, int parent, bool first) {
  PgChild x;
  x.parent = parent;
  x.first = first;
  x.rows = parent >= 0 ? pg_clamped(p.from.lens[static_cast<int64_t>(l) * p.from_batch + parent], p) : 0;
  x.full = x.rows / p.page_size;
  x.part = x.rows - x.full * p.page_size;
  x.keeps = x.full + (x.part > 0 && first ? 1 : 0);
  const int add = p.add ? max(p.add[l * p.add_stride + c], 0) : 0;
  x.rows_new = static_cast<uint32_t>(x.rows) + static_cast<uint32_t>(add);
  const uint32_t pages = x.rows_new / static_cast<uint32_t>(p.page_size);
  x.pages = static_cast<int>(min(pages + (pages * p.page_size < x.rows_new ? 1u : 0u), static_cast<uint32_t>(INT32_MAX)));
  return x;
}

// ------------------------------------------------------------------ staging of a call that works in place
// grid-stride copy of from's own arrays to the staged ones.
__global__ void __launch_bounds__(kPgCarryThreads) pages_stage_kernel(const __grid_constant__ PagesParams p) {
  pdl_trigger();
  pdl_wait();
  const int64_t entries = static_cast<int64_t>(p.layers) * p.from_batch * p.num_kv_heads * p.max_pages;
  const int64_t lens = static_cast<int64_t>(p.layers) * p.from_batch;
  const int64_t at = static_cast<int64_t>(blockIdx.x) * kPgCarryThreads + threadIdx.x, step = static_cast<int64_t>(gridDim.x) * kPgCarryThreads;
  for (int64_t i = at; i < entries; i += step) p.from.tables[i] = p.home.tables[i];
  for (int64_t i = at; i < lens; i += step) p.from.lens[i] = p.home.lens[i];
  for (int64_t i = at; i < p.num_pages; i += step) p.from.refs[i] = p.home.refs[i];
}

// refs of `to` from those of `from`: ahead of the next kernel where that one adjusts counts.
__global__ void __launch_bounds__(kPgCarryThreads) pages_refs_kernel(const __grid_constant__ PagesParams p) {
  pdl_trigger();
  pdl_wait();
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * kPgCarryThreads + threadIdx.x; i < p.num_pages; i += static_cast<int64_t>(gridDim.x) * kPgCarryThreads)
    p.to.refs[i] = p.from.refs[i];
}

// ------------------------------------------------------------------ 1. what is carried over
// grid (sequences of `to` and, where there are parents, of `from`; layers).  Entries that children keep are written to `to`;
// a page gains a count for every child behind its first and loses one for a sequence without children.
__global__ void __launch_bounds__(kPgCarryThreads) pages_carry_kernel(const __grid_constant__ PagesParams p) {
  __shared__ int s_first;
  pdl_trigger();
  pdl_wait();
  const int l = blockIdx.y, c = blockIdx.x;
  if (!p.parents && !p.in_place) {         // no count changes: they are copied on the way
    const int64_t at = (static_cast<int64_t>(l) * gridDim.x + c) * kPgCarryThreads + threadIdx.x;
    for (int64_t i = at; i < p.num_pages; i += static_cast<int64_t>(gridDim.x) * gridDim.y * kPgCarryThreads) p.to.refs[i] = p.from.refs[i];
  }
  if (c < p.to_batch) {
    const int parent = pg_parent(p, c);
    bool first = true;
    if (p.parents) {
      if (threadIdx.x == 0) s_first = 1;
      __syncthreads();
      for (int i = threadIdx.x; i < c; i += kPgCarryThreads)
        if (p.parents[i] == parent) s_first = 0;
      __syncthreads();
      first = s_first != 0;
    }
    const PgChild x = pg_child(p, l, c, parent, first);
    if (parent < 0) return;
    const int64_t src = (static_cast<int64_t>(l) * p.from_batch + parent) * p.num_kv_heads * p.max_pages;
    const int64_t dst = (static_cast<int64_t>(l) * p.to_batch + c) * p.num_kv_heads * p.max_pages;
    for (int h = threadIdx.x >> 5; h < p.num_kv_heads; h += kPgCarryThreads / 32) {        // a warp per head
      const int32_t* from = p.from.tables + src + static_cast<int64_t>(h) * p.max_pages;
      int32_t* to = p.to.tables + dst + static_cast<int64_t>(h) * p.max_pages;
      for (int j = threadIdx.x & 31; j < x.keeps; j += 32) {
        const int entry = from[j];
        to[j] = entry;
        if (!x.first && entry >= 0 && entry < p.num_pages) atomicAdd(p.to.refs + entry, 1);
      }
    }
    return;
  }
  // a sequence of `from` that nobody goes on with: its pages are let go
  const int b = c - p.to_batch;
  if (threadIdx.x == 0) s_first = 1;
  __syncthreads();
  for (int i = threadIdx.x; i < p.to_batch; i += kPgCarryThreads)
    if (p.parents[i] == b) s_first = 0;
  __syncthreads();
  if (!s_first) return;
  const int rows = pg_clamped(p.from.lens[static_cast<int64_t>(l) * p.from_batch + b], p);
  const int pages = pg_pages(p, rows);
  const int64_t src = (static_cast<int64_t>(l) * p.from_batch + b) * p.num_kv_heads * p.max_pages;
  for (int h = threadIdx.x >> 5; h < p.num_kv_heads; h += kPgCarryThreads / 32)
    for (int j = threadIdx.x & 31; j < pages; j += 32) {
      const int entry = p.from.tables[src + static_cast<int64_t>(h) * p.max_pages + j];
      if (entry >= 0 && entry < p.num_pages) atomicSub(p.to.refs + entry, 1);
    }
}

// ------------------------------------------------------------------ 2. sums and ranks over a cluster
struct PgShared {
  long long warp[32];
  int32_t need[kPgCluster], free[kPgCluster], flag[kPgCluster];  // of every CTA, written by it ahead of the cluster's barrier
  int32_t bad;
};

// Exclusive running sum over the CTA's threads; *total: the CTA's sum.  Everybody takes part.
template <typename I>
__device__ __forceinline__ I pg_scan(PgShared& s, I x, I* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  I run = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const I y = __shfl_up_sync(0xffffffffu, run, o);
    if (lane >= o) run += y;
  }
  __syncthreads();                         // the last call's sums have been read
  if (lane == 31) s.warp[warp] = run;
  __syncthreads();
  I w = static_cast<I>(s.warp[lane]);
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const I y = __shfl_up_sync(0xffffffffu, w, o);
    if (lane >= o) w += y;
  }
  *total = __shfl_sync(0xffffffffu, w, 31);
  const I ahead = __shfl_sync(0xffffffffu, w, warp ? warp - 1 : 0);
  return run - x + (warp ? ahead : I(0));
}

// Every CTA gets this one's number; there behind a barrier of the cluster.  (Read from the others behind it: 1.6 us for three.)
__device__ __forceinline__ void pg_tell(int32_t (&of)[kPgCluster], int32_t x) {
  namespace cg = cooperative_groups;
  cg::cluster_group cluster = cg::this_cluster();
  if (threadIdx.x < kPgCluster) *cluster.map_shared_rank(&of[cluster.block_rank()], threadIdx.x) = x;
}

// What the CTAs ahead have of a number, and all of them.
__device__ __forceinline__ void pg_cluster(const int32_t (&of)[kPgCluster], int rank, int* ahead, int* total) {
  *ahead = *total = 0;
#pragma unroll
  for (int c = 0; c < kPgCluster; ++c) {
    const int x = of[c];
    if (c < rank) *ahead += x;
    *total += x;
  }
}

// Four consecutive refs from `i` on (a multiple of four) as bits of free pages; pages behind `end` are not free.
__device__ __forceinline__ uint32_t pg_free4(const int32_t* refs, bool aligned, int64_t i, int64_t end) {
  uint32_t bits = 0;
  if (aligned && i + 4 <= end) {
    const int4 v = __ldcg(reinterpret_cast<const int4*>(refs + i));
    bits = (v.x <= 0 ? 1u : 0u) | (v.y <= 0 ? 2u : 0u) | (v.z <= 0 ? 4u : 0u) | (v.w <= 0 ? 8u : 0u);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (i + e < end && __ldcg(refs + i + e) <= 0) bits |= 1u << e;
  }
  return bits;
}

// A warp's share of the pool: tiles of 128 pages, four to a lane.
constexpr int kPgTile = 128;
constexpr int kPgWarps = kPgCluster * kPgThreads / 32;
__device__ __forceinline__ void pg_share(int64_t pages, int rank, int64_t* lo, int64_t* hi) {
  const int64_t per = ((pages + kPgWarps - 1) / kPgWarps + kPgTile - 1) / kPgTile * kPgTile;
  const int64_t worker = rank * (kPgThreads / 32) + (threadIdx.x >> 5);
  *lo = min(pages, per * worker);
  *hi = min(pages, per * (worker + 1));
}

// Free pages of a warp's share.  The bits of its first eight tiles stay with the lane, so that a second look needs no loads there.
struct PgFree {
  uint32_t bits = 0;
  __device__ __forceinline__ int count(const int32_t* refs, bool aligned, int64_t lo, int64_t hi) {
    int free = 0;
    const int64_t mine = lo + (threadIdx.x & 31) * 4;
#pragma unroll
    for (int t = 0; t < 8; ++t) bits |= pg_free4(refs, aligned, mine + t * kPgTile, hi) << (4 * t);
    free = __popc(bits);
#pragma unroll 4
    for (int64_t i = mine + 8 * kPgTile; i < hi; i += kPgTile) free += __popc(pg_free4(refs, aligned, i, hi));
    return __reduce_add_sync(0xffffffffu, free);
  }
  __device__ __forceinline__ uint32_t tile(const int32_t* refs, bool aligned, int64_t i, int64_t hi, int t) const {
    return t < 8 ? (bits >> (4 * t)) & 15u : pg_free4(refs, aligned, i, hi);
  }
};

// What the lanes ahead have; *total: all of them.
__device__ __forceinline__ int pg_lanes_ahead(int mine, int* total) {
  const int lane = threadIdx.x & 31;
  int run = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, run, o);
    if (lane >= o) run += y;
  }
  *total = __shfl_sync(0xffffffffu, run, 31);
  return run - mine;
}

// One cluster.  Requests are counted, free pages found and dealt out; lens, granted and the new table entries of `to` are written.
__global__ void __launch_bounds__(kPgThreads) pages_deal_kernel(const __grid_constant__ PagesParams p) {
  namespace cg = cooperative_groups;
  cg::cluster_group cluster = cg::this_cluster();
  __shared__ PgShared s;
  __shared__ int32_t s_parent[PKV_MAX_CACHE_BATCH];              // bit 30: not the parent's first child
  __shared__ int32_t s_child[PKV_MAX_CACHE_BATCH];               // a parent's first child
  pdl_trigger();
  const int rank = static_cast<int>(cluster.block_rank()), tid = threadIdx.x;
  asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");  // this CTA's shared memory may be written
  pdl_wait();
  if (tid == 0) s.bad = 0;
  const bool aligned = reinterpret_cast<uintptr_t>(p.to.refs) % 16 == 0;
  int64_t lo, hi;
  pg_share(p.num_pages, rank, &lo, &hi);
  PgFree free;
  const int my_free = free.count(p.to.refs, aligned, lo, hi);
  int bad = 0;                             // bit 0: a parent outside the batch, bit 1: a sequence too long for its table
  if (p.parents) {
    for (int b = tid; b < p.from_batch; b += kPgThreads) s_child[b] = INT32_MAX;
    __syncthreads();
    for (int c = tid; c < p.to_batch; c += kPgThreads) {
      const int parent = pg_parent(p, c);
      if (parent < 0 && p.parents[c] != -1) bad |= 1;
      if (parent >= 0) atomicMin(&s_child[parent], c);
      s_parent[c] = parent;
    }
    __syncthreads();
    for (int c = tid; c < p.to_batch; c += kPgThreads)
      if (s_parent[c] >= 0 && s_child[s_parent[c]] != c) s_parent[c] |= 1 << 30;
  }
  __syncthreads();
  const int units = p.layers * p.to_batch;
  auto child = [&](int unit) {
    const int l = unit / p.to_batch, c = unit - l * p.to_batch;
    const int x = p.parents ? s_parent[c] : c;
    return pg_child(p, l, c, x < 0 ? -1 : x & ~(1 << 30), x >= 0 && !(x >> 30));
  };
  // requests of every unit; each thread has consecutive ones
  constexpr int kWorkers = kPgCluster * kPgThreads;
  const int per = (units + kWorkers - 1) / kWorkers, u0 = min(units, per * (rank * kPgThreads + tid)), u1 = min(units, u0 + per);
  int64_t mine = 0;
  for (int u = u0; u < u1; ++u) {
    const PgChild x = child(u);
    if (x.pages > p.max_pages) bad |= 2;
    else mine += static_cast<int64_t>(x.pages - x.keeps) * p.num_kv_heads;
  }
  // more requests than pages cannot be met; sums stay within bounds that way
  if (mine > p.num_pages) { bad |= 2; mine = 0; }
  if (bad) atomicOr(&s.bad, bad);
  // one scan for both: requests (at most 2^27 of 1024 threads) in 38 bits, free pages (at most 2^24 of a CTA) above
  constexpr int kBits = 38;
  const long long ours = mine + (static_cast<long long>((tid & 31) == 0 ? my_free : 0) << kBits);
  long long cta;
  const long long run = pg_scan<long long>(s, ours, &cta);
  const long long run_need = run & ((1ll << kBits) - 1), cta_need = cta & ((1ll << kBits) - 1);
  const int run_free = __shfl_sync(0xffffffffu, static_cast<int>(run >> kBits), 0);
  asm volatile("barrier.cluster.wait.acquire;" ::: "memory");    // and everybody else's
  pg_tell(s.need, cta_need > p.num_pages ? 0 : static_cast<int>(cta_need));
  pg_tell(s.free, static_cast<int>(cta >> kBits));
  pg_tell(s.flag, s.bad | (cta_need > p.num_pages ? 2 : 0));
  cluster.sync();
  int ahead, need, place, free_all, flags = 0;
  pg_cluster(s.need, rank, &ahead, &need);
  pg_cluster(s.free, rank, &place, &free_all);
  place += run_free;                       // the rank of this warp's first free page
#pragma unroll
  for (int c = 0; c < kPgCluster; ++c) flags |= s.flag[c];
  const bool met = flags == 0 && need <= free_all;               // (sums of eight shares of at most 2^27)
  if (rank == 0 && tid == 0) {
    p.state[0] = met ? 1 : 0;
    if (!met) atomicOr(p.status, (flags & 1 ? kStatusBadIndex : 0u) | ((flags & 2) || flags == 0 ? kStatusNoRoom : 0u));
  }
  if (!met) {                              // the same in the whole cluster
    if (p.granted)
      for (int u = u0; u < u1; ++u) p.granted[u] = 0;
    return;
  }
  int t = 0;
  for (int64_t base = lo; base < hi && my_free && place < need; base += kPgTile, ++t) {    // (uniform over the warp)
    const int64_t i = base + (tid & 31) * 4;
    const uint32_t bits = free.tile(p.to.refs, aligned, i, hi, t);
    int total;
    int r = place + pg_lanes_ahead(__popc(bits), &total);
    place += total;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if ((bits >> e) & 1u) {
        if (r < need) {
          p.list[r] = static_cast<int32_t>(i + e);
          p.to.refs[i + e] = 1;
        }
        ++r;
      }
  }
  cluster.sync();                          // the list is there (and so are everybody's reads of parents' lens)
  // Table entries of this thread's units, their pages one after another in the list, head by head.  Many of them: by the whole warp.
  // (A warp per head of a unit, one after another: 79 us for 64 sequences x 32 layers x 8 heads, 19 with a lane per head, 15 this way, all with a cold L2.)
  constexpr int kAlone = 32;
  int64_t off = ahead + run_need;
  for (int i = 0; i < per; ++i) {          // (uniform over the warp)
    const int u = u0 + i;
    const int32_t* pages = p.list + off;
    int32_t* table = p.to.tables;
    int fresh = 0, all = 0;
    if (u < u1) {
      const PgChild x = child(u);
      fresh = x.pages - x.keeps;
      all = fresh * p.num_kv_heads;        // (at most num_pages)
      off += all;
      table += static_cast<int64_t>(u) * p.num_kv_heads * p.max_pages + x.keeps;
      p.to.lens[u] = static_cast<int32_t>(x.rows_new);
      if (p.granted) p.granted[u] = static_cast<int32_t>(x.rows_new) - x.rows;
    }
    if (all <= kAlone) {
      constexpr int kAhead = 8;            // entries on their way at a time
      for (int e = 0, h = 0, j = 0; e < all; e += kAhead) {
        int32_t page[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) page[i] = __ldcg(pages + min(e + i, all - 1));
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
          if (e + i < all) {
            table[static_cast<int64_t>(h) * p.max_pages + j] = page[i];
            if (++j == fresh) {
              j = 0;
              ++h;
            }
          }
      }
    }
    for (unsigned many = __ballot_sync(0xffffffffu, all > kAlone); many; many &= many - 1) {
      const int l = __ffs(many) - 1, n = __shfl_sync(0xffffffffu, fresh, l), sum = __shfl_sync(0xffffffffu, all, l);
      const int32_t* from = reinterpret_cast<const int32_t*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(pages), l));
      int32_t* to = reinterpret_cast<int32_t*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(table), l));
      for (int e = tid & 31; e < sum; e += 32) {
        const int h = e / n;
        to[static_cast<int64_t>(h) * p.max_pages + (e - h * n)] = __ldcg(from + e);
      }
    }
  }
}

// ------------------------------------------------------------------ 3. rows of a part-filled page to its copies
// grid (sequences of `to`, layers).  If the call was not met: puts `to` back (in place), a share per CTA.
__global__ void __launch_bounds__(kPgCarryThreads) pages_copy_kernel(const __grid_constant__ PagesParams p) {
  __shared__ int s_first;
  pdl_trigger();
  pdl_wait();
  const int c = blockIdx.x, l = blockIdx.y;
  if (!p.state[0]) {
    if (!p.in_place) return;
    const int64_t at = (static_cast<int64_t>(l) * gridDim.x + c) * kPgCarryThreads + threadIdx.x;
    const int64_t step = static_cast<int64_t>(gridDim.x) * gridDim.y * kPgCarryThreads;
    const int64_t entries = static_cast<int64_t>(p.layers) * p.from_batch * p.num_kv_heads * p.max_pages;
    for (int64_t i = at; i < entries; i += step) p.home.tables[i] = p.from.tables[i];
    for (int64_t i = at; i < p.num_pages; i += step) p.home.refs[i] = p.from.refs[i];
    return;                                // lens were not written
  }
  const int parent = pg_parent(p, c);
  if (parent < 0) return;
  if (threadIdx.x == 0) s_first = 1;
  __syncthreads();
  for (int i = threadIdx.x; i < c; i += kPgCarryThreads)
    if (p.parents[i] == parent) s_first = 0;
  __syncthreads();
  const PgChild x = pg_child(p, l, c, parent, s_first != 0);
  if (x.first || !x.part) return;
  const int32_t* src_table = p.from.tables + (static_cast<int64_t>(l) * p.from_batch + parent) * p.num_kv_heads * p.max_pages + x.full;
  const int32_t* dst_table = p.to.tables + (static_cast<int64_t>(l) * p.to_batch + c) * p.num_kv_heads * p.max_pages + x.full;
  const int64_t page = static_cast<int64_t>(p.page_size) * p.row_pieces;
  const int64_t pieces = static_cast<int64_t>(x.part) * p.row_pieces;
  const int lane = threadIdx.x & 31;
  for (int h = threadIdx.x >> 5; h < p.num_kv_heads; h += kPgCarryThreads / 32) {          // a warp per head
    const int src = src_table[static_cast<int64_t>(h) * p.max_pages], dst = dst_table[static_cast<int64_t>(h) * p.max_pages];
    if (src < 0 || src >= p.num_pages) {
      if (lane == 0) atomicOr(p.status, kStatusBadPage);
      continue;
    }
    const uint4* ks = static_cast<const uint4*>(p.k_pool) + src * page;
    const uint4* vs = static_cast<const uint4*>(p.v_pool) + src * page;
    uint4* kd = static_cast<uint4*>(p.k_pool) + dst * page;
    uint4* vd = static_cast<uint4*>(p.v_pool) + dst * page;
    constexpr int kAhead = 4;
    for (int64_t i = lane; i < pieces; i += 32 * kAhead) {
      uint4 a[kAhead], b[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const int64_t at = min(i + j * 32, pieces - 1);          // (the last piece again behind it)
        a[j] = ks[at];
        b[j] = vs[at];
      }
#pragma unroll
      for (int j = 0; j < kAhead; ++j)
        if (i + j * 32 < pieces) {
          kd[i + j * 32] = a[j];
          vd[i + j * 32] = b[j];
        }
    }
    if (p.pos_pool)
      for (int i = lane; i < x.part; i += 32)
        p.pos_pool[static_cast<int64_t>(dst) * p.page_size + i] = p.pos_pool[static_cast<int64_t>(src) * p.page_size + i];
  }
}

// ------------------------------------------------------------------ compaction
// One cluster.  With u pages in use, the free pages below u (list) and the used ones from u on (second) are as many; the i-th
// of the latter moves to the i-th of the former.
__global__ void __launch_bounds__(kPgThreads) pages_pair_kernel(const __grid_constant__ PagesParams p) {
  namespace cg = cooperative_groups;
  cg::cluster_group cluster = cg::this_cluster();
  __shared__ PgShared s;
  pdl_trigger();
  const int rank = static_cast<int>(cluster.block_rank()), tid = threadIdx.x;
  asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");  // this CTA's shared memory may be written
  pdl_wait();
  const int32_t* refs = p.from.refs;
  const bool aligned = reinterpret_cast<uintptr_t>(refs) % 16 == 0;
  int64_t lo, hi;                          // this warp's pages
  pg_share(p.num_pages, rank, &lo, &hi);
  PgFree free;
  const int mine = free.count(refs, aligned, lo, hi);
  int cta, ahead, all;
  const int run = __shfl_sync(0xffffffffu, pg_scan<int>(s, (tid & 31) == 0 ? mine : 0, &cta), 0);
  asm volatile("barrier.cluster.wait.acquire;" ::: "memory");    // and everybody else's
  pg_tell(s.free, cta);
  cluster.sync();
  pg_cluster(s.free, rank, &ahead, &all);
  ahead += run;                            // free pages ahead of this warp's
  const int used = p.num_pages - all;
  // The warp whose share the border lies in (the last one with pages, if that is the pool's end) counts the free pages below it.
  if (lo <= used && (used < hi || (hi == p.num_pages && lo < hi))) {
    int below = 0;
    int t = 0;
    for (int64_t base = lo; base < used; base += kPgTile, ++t) {
      const int64_t i = base + (tid & 31) * 4;
      const uint32_t in = i >= used ? 0u : (i + 4 <= used ? 15u : (1u << (used - i)) - 1u);
      below += __popc(free.tile(refs, aligned, i, hi, t) & in);
    }
    below = __reduce_add_sync(0xffffffffu, below);
    if ((tid & 31) == 0) {
      p.state[0] = used;
      p.state[1] = ahead + below;
      if (p.used) *p.used = used;
    }
  }
  cluster.sync();
  const int moves = __ldcg(p.state + 1);
  int hole = ahead;                        // rank of this warp's first free page below the border,
  int mover = static_cast<int>(max(static_cast<int64_t>(0), lo - used)) - max(0, ahead - moves);   // and of its first used one above
  int t = 0;
  for (int64_t base = lo; base < hi; base += kPgTile, ++t) {
    const int64_t i = base + (tid & 31) * 4;
    const uint32_t free4 = free.tile(refs, aligned, i, hi, t);
    const uint32_t there = i >= hi ? 0u : (i + 4 <= hi ? 15u : (1u << (hi - i)) - 1u);
    const uint32_t below = i >= used ? 0u : (i + 4 <= used ? 15u : (1u << (used - i)) - 1u);
    const uint32_t hole4 = free4 & below, mover4 = there & ~below & ~free4;
    int total;
    int h = pg_lanes_ahead(__popc(hole4) | __popc(mover4) << 16, &total);
    int m = mover + (h >> 16);
    h = hole + (h & 0xffff);
    hole += total & 0xffff;
    mover += total >> 16;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int32_t page = static_cast<int32_t>(i + e);
      if ((hole4 >> e) & 1u) p.list[h++] = page;
      if ((mover4 >> e) & 1u) p.second[m++] = page;
      if (((free4 & ~below) >> e) & 1u) p.place[page] = page;     // nothing should name it
    }
  }
  cluster.sync();                          // both lists are there
  constexpr int kAhead = 4;
  for (int m0 = rank * kPgThreads + tid; m0 < moves; m0 += kAhead * kPgCluster * kPgThreads) {
    int from[kAhead], to[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int m = min(m0 + j * kPgCluster * kPgThreads, moves - 1);
      from[j] = __ldcg(p.second + m);
      to[j] = __ldcg(p.list + m);
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) p.place[from[j]] = to[j];  // (the last one again behind it)
  }
}

// Three independent jobs, each dealt out over the grid: pages to their new places, tables with the new places, refs of `to`.
__global__ void __launch_bounds__(kPgCopyThreads) pages_move_kernel(const __grid_constant__ PagesParams p) {
  pdl_trigger();
  pdl_wait();
  const int used = p.state[0], moves = p.state[1];
  const int64_t page = static_cast<int64_t>(p.page_size) * p.row_pieces;
  for (int m = blockIdx.x; m < moves; m += gridDim.x) {
    const int dst = p.list[m], src = p.second[m];
    const uint4* ks = static_cast<const uint4*>(p.k_pool) + src * page;
    const uint4* vs = static_cast<const uint4*>(p.v_pool) + src * page;
    uint4* kd = static_cast<uint4*>(p.k_pool) + dst * page;
    uint4* vd = static_cast<uint4*>(p.v_pool) + dst * page;
    for (int64_t i = threadIdx.x; i < page; i += 2 * kPgCopyThreads) {
      const bool two = i + kPgCopyThreads < page;
      const uint4 a = ks[i], b = vs[i];
      uint4 c = make_uint4(0, 0, 0, 0), d = c;
      if (two) {
        c = ks[i + kPgCopyThreads];
        d = vs[i + kPgCopyThreads];
      }
      kd[i] = a;
      vd[i] = b;
      if (two) {
        kd[i + kPgCopyThreads] = c;
        vd[i + kPgCopyThreads] = d;
      }
    }
    if (p.pos_pool)
      for (int i = threadIdx.x; i < p.page_size; i += kPgCopyThreads)
        p.pos_pool[static_cast<int64_t>(dst) * p.page_size + i] = p.pos_pool[static_cast<int64_t>(src) * p.page_size + i];
  }
  const int64_t units = static_cast<int64_t>(p.layers) * p.from_batch;
  for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
    const int rows = p.from.lens[unit];
    const int pages = pg_pages(p, pg_clamped(rows, p));
    for (int h = threadIdx.x >> 5; h < p.num_kv_heads; h += kPgCopyThreads / 32)
      for (int j = threadIdx.x & 31; j < pages; j += 32) {
        const int64_t e = (unit * p.num_kv_heads + h) * p.max_pages + j;
        const int entry = p.from.tables[e];
        const int place = entry >= used && entry < p.num_pages ? p.place[entry] : entry;
        if (!p.in_place || place != entry) p.to.tables[e] = place;
      }
    if (!p.in_place && threadIdx.x == 0) p.to.lens[unit] = rows;
  }
  // A free page below the border has its new tenant's count, a page from the border on none.
  const int64_t at = static_cast<int64_t>(blockIdx.x) * kPgCopyThreads + threadIdx.x, step = static_cast<int64_t>(gridDim.x) * kPgCopyThreads;
  if (!p.in_place)
    for (int64_t i = at; i < p.num_pages; i += step) {
      const int count = i < used ? p.from.refs[i] : 0;
      if (i >= used || count > 0) p.to.refs[i] = count;
    }
  for (int64_t m = at; m < moves; m += step) {
    p.to.refs[p.list[m]] = p.from.refs[p.second[m]];
    if (p.in_place) p.to.refs[p.second[m]] = 0;
  }
}

}  // namespace pkv
