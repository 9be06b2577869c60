// Who holds the pages of a pool (quoka_pages_resize, quoka_pages_fork): a count of holders for each page (0: free), and for each sequence a row
// of the page table and the number of its entries in use.
//
// Pages are handed out lowest first, in the order of the sequences and of their entries, so that a call's result depends on nothing but its
// arguments: counts are changed by integer atomics, whose order does not matter, and the rank of a free page among the free ones names the
// entry that gets it.  Three steps, each of which uses what the one before has completed: entries that go or are shared, free pages counted
// beside the sum of what the sequences lack, free pages to entries.  Small pools and batches take them in one launch of one block, small pools of
// larger batches in two (a block a sequence, then one block), others in three (a block a sequence, a tile of pages a block twice).
// Bound by the chain: lengths, table, counts' atomics, counts, table.  Measured: a step of 16 sequences over 8192 pages 3 - 4 us, of 256 over 262144
// 2.7 + 2.5 + 4.3; forks that change only last pages, of 16 sequences 6.2, of 256 with tables of 130816 entries 3.3 + 5.1 (a call 9.9, and 10.5 where nearly
// every entry changes; of the 16 the same).  With many tiles, each block of the last launch adds up the counts of those before its own, which grows with the
// square of the pool: steps that want nothing, over 2^18 and 2^22 pages 11.6 us, 2^26 101, 2^28 1012, 2^30 13500.  (Counts fetched ahead of the scans,
// whether pages are wanted or not: 0.6 us more for a step that wants none, which most are, otherwise the same.)
#include <type_traits>

#include "common.hip.h"
#include "kernels.h"

namespace quoka {

constexpr int kOwThreads = 256, kOwRun = 16, kOwTile = kOwThreads * kOwRun;   // pages of a thread, of a tile
constexpr int kOwBatch = 4096;   // sequences whose sums a block keeps in LDS

// What a call leaves for its later launches.
struct OwWs {
  int32_t* start;    // [b] entries in use after the first launch
  int32_t* need;     // [b] entries that want a page
  int32_t* prefix;   // [b + 1] of need
  int32_t* counts;   // [tiles] free pages
};
static int ow_tiles(int n_pages) { return (n_pages + kOwTile - 1) / kOwTile; }
size_t owners_ws_bytes(const Owners& o) { return ((size_t)3 * o.b + 1 + ow_tiles(o.n_pages)) * sizeof(int32_t); }
static OwWs ow_ws(const Owners& o, void* ws) {
  int32_t* p = static_cast<int32_t*>(ws);
  return {p, p + o.b, p + 2 * (size_t)o.b, p + 3 * (size_t)o.b + 1};
}

__device__ __forceinline__ void add_holder(const Owners& o, int32_t page, int by) {
  if ((uint32_t)page < (uint32_t)o.n_pages) atomicAdd(o.ref + page, by);   // (others: no page of the pool)
}
__device__ __forceinline__ int held_by(const Owners& o, int b) { return min(max(o.held[b], 0), o.max_pages); }

// What sequence b holds after a cut, and lacks; `lane` of `width` threads that share its entries.
__device__ __forceinline__ void cut_sequence(const Owners& o, const int32_t* __restrict__ lens, int b, int lane, int width, int& start, int& need) {
  const int len = lens[b], had = held_by(o, b);
  const int n = len <= 0 ? 0 : min(((len - 1) >> o.shift) + 1, o.max_pages);
  int32_t* row = o.table + (long long)b * o.max_pages;
  start = min(had, n);
  need = n - start;
  for (int e = n + lane; e < had; e += width) {
    add_holder(o, row[e], -1);
    row[e] = -1;
  }
}

// Likewise for a child that goes on from its parent.
__device__ __forceinline__ void share_sequence(const Owners& from, const Owners& o, const ForkArgs& f, int b, int lane, int width, int& start,
                                               int& need) {
  const int had = held_by(o, b), parent = f.parents[b];
  const bool has_parent = (uint32_t)parent < (uint32_t)from.b;
  // (at most what the parent holds and the child has room for: 64 bits)
  long long len = 0;
  if (has_parent) len = min((long long)max(f.lens[parent], 0), (long long)min(held_by(from, parent), o.max_pages) << o.shift);
  const int whole = (int)(len >> o.shift);
  start = whole;
  need = (len & ((1 << o.shift) - 1)) != 0 ? 1 : 0;
  int32_t* row = o.table + (long long)b * o.max_pages;
  const int32_t* theirs = from.table + (long long)(has_parent ? parent : 0) * from.max_pages;
  for (int e = lane; e < max(whole, had); e += width) {
    const int32_t old = e < had ? row[e] : -1, page = e < whole ? theirs[e] : -1;
    if (e < had && old == page) continue;   // (shared as it was: beams that swap between two tables keep most of their pages)
    add_holder(o, old, -1);
    add_holder(o, page, 1);
    row[e] = page;
  }
  if (lane == 0) {
    f.first[b] = whole << o.shift;
    f.child_lens[b] = (int)len;
  }
}

__global__ __launch_bounds__(kOwThreads) void owners_cut(Owners o, const int32_t* __restrict__ lens, OwWs ws) {
  const int b = blockIdx.x;
  int start, need;
  cut_sequence(o, lens, b, threadIdx.x, kOwThreads, start, need);
  if (threadIdx.x == 0) {
    ws.start[b] = start;
    ws.need[b] = need;
  }
}

__global__ __launch_bounds__(kOwThreads) void owners_share(Owners from, Owners o, ForkArgs f, OwWs ws) {
  const int b = blockIdx.x;
  int start, need;
  share_sequence(from, o, f, b, threadIdx.x, kOwThreads, start, need);
  if (threadIdx.x == 0) {
    ws.start[b] = start;
    ws.need[b] = need;
  }
}

// Which of the pages page0 .. page0 + kOwRun - 1 are free.
__device__ __forceinline__ uint32_t free_pages(const Owners& o, int page0) {
  typedef int32_t four __attribute__((ext_vector_type(4), aligned(4)));
  uint32_t is = 0;
  if (page0 + kOwRun <= o.n_pages) {
    four r[kOwRun / 4];
#pragma unroll
    for (int i = 0; i < kOwRun / 4; ++i) r[i] = *reinterpret_cast<const four*>(o.ref + page0 + 4 * i);
#pragma unroll
    for (int i = 0; i < kOwRun; ++i) is |= r[i / 4][i % 4] <= 0 ? 1u << i : 0u;
  } else {
#pragma unroll
    for (int i = 0; i < kOwRun; ++i) is |= page0 + i < o.n_pages && o.ref[min(page0 + i, o.n_pages - 1)] <= 0 ? 1u << i : 0u;
  }
  return is;
}

// Free pages `is` of page0 .. page0 + kOwRun - 1, the first of which is number `rank` of all free ones, to the entries that want them.
// prefix [b + 1], start [b]: what the sequences before each one lack, and its entries in use.
template <typename P, typename S>
__device__ __forceinline__ void give_pages(const Owners& o, int page0, uint32_t is, uint32_t rank, uint32_t wanted, const P* prefix, const S* start) {
  if (is == 0 || rank >= wanted) return;
  int lo = 0, hi = o.b - 1;   // the last sequence whose first rank is not above `rank` (one that wants none has the next one's)
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if ((uint32_t)prefix[mid] <= rank) lo = mid;
    else hi = mid - 1;
  }
  for (; is != 0 && rank < wanted; is &= is - 1, ++rank) {
    while ((uint32_t)prefix[lo + 1] <= rank) ++lo;   // (rank < wanted, the last of them)
    const int page = page0 + __builtin_ctz(is);
    o.ref[page] = 1;
    o.table[(long long)lo * o.max_pages + (int)start[lo] + (int)(rank - (uint32_t)prefix[lo])] = page;
  }
}

// The last block: the sums of what the sequences before each one lack.
__global__ __launch_bounds__(kOwThreads) void owners_count(Owners o, OwWs ws) {
  __shared__ uint32_t scan[kOwThreads / kWave + 1];
  const int tid = threadIdx.x;
  uint32_t total;
  if (blockIdx.x == gridDim.x - 1) {
    uint32_t before = 0;
    for (int b0 = 0; b0 < o.b; b0 += kOwThreads) {
      const uint32_t mine = b0 + tid < o.b ? (uint32_t)ws.need[b0 + tid] : 0u;
      const uint32_t excl = block_excl_scan<kOwThreads>(mine, scan, &total);
      if (b0 + tid < o.b) ws.prefix[b0 + tid] = (int32_t)(before + excl);
      before += total;
    }
    if (tid == 0) ws.prefix[o.b] = (int32_t)before;
    return;
  }
  block_excl_scan<kOwThreads>((uint32_t)__popc(free_pages(o, (int)blockIdx.x * kOwTile + tid * kOwRun)), scan, &total);
  if (tid == 0) ws.counts[blockIdx.x] = (int32_t)total;
}

// Block t: the free pages of tile t.  The last block: what every sequence holds now.  (fork: a child whose last page is lacking has its whole
// pages.)
__global__ __launch_bounds__(kOwThreads) void owners_take(Owners o, ForkArgs f, OwWs ws, int32_t* __restrict__ lacking) {
  __shared__ uint32_t scan[kOwThreads / kWave + 1];
  const int tid = threadIdx.x, tiles = (int)gridDim.x - 1;
  const uint32_t wanted = (uint32_t)ws.prefix[o.b];
  uint32_t mine = 0, before;
  for (int t = tid; t < (int)blockIdx.x; t += kOwThreads) mine += (uint32_t)ws.counts[t];   // (the last block: all)
  block_excl_scan<kOwThreads>(mine, scan, &before);
  if ((int)blockIdx.x == tiles) {
    for (int b = tid; b < o.b; b += kOwThreads) {
      const int need = ws.need[b], got = min(max((int)(before - (uint32_t)ws.prefix[b]), 0), need);
      o.held[b] = ws.start[b] + got;
      if (f.child_lens != nullptr && got < need) f.child_lens[b] = f.first[b];
    }
    if (tid == 0) *lacking = (int32_t)(wanted > before ? wanted - before : 0u);
    return;
  }
  if (before >= wanted) return;   // block-uniform
  uint32_t total;
  const int page0 = (int)blockIdx.x * kOwTile + tid * kOwRun;
  const uint32_t is = free_pages(o, page0);
  const uint32_t rank = before + block_excl_scan<kOwThreads>((uint32_t)__popc(is), scan, &total);
  if (o.b <= kOwBatch) {   // (a search is some ten look-ups one after the other)
    __shared__ int32_t prefix[kOwBatch + 1], start[kOwBatch];
    for (int b = tid; b <= o.b; b += kOwThreads) {
      prefix[b] = ws.prefix[b];
      if (b < o.b) start[b] = ws.start[b];
    }
    __syncthreads();
    give_pages(o, page0, is, rank, wanted, prefix, start);
  } else {
    give_pages(o, page0, is, rank, wanted, ws.prefix, ws.start);
  }
}

// Free pages counted and handed out by one block, RUNS times 16 of every thread at once.  A thread has the sequence of its number: `need` entries
// that want a page behind the `start_of` ones in use.
constexpr int kOsThreads = 1024;
template <bool FORK, int RUNS>
__device__ __forceinline__ void hand_out(const Owners& o, const ForkArgs& f, int start_of, int need, int32_t* lacking) {
  __shared__ uint32_t scan[kOsThreads / kWave + 1];
  __shared__ int32_t prefix[kOsThreads + 1], start[kOsThreads];
  const int tid = threadIdx.x;
  uint32_t wanted, total;
  const uint32_t mine = block_excl_scan<kOsThreads>((uint32_t)need, scan, &wanted);
  prefix[tid] = (int32_t)mine;   // (past the batch: `wanted`)
  start[tid] = start_of;
  if (tid == kOsThreads - 1) prefix[kOsThreads] = (int32_t)wanted;
  __syncthreads();
  uint32_t before = 0;
  for (int of_block = 0; before < wanted && of_block < o.n_pages; of_block += kOsThreads * kOwRun * RUNS) {   // block-uniform
    constexpr int kStep = kOsThreads * kOwRun;   // pages of a run of all threads (16 bits hold their number: two runs a scan)
    uint32_t is[RUNS];
#pragma unroll
    for (int i = 0; i < RUNS; ++i) is[i] = free_pages(o, of_block + i * kStep + tid * kOwRun);
#pragma unroll
    for (int i = 0; i < RUNS; i += 2) {
      const uint32_t second = i + 1 < RUNS ? (uint32_t)__popc(is[i + 1]) : 0u;
      const uint32_t excl = block_excl_scan<kOsThreads>((uint32_t)__popc(is[i]) | second << 16, scan, &total);
      give_pages(o, of_block + i * kStep + tid * kOwRun, is[i], before + (excl & 0xFFFFu), wanted, prefix, start);
      before += total & 0xFFFFu;
      if (i + 1 < RUNS) give_pages(o, of_block + (i + 1) * kStep + tid * kOwRun, is[i + 1], before + (excl >> 16), wanted, prefix, start);
      before += total >> 16;
    }
  }
  if (tid < o.b) {
    const int got = min(max((int)(before - mine), 0), need);
    o.held[tid] = start_of + got;
    if (FORK && got < need) f.child_lens[tid] = f.first[tid];
  }
  if (tid == 0) *lacking = (int32_t)(wanted > before ? wanted - before : 0u);
}

// All of it in one block.  Counts are fetched when the atomics of the first step have reached them, and not from the first-level cache, where a
// line may be that has table entries of the first step and counts in it.
template <bool FORK, int RUNS>
__global__ __launch_bounds__(kOsThreads) void owners_one(Owners from, Owners o, ForkArgs f, const int32_t* __restrict__ lens,
                                                         int32_t* __restrict__ lacking) {
  __shared__ int32_t starts[kOsThreads], needs[kOsThreads];
  const int tid = threadIdx.x, lane = tid & 63;
  for (int b = tid >> 6; b < o.b; b += kOsThreads / kWave) {   // a wave a sequence
    int start, need;
    if constexpr (FORK) share_sequence(from, o, f, b, lane, kWave, start, need);
    else cut_sequence(o, lens, b, lane, kWave, start, need);
    if (lane == 0) {
      starts[b] = start;
      needs[b] = need;
    }
  }
  wait_vmcnt<0>();
  __syncthreads();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
  hand_out<FORK, RUNS>(o, f, tid < o.b ? starts[tid] : 0, tid < o.b ? needs[tid] : 0, lacking);
}

// The second and third step.
template <bool FORK, int RUNS>
__global__ __launch_bounds__(kOsThreads) void owners_rest(Owners o, ForkArgs f, OwWs ws, int32_t* __restrict__ lacking) {
  const int b = min((int)threadIdx.x, o.b - 1);
  const int start = ws.start[b], need = ws.need[b];
  hand_out<FORK, RUNS>(o, f, start, (int)threadIdx.x < o.b ? need : 0, lacking);
}

// Which launches: one block for all, its last two steps, or many blocks throughout.  Us a call, in one block (the steps that the rule below gives it) and in
// many; a resize by 40 tokens, one that gives back or takes every page, a fork: 16 sequences of 260 pages 3.3 / 6.8, 5.5 / 8.5, 8.8 / 11.0; of
// 1004 pages 3.4 / 6.9, 12.8 / 9.1, 10.4 / 11.8 (two steps in one block; all three 14.7); 64 of 254 4.7 / 7.6, 13.7 / 9.0, 9.4 / 11.0 (all three 16.1);
// 256 of 67 6.5 / 7.5, 14.5 / 9.2, 11.4 / 11.2.  The step that a generated token takes is what counts, so a resize goes by it.  The block's time
// grows by 0.7 us for every 16384 pages that are looked through (4.4 for 65536), that of the many not: a step over 65536 pages 5.4 - 5.9 / 5.8 - 6.6 us
// (16 sequences or fewer) and 7.0 / 7.3 (256), over 131072 5.5 - 8.5 / 6.6 by where the free ones are, and where calls are enqueued one by one, at 3 us
// a launch, 5.5 - 8.7 / 11.0; forks of 16 over 65536 11.8 / 10.4.
constexpr int kOwSmall = 32768;
struct OwPlan {
  bool one, rest;
};
static OwPlan ow_plan(const Owners& o, bool fork) {
  const bool small_pool = o.n_pages <= (fork ? kOwSmall : 4 * kOwSmall);
  const long long entries = (long long)o.b * o.max_pages;
  return {small_pool && (fork ? o.b <= 64 && entries <= 8192 : o.b <= 128 && entries <= 16384), small_pool && o.b <= kOsThreads};
}

static hipError_t launch_take(const Owners& o, const ForkArgs& f, const OwWs& w, int32_t* lacking, bool fork, hipStream_t st) {
  if (ow_plan(o, fork).rest) {
    if (fork) hipLaunchKernelGGL((owners_rest<true, 1>), dim3(1), dim3(kOsThreads), 0, st, o, f, w, lacking);
    else if (o.n_pages <= kOwSmall) hipLaunchKernelGGL((owners_rest<false, 1>), dim3(1), dim3(kOsThreads), 0, st, o, f, w, lacking);
    else hipLaunchKernelGGL((owners_rest<false, 4>), dim3(1), dim3(kOsThreads), 0, st, o, f, w, lacking);
    return hipGetLastError();
  }
  const int tiles = ow_tiles(o.n_pages);
  hipLaunchKernelGGL(owners_count, dim3(tiles + 1), dim3(kOwThreads), 0, st, o, w);
  hipLaunchKernelGGL(owners_take, dim3(tiles + 1), dim3(kOwThreads), 0, st, o, f, w, lacking);
  return hipGetLastError();
}

hipError_t launch_pages_resize(const Owners& o, const int32_t* lens, int32_t* lacking, void* ws, hipStream_t st) {
  if (ow_plan(o, false).one) {
    if (o.n_pages <= kOwSmall) hipLaunchKernelGGL((owners_one<false, 1>), dim3(1), dim3(kOsThreads), 0, st, o, o, ForkArgs{}, lens, lacking);
    else hipLaunchKernelGGL((owners_one<false, 4>), dim3(1), dim3(kOsThreads), 0, st, o, o, ForkArgs{}, lens, lacking);
    return hipGetLastError();
  }
  const OwWs w = ow_ws(o, ws);
  hipLaunchKernelGGL(owners_cut, dim3(o.b), dim3(kOwThreads), 0, st, o, lens, w);
  return launch_take(o, ForkArgs{}, w, lacking, false, st);
}

hipError_t launch_pages_fork(const Owners& from, const Owners& o, const ForkArgs& f, int32_t* lacking, void* ws, hipStream_t st) {
  if (ow_plan(o, true).one) {
    hipLaunchKernelGGL((owners_one<true, 1>), dim3(1), dim3(kOsThreads), 0, st, from, o, f, nullptr, lacking);
    return hipGetLastError();
  }
  const OwWs w = ow_ws(o, ws);
  hipLaunchKernelGGL(owners_share, dim3(o.b), dim3(kOwThreads), 0, st, from, o, f, w);
  return launch_take(o, f, w, lacking, true, st);
}

}  // namespace quoka
