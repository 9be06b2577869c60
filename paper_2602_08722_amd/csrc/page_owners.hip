// Who holds the pages of a pool (quoka_pages_resize, quoka_pages_fork): a count of holders for each page (0: free), and for each sequence a row
// of the page table and the number of its entries in use.
//
// Pages are handed out lowest first, in the order of the sequences and of their entries, so that a call's result depends on nothing but its
// arguments: counts are changed by integer atomics, whose order does not matter, and the rank of a free page among the free ones names the
// entry that gets it.  Three launches, each of which uses what the one before has completed: entries that go or are shared (a wave a
// sequence), free pages counted (a tile of pages a block) beside the sum of what the sequences lack, free pages to entries.
#include "common.hip.h"
#include "kernels.h"

namespace quoka {

constexpr int kOwThreads = 256, kOwRun = 16, kOwTile = kOwThreads * kOwRun;   // pages of a thread, of a tile

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

__global__ __launch_bounds__(kOwThreads) void owners_cut(Owners o, const int32_t* __restrict__ lens, OwWs ws) {
  const int b = (int)blockIdx.x * (kOwThreads / kWave) + (int)(threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (b >= o.b) return;
  const int len = lens[b], had = held_by(o, b);
  const int n = len <= 0 ? 0 : min(((len - 1) >> o.shift) + 1, o.max_pages), stay = min(had, n);
  int32_t* row = o.table + (long long)b * o.max_pages;
  for (int e = n + lane; e < had; e += kWave) {
    add_holder(o, row[e], -1);
    row[e] = -1;
  }
  if (lane == 0) {
    ws.start[b] = stay;
    ws.need[b] = n - stay;
  }
}

__global__ __launch_bounds__(kOwThreads) void owners_share(Owners from, Owners o, ForkArgs f, OwWs ws) {
  const int b = (int)blockIdx.x * (kOwThreads / kWave) + (int)(threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (b >= o.b) return;
  const int had = held_by(o, b), parent = f.parents[b];
  const bool has_parent = (uint32_t)parent < (uint32_t)from.b;
  // (at most what the parent holds and the child has room for: 64 bits)
  long long len = 0;
  if (has_parent) len = min((long long)max(f.lens[parent], 0), (long long)min(held_by(from, parent), o.max_pages) << o.shift);
  const int whole = (int)(len >> o.shift), need = (len & ((1 << o.shift) - 1)) != 0 ? 1 : 0;
  int32_t* row = o.table + (long long)b * o.max_pages;
  const int32_t* theirs = from.table + (long long)(has_parent ? parent : 0) * from.max_pages;
  for (int e = lane; e < max(whole, had); e += kWave) {
    if (e < had) add_holder(o, row[e], -1);
    int32_t page = -1;
    if (e < whole) {
      page = theirs[e];
      add_holder(o, page, 1);
    }
    row[e] = page;
  }
  if (lane == 0) {
    ws.start[b] = whole;
    ws.need[b] = need;
    f.first[b] = whole << o.shift;
    f.child_lens[b] = (int)len;
  }
}

__device__ __forceinline__ bool is_free(const Owners& o, int page) { return page < o.n_pages && o.ref[page] <= 0; }

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
  uint32_t n = 0;
#pragma unroll
  for (int i = 0; i < kOwRun; ++i) n += is_free(o, (int)blockIdx.x * kOwTile + i * kOwThreads + tid) ? 1u : 0u;
  block_excl_scan<kOwThreads>(n, scan, &total);
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
  uint32_t is = 0, total;
  const int page0 = (int)blockIdx.x * kOwTile + tid * kOwRun;
#pragma unroll
  for (int i = 0; i < kOwRun; ++i) is |= is_free(o, page0 + i) ? 1u << i : 0u;
  uint32_t rank = before + block_excl_scan<kOwThreads>((uint32_t)__popc(is), scan, &total);
  for (; is != 0 && rank < wanted; is &= is - 1, ++rank) {
    const int page = page0 + __builtin_ctz(is);
    int lo = 0, hi = o.b - 1;   // the last sequence whose first rank is not above `rank` (one that wants none has the next one's)
    while (lo < hi) {
      const int mid = (lo + hi + 1) / 2;
      if ((uint32_t)ws.prefix[mid] <= rank) lo = mid;
      else hi = mid - 1;
    }
    o.ref[page] = 1;
    o.table[(long long)lo * o.max_pages + ws.start[lo] + (int)(rank - (uint32_t)ws.prefix[lo])] = page;
  }
}

static hipError_t launch_take(const Owners& o, const ForkArgs& f, const OwWs& w, int32_t* lacking, hipStream_t st) {
  const int tiles = ow_tiles(o.n_pages);
  hipLaunchKernelGGL(owners_count, dim3(tiles + 1), dim3(kOwThreads), 0, st, o, w);
  hipLaunchKernelGGL(owners_take, dim3(tiles + 1), dim3(kOwThreads), 0, st, o, f, w, lacking);
  return hipGetLastError();
}

hipError_t launch_pages_resize(const Owners& o, const int32_t* lens, int32_t* lacking, void* ws, hipStream_t st) {
  const OwWs w = ow_ws(o, ws);
  constexpr int per_block = kOwThreads / kWave;
  hipLaunchKernelGGL(owners_cut, dim3((o.b + per_block - 1) / per_block), dim3(kOwThreads), 0, st, o, lens, w);
  return launch_take(o, ForkArgs{}, w, lacking, st);
}

hipError_t launch_pages_fork(const Owners& from, const Owners& o, const ForkArgs& f, int32_t* lacking, void* ws, hipStream_t st) {
  const OwWs w = ow_ws(o, ws);
  constexpr int per_block = kOwThreads / kWave;
  hipLaunchKernelGGL(owners_share, dim3((o.b + per_block - 1) / per_block), dim3(kOwThreads), 0, st, from, o, f, w);
  return launch_take(o, f, w, lacking, st);
}

}  // namespace quoka
