// Verification of drafted tokens against the target's probabilities (quoka_verify_draft).
//
// Token i of a sequence is accepted while u_i q_i(x_i) < p_i(x_i); the product of two float32 numbers is exact in 64 bits.  The token after
// the a accepted ones is the lowest v of positive weight w_v with w_0 + ... + w_v > u_n (w_0 + w_1 + ...), w = max(p_a - q_a, 0) behind a refusal
// (p_a, should nothing be left of it), else p_a.  Sums are in 64 bits: a token's part of that line is as narrow as its probability.
//
// Bound by memory where there are many sequences (two rows of the vocabulary each), by a chain of fetches where there are few (tokens, their
// probabilities, the rows).  Every block works out `a` for itself.  verify_parts leaves the sums of tiles of kVfTile entries,
// verify_pick finds the tile and the token in it.
#include <type_traits>

#include "common.hip.h"
#include "kernels.h"

namespace quoka {

constexpr int kVfThreads = 256, kVfRun = 16, kVfTile = kVfThreads * kVfRun;   // entries of a thread, of a tile

__device__ __forceinline__ double wave64_sum(double x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o, kWave);
  return x;
}
__device__ __forceinline__ double wave_incl_scan(double x) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const double y = __shfl_up(x, o, kWave);
    if (lane >= o) x += y;
  }
  return x;
}

// What an entry weighs: nothing unless it is a positive number.
__device__ __forceinline__ double weight_of(double x) { return x > 0.0 && x < (double)INFINITY ? x : 0.0; }

// Accepted tokens of sequence b.  Every wave works it out for itself, 64 tokens at a time.
template <typename T>
__device__ __forceinline__ int accepted(const VerifyArgs& a, int b) {
  const int lane = threadIdx.x & 63;
  const int n = a.draft_lens == nullptr ? a.n : min(max(a.draft_lens[b], 0), a.n);
  for (int i0 = 0; i0 < n; i0 += kWave) {
    const int i = i0 + lane;
    bool good = false;
    if (i < n) {
      const int x = a.tokens[(long long)b * a.n + i];
      if (x >= 0 && x < a.V) {
        const double u = a.uniform[(long long)b * (a.n + 1) + i];
        const double p = Elem<T>::load1(static_cast<const T*>(a.target) + b * a.ts[0] + i * a.ts[1] + x);
        const double q = a.draft == nullptr ? 1.0 : Elem<T>::load1(static_cast<const T*>(a.draft) + b * a.ds[0] + i * a.ds[1] + x);
        good = u * q < p;
      }
    }
    const unsigned long long stops = __builtin_amdgcn_ballot_w64(!good);
    if (stops != 0) return i0 + (int)__builtin_ctzll(stops);   // (lanes past n stop too)
  }
  return n;
}

// The two rows that the next token of sequence b comes from.
template <typename T>
struct VfRows {
  const T *p, *q;   // q: nullptr where nothing is taken off, or only
  int x;            // the refused token, whose weight loses 1 (-1: none)
};
template <typename T>
__device__ __forceinline__ VfRows<T> rows_of(const VerifyArgs& a, int b, int acc) {
  const int n = a.draft_lens == nullptr ? a.n : min(max(a.draft_lens[b], 0), a.n);
  VfRows<T> r;
  r.p = static_cast<const T*>(a.target) + b * a.ts[0] + acc * a.ts[1];
  r.q = nullptr;
  r.x = -1;
  if (acc < n) {
    if (a.draft != nullptr) r.q = static_cast<const T*>(a.draft) + b * a.ds[0] + acc * a.ds[1];
    else r.x = a.tokens[(long long)b * a.n + acc];
  }
  return r;
}

// Entries v0 .. v0 + kVfRun - 1: `left` what remains of p, `all` p itself.
template <typename T>
__device__ __forceinline__ void weights(const VfRows<T>& r, int V, int v0, double (&left)[kVfRun], double (&all)[kVfRun]) {
  float p[kVfRun], q[kVfRun];
#pragma unroll
  for (int e = 0; e < kVfRun; ++e) {
    p[e] = v0 + e < V ? Elem<T>::load1(r.p + v0 + e) : 0.f;
    q[e] = r.q != nullptr && v0 + e < V ? Elem<T>::load1(r.q + v0 + e) : v0 + e == r.x ? 1.f : 0.f;
  }
#pragma unroll
  for (int e = 0; e < kVfRun; ++e) {
    all[e] = weight_of((double)p[e]);
    left[e] = weight_of((double)p[e] - (double)q[e]);
  }
}

// parts: [b, tiles] sums of what is left and of p.
template <typename T>
__global__ __launch_bounds__(kVfThreads) void verify_parts(VerifyArgs a, double2* __restrict__ parts) {
  __shared__ double2 of_wave[kVfThreads / kWave];
  const int b = blockIdx.y, tid = threadIdx.x;
  const VfRows<T> r = rows_of<T>(a, b, accepted<T>(a, b));
  double left[kVfRun], all[kVfRun], sl = 0.0, sa = 0.0;
  weights<T>(r, a.V, (int)blockIdx.x * kVfTile + tid * kVfRun, left, all);
#pragma unroll
  for (int e = 0; e < kVfRun; ++e) {
    sl += left[e];
    sa += all[e];
  }
  sl = wave64_sum(sl);
  sa = wave64_sum(sa);
  if ((tid & 63) == 0) of_wave[tid >> 6] = make_double2(sl, sa);
  __syncthreads();
  if (tid != 0) return;
#pragma unroll
  for (int w = 1; w < kVfThreads / kWave; ++w) {
    sl += of_wave[w].x;
    sa += of_wave[w].y;
  }
  parts[(size_t)b * gridDim.x + blockIdx.x] = make_double2(sl, sa);
}

template <typename T>
__global__ __launch_bounds__(kVfThreads) void verify_pick(VerifyArgs a, const double2* __restrict__ parts, int tiles) {
  __shared__ double of_wave[kVfThreads / kWave];
  __shared__ int first_of[kVfThreads / kWave], last_of[kVfThreads / kWave];
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int acc = accepted<T>(a, b);
  const VfRows<T> r = rows_of<T>(a, b, acc);
  // every wave: the sums of the whole row, then the tile that the random number points into
  const double2* mine = parts + (size_t)b * tiles;
  double sl = 0.0, sa = 0.0;
  for (int t = lane; t < tiles; t += kWave) {
    sl += mine[t].x;
    sa += mine[t].y;
  }
  const bool use_left = wave64_sum(sl) > 0.0;
  (void)sa;
  auto part_of = [&](int t) { return t < tiles ? use_left ? mine[t].x : mine[t].y : 0.0; };
  double total = 0.0;
  for (int t0 = 0; t0 < tiles; t0 += kWave) total += __shfl(wave_incl_scan(part_of(t0 + lane)), 63, kWave);
  const float u = fminf(fmaxf(a.uniform[(long long)b * (a.n + 1) + a.n], 0.f), 1.f - 0x1p-24f);
  const double point = (double)u * total;
  double before = 0.0;
  int tile = -1;
  for (int t0 = 0; t0 < tiles && tile < 0; t0 += kWave) {
    const double incl = wave_incl_scan(part_of(t0 + lane));
    const unsigned long long hit = __builtin_amdgcn_ballot_w64(before + incl > point);
    if (hit != 0) {
      const int at = (int)__builtin_ctzll(hit);
      tile = t0 + at;
      before += __shfl(incl, at, kWave) - __shfl(part_of(t0 + lane), at, kWave);
    } else {
      before += __shfl(incl, 63, kWave);
    }
  }
  int y = -1;
  if (tile >= 0) {   // block-uniform (-1: nothing has any weight)
    double left[kVfRun], all[kVfRun], s = 0.0;
    const int v0 = tile * kVfTile + tid * kVfRun;
    weights<T>(r, a.V, v0, left, all);
#pragma unroll
    for (int e = 0; e < kVfRun; ++e) {
      if (!use_left) left[e] = all[e];
      s += left[e];
    }
    const double incl = wave_incl_scan(s);
    if (lane == 63) of_wave[w] = incl;
    __syncthreads();
    double run = before + (incl - s);
    for (int i = 0; i < w; ++i) run += of_wave[i];
    int first = INT32_MAX, last = -1;
#pragma unroll
    for (int e = 0; e < kVfRun; ++e) {
      run += left[e];
      if (left[e] > 0.0) {
        last = v0 + e;
        if (run > point && first == INT32_MAX) first = v0 + e;
      }
    }
    first = (int)wave_min_u32((uint32_t)first);
    last = (int)wave_max_u32((uint32_t)(last + 1)) - 1;
    if (lane == 0) {
      first_of[w] = first;
      last_of[w] = last;
    }
    __syncthreads();
    for (int i = 0; i < kVfThreads / kWave; ++i) {
      first = min(first, first_of[i]);
      last = max(last, last_of[i]);
    }
    y = first != INT32_MAX ? first : last;   // (sums of two orders may leave the point a rounding past the tile's end)
  }
  if (tid == 0) a.n_accepted[b] = acc;
  for (int i = tid; i <= a.n; i += kVfThreads)
    a.tokens_out[(long long)b * (a.n + 1) + i] = i < acc ? a.tokens[(long long)b * a.n + i] : i == acc ? y : -1;
}

static int vf_tiles(int vocab) { return (vocab + kVfTile - 1) / kVfTile; }

size_t verify_ws_bytes(int batch, int vocab) { return (size_t)batch * vf_tiles(vocab) * sizeof(double2); }

hipError_t launch_verify(const VerifyArgs& a, int dtype, void* ws, hipStream_t st) {
  auto launch = [&](auto one) {
    using T = decltype(one);
    const int tiles = vf_tiles(a.V);
    hipLaunchKernelGGL((verify_parts<T>), dim3(tiles, a.b), dim3(kVfThreads), 0, st, a, static_cast<double2*>(ws));
    hipLaunchKernelGGL((verify_pick<T>), dim3(a.b), dim3(kVfThreads), 0, st, a, static_cast<const double2*>(ws), tiles);
    return hipGetLastError();
  };
  return dtype == QUOKA_BF16 ? launch(uint16_t{}) : launch(float{});
}

}  // namespace quoka
