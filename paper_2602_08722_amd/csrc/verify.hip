// Verification of drafted tokens against the target's probabilities (quoka_verify_draft).
//
// Token i of a sequence is accepted while u_i q_i(x_i) < p_i(x_i), a positive number; the product of two float32 numbers is exact in 64 bits.  The token after
// the a accepted ones is the lowest v of positive weight w_v with w_0 + ... + w_v > u_n (w_0 + w_1 + ...), w = max(p_a - q_a, 0) behind a refusal
// (p_a, should nothing be left of it), else p_a.  Sums are in 64 bits: a token's part of that line is as narrow as its probability.
//
// Bound by memory where there are many sequences (two rows of the vocabulary each), by a chain of fetches where there are few (tokens, their
// probabilities, the rows).  Lanes take neighbouring pieces of 16 bytes, wherever a row starts (an odd vocabulary's rows are aligned to an
// element), and a wave a run of neighbouring entries: the sums of whole waves say which one the random number points into, and that one
// alone adds up its entries in order.
// Measured: one sequence, 4 tokens that were looked up, vocabulary 32003, 3.7 us and 3.3 (two launches of a chain of fetches each: 8.3 a call);
// 64 sequences of up to 7, 131072 float32, 12.3 and 5.1 (67 MB in the first: 5.5 TB/s).  One launch, a block a sequence, 16 us where this takes 7.
#include <type_traits>

#include "common.hip.h"
#include "kernels.h"

namespace quoka {

// Sums over the wave's lanes, by moves between neighbouring lanes as in common.hip.h (through LDS, a step takes several times as long).
__device__ __forceinline__ double lane_of(double x, int lane) {
  const unsigned long long u = __double_as_longlong(x);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)u, lane), hi = (uint32_t)__builtin_amdgcn_readlane((int)(u >> 32), lane);
  return __longlong_as_double((long long)((unsigned long long)hi << 32 | lo));
}
template <int CTRL, int ROW_MASK = 0xF>
__device__ __forceinline__ double plus_lane(double x) {
  const unsigned long long u = __double_as_longlong(x);
  const uint32_t lo = dpp_take<CTRL, ROW_MASK>(0u, (uint32_t)u), hi = dpp_take<CTRL, ROW_MASK>(0u, (uint32_t)(u >> 32));
  return x + __longlong_as_double((long long)((unsigned long long)hi << 32 | lo));
}
__device__ __forceinline__ double wave_incl_scan(double x) {
  x = plus_lane<0x111>(x);
  x = plus_lane<0x112>(x);
  x = plus_lane<0x114>(x);
  x = plus_lane<0x118>(x);
  x = plus_lane<0x142, 0xA>(x);
  return plus_lane<0x143, 0xC>(x);
}
__device__ __forceinline__ double last_lane(double x) { return lane_of(x, 63); }
__device__ __forceinline__ double wave64_sum(double x) { return last_lane(wave_incl_scan(x)); }

// What an entry weighs: nothing unless it is a positive number.
__device__ __forceinline__ double weight_of(double x) { return x > 0.0 && x < (double)INFINITY ? x : 0.0; }

__device__ __forceinline__ int drafted(const VerifyArgs& a, int b) {
  return a.draft_lens == nullptr ? a.n : min(max(a.draft_lens[b], 0), a.n);
}

// Accepted tokens of sequence b, n of which are drafted.  Every wave works it out for itself, 64 tokens at a time.
template <typename T>
__device__ __forceinline__ int accepted(const VerifyArgs& a, int b, int n) {
  const int lane = threadIdx.x & 63;
  for (int i0 = 0; i0 < n; i0 += kWave) {
    const int i = i0 + lane;
    bool good = false;
    if (i < n) {
      const int x = a.tokens[(long long)b * a.n + i];
      const double u = a.uniform[(long long)b * (a.n + 1) + i];
      if (x >= 0 && x < a.V) {
        const double p = Elem<T>::load1(static_cast<const T*>(a.target) + b * a.ts[0] + i * a.ts[1] + x);
        const double q = a.draft == nullptr ? 1.0 : Elem<T>::load1(static_cast<const T*>(a.draft) + b * a.ds[0] + i * a.ds[1] + x);
        good = u * q < p && weight_of(p) > 0.0;   // (a NaN compares false)
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
__device__ __forceinline__ VfRows<T> rows_of(const VerifyArgs& a, int b, int n, int acc) {
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

// 16 bytes of a row, at an element's alignment.
template <typename T>
struct Piece {
  static constexpr int N = 16 / sizeof(T);
  typedef T vec __attribute__((ext_vector_type(N), aligned(sizeof(T))));
  vec x;
  __device__ __forceinline__ void load(const T* row, int v0, int V) {   // entries past V are zeros
    if (v0 + N <= V) {
      x = *reinterpret_cast<const vec*>(row + v0);
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] = v0 + e < V ? row[v0 + e] : T(0);
    }
  }
  __device__ __forceinline__ double at(int e) const {
    if constexpr (sizeof(T) == 4) return (double)x[e];
    else return (double)bf16_bits_to_f32(x[e]);
  }
};

// J pieces of a lane, 64 lanes' pieces one behind the other: N * 64 * J neighbouring entries of a wave, from v0 on (the lane's own start in it).
template <typename T, int J>
struct Run {
  static constexpr int N = Piece<T>::N, kEntries = N * kWave * J;
  Piece<T> p[J], q[J];
  int x;   // place of the refused token among the wave's entries, as seen from this lane (negative or large: elsewhere)
  bool has_q;
  __device__ __forceinline__ void load(const VfRows<T>& r, int first, int V) {
    const int v0 = first + (int)(threadIdx.x & 63) * N;
    has_q = r.q != nullptr;
    x = r.x < 0 ? -1 : r.x - v0;
#pragma unroll
    for (int j = 0; j < J; ++j) p[j].load(r.p, v0 + j * N * kWave, V);
    if (has_q) {   // (the same for all lanes)
#pragma unroll
      for (int j = 0; j < J; ++j) q[j].load(r.q, v0 + j * N * kWave, V);
    }
  }
  __device__ __forceinline__ double all(int j, int e) const { return weight_of(p[j].at(e)); }
  __device__ __forceinline__ double left(int j, int e) const {   // what remains of p
    return weight_of(p[j].at(e) - (has_q ? q[j].at(e) : x == j * N * kWave + e ? 1.0 : 0.0));
  }
  __device__ __forceinline__ double weight(bool use_left, int j, int e) const { return use_left ? left(j, e) : all(j, e); }

  // The lowest entry of positive weight behind which `before` and the entries up to it are more than `point`; should there be none, the last
  // one of positive weight (sums of two orders may leave the point a rounding past the end); as a place in the row, -1: nothing weighs.
  __device__ __forceinline__ int find(bool use_left, double before, double point, int first) const {
    const int lane = threadIdx.x & 63;
    double w[J][N], s[J], incl[J];
#pragma unroll
    for (int j = 0; j < J; ++j) {
      s[j] = 0.0;
#pragma unroll
      for (int e = 0; e < N; ++e) s[j] += w[j][e] = weight(use_left, j, e);
      incl[j] = wave_incl_scan(s[j]);
    }
    int last = -1;
#pragma unroll
    for (int j = 0; j < J; ++j) {
      double run = before + (incl[j] - s[j]);
      int hit = -1, mine = -1;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        run += w[j][e];
        if (w[j][e] > 0.0) {
          mine = e;
          if (run > point && hit < 0) hit = e;
        }
      }
      const int at = first + j * N * kWave + lane * N;
      const unsigned long long hits = __builtin_amdgcn_ballot_w64(hit >= 0);
      if (hits != 0) return __builtin_amdgcn_readlane(at + hit, (int)__builtin_ctzll(hits));
      const unsigned long long some = __builtin_amdgcn_ballot_w64(mine >= 0);
      if (some != 0) last = __builtin_amdgcn_readlane(at + mine, 63 - (int)__builtin_clzll(some));
      before += last_lane(incl[j]);
    }
    return last;
  }
};

// The random number, cut to [0, 1).
__device__ __forceinline__ double draw_of(const VerifyArgs& a, int b) {
  return (double)fminf(fmaxf(a.uniform[(long long)b * (a.n + 1) + a.n], 0.f), 1.f - 0x1p-24f);
}
__device__ __forceinline__ void put_tokens(const VerifyArgs& a, int b, int acc, int y, int lane) {   // one wave
  for (int i = lane; i <= a.n; i += kWave)
    a.tokens_out[(long long)b * (a.n + 1) + i] = i < acc ? a.tokens[(long long)b * a.n + i] : i == acc ? y : -1;
}

// Two launches: the sums of parts of kVfPart entries, a wave each; then the part that the random number points into, and the token in it.
constexpr int kVfThreads = 256, kVfPart = 1024;

// sums: [b, parts] of what is left and of p
template <typename T>
__global__ __launch_bounds__(kVfThreads) void verify_parts(VerifyArgs a, double2* __restrict__ sums, int parts) {
  constexpr int J = kVfPart / (Piece<T>::N * kWave);
  const int b = blockIdx.y, part = (int)blockIdx.x * (kVfThreads / kWave) + (int)(threadIdx.x >> 6);
  if (part >= parts) return;
  const int n = drafted(a, b), acc = accepted<T>(a, b, n);
  if (part == 0 && (threadIdx.x & 63) == 0) a.n_accepted[b] = acc;   // (what the next launch goes by, too)
  Run<T, J> run;
  run.load(rows_of<T>(a, b, n, acc), part * kVfPart, a.V);
  double left = 0.0, all = 0.0;
#pragma unroll
  for (int j = 0; j < J; ++j)
#pragma unroll
    for (int e = 0; e < Piece<T>::N; ++e) {
      left += run.left(j, e);
      all += run.all(j, e);
    }
  left = wave64_sum(left);
  all = wave64_sum(all);
  if ((threadIdx.x & 63) == 0) sums[(size_t)b * parts + part] = make_double2(left, all);
}

// A wave a sequence; a lane has K neighbouring sums at a time.
template <typename T>
__global__ __launch_bounds__(kWave) void verify_pick(VerifyArgs a, const double2* __restrict__ sums, int parts) {
  constexpr int J = kVfPart / (Piece<T>::N * kWave), K = 4;
  const int b = blockIdx.x, lane = threadIdx.x;
  const double2* mine = sums + (size_t)b * parts;
  double2 s[K];
  auto load = [&](int t0) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int t = t0 + lane * K + k;
      s[k] = t < parts ? mine[t] : make_double2(0.0, 0.0);
    }
  };
  load(0);
  const double u = draw_of(a, b);
  const int n = drafted(a, b), acc = min(max(a.n_accepted[b], 0), n);
  const VfRows<T> r = rows_of<T>(a, b, n, acc);
  double left = 0.0, all = 0.0;
  for (int t0 = 0; t0 < parts; t0 += K * kWave) {
    if (t0 > 0) load(t0);
    double l = 0.0, p = 0.0;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      l += s[k].x;
      p += s[k].y;
    }
    left += last_lane(wave_incl_scan(l));   // (in the order of the search below: the line's end is its last sum)
    all += last_lane(wave_incl_scan(p));
  }
  const bool use_left = left > 0.0;
  const double point = u * (use_left ? left : all);
  double before = 0.0;
  int y = -1;
  if (left > 0.0 || all > 0.0) {   // (the same for all lanes)
    int part = -1, last = -1;
    double before_last = 0.0;
    for (int t0 = 0; t0 < parts && part < 0; t0 += K * kWave) {
      if (parts > K * kWave) load(t0);
      double w[K], sum = 0.0;
#pragma unroll
      for (int k = 0; k < K; ++k) {
        w[k] = use_left ? s[k].x : s[k].y;
        sum += w[k];
      }
      const double incl = wave_incl_scan(sum);
      double run = before + (incl - sum), at = run, at_some = run;
      int hit = -1, some = -1;
#pragma unroll
      for (int k = 0; k < K; ++k) {
        if (w[k] > 0.0) {
          some = k;
          at_some = run;
          if (hit < 0 && run + w[k] > point) {
            hit = k;
            at = run;
          }
        }
        run += w[k];
      }
      const unsigned long long hits = __builtin_amdgcn_ballot_w64(hit >= 0), any = __builtin_amdgcn_ballot_w64(some >= 0);
      if (hits != 0) {
        const int of = (int)__builtin_ctzll(hits);
        part = t0 + of * K + __builtin_amdgcn_readlane(hit, of);
        before = lane_of(at, of);
      } else {
        if (any != 0) {
          const int of = 63 - (int)__builtin_clzll(any);
          last = t0 + of * K + __builtin_amdgcn_readlane(some, of);
          before_last = lane_of(at_some, of);
        }
        before += last_lane(incl);
      }
    }
    if (part < 0) {
      part = last;
      before = before_last;
    }
    Run<T, J> run;
    run.load(r, part * kVfPart, a.V);
    y = run.find(use_left, before, point, part * kVfPart);
  }
  put_tokens(a, b, acc, y, lane);
}

static int vf_parts(int vocab) { return (vocab + kVfPart - 1) / kVfPart; }

size_t verify_ws_bytes(int batch, int vocab) { return (size_t)batch * vf_parts(vocab) * sizeof(double2); }

hipError_t launch_verify(const VerifyArgs& a, int dtype, void* ws, hipStream_t st) {
  auto launch = [&](auto one) {
    using T = decltype(one);
    const int parts = vf_parts(a.V), waves = kVfThreads / kWave;
    hipLaunchKernelGGL((verify_parts<T>), dim3((parts + waves - 1) / waves, a.b), dim3(kVfThreads), 0, st, a, static_cast<double2*>(ws), parts);
    hipLaunchKernelGGL((verify_pick<T>), dim3(a.b), dim3(kWave), 0, st, a, static_cast<const double2*>(ws), parts);
    return hipGetLastError();
  };
  return dtype == QUOKA_BF16 ? launch(uint16_t{}) : launch(float{});
}

}  // namespace quoka
