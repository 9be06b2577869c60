// Verification of drafted tokens against the target's probabilities (quoka_verify_draft).
//
// Token i of a sequence is accepted while u_i q_i(x_i) < p_i(x_i), a positive number, and q_i(x_i) is finite; the product of two float32 numbers is
// exact in 64 bits.  The token after the a accepted ones is the lowest v of positive weight w_v with w_0 + ... + w_v > u_n (w_0 + w_1 + ...), w = max(p_a - q_a, 0) behind a refusal
// (p_a, should nothing be left of it), else p_a.  Sums are in 64 bits: a token's part of that line is as narrow as its probability.
//
// Bound by memory where there are many sequences (two rows of the vocabulary each), by a chain of fetches where there are few (tokens, their
// probabilities, the rows).  Lanes take neighbouring pieces of 16 bytes, wherever a row starts (an odd vocabulary's rows are aligned to an
// element), and a wave a run of neighbouring entries: the sums of whole waves say which one the random number points into, and that one
// alone adds up its entries in order.
// Measured: one sequence, 4 tokens that were looked up, vocabulary 32003, 4.0 us and 3.4 (two launches of a chain of fetches each: 8.3 a call);
// 64 sequences of up to 7, 131072 float32, 12.8 and 4.6 (67 MB in the first: 5.2 TB/s); vocabulary 1000 in one launch 3.3.
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
        good = u * q < p && weight_of(p) > 0.0 && fabs(q) < (double)INFINITY;   // (a NaN compares false)
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
  // Values worked out before this line are not kept for use after it (twice as wide as what they come from, they would not fit the registers).
  __device__ __forceinline__ void forget() {
    typedef uint32_t four __attribute__((ext_vector_type(4)));
    four bits = __builtin_bit_cast(four, x);
    asm volatile("" : "+v"(bits));
    x = __builtin_bit_cast(vec, bits);
  }
  __device__ __forceinline__ float at(int e) const {
    if constexpr (sizeof(T) == 4) return x[e];
    else return bf16_bits_to_f32(x[e]);
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
    __builtin_amdgcn_sched_barrier(0);   // (all on the way before any is used)
  }
  __device__ __forceinline__ void forget() {
#pragma unroll
    for (int j = 0; j < J; ++j) {
      p[j].forget();
      q[j].forget();
    }
  }
  // What entry e of piece j weighs: p, or (LEFT) what remains of it, weight_of((double)p - (double)q).
  template <typename LEFT>
  __device__ __forceinline__ double weight(LEFT, int j, int e) const {
    const float from = p[j].at(e);
    if constexpr (!LEFT::value) return weight_of(from);
    const float off = has_q ? q[j].at(e) : x == j * N * kWave + e ? 1.f : 0.f;
    return from > off && from < INFINITY && off > -INFINITY ? (double)from - (double)off : 0.0;
  }
  // This lane's entries of piece j.
  template <typename LEFT>
  __device__ __forceinline__ double sum(LEFT left, int j) const {
    double s = 0.0;
#pragma unroll
    for (int e = 0; e < N; ++e) s += weight(left, j, e);
    return s;
  }

  // The lowest entry of positive weight behind which `before` and the entries up to it are more than `point`; should there be none, the last
  // one of positive weight (sums of two orders may leave the point a rounding past the end); as a place in the row, -1: nothing weighs.
  // s: sums of the pieces, which name the lane; its entries are added up in order.
  template <typename LEFT>
  __device__ __forceinline__ int find(LEFT left, const double (&s)[J], double before, double point, int first) const {
    const int lane = threadIdx.x & 63;
    double incl[J];
#pragma unroll
    for (int j = 0; j < J; ++j) incl[j] = wave_incl_scan(s[j]);
    int piece = -1, of = 0;   // (the same for all lanes)
    double start = 0.0;
    bool found = false;
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const unsigned long long hits = __builtin_amdgcn_ballot_w64(s[j] > 0.0 && before + incl[j] > point), some = __builtin_amdgcn_ballot_w64(s[j] > 0.0);
      if (!found && some != 0) {
        found = hits != 0;
        piece = j;
        of = found ? (int)__builtin_ctzll(hits) : 63 - (int)__builtin_clzll(some);
        start = before + (incl[j] - s[j]);
      }
      before += last_lane(incl[j]);
    }
    if (piece < 0) return -1;
    int hit = -1, last = 0;
#pragma unroll
    for (int j = 0; j < J; ++j) {
      if (piece != j) continue;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const double w = weight(left, j, e);
        start += w;
        if (w > 0.0) {
          last = e;
          if (start > point && hit < 0) hit = e;
        }
      }
    }
    return first + piece * N * kWave + __builtin_amdgcn_readlane(lane * N + (hit >= 0 ? hit : last), of);
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

// Longer vocabularies in two launches: the sums of parts of kVfPart entries, a wave each; then the part that the random number points into, and the token in it.
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
  for (int j = 0; j < J; ++j) {
    left += run.sum(std::true_type{}, j);
    all += run.sum(std::false_type{}, j);
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
    auto search = [&](auto of) __attribute__((always_inline)) {
      double pieces[J];
#pragma unroll
      for (int j = 0; j < J; ++j) pieces[j] = run.sum(of, j);
      return run.find(of, pieces, before, point, part * kVfPart);
    };
    y = use_left ? search(std::true_type{}) : search(std::false_type{});
  }
  put_tokens(a, b, acc, y, lane);
}

// Short vocabularies in one launch: a block a sequence, a wave a run of J pieces; the entries stay in registers from their sums to the search.
constexpr int kVoThreads = 1024, kVoWaves = kVoThreads / kWave;

template <typename T, int J>
__global__ __launch_bounds__(kVoThreads) void verify_one(VerifyArgs a) {
  constexpr int N = Piece<T>::N, kRun = N * kWave * J;
  __shared__ double sums[kVoWaves];
  const int b = blockIdx.x, lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const double u = draw_of(a, b);
  const int n = drafted(a, b), acc = accepted<T>(a, b, n), first = w * kRun;
  Run<T, J> run;
  run.load(rows_of<T>(a, b, n, acc), first, a.V);
  double total, before, s[J];   // s: of this lane's pieces
  int chosen;                   // the wave that the random number points into
  auto add_up = [&](auto left) __attribute__((always_inline)) {
    double mine = 0.0;
#pragma unroll
    for (int j = 0; j < J; ++j) mine += s[j] = run.sum(left, j);
    run.forget();
    mine = wave64_sum(mine);
    __syncthreads();
    if (lane == 0) sums[w] = mine;
    __syncthreads();
    mine = lane < kVoWaves ? sums[lane] : 0.0;
    const double incl = wave_incl_scan(mine);
    total = last_lane(incl);
    before = incl - mine;
    const unsigned long long hits = __builtin_amdgcn_ballot_w64(mine > 0.0 && before + mine > u * total), some = __builtin_amdgcn_ballot_w64(mine > 0.0);
    chosen = hits != 0 ? (int)__builtin_ctzll(hits) : some != 0 ? 63 - (int)__builtin_clzll(some) : 0;
  };
  add_up(std::true_type{});
  const bool use_left = total > 0.0 || acc >= n;
  if (!use_left) add_up(std::false_type{});   // (nothing is left behind a refusal; the same for all waves)
  if (w != chosen) return;
  if (lane == 0) a.n_accepted[b] = acc;
  int y = -1;
  before = lane_of(before, chosen);
  if (total > 0.0) y = use_left ? run.find(std::true_type{}, s, before, u * total, first) : run.find(std::false_type{}, s, before, u * total, first);
  put_tokens(a, b, acc, y, lane);
}

static int vf_parts(int vocab) { return (vocab + kVfPart - 1) / kVfPart; }

size_t verify_ws_bytes(int batch, int vocab) { return (size_t)batch * vf_parts(vocab) * sizeof(double2); }

hipError_t launch_verify(const VerifyArgs& a, int dtype, void* ws, hipStream_t st) {
  auto launch = [&](auto one) {
    using T = decltype(one);
    // One launch up to 24576 float32 entries, 16384 bfloat16 ones, and of 64 sequences or more up to 32768.  Us of one and of two launches, 1 to 128
    // sequences: float32, 4096 entries 3.2 - 4.3 / 6.8 - 8.6, 8000 3.9 - 4.7 / 6.2 - 8.3, 16000 4.9 - 5.9 / 6.0 - 8.7, 24000 5.8 - 7.4 / 6.6 - 10.3, 32003
    // 6.9 - 8.2 / 6.5 - 8.0 (8 sequences or fewer), 7.7 - 9.5 / 8.1 - 12.0 (64 and 128); bfloat16, 8000 4.2 - 5.0 / 6.8 - 8.5, 16000 4.9 - 6.1 / 7.0 -
    // 8.5, 32003 6.9 - 9.3 / 6.8 - 8.2, 8.0 - 9.6 / 8.3 - 10.4.
    constexpr int kStep = Piece<T>::N * kWave * kVoWaves;   // entries of a block whose waves have one piece
    auto one_launch = [&](auto pieces) {
      hipLaunchKernelGGL((verify_one<T, decltype(pieces)::value>), dim3(a.b), dim3(kVoThreads), 0, st, a);
      return hipGetLastError();
    };
    using std::integral_constant;
    if (a.V <= kStep) return one_launch(integral_constant<int, 1>{});
    if (a.V <= 2 * kStep) return one_launch(integral_constant<int, 2>{});
    if constexpr (sizeof(T) == 4) {
      if (a.V <= 4 * kStep) return one_launch(integral_constant<int, 4>{});
      if (a.V <= 6 * kStep) return one_launch(integral_constant<int, 6>{});
      if (a.V <= 8 * kStep && a.b >= 64) return one_launch(integral_constant<int, 8>{});
    } else {
      if (a.V <= 4 * kStep && a.b >= 64) return one_launch(integral_constant<int, 4>{});
    }
    const int parts = vf_parts(a.V), waves = kVfThreads / kWave;
    hipLaunchKernelGGL((verify_parts<T>), dim3((parts + waves - 1) / waves, a.b), dim3(kVfThreads), 0, st, a, static_cast<double2*>(ws), parts);
    hipLaunchKernelGGL((verify_pick<T>), dim3(a.b), dim3(kWave), 0, st, a, static_cast<const double2*>(ws), parts);
    return hipGetLastError();
  };
  return dtype == QUOKA_BF16 ? launch(uint16_t{}) : launch(float{});
}

}  // namespace quoka
