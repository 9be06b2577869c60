// Cross attention of single tokens and a few (at most 32 query rows per KV head) over states in pages, bfloat16, where the states are not
// many: a block has a sequence and a KV head to itself and writes the rows whole, so there are no partials and no second launch.
//
// Rows, products and the way of a tile to LDS are those of paged_decode.hip; the waves of the block take tiles of 32 states in turn, and
// their sums meet in LDS.  Without a mask, every token sees every state.
// Bound by a chain of fetches (length, pages, rows: 4 us until a block of one round of tiles has ended) and by the waves' way through a round
// of tiles, 1.2 us at d 64, 1.4 at d 128, whatever the bytes: LDS, which takes every row and gives it back, and the products' latency.  Two
// tiles of each wave on the way at once, and rows in four registers in the place of sixteen (at most eight query rows, states on lanes, P by
// way of LDS), left a round as it was; K as operands straight from memory and 16 waves a block made it longer (rows as they are 2.4 us).
#include "decode_tile.hip.h"

namespace quoka {

template <int D, bool FP8, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void cross_few(Dims dm, PagedArgs a) {
  using Cfg = PdTile<D, FP8, WAVES>;
  constexpr int KS = Cfg::KS, DB = Cfg::DB, LPR = Cfg::LPR, NLD = Cfg::NLD, LD = Cfg::LD, LDV = Cfg::LDV, LDO = Cfg::LDO;
  constexpr int THREADS = 64 * WAVES;
  extern __shared__ __align__(16) unsigned char smem[];
  const Pages& pg = a.pg;
  const int b = blockIdx.x, kv = blockIdx.y;
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int li = lane & 31, hf = lane >> 5;
  const int g = dm.g;
  const int C = a.chunk_lens == nullptr ? dm.C : max(min(a.chunk_lens[b], dm.C), 0);
  const int n = min(max(a.kv_lens[b], 0), dm.T_max), n_rows = n > 0 ? C * g : 0;   // n_rows <= 32, checked by the launcher
  // rows past the chunk, and all where there is nothing to see: zeros and no weight
  for (int i = n_rows * (D / 8) + tid; i < dm.C * g * (D / 8); i += THREADS) {
    const int r = i / (D / 8), c8 = i % (D / 8), tok = r / g, h = kv * g + r % g;
    *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(a.out) + b * dm.os[0] + h * dm.os[1] + (size_t)tok * dm.os[2] + 8 * c8) =
        u32x4{0u, 0u, 0u, 0u};
    if (c8 == 0 && a.lse != nullptr) a.lse[(size_t)(b * dm.n_q + h) * dm.C + tok] = -INFINITY;
  }
  if (n_rows == 0) return;   // block-uniform
  const int tiles = (n + kPdTile - 1) / kPdTile;

  const int32_t* table = pg.table + (size_t)b * pg.max_pages;
  constexpr int es = FP8 ? 1 : 2;
  const int c = lane % LPR, group = lane / LPR;   // 16 bytes of a row
  const uint64_t k_pool = reinterpret_cast<uint64_t>(pg.k) + (uint64_t)kv * pg.st[1] * es;
  const uint64_t v_pool = reinterpret_cast<uint64_t>(pg.v) + (uint64_t)kv * pg.st[1] * es;
  const uint8_t* k_scales = pg.k_scale + ((size_t)kv << pg.shift);
  const uint8_t* v_scales = pg.v_scale + ((size_t)kv << pg.shift);
  const uint32_t page_units = (uint32_t)(pg.st[0] / (16 / es)), slot_units = (uint32_t)(pg.st[2] / (16 / es)), page_scales = (uint32_t)pg.n_kv << pg.shift;
  const int row0 = Cfg::first_row(group), my_slot = row0 + lane % NLD;   // the group's rows; the one that this lane looks up
  uint32_t pos = 0, page = 0;   // of the tile whose rows are fetched next
  auto look_up_page = [&](int tt) __attribute__((always_inline)) {
    pos = (uint32_t)min(tt * kPdTile + my_slot, n - 1);   // (tail slots repeat a real row)
    page = (uint32_t)table[min((int)(pos >> pg.shift), pg.max_pages - 1)];
  };
  struct Rows {
    u32x4 k[NLD], v[NLD];
    uint32_t k_ex, v_ex;   // exponents of the slot that this lane looked up
  };
  // Requests the rows whose pages have been looked up last, and looks up the pages of tile tt: ahead of the rows, since fetches arrive in
  // order and the next call waits for the pages.
  auto issue = [&](Rows& r, int tt) __attribute__((always_inline)) {
    const uint32_t at_page = min(page, (uint32_t)(pg.n_pages - 1)), slot = pos & ((1u << pg.shift) - 1u);
    const uint32_t off = at_page * page_units + slot * slot_units;
    look_up_page(tt);
    if constexpr (FP8) {
      const uint32_t s = at_page * page_scales + slot;
      r.k_ex = k_scales[s];
      r.v_ex = v_scales[s];
    }
    __builtin_amdgcn_sched_barrier(0);
    typedef const u32x4 __attribute__((address_space(1))) * global_row;
#pragma unroll
    for (int i = 0; i < NLD; ++i) {
      const uint64_t o = (uint64_t)(group_lane<LPR>(off, i) + (uint32_t)c) << 4;
      r.k[i] = *(global_row)(k_pool + o);
      r.v[i] = *(global_row)(v_pool + o);
    }
  };
  uint16_t* kt = reinterpret_cast<uint16_t*>(smem + (size_t)w * Cfg::kWaveBytes);
  uint16_t* vt = reinterpret_cast<uint16_t*>(smem + (size_t)w * Cfg::kWaveBytes + Cfg::kKBytes);
  const int turn = (D == 128 ? c / 4 : row0 / 4) % 2 * 8;   // FP8: where a lane's first piece of V goes
  auto to_lds = [&](const Rows& r) __attribute__((always_inline)) {
    const uint32_t both = FP8 ? r.k_ex | r.v_ex << 8 : 0u;
#pragma unroll
    for (int i = 0; i < NLD; ++i) {
      uint16_t* kd = kt + (row0 + i) * LD + c * 8;
      uint16_t* vd = vt + (row0 + i) * LDV + c * (16 / es);
      if constexpr (FP8) {
        const uint32_t ex = group_lane<LPR>(both, i);
        const float ks = row_scale(ex & 255u), vs = row_scale(ex >> 8);
        *reinterpret_cast<u32x4*>(kd) = widen_bf16(u32x2{r.k[i][0], r.k[i][1]}, ks);
        *reinterpret_cast<u32x4*>(kd + D / 2) = widen_bf16(u32x2{r.k[i][2], r.k[i][3]}, ks);
        *reinterpret_cast<u32x4*>(vd + turn) = widen_bf16(u32x2{r.v[i][0], r.v[i][1]}, vs);
        *reinterpret_cast<u32x4*>(vd + (8 - turn)) = widen_bf16(u32x2{r.v[i][2], r.v[i][3]}, vs);
      } else {
        *reinterpret_cast<u32x4*>(kd) = r.k[i];
        *reinterpret_cast<u32x4*>(vd) = r.v[i];
      }
    }
  };

  Rows rows;
  int t = w;   // this wave's tiles: every WAVES-th
  if (t < tiles) {
    look_up_page(t);
    issue(rows, t + WAVES);
  }

  // Q operand: row li -> (token li / g, head li % g); padding rows repeat row 0 and are never stored
  const int row = li < n_rows ? li : 0;
  bf16x8 qreg[KS];
  {
    const uint16_t* qrow = static_cast<const uint16_t*>(a.q) + b * dm.qs[0] + (size_t)(kv * g + row % g) * dm.qs[1] +
                           (size_t)(row / g) * dm.qs[2] + (FP8 ? 16 : 8) * hf;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)   // (FP8: piece j of a row in LDS holds elements 16 j .. + 7, or 16 (j - D / 16) + 8 .. + 15)
      qreg[ks] = *reinterpret_cast<const bf16x8*>(qrow + (!FP8 ? ks * 16 : ks < KS / 2 ? ks * 32 : (ks - KS / 2) * 32 + 8));
  }

  f32x16 o[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int v = 0; v < 16; ++v) o[db][v] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;
  constexpr float kLazy = 8.0f;   // the reference point only moves when a row's maximum exceeds it by more than 2^8
  const float sl2 = 1.4426950408889634f / sqrtf((float)D);   // the softmax scale and the change to base 2
  for (; t < tiles; t += WAVES) {
    to_lds(rows);   // (this wave's own piece of LDS: its accesses stay in order, no barrier)
    __builtin_amdgcn_wave_barrier();
    if (t + WAVES < tiles) issue(rows, t + 2 * WAVES);
    // ---- S^T = K Q^T ----
    f32x16 s;
#pragma unroll
    for (int v = 0; v < 16; ++v) s[v] = 0.f;
    const uint16_t* kp = kt + li * LD + 8 * hf;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8*>(kp + ks * 16), qreg[ks], s, 0, 0, 0);
    const int limit = n - t * kPdTile;   // states of the tile
    if (limit < kPdTile) {                // wave-uniform
#pragma unroll
      for (int v = 0; v < 16; ++v)
        if (8 * (v / 4) + 4 * hf + v % 4 >= limit) s[v] = -INFINITY;
    }
    // ---- online softmax ----
    float mx = -INFINITY;
#pragma unroll
    for (int v = 0; v < 16; ++v) mx = fmaxf(mx, s[v]);
    mx = fmaxf(mx, other_half(mx)) * sl2;
    if (__builtin_amdgcn_ballot_w64(mx > m_run + kLazy) != 0) {   // wave-uniform branch
      const float m_new = mx > m_run + kLazy ? mx : m_run;
      const float alpha = __builtin_amdgcn_exp2f(m_run - (m_new == -INFINITY ? 0.f : m_new));
      m_run = m_new;
      l_run *= alpha;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int v = 0; v < 16; ++v) o[db][v] *= alpha;
    }
    const float neg_m = m_run == -INFINITY ? 0.f : -m_run;
    float psum = 0.f;   // (of the probabilities before they are rounded: what lse shows; the weights add up to 1 within the roundings)
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      s[v] = __builtin_amdgcn_exp2f(fmaf(s[v], sl2, neg_m));
      psum += s[v];
    }
    l_run += psum;
    // ---- O^T += V^T P^T ----
    // (FP8, where pieces are the other way round: D = 128 dims 64 .. 127, D = 64 rows 4 .. 7 of 8)
    const int v_at = (4 * hf + ((lane & 15) >> 2)) * LDV + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
    const tr_ptr vtr = (tr_ptr)(vt + (FP8 && D == 64 ? v_at ^ (8 * hf) : v_at)), vtr_upper = (tr_ptr)(vt + (FP8 && D == 128 ? v_at ^ 8 : v_at));
#pragma unroll
    for (int t2 = 0; t2 < 2; ++t2) {
      bf16x8 p;
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] = (__bf16)s[8 * t2 + e];   // (the operands of a product are bfloat16: one rounding)
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const int e0 = 16 * t2 * LDV + db * 32;
        const tr_ptr at_v = (FP8 && D == 128 && db >= 2 ? vtr_upper : vtr) + e0 / 4;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(at_v);
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(at_v + 8 * LDV / 4);
        const s16x8 both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, both), p, o[db], 0, 0, 0);
      }
    }
    __builtin_amdgcn_wave_barrier();
  }

  // ---- the waves' sums of the real rows meet in LDS ----
  const float l_wave = l_run + other_half(l_run);
  __syncthreads();   // the waves' pieces may be reused
  float* mo = reinterpret_cast<float*>(smem);   // [WAVES][32 rows][LDO]
  float* mm = mo + WAVES * 32 * LDO;            // [WAVES][32]
  float* ml = mm + WAVES * 32;
  float* mw = ml + WAVES * 32;
  if (li < n_rows) {
    if (hf == 0) {
      mm[w * 32 + li] = m_run;
      ml[w * 32 + li] = l_wave;
    }
    float* rec = mo + ((size_t)w * 32 + li) * LDO + 4 * hf;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int v4 = 0; v4 < 4; ++v4)   // registers 4*v4 .. 4*v4+3 are four consecutive dims
        *reinterpret_cast<float4*>(rec + 32 * db + 8 * v4) = make_float4(o[db][4 * v4], o[db][4 * v4 + 1], o[db][4 * v4 + 2], o[db][4 * v4 + 3]);
  }
  __syncthreads();
  if (tid < n_rows) {   // the weights of a row's waves, divided by its sum (some wave has seen a state: finite)
    float m = mm[tid], l = 0.f, e[WAVES];
#pragma unroll
    for (int u = 1; u < WAVES; ++u) m = fmaxf(m, mm[u * 32 + tid]);
#pragma unroll
    for (int u = 0; u < WAVES; ++u) {
      e[u] = mm[u * 32 + tid] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mm[u * 32 + tid] - m);
      l += e[u] * ml[u * 32 + tid];
    }
#pragma unroll
    for (int u = 0; u < WAVES; ++u) mw[u * 32 + tid] = e[u] / l;
    if (a.lse != nullptr) a.lse[(size_t)(b * dm.n_q + kv * g + tid % g) * dm.C + tid / g] = (m + log2f(l)) * 0.6931471805599453f;
  }
  __syncthreads();
  for (int i = tid; i < n_rows * (D / 4); i += THREADS) {
    const int r = i / (D / 4), c4 = i % (D / 4);
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int u = 0; u < WAVES; ++u) {
      const float wgt = mw[u * 32 + r];
      const float4 x = *reinterpret_cast<const float4*>(mo + ((size_t)u * 32 + r) * LDO + 4 * c4);
      acc.x += wgt * x.x;
      acc.y += wgt * x.y;
      acc.z += wgt * x.z;
      acc.w += wgt * x.w;
    }
    const bf16x2 lo = {(__bf16)acc.x, (__bf16)acc.y}, hi = {(__bf16)acc.z, (__bf16)acc.w};
    *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.out) + b * dm.os[0] + (kv * g + r % g) * dm.os[1] + (size_t)(r / g) * dm.os[2] + 4 * c4) =
        u32x2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
  }
}

template <int D>
constexpr int kFewWaves = D == 64 ? 12 : 8;   // as many as LDS has room for

// (One row, and two, over fewer states yet: cross_rows.hip.)
// Which lists are few, by rounds of tiles and blocks (a compute unit has one at a time); us of this kernel and of the two launches that share
// lists (paged_decode), all lists equal, and of lists between an eighth of it and the longest.
//   Few blocks: three rounds (two at d 128).  12 heads, d 64, one or eight sequences of 64 states 5.0 / 7.4, 500 6.3 / 7.8, 1000 7.7 / 8.0,
//   2000 11.0 / 8.2; 8 heads of 4, d 128, 64 5.0 / 7.5, 500 8.0 / 8.5, 1000 10.8 / 8.6.
//   96 blocks: four; 128 to 256, half of the compute units and all of them: eight.  32 sequences, d 64, 8 heads of 4, 1500 states 19.0 / 22.4 and
//   14.6 / 17.4 (200 at least); of up to 3000 0.83 - 0.97 of the time, of 6000 0.85 - 1.15; d 128, 1500 31.8 / 35.8 and 24.7 / 26.5, of up to 2000
//   0.85 - 1.03, of 4000 0.8 - 1.08.  The most that such a batch may lose are lists that differ at 100 blocks, 1.04 (four rounds; eight 1.14).
//   More than 256: three (two) again, up to 768.  12 heads, d 64, 500 states, 300 blocks 0.8 - 0.92 of the time, 700 1.0 - 1.02, 1030 1.11 - 1.23,
//   2000 1.23 - 1.27, since blocks with 129 or 152 KB of LDS leave a compute unit to one sequence after another.
bool cross_few_applies(const Dims& dm) {
  const int tiles = (dm.T_max + kPdTile - 1) / kPdTile, waves = dm.d == 64 ? kFewWaves<64> : kFewWaves<128>;
  const long long blocks = (long long)dm.b * dm.n_kv;
  if (blocks > 768) return false;
  const int rounds = blocks > 256 || blocks < 96 ? (dm.d == 64 ? 3 : 2) : blocks < 128 ? 4 : 8;
  return tiles <= rounds * waves;
}

hipError_t launch_cross_few(const Dims& dm, bool fp8, const PagedArgs& a, hipStream_t st) {
  auto launch = [&](auto d, auto eight_bit) -> hipError_t {
    constexpr int D = decltype(d)::value, WAVES = kFewWaves<D>;
    constexpr bool FP8 = decltype(eight_bit)::value;
    constexpr size_t lds = PdTile<D, FP8, WAVES>::kLdsBytes;
    static_assert(lds <= 160 * 1024, "the LDS of a compute unit");
    static std::atomic<uint64_t> lds_done{0};
    const hipError_t e = ensure_dynamic_lds(reinterpret_cast<const void*>(&cross_few<D, FP8, WAVES>), lds, lds_done);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((cross_few<D, FP8, WAVES>), dim3(dm.b, dm.n_kv), dim3(64 * WAVES), lds, st, dm, a);
    return hipGetLastError();
  };
  using d64 = std::integral_constant<int, 64>;
  using d128 = std::integral_constant<int, 128>;
  if (dm.d == 64) return fp8 ? launch(d64{}, std::true_type{}) : launch(d64{}, std::false_type{});
  return fp8 ? launch(d128{}, std::true_type{}) : launch(d128{}, std::false_type{});
}

}  // namespace quoka
