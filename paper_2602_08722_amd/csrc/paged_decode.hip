// Attention of single tokens and a few over a cache in pages, bfloat16 (quoka_paged_attn with at most 32 query rows per KV head): as in
// attn_decode.hip the rows of a KV head are one block of 32 for the matrix instructions, the key list is split over blocks, and a second
// launch merges their partials (m, l, O); only the summation is regrouped.
//
// Rows: row r = c * g + j is chunk token c of q-head kv * g + j.  Keys: slot n of a list is its entry (whole sequences: position n), from
// the list's length on the chunk's own tokens; token c sees slot n iff n <= length + c.
//
// Bound by memory: every row of K and V is used once, by one wave, which works by itself on 32 slots at a time.  A load takes 16
// bytes a lane and whole rows by LPR neighbouring lanes (16, 8 or 4 of them); such a group fetches NLD neighbouring slots, one a load, so
// each of its lanes looks up one slot's row and hands it to the others by a cross-lane move.  Rows are fetched one tile ahead, pages two,
// entries three; 8-bit rows are widened on their way to LDS.
// Measured: one token for 32 sequences of 1024 - 32768, 8-bit rows of 8 heads of 128 (1.15 GB), 204 us (5.6 TB/s); for 8 of 4096 - 65536,
// 16-bit rows (1.32 GB), 231 (5.7 TB/s).  One sequence of 8192 in 8 bits 12.8: 7 until the last partial has left (1.6 arguments and length,
// 0.5 pages, 1 the first rows, then one or two tiles and the merge of the block's waves), the rest the second launch.
// Over states (quoka_cross_attn; the chunk's own rows are not among the keys): the 32 above 196 us (1.09 GB, 5.6 TB/s).
//
// The tiles of all sequences lie one behind the other, and every block of a KV head takes as many of them: the end of one
// sequence, whole ones, the beginning of another, or, where that costs nothing, a part of one (PdPlan).  A part of a sequence leaves a
// partial.  (With an equal number of blocks for each sequence the 32 above took 262 us.)
#include "decode_tile.hip.h"

namespace quoka {

constexpr int kPdWaves = 4;
constexpr int kPdThreads = 64 * kPdWaves;
constexpr int kPdMaxSlots = 512;   // blocks per KV head: two for every compute unit, which are resident together
constexpr int kPdFew = 16;         // partials of a sequence that one thread adds up

template <int D, bool FP8>
using PdCfg = PdTile<D, FP8, kPdWaves>;

struct PdSeq {
  int n_list, n_before, C;   // entries (cached tokens) attended, cached tokens, chunk tokens
};
// `sparse`: whether there are lists.
__device__ __forceinline__ PdSeq pd_seq(const Dims& dm, const PagedArgs& a, int b, int kv, bool sparse) {
  PdSeq s;
  s.C = a.chunk_lens == nullptr ? dm.C : max(min(a.chunk_lens[b], dm.C), 0);
  s.n_before = min(max(a.kv_lens[b], 0), dm.T_max);
  s.n_list = !sparse ? s.n_before : max(min(a.k_cnt[b * dm.n_kv + kv], dm.B_max), 0);
  return s;
}

// 64 sequences from b0 on, one a lane, and their tiles (a sequence without a token in this chunk has none).
template <bool OWN>
struct PdLine {
  PdSeq seq;
  uint32_t end;   // and where their room in the line of tiles ends (pd_place)
  int b0;
  __device__ __forceinline__ uint32_t tiles() const {
    return seq.C > 0 ? (uint32_t)(seq.n_list + (OWN ? seq.C : 0) + kPdTile - 1) / kPdTile : 0u;
  }
};
template <bool OWN>
__device__ __forceinline__ PdLine<OWN> pd_line(const Dims& dm, const PagedArgs& a, int kv, int b0, bool sparse) {
  PdLine<OWN> line;
  line.b0 = b0;
  const int b = b0 + (threadIdx.x & 63);
  line.seq = dm.b == 1 ? pd_seq(dm, a, 0, kv, sparse) : pd_seq(dm, a, min(b, dm.b - 1), kv, sparse);   // (one sequence: scalar fetches)
  if (b >= dm.b) line.seq.C = 0;
  return line;
}
__device__ __forceinline__ uint32_t last_lane(uint32_t x) { return (uint32_t)__builtin_amdgcn_readlane((int)x, 63); }
// (both below 2^23: the float quotient's integer part is the quotient's)
__device__ __forceinline__ uint32_t blocks_of(uint32_t tiles, uint32_t quota) { return (uint32_t)((float)(tiles + quota - 1) / (float)quota); }

// Tiles of a block, `quota`, and how many the line has.  All tiles over the blocks, at least one for each wave; or, where that takes no wave
// another tile, a whole number of blocks for each sequence, since a block's second part is another chain of fetches (one token, 8-bit rows, us:
// 16 sequences of 60 keys, 16/4 heads of 128 12.4 -> 10.9, 16 of 1100, 32/8 heads 17.5 -> 16.5, 8 of 3000 19.1 -> 18.4; with another tile a
// wave 32 of 200 - 2000 31.6 -> 32.7).
struct PdPlan {
  uint32_t quota, total;
  bool whole;
};
template <bool OWN>
__device__ __forceinline__ PdPlan pd_plan(const Dims& dm, const PagedArgs& a, int kv, const PdLine<OWN>& start, int n_slots, bool sparse) {   // start: b0 = 0
  uint32_t total = dm.b == 1 ? (uint32_t)__builtin_amdgcn_readfirstlane((int)start.tiles()) : last_lane(wave_incl_scan_u32(start.tiles()));
  for (int b0 = kWave; b0 < dm.b; b0 += kWave) total += last_lane(wave_incl_scan_u32(pd_line<OWN>(dm, a, kv, b0, sparse).tiles()));
  const uint32_t even = max((total + (uint32_t)n_slots - 1) / (uint32_t)n_slots, 1u);
  if (dm.b > 1 && dm.b <= kWave && 2 * dm.b <= n_slots) {   // (with more sequences it is rarely so, and the question costs 2 - 3 %)
    const uint32_t quota = (even + kPdWaves - 1) / kPdWaves * kPdWaves, blocks = last_lane(wave_incl_scan_u32(blocks_of(start.tiles(), quota)));
    if (blocks <= (uint32_t)n_slots) return {quota, blocks * quota, true};
  }
  return {max(even, (uint32_t)kPdWaves), total, false};
}
// The room that a sequence's tiles take.
__device__ __forceinline__ uint32_t pd_room(const PdPlan& plan, uint32_t tiles) {
  return plan.whole ? blocks_of(tiles, plan.quota) * plan.quota : tiles;
}
template <bool OWN>
__device__ __forceinline__ void pd_place(const Dims& dm, const PdPlan& plan, PdLine<OWN>& line, uint32_t before) {
  const uint32_t room = pd_room(plan, line.tiles());
  line.end = before + (dm.b == 1 ? (uint32_t)__builtin_amdgcn_readfirstlane((int)room) : wave_incl_scan_u32(room));
}

// part: [n_kv, n_slots + batch, kRec] float32.  The partial of sequence b from block s is s + b: along the line of tiles either grows with every
// part of a sequence.  parts: [n_kv, batch], the block of a sequence's first part and how many there are, for the merge.
// OWN: the chunk's own rows come behind the list, and token c sees those up to its own; otherwise every token sees the list and no more.
template <int D, bool FP8, bool LIST, bool OWN>
__global__ __launch_bounds__(kPdThreads, 2) void paged_decode(Dims dm, PagedArgs a, float* __restrict__ part, u32x2* __restrict__ parts,
                                                              int n_slots) {
  using Cfg = PdCfg<D, FP8>;
  constexpr int KS = Cfg::KS, DB = Cfg::DB, LPR = Cfg::LPR, NLD = Cfg::NLD, LD = Cfg::LD, LDV = Cfg::LDV, LDO = Cfg::LDO;
  extern __shared__ __align__(16) unsigned char smem[];
  const Pages& pg = a.pg;
  const int kv = blockIdx.y;
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int li = lane & 31, hf = lane >> 5;
  const int g = dm.g;
  PdLine<OWN> line = pd_line<OWN>(dm, a, kv, 0, LIST);
  const PdPlan plan = pd_plan(dm, a, kv, line, n_slots, LIST);
  pd_place(dm, plan, line, 0u);
  uint32_t at = blockIdx.x * plan.quota;   // (blocks x quota < total + a block's share: 32 bits)
  const uint32_t at_end = min(at + plan.quota, plan.total);
  while (at < at_end) {   // block-uniform: the sequences that the block has a part of
    unsigned long long hit;
    while ((hit = __builtin_amdgcn_ballot_w64(at < line.end)) == 0) {   // (at < total: some sequence has it)
      const uint32_t before = last_lane(line.end);
      line = pd_line<OWN>(dm, a, kv, line.b0 + kWave, LIST);
      pd_place(dm, {0u, 0u, false}, line, before);   // (more than 64 sequences: not by whole blocks)
    }
    const int of = (int)__builtin_ctzll(hit), b = line.b0 + of;
    PdSeq seq;
    seq.n_list = __builtin_amdgcn_readlane(line.seq.n_list, of);
    seq.n_before = __builtin_amdgcn_readlane(line.seq.n_before, of);
    seq.C = __builtin_amdgcn_readlane(line.seq.C, of);
    const uint32_t first = (uint32_t)__builtin_amdgcn_readlane((int)(line.end - pd_room(plan, line.tiles())), of),
                   end = first + (uint32_t)__builtin_amdgcn_readlane((int)line.tiles(), of);
    const int n_list = seq.n_list, n_keys = n_list + (OWN ? seq.C : 0), n_rows = seq.C * g;   // n_rows <= 32, checked by the launcher
    const int t_end = (int)(min(at_end, end) - first);
    if (at == first && tid == 0) parts[kv * dm.b + b] = u32x2{blockIdx.x, (end - 1) / plan.quota - blockIdx.x + 1};
    int t = (int)(at - first) + w;   // this wave's tiles: every fourth
    at = plan.whole ? at_end : first + t_end;

    const int32_t* table = pg.table + (size_t)b * pg.max_pages;
    const int32_t* list = LIST ? a.k_idx + (size_t)(b * dm.n_kv + kv) * dm.B_max : nullptr;
    constexpr int es = FP8 ? 1 : 2;
    const int c = lane % LPR, group = lane / LPR;   // 16 bytes of a row
    const uint64_t k_pool = reinterpret_cast<uint64_t>(pg.k) + (uint64_t)kv * pg.st[1] * es;
    const uint64_t v_pool = reinterpret_cast<uint64_t>(pg.v) + (uint64_t)kv * pg.st[1] * es;
    const uint8_t* k_scales = pg.k_scale + ((size_t)kv << pg.shift);
    const uint8_t* v_scales = pg.v_scale + ((size_t)kv << pg.shift);
    const uint32_t page_units = (uint32_t)(pg.st[0] / (16 / es)), slot_units = (uint32_t)(pg.st[2] / (16 / es)), page_scales = (uint32_t)pg.n_kv << pg.shift;
    const int row0 = Cfg::first_row(group), my_slot = row0 + lane % NLD;   // the group's rows; the one that this lane looks up
    auto slot_of_tile = [&](int tt) __attribute__((always_inline)) { return min(tt * kPdTile + my_slot, n_keys - 1); };   // (tail slots repeat a real one)

    uint32_t entry = 0;          // of the tile after the one whose page is looked up
    uint32_t pos = 0, page = 0;  // of the tile whose rows are fetched next
    auto look_up_entry = [&](int tt) __attribute__((always_inline)) {
      if constexpr (LIST) entry = (uint32_t)list[max(min(slot_of_tile(tt), n_list - 1), 0)];
    };
    auto look_up_page = [&](int tt) __attribute__((always_inline)) {
      const int n = slot_of_tile(tt);
      if constexpr (LIST) pos = n < n_list ? min(entry, (uint32_t)max(dm.T_max - 1, 0)) : (uint32_t)(seq.n_before + n - n_list);
      else pos = (uint32_t)n;
      page = (uint32_t)table[min((int)(pos >> pg.shift), pg.max_pages - 1)];
    };
    struct Rows {
      u32x4 k[NLD], v[NLD];
      uint32_t k_ex, v_ex;   // exponents of the slot that this lane looked up
    };
    // Requests the rows whose pages have been looked up last, and looks up the pages of tile tt and the entries of the one after it: ahead
    // of the rows, since fetches arrive in order and the next call waits for the pages.
    auto issue = [&](Rows& r, int tt) __attribute__((always_inline)) {
      const uint32_t at_page = min(page, (uint32_t)(pg.n_pages - 1)), slot = pos & ((1u << pg.shift) - 1u);
      const uint32_t off = at_page * page_units + slot * slot_units;
      look_up_page(tt);
      look_up_entry(tt + kPdWaves);
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
    if (t < t_end) {
      look_up_entry(t);
      look_up_page(t);
      look_up_entry(t + kPdWaves);
      issue(rows, t + kPdWaves);
    }

    // Q operand: row li -> (token li / g, head li % g); padding rows repeat row 0 and are never stored
    const int row = li < n_rows ? li : 0;
    const int tok = row / g, hj = row % g;
    bf16x8 qreg[KS];
    {
      const uint16_t* qrow = static_cast<const uint16_t*>(a.q) + b * dm.qs[0] + (size_t)(kv * g + hj) * dm.qs[1] +
                             (size_t)tok * dm.qs[2] + (FP8 ? 16 : 8) * hf;
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
    const float sl2 = 1.4426950408889634f / sqrtf((float)D);   // the softmax scale and the change to base 2
    for (; t < t_end; t += kPdWaves) {
      to_lds(rows);   // (this wave's own piece of LDS: its accesses stay in order, no barrier)
      __builtin_amdgcn_wave_barrier();
      if (t + kPdWaves < t_end) issue(rows, t + 2 * kPdWaves);
      const int slot0 = t * kPdTile;
      // ---- S^T = K Q^T ----
      f32x16 s;
#pragma unroll
      for (int v = 0; v < 16; ++v) s[v] = 0.f;
      const uint16_t* kp = kt + li * LD + 8 * hf;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8*>(kp + ks * 16), qreg[ks], s, 0, 0, 0);
      if (slot0 + kPdTile > n_list) {   // wave-uniform: the tile touches the chunk's rows or the end
        const int limit = n_list + (OWN ? tok + 1 : 0) - slot0;   // keys kk < limit of the tile are visible
#pragma unroll
        for (int v = 0; v < 16; ++v)
          if (8 * (v / 4) + 4 * hf + v % 4 >= limit) s[v] = -INFINITY;
      }
      // ---- online softmax ----
      float mx = -INFINITY;
#pragma unroll
      for (int v = 0; v < 16; ++v) mx = fmaxf(mx, s[v]);
      mx = fmaxf(mx, other_half(mx)) * sl2;
      // the reference point only moves when the tile's maximum exceeds it by more than 2^8
      constexpr float kLazy = 8.0f;
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

    // ---- the four waves' partials of the real rows are merged through LDS, then the block's partial goes out ----
    const float l_wave = l_run + other_half(l_run);
    __syncthreads();   // the waves' pieces may be reused
    float* mo = reinterpret_cast<float*>(smem);      // [4 waves][32 rows][LDO]
    float* mm = mo + kPdWaves * 32 * LDO;             // [4][32]
    float* ml = mm + kPdWaves * 32;
    float* mw = ml + kPdWaves * 32;
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
    float* my_part = part + ((size_t)kv * (n_slots + dm.b) + blockIdx.x + b) * Cfg::kRec;
    if (tid < kPdWaves * 32 && li < n_rows) {   // thread (wave tid / 32, row tid % 32 == li)
      float m = mm[li];
#pragma unroll
      for (int u = 1; u < kPdWaves; ++u) m = fmaxf(m, mm[u * 32 + li]);
      mw[tid] = mm[tid] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mm[tid] - m);
      if (tid < 32) my_part[32 * D + li] = m;
    }
    __syncthreads();
    if (tid < n_rows) {
      float l = 0.f;
#pragma unroll
      for (int u = 0; u < kPdWaves; ++u) l += mw[u * 32 + tid] * ml[u * 32 + tid];
      my_part[32 * D + 32 + tid] = l;
    }
    for (int i = tid; i < n_rows * (D / 4); i += kPdThreads) {
      const int r = i / (D / 4), c4 = i % (D / 4);
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int u = 0; u < kPdWaves; ++u) {
        const float wgt = mw[u * 32 + r];
        const float4 x = *reinterpret_cast<const float4*>(mo + ((size_t)u * 32 + r) * LDO + 4 * c4);
        acc.x += wgt * x.x;
        acc.y += wgt * x.y;
        acc.z += wgt * x.z;
        acc.w += wgt * x.w;
      }
      *reinterpret_cast<float4*>(my_part + r * D + 4 * c4) = acc;
    }
    __syncthreads();   // LDS is free for the next sequence
  }
}

// Tokens of sequence b's chunk that see any row (not OWN: none where nothing is cached, and then there are no partials).
template <bool OWN>
__device__ __forceinline__ int pd_live(const Dims& dm, const PagedArgs& a, int b) {
  const int C = a.chunk_lens == nullptr ? dm.C : max(min(a.chunk_lens[b], dm.C), 0);
  if constexpr (OWN) return C;
  return a.kv_lens[b] > 0 && dm.T_max > 0 ? C : 0;
}

// Many partials: a block merges row r of sequence b.  Threads weigh a partial each, or two; thread (four dims c4, group sg) adds up the outputs of
// every NG-th split, four of them on the way at a time, and the groups' sums meet in LDS, in a fixed order.
template <int D, bool OWN>
__device__ __forceinline__ void merge_row(const Dims& dm, const PagedArgs& a, const float* __restrict__ part, const u32x2* __restrict__ parts,
                                          int n_slots, int r, int kv, int b) {
  constexpr int TPR = D / 4, NG = kPdThreads / TPR, RUN = 4;
  static_assert(kPdMaxSlots <= 2 * kPdThreads, "two partials a thread");
  constexpr size_t REC = PdCfg<D, false>::kRec;
  __shared__ float wgt[2 * kPdThreads];
  __shared__ float4 red[NG][TPR];
  __shared__ float wm[kPdWaves], wl[kPdWaves];
  const int tid = threadIdx.x;
  const int C = pd_live<OWN>(dm, a, b);
  if (r >= C * dm.g) {   // block-uniform: a row past the sequence's chunk, or without a row to see
    const int tok = r / dm.g, h = kv * dm.g + r % dm.g;
    uint16_t* orow = static_cast<uint16_t*>(a.out) + b * dm.os[0] + h * dm.os[1] + (size_t)tok * dm.os[2];
    if (tid < TPR) *reinterpret_cast<u32x2*>(orow + 4 * tid) = u32x2{0u, 0u};
    if (tid == 0 && a.lse != nullptr) a.lse[(size_t)(b * dm.n_q + h) * dm.C + tok] = -INFINITY;
    return;
  }
  const int records = n_slots + dm.b;   // of a KV head
  int s_first = 0, n = 0;
  const int c4 = tid % TPR, sg = tid / TPR;
  float4 x[RUN];
  float m_s[2], l_s[2];
  const float* base = part + (size_t)kv * records * REC;
  // (a part past the sequence's last is some record of the KV head, and is not used)
  auto load = [&](int s0) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < RUN; ++u)
      x[u] = *reinterpret_cast<const float4*>(base + (size_t)min(s_first + b + s0 + u * NG, records - 1) * REC + r * D + 4 * c4);
  };
  auto load_weights = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const float* rec = base + (size_t)min(s_first + b + tid + u * kPdThreads, records - 1) * REC + 32 * D;
      m_s[u] = rec[r];
      l_s[u] = rec[32 + r];
    }
  };
  // the sequence's partials: n of them from s_first + b on
  if (dm.b > 1) s_first = (int)parts[kv * dm.b + b][0];   // (of one sequence they begin at the first: requested beside their number)
  load_weights();
  load(sg);
  __builtin_amdgcn_sched_barrier(0);
  n = (int)parts[kv * dm.b + b][1];
#pragma unroll
  for (int u = 0; u < 2; ++u)
    if (tid + u * kPdThreads >= n) {
      m_s[u] = -INFINITY;
      l_s[u] = 0.f;
    }
  const float m_wave = wave64_max(fmaxf(m_s[0], m_s[1]));
  if ((tid & 63) == 0) wm[tid >> 6] = m_wave;
  __syncthreads();
  float m = wm[0];
#pragma unroll
  for (int u = 1; u < kPdWaves; ++u) m = fmaxf(m, wm[u]);   // (every row sees its own key: finite)
  float l_mine = 0.f;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const float w = m_s[u] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_s[u] - m);
    wgt[tid + u * kPdThreads] = w;
    l_mine += w * l_s[u];
  }
  const float l_wave = wave64_sum(l_mine);
  if ((tid & 63) == 0) wl[tid >> 6] = l_wave;
  __syncthreads();
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int s0 = sg; s0 < n; s0 += RUN * NG) {
    float4 y[RUN];
#pragma unroll
    for (int u = 0; u < RUN; ++u) y[u] = x[u];
    if (s0 + RUN * NG < n) load(s0 + RUN * NG);
#pragma unroll
    for (int u = 0; u < RUN; ++u) {
      if (s0 + u * NG < n) {
        const float k = wgt[s0 + u * NG];
        acc.x += k * y[u].x;
        acc.y += k * y[u].y;
        acc.z += k * y[u].z;
        acc.w += k * y[u].w;
      }
    }
  }
  red[sg][c4] = acc;
  __syncthreads();
  if (tid < TPR) {
    float l = wl[0];
#pragma unroll
    for (int u = 1; u < kPdWaves; ++u) l += wl[u];
    float4 sum = red[0][tid];
#pragma unroll
    for (int u = 1; u < NG; ++u) {
      sum.x += red[u][tid].x;
      sum.y += red[u][tid].y;
      sum.z += red[u][tid].z;
      sum.w += red[u][tid].w;
    }
    const int tok = r / dm.g, h = kv * dm.g + r % dm.g;
    uint16_t* orow = static_cast<uint16_t*>(a.out) + b * dm.os[0] + h * dm.os[1] + (size_t)tok * dm.os[2];
    const bf16x2 lo = {(__bf16)(sum.x / l), (__bf16)(sum.y / l)}, hi = {(__bf16)(sum.z / l), (__bf16)(sum.w / l)};
    *reinterpret_cast<u32x2*>(orow + 4 * tid) = u32x2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
    if (tid == 0 && a.lse != nullptr) a.lse[(size_t)(b * dm.n_q + h) * dm.C + tok] = (m + log2f(l)) * 0.6931471805599453f;
  }
}

// The sequence of a KV head that is number `rank` of those with more than kPdFew partials, or -1.  Every wave finds it for itself, 256
// sequences at a time.
template <bool OWN>
__device__ __forceinline__ int long_sequence(const Dims& dm, const PagedArgs& a, const u32x2* __restrict__ parts, int kv, int rank) {
  constexpr int RUN = 4;
  const int lane = threadIdx.x & 63;
  for (int b0 = 0; b0 < dm.b; b0 += RUN * kWave) {
    bool is_long[RUN];
#pragma unroll
    for (int u = 0; u < RUN; ++u) {
      const int b = b0 + u * kWave + lane, at = min(b, dm.b - 1);
      const int C = OWN ? a.chunk_lens == nullptr ? dm.C : a.chunk_lens[at] : pd_live<OWN>(dm, a, at);   // (without a token the parts are not this call's)
      is_long[u] = b < dm.b && C > 0 && (int)parts[kv * dm.b + at][1] > kPdFew;
    }
#pragma unroll
    for (int u = 0; u < RUN; ++u) {
      unsigned long long hits = __builtin_amdgcn_ballot_w64(is_long[u]);
      const int n = (int)__builtin_popcountll(hits);
      if (rank < n) {
        for (; rank > 0; --rank) hits &= hits - 1;
        return b0 + u * kWave + (int)__builtin_ctzll(hits);
      }
      rank -= n;
    }
  }
  return -1;
}

// Many partials a sequence: one block per (row, KV head, sequence).
template <int D, bool OWN>
__global__ __launch_bounds__(kPdThreads) void paged_decode_merge(Dims dm, PagedArgs a, const float* __restrict__ part,
                                                               const u32x2* __restrict__ parts, int n_slots) {
  merge_row<D, OWN>(dm, a, part, parts, n_slots, blockIdx.x, blockIdx.y, blockIdx.z);
}

// Few partials a sequence: a thread adds up four dims of a row over all of them, eight on the way at a time, and D / 4 threads are a row, so that
// a block has eight rows (d 64: 16), which counts in large batches.  The two launches, the other's time first, us: 128 sequences of 500 keys,
// 32/8 heads of 128 8.8 and 4.1, 32/4 of 64 10.6 and 3.6; 32 of 500 4.0 and 3.9, 5.0 and 3.7; one of 500 (five partials) 3.6 and 3.4, of
// 2000 (16) 3.8 and 4.8; batches of 2 - 8 of 2000 (9 - 16) 3.7 - 4.2 and 4.0 - 4.8.
// Few on the mean, that is: a sequence far longer than the others has nearly all blocks' partials.  Those of more than kPdFew are left to the
// launch's first `n_long` layers, where a block is a row as above (one sequence of 100000 keys among 73 of 100, whole calls, 16/1 heads of 128
// 70.9 -> 24.9 us, 16/2 49.0 -> 26.8, 32/4 of 64 41.8 -> 29.4, 32/8 68.8 -> 63.8; 32 - 128 of 500 the same within 1 %, and so with kPdFew 8 or 32).
template <int D, bool OWN>
__global__ __launch_bounds__(kPdThreads) void paged_decode_merge_few(Dims dm, PagedArgs a, const float* __restrict__ part,
                                                                   const u32x2* __restrict__ parts, int n_slots, int n_long) {
  constexpr int TPR = D / 4, RUN = 8;
  constexpr size_t REC = PdCfg<D, false>::kRec;
  const int kv = blockIdx.y, rows = dm.C * dm.g;
  if ((int)blockIdx.z < n_long) {
    const int unit = (int)blockIdx.z * (int)gridDim.x + (int)blockIdx.x, rank = unit / rows;
    const int b = long_sequence<OWN>(dm, a, parts, kv, rank);
    if (b >= 0) merge_row<D, OWN>(dm, a, part, parts, n_slots, unit - rank * rows, kv, b);   // block-uniform
    return;
  }
  const int r = (int)blockIdx.x * (kPdThreads / TPR) + (int)threadIdx.x / TPR, c4 = threadIdx.x % TPR, b = (int)blockIdx.z - n_long;
  if (r >= rows) return;
  const int C = pd_live<OWN>(dm, a, b);
  const u32x2 of = parts[kv * dm.b + b];   // (a sequence without a token in this chunk has none, and uses none)
  if (n_long > 0 && C > 0 && (int)of[1] > kPdFew) return;
  const int tok = r / dm.g, h = kv * dm.g + r % dm.g;
  uint16_t* orow = static_cast<uint16_t*>(a.out) + b * dm.os[0] + h * dm.os[1] + (size_t)tok * dm.os[2];
  float* lse = a.lse != nullptr && c4 == 0 ? a.lse + (size_t)(b * dm.n_q + h) * dm.C + tok : nullptr;
  if (tok >= C) {   // a row past the sequence's chunk
    *reinterpret_cast<u32x2*>(orow + 4 * c4) = u32x2{0u, 0u};
    if (lse != nullptr) *lse = -INFINITY;
    return;
  }
  const int n = (int)of[1];
  const float* rec = part + ((size_t)kv * (n_slots + dm.b) + of[0] + b) * REC;
  float m = -INFINITY, l = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int s0 = 0; s0 < n; s0 += RUN) {
    float ms[RUN], ls[RUN];
    float4 x[RUN];
#pragma unroll
    for (int u = 0; u < RUN; ++u) {
      const float* p = rec + (size_t)min(s0 + u, n - 1) * REC;
      ms[u] = p[32 * D + r];
      ls[u] = p[32 * D + 32 + r];
      x[u] = *reinterpret_cast<const float4*>(p + r * D + 4 * c4);
    }
    float m_new = m;
#pragma unroll
    for (int u = 0; u < RUN; ++u) m_new = fmaxf(m_new, s0 + u < n ? ms[u] : -INFINITY);
    const float m_fin = m_new == -INFINITY ? 0.f : m_new, old = __builtin_amdgcn_exp2f(m - m_fin);
    m = m_new;
    l *= old;
    acc.x *= old;
    acc.y *= old;
    acc.z *= old;
    acc.w *= old;
#pragma unroll
    for (int u = 0; u < RUN; ++u) {
      if (s0 + u < n) {
        const float w = __builtin_amdgcn_exp2f(ms[u] - m_fin);
        l += w * ls[u];
        acc.x += w * x[u].x;
        acc.y += w * x[u].y;
        acc.z += w * x[u].z;
        acc.w += w * x[u].w;
      }
    }
  }
  const bf16x2 lo = {(__bf16)(acc.x / l), (__bf16)(acc.y / l)}, hi = {(__bf16)(acc.z / l), (__bf16)(acc.w / l)};
  *reinterpret_cast<u32x2*>(orow + 4 * c4) = u32x2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
  if (lse != nullptr) *lse = (m + log2f(l)) * 0.6931471805599453f;
}

// ---------------------------------------------------------------------------------------------
static int pd_slots(const Dims& dm) { return (kPdMaxSlots + dm.n_kv - 1) / dm.n_kv; }

// Cross attention: no more than that are resident (12 x 1 heads, 43 and 42 blocks a head: 44 sequences of 3000 states, d 64, 0.86 of the time,
// d 128 0.87, 86 of 6000 0.85; one sequence the same).
static int pd_state_slots(const Dims& dm) { return dm.n_kv < kPdMaxSlots ? kPdMaxSlots / dm.n_kv : 1; }
static size_t pd_part_floats(const Dims& dm) { return (size_t)dm.n_kv * (pd_slots(dm) + dm.b) * 32 * (dm.d + 2); }
size_t paged_decode_ws_floats(const Dims& dm) { return pd_part_floats(dm) + (size_t)2 * dm.n_kv * dm.b; }

hipError_t launch_paged_decode(const Dims& dm, bool fp8, const PagedArgs& a, float* part, hipStream_t st, bool own) {
  const int n_slots = own ? pd_slots(dm) : pd_state_slots(dm);
  u32x2* parts = reinterpret_cast<u32x2*>(part + pd_part_floats(dm));
  const long long tiles = ((long long)attended_cap(dm, a.k_idx != nullptr) + (own ? dm.C : 0) + kPdTile - 1) / kPdTile;
  if (dm.b * tiles >= 1ll << 31) return hipErrorInvalidValue;   // (refused by the entry point)
  const long long most = dm.b * ((tiles + kPdWaves - 1) / kPdWaves);   // (blocks that short lists leave without work)
  auto launch = [&](auto d, auto eight_bit, auto is_list, auto own_rows) -> hipError_t {
    constexpr int D = decltype(d)::value;
    constexpr bool FP8 = decltype(eight_bit)::value, LIST = decltype(is_list)::value, OWN = decltype(own_rows)::value;
    constexpr size_t lds = PdCfg<D, FP8>::kLdsBytes;
    static std::atomic<uint64_t> lds_done{0};
    const hipError_t e = ensure_dynamic_lds(reinterpret_cast<const void*>(&paged_decode<D, FP8, LIST, OWN>), lds, lds_done);
    if (e != hipSuccess) return e;
    if (most > 0)   // (states of no length at all leave the merge alone, which writes the rows that see nothing)
      hipLaunchKernelGGL((paged_decode<D, FP8, LIST, OWN>), dim3(n_slots < most ? n_slots : (int)most, dm.n_kv), dim3(kPdThreads), lds, st,
                         dm, a, part, parts, n_slots);
    const int rows = dm.C * dm.g, of_block = kPdThreads / (D / 4);
    // partials of a sequence: at most those of the longest list there can be; on the mean one more than its share of the blocks
    const long long of_list = (tiles + kPdWaves - 1) / kPdWaves, of_batch = n_slots / dm.b + 1;
    if ((of_list < of_batch ? of_list : of_batch) <= 8) {
      // Sequences of more than kPdFew: each has kPdFew - 1 blocks or more of the n_slots to itself.  (A list's tiles may lie in one block more than
      // they fill.)
      const int blocks = (rows + of_block - 1) / of_block, most_long = of_list < kPdFew || n_slots <= kPdFew ? 0 : n_slots / (kPdFew - 1);
      int n_long = ((most_long < dm.b ? most_long : dm.b) * rows + blocks - 1) / blocks;
      if (n_long + dm.b > 65535) n_long = 0;   // (layers of a grid)
      hipLaunchKernelGGL((paged_decode_merge_few<D, OWN>), dim3(blocks, dm.n_kv, n_long + dm.b), dim3(kPdThreads), 0, st, dm, a, part, parts,
                         n_slots, n_long);
    } else {
      hipLaunchKernelGGL((paged_decode_merge<D, OWN>), dim3(rows, dm.n_kv, dm.b), dim3(kPdThreads), 0, st, dm, a, part, parts, n_slots);
    }
    return hipGetLastError();
  };
  using std::false_type;
  using std::true_type;
  using d64 = std::integral_constant<int, 64>;
  using d128 = std::integral_constant<int, 128>;
  auto with_list = [&](auto d, auto eight_bit) {
    if (!own) return launch(d, eight_bit, false_type{}, false_type{});   // (cross attention takes no lists)
    return a.k_idx != nullptr ? launch(d, eight_bit, true_type{}, true_type{}) : launch(d, eight_bit, false_type{}, true_type{});
  };
  if (dm.d == 64) return fp8 ? with_list(d64{}, true_type{}) : with_list(d64{}, false_type{});
  return fp8 ? with_list(d128{}, true_type{}) : with_list(d128{}, false_type{});
}

}  // namespace quoka
