// Attention over a prefix that the whole batch shares.
//
// Every query row (sequence b, head h, token t) attends to the first prefix_len[b] rows of one
// K/V block Kp, Vp [Hkv][P][d] and to keys of its own (the sequence's cache, or the kept tokens of
// its own row).  The two sets are disjoint, so the softmax over both is joined from partial
// results: with reference exponents m_i, sums l_i and unnormalised values a_i,
//   O = sum a_i 2^(m_i-M) / sum l_i 2^(m_i-M),  M = max m_i.
// This file has the prefix part: the rows of all sequences, tokens and heads that read one kv head
// are the rows of one matrix product, 128 to a tile, so the prefix is read once per 256 rows instead
// of once per sequence.
//
// What bounds it: 4 d operations per (row, key) on the tensor pipe and one exponential, which take
// 2048 and 2087 cycles for the 2 x 128 rows and 128 keys of a step at d = 128.  Measured: 3400 cycles
// a step, 55 to 62 % of the tensor pipe while a CTA runs (168 GFLOP of 8192 rows x 40 000 keys in
// 157 us on all SMs); what is left is the chain of a slot's softmax (maximum 400, exponentials 1500,
// P to shared memory and its fence 550 cycles), not a saturated unit.  A run has about 8 us of its own
// (start 3 us, the drain and output of a segment 2 to 6 us).  Why equal runs: with whole units to a
// CTA, 256 units on 148 SMs took 325 us, in equal runs 274 (and 248 with P in shared memory and the
// turns at the exponentials).
#include <algorithm>
#include <cmath>

#include "attn_common.cuh"
#include "prefix_sync.h"

namespace sepllm {

namespace {

constexpr int kPfxThreads = 384;
constexpr int kMaxPairs = 128;    // pairs of row tiles per launch (their lengths sit in shared memory)

template <int D>
struct PfxCfg {
  static constexpr int NB = D / 64;               // 64-column blocks per row
  static constexpr int NST = (D == 128) ? 3 : 7;  // ring of K and V tiles
  static constexpr uint32_t kTile = NB * kTileBlockBytes;
  static constexpr uint32_t kPTile = 2 * kTileBlockBytes;   // 128 rows x 128 keys
  static constexpr uint32_t kQ = 0;                         // 2 slots
  static constexpr uint32_t kP = kQ + 2 * kTile;            // 2 slots
  static constexpr uint32_t kKV = kP + 2 * kPTile;
  static constexpr uint32_t kTab = kKV + NST * kTile;
  static constexpr uint32_t kBar = kTab + kMaxPairs * 8;
  static constexpr uint32_t kTotal = kBar + 1024;
  static constexpr uint32_t kRequest = kTotal + 1024;
  static constexpr uint32_t kS0 = 0, kS1 = 128, kO0 = 256, kO1 = 256 + D;  // tensor-memory columns
};
static_assert(PfxCfg<128>::kRequest <= 227 * 1024 && PfxCfg<64>::kRequest <= 227 * 1024 &&
                  PfxCfg<64>::kRequest > 114 * 1024,
              "one CTA per SM owns all 512 tensor-memory columns");

// Row tile i holds rows (b, t, g) of one kv head: bt sequences x tt tokens x gt heads of the group,
// heads fastest.
struct RowTile {
  int b0, t0, g0;
};
__device__ __forceinline__ RowTile row_tile(const PrefixParams& p, int i) {
  RowTile r;
  r.g0 = (i % p.g_tiles) * p.gt;
  i /= p.g_tiles;
  r.t0 = (i % p.t_tiles) * p.tt;
  r.b0 = (i / p.t_tiles) * p.bt;
  return r;
}
// Longest prefix that sequence b's rows of a tile see; -1: the tile holds none of its tokens.
__device__ __forceinline__ int seen_length(const PrefixParams& p, int b, int t0) {
  if (b >= p.B || (p.seq_len && t0 >= p.seq_len[b])) return -1;
  return p.prefix_len ? max(0, min(p.P, p.prefix_len[b])) : p.P;
}
// Key tiles of a pair of row tiles whose longest prefixes are len[0] and len[1].  A pair that sees nothing of the
// prefix still takes one (wholly masked) tile: its rows have to be finished by someone.
__device__ __forceinline__ int pair_tiles(const int* len) {
  const int m = max(len[0], len[1]);
  return m < 0 ? 0 : max(1, (m + kBN - 1) / kBN);
}

// The row's own part in FwdParams::O32: four columns k at [k * 128].
template <int D>
__device__ __forceinline__ const float4* own_row(const PrefixParams& p, int b, int h, int t) {
  return reinterpret_cast<const float4*>(p.own_O) +
         ((size_t(b) * p.Hkv * p.G + h) * ((p.T + 127) / 128) + t / 128) * (D / 4) * 128 + t % 128;
}

// The work is the key tiles of every (kv head, pair) in that order, cut into equal runs, one per
// CTA: a CTA's run is a sequence of segments, each a range of key tiles of one (kv head, pair).
// Every warp walks the run by itself; its place sits in shared memory (a warp's copy each), so that
// nothing of it takes registers in the softmax loop.
struct Segment {
  int left;         // key tiles of the run behind this segment
  int hk, pair;
  int j0, j1, nt;   // key tiles [j0, j1) of nt
  int len[2];       // longest prefix of the row tile in slot x (-1: no rows)
};
// Advances to the next segment (false: none left).  WARP: called by all lanes of a warp, else by one
// thread.
template <bool WARP>
__device__ __forceinline__ bool next_segment(Segment* sg, const int* tab, int pairs) {
  const int left = sg->left;
  int hk = sg->hk, pair = sg->pair, off = sg->j1, nt;
  if (WARP) __syncwarp();
  if (left <= 0) return false;
  while ((nt = pair_tiles(tab + 2 * pair)) <= off) {   // finished
    off = 0;
    if (++pair == pairs) { pair = 0; ++hk; }
  }
  if (!WARP || (threadIdx.x & 31) == 0) {
    sg->hk = hk; sg->pair = pair; sg->j0 = off; sg->nt = nt;
    sg->j1 = min(nt, off + left);
    sg->left = left - (sg->j1 - off);
    sg->len[0] = tab[2 * pair];
    sg->len[1] = tab[2 * pair + 1];
  }
  if (WARP) __syncwarp();
  return true;
}
// Key tiles of the segment that slot x works on: in pair mode the first ones (as far as its longest
// prefix goes), in alternate mode those with j % 2 = x.
__device__ __forceinline__ int slot_tiles(const Segment* sg, bool alt, int x) {
  const int n = sg->j1 - sg->j0, len = sg->len[x];
  if (alt) return (n - x + 1) / 2;
  return len < 0 ? 0 : max(0, min(n, max(1, (len + kBN - 1) / kBN) - sg->j0));
}
// The segment's last tile holds the end of the longest prefix: V rows behind it may hold anything
// (rows behind P are zero already).
__device__ __forceinline__ bool ends_inside(const Segment* sg, int P) {
  const int m = max(sg->len[0], sg->len[1]);
  return m < P && sg->j1 * kBN > m;
}

// One CTA: two slots of 128 query rows, walked over the segments of its run.
//   pair mode        slot x holds the x-th row tile of a pair; both slots walk the same key tiles
//   alternate mode   (one row tile in all) both slots hold that tile and take the key tiles in turn,
//                    so that one slot's softmax runs under the other's loads and products; each
//                    slot leaves a partial result of its own
// Warps: 0 TMA; 1 and 2 MMA issue of slot 0 and 1; 3 clears V rows behind the prefix; 4-7 and 8-11
// softmax of slot 0 and 1, one thread per row.  P goes to shared memory as bf16: S is free as soon as
// it is in registers, so S of the slot's next key tile is issued at once and the softmax threads go
// from tile to tile without waiting for the tensor pipe.  K and V tiles share one ring in the order in
// which they are used: K0, K1, V0, K2, V1, ...
template <int D>
__global__ void __launch_bounds__(kPfxThreads, 1)
prefix_attn(const __grid_constant__ CUtensorMap mapQ, const __grid_constant__ CUtensorMap mapK,
            const __grid_constant__ CUtensorMap mapV, const PrefixParams p) {
  using C = PfxCfg<D>;
  constexpr int NB = C::NB, NST = C::NST;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~uintptr_t(1023));
  uint8_t* sQ = smem + C::kQ;
  uint8_t* sP = smem + C::kP;
  uint8_t* sKV = smem + C::kKV;
  int* tab = reinterpret_cast<int*>(smem + C::kTab);   // [2 * pairs] longest prefix of each row tile that
                                                       // has rows, two and two a pair
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::kBar);
  uint64_t* bar_q = bars;          // [2]   Q of slot x landed
  uint64_t* bar_qe = bars + 2;     // [2]   slot x has read the segment's Q for the last time
  uint64_t* bar_s = bars + 4;      // [2]   S_x complete
  uint64_t* bar_sl = bars + 6;     // [2]   S_x read into registers by the 4 softmax warps
  uint64_t* bar_p = bars + 8;      // [2]   P_x written
  uint64_t* bar_pv = bars + 10;    // [2]   P_x V complete: P_x may be rewritten, O_x is at rest
  uint64_t* bar_g = bars + 12;     // [2]   slot x asks for the rows of V behind the prefix to be cleared
  uint64_t* bar_z = bars + 14;     // [2]   they are, for slot x
  uint64_t* bar_d = bars + 16;     // [2]   every product and arrival of slot x done
  uint64_t* bar_f = bars + 18;     // [NST] ring stage full
  uint64_t* bar_r = bar_f + NST;   // [NST] ring stage free (both slots)
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 18 + 2 * NST);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 2);
  int* s_warp = reinterpret_cast<int*>(tmem_slot + 4);   // [12] key tiles per warp of the scan
  int* s_start = s_warp + 12;                            // [2] pair and offset where the run starts
  int* s_run = s_warp + 14;                              // end of the run, tiles per run, longer runs, pairs
  Segment* s_seg = reinterpret_cast<Segment*>(s_run + 4);    // [12] place of each warp in the run
  uint8_t* s_id = reinterpret_cast<uint8_t*>(s_seg + 12);    // [2 * pairs] number of those row tiles
  static_assert((18 + 2 * NST) * 8 + 16 + 18 * 4 + 12 * sizeof(Segment) + 2 * kMaxPairs <= C::kTotal - C::kBar,
                "barriers, places and tile numbers fit behind kBar");

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const bool alt = p.alternate != 0;
  const int rows = p.gt * p.tt * p.bt;

  if (p.reset_status) {   // a decode: its own part may share the GPU with this kernel
    let_dependents_start();
    if (blockIdx.x == 0 && tid == 0) *p.status = SEPLLM_OK;
  }
  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(bar_q + i, 1); mbar_init(bar_qe + i, 1); mbar_init(bar_s + i, 1);
      mbar_init(bar_sl + i, 4); mbar_init(bar_p + i, 4); mbar_init(bar_pv + i, 1);
      mbar_init(bar_g + i, 1); mbar_init(bar_z + i, 1); mbar_init(bar_d + i, 1);
    }
    for (int i = 0; i < NST; ++i) { mbar_init(bar_f + i, 1); mbar_init(bar_r + i, 2); }
    *abort_flag = 0;
    fence_mbar_init();
    tma_prefetch_desc(&mapQ); tma_prefetch_desc(&mapK); tma_prefetch_desc(&mapV);
  }
  if (warp == 0) {
    __syncwarp();
    tmem_alloc(tmem_slot, 512);
    tmem_relinquish();
  }
  // rows of a tile that no load fills are zero: their scores are finite and nothing of them is stored
  for (int i = tid; i < (128 - rows) * 8 * NB * 2; i += kPfxThreads) {
    const int ch = i & 7, blk = (i >> 3) % (2 * NB), r = rows + (i >> 3) / (2 * NB);
    *reinterpret_cast<uint4*>(sQ + blk * kTileBlockBytes + r * 128 + ch * 16) = make_uint4(0, 0, 0, 0);
  }
  fence_proxy_async_smem();

  // longest prefix of every row tile: a warp per tile with its lanes over the sequences, or, where a
  // tile has few of them (and there may be many tiles), a thread per tile
  const bool by_warp = p.bt > 8;
  for (int i = by_warp ? warp : tid; i < 2 * p.pairs; i += by_warp ? kPfxThreads / 32 : kPfxThreads) {
    int len = -1;
    const int ti = 2 * p.pair_base + i;
    if (ti < p.m_tiles) {
      const RowTile rt = row_tile(p, ti);
      for (int k = by_warp ? lane : 0; k < p.bt; k += by_warp ? 32 : 1)
        len = max(len, seen_length(p, rt.b0 + k, rt.t0));
    }
    if (by_warp) len = __reduce_max_sync(0xffffffffu, len);
    if (!by_warp || lane == 0) tab[i] = len;
  }
  __syncthreads();
  int n_pairs = p.pairs;
  {
    // tiles of padding drop out, so that every pair but the last has two tiles with rows
    const int len = tid < 2 * p.pairs ? tab[tid] : -1;
    const uint32_t with_rows = __ballot_sync(0xffffffffu, len >= 0);
    if (lane == 0) s_warp[warp] = __popc(with_rows);
    __syncthreads();
    int at = __popc(with_rows & ((1u << lane) - 1)), all = 0;
    for (int w = 0; w < kPfxThreads / 32; ++w) {
      if (w < warp) at += s_warp[w];
      all += s_warp[w];
    }
    n_pairs = (all + 1) / 2;
    if (len >= 0) { tab[at] = len; s_id[at] = uint8_t(tid); }
    if (tid == 0 && all % 2) tab[all] = -1;
    __syncthreads();
  }
  // where the run starts: key tiles of one kv head summed over the pairs
  static_assert(2 * kMaxPairs <= kPfxThreads && 2 * kMaxPairs <= 256, "a thread per row tile, its number in a byte");
  const int mine = tid < n_pairs ? pair_tiles(tab + 2 * tid) : 0;
  int incl = mine;
#pragma unroll
  for (int k = 1; k < 32; k <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, incl, k);
    if (lane >= k) incl += v;
  }
  if (lane == 31) s_warp[warp] = incl;
  __syncthreads();
  int before = incl - mine, per_head = 0;
  for (int w = 0; w < kPfxThreads / 32; ++w) {
    if (w < warp) before += s_warp[w];
    per_head += s_warp[w];
  }
  const int total = per_head * p.Hkv;
  // CTAs that get a run: none an empty one, in alternate mode one tile for each slot.  With one
  // pair in all and short runs, a whole number of runs per kv head: a run that straddles two heads
  // loads queries and leaves parts twice (costs about two tiles, saves less than one).
  int n_runs = min(int(gridDim.x), alt ? (total + 1) / 2 : total);
  if (p.pairs == 1 && n_runs >= p.Hkv && total < 16 * n_runs) n_runs -= n_runs % p.Hkv;
  // runs of `run` tiles, the first `longer` of them of one more
  const int blk = blockIdx.x, run = n_runs > 0 ? total / n_runs : 0, longer = total - run * n_runs;
  const int run0 = blk < n_runs ? blk * run + min(blk, longer) : 0;
  const int run1 = blk < n_runs ? run0 + run + (blk < longer) : 0;
  const int hk0 = per_head > 0 ? run0 / per_head : 0, in_head = run0 - hk0 * per_head;
  if (run0 < run1 && in_head >= before && in_head < before + mine) {
    s_start[0] = tid;
    s_start[1] = in_head - before;
  }
  if (tid == 0) { s_run[0] = run1; s_run[1] = run; s_run[2] = longer; s_run[3] = n_pairs; }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  Segment* sg = s_seg + warp;
  if (lane == 0) {
    sg->left = run1 - run0;
    sg->hk = hk0;
    sg->pair = s_start[0];
    sg->j1 = s_start[1];
  }
  __syncwarp();

  bool ok = true;
  auto wait = [&](uint64_t* bar, uint32_t parity) {
    if (!mbar_wait(bar, parity, abort_flag)) {
      if (ok) set_status(p.status, SEPLLM_TIMEOUT);
      ok = false;
    }
  };

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    // place of K(j) and V(j) of a segment of n key tiles in the order of the loads
    auto k_place = [](int j) { return j == 0 ? 0 : 2 * j - 1; };
    auto v_place = [](int j, int n) { return j < n - 1 ? 2 * j + 2 : 2 * n - 1; };
    if (warp == 0 && lane == 0) {
      // ---------------- TMA producer ----------------
      int at = 0;  // tiles loaded
      for (int n = 0; next_segment<false>(sg, tab, s_run[3]); ++n) {
        const int hk = sg->hk, j0 = sg->j0, n_tiles = sg->j1 - j0;
        for (int i = 0; i < 2 * n_tiles; ++i, ++at) {
          // 0: K(0), odd: K((i + 1) / 2), even: V(i / 2 - 1), and the last one V(n - 1)
          const bool is_v = i == 2 * n_tiles - 1 || (i > 0 && i % 2 == 0);
          const int j = is_v ? (i % 2 ? n_tiles - 1 : i / 2 - 1) : (i + 1) / 2;
          const int st = at % NST, use = at / NST;
          if (use > 0) wait(bar_r + st, (use - 1) & 1);
          mbar_expect_tx(bar_f + st, C::kTile);
          for (int nb = 0; nb < NB; ++nb)
            tma_load_3d(sKV + st * C::kTile + nb * kTileBlockBytes, is_v ? &mapV : &mapK, bar_f + st, nb * 64,
                        (j0 + j) * kBN, hk);
          if (i == 0) {
            if (n > 0) { wait(bar_qe, (n - 1) & 1); wait(bar_qe + 1, (n - 1) & 1); }
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              if (alt ? x == 1 : slot_tiles(sg, false, x) == 0) continue;   // a slot without work loads nothing
              const RowTile rt = row_tile(p, 2 * p.pair_base + s_id[2 * sg->pair + x]);
              mbar_expect_tx(bar_q + x, uint32_t(NB * rows) * 128u);
              for (int nb = 0; nb < NB; ++nb)
                tma_load_5d(sQ + x * C::kTile + nb * kTileBlockBytes, &mapQ, bar_q + x, nb * 64, rt.g0, rt.t0,
                            hk, rt.b0);
            }
          }
        }
      }
    } else if ((warp == 1 || warp == 2) && lane == 0) {
      // ---------------- MMA issuers: one thread per slot ----------------
      // A slot's products go in its own order: S(j+1) as soon as S(j) has been read, P V(j) as soon as
      // P(j) is written.  A stage of the ring is free when both slots are through with it; a slot that
      // does not use a tile lets it go as soon as it has landed.
      const int x = warp - 1, qx = alt ? 0 : x;
      constexpr uint32_t idesc_s = make_idesc_bf16(128, 128, 0, 0);
      constexpr uint32_t idesc_o = make_idesc_bf16(128, D, 0, 1);
      const uint32_t q_lo = desc_lo(smem_u32(sQ + qx * C::kTile), 16);
      const uint32_t p_lo = desc_lo(smem_u32(sP + x * C::kPTile), 16);
      const uint32_t k_lo0 = desc_lo(smem_u32(sKV), 16), v_lo0 = desc_lo(smem_u32(sKV), kTileBlockBytes);
      const uint32_t tS = tmem + (x ? C::kS1 : C::kS0), tO = tmem + (x ? C::kO1 : C::kO0);
      uint32_t ph_sl = 0, ph_p = 0, ph_q = 0, ph_z = 0;   // phases
      int at0 = 0;                                        // tiles loaded for earlier segments
      for (int n = 0; next_segment<false>(sg, tab, s_run[3]); ++n) {
        const int n_tiles = sg->j1 - sg->j0, n_mine = slot_tiles(sg, alt, x);
        const bool ask = ends_inside(sg, p.P) && uses_last(alt, x, n_tiles, n_mine);
        auto mine = [&](int j) { return alt ? (j & 1) == x : j < n_mine; };
        int left_s = n_mine;      // S products still to issue
        bool s_out = false;       // an S product has been issued in this segment
        auto scores = [&](int j) {
          const int at = at0 + k_place(j), st = at % NST;
          if (mine(j)) {
            if (!s_out) { wait(bar_q + qx, ph_q); ph_q ^= 1; }
            else { wait(bar_sl + x, ph_sl); ph_sl ^= 1; }
            s_out = true;
          }
          wait(bar_f + st, (at / NST) & 1);
          if (!mine(j)) { mbar_arrive(bar_r + st); return; }
          tc_fence_after();
          const uint32_t k_lo = k_lo0 + st * (C::kTile >> 4);
#pragma unroll
          for (int k = 0; k < D / 16; ++k)
            umma_ss_lo(tS, q_lo + kmajor_step(k, kTileBlockBytes), k_lo + kmajor_step(k, kTileBlockBytes),
                       idesc_s, k > 0);
          tc_commit(bar_s + x);
          tc_commit(bar_r + st);
          if (--left_s == 0) tc_commit(bar_qe + x);
        };
        bool o_begun = false;
        auto values = [&](int j) {
          const int at = at0 + v_place(j, n_tiles), st = at % NST;
          wait(bar_f + st, (at / NST) & 1);
          if (!mine(j)) { mbar_arrive(bar_r + st); return; }
          const bool cleared = ask && j == n_tiles - 1;
          if (cleared) mbar_arrive(bar_g + x);   // (the clearing runs under this tile's softmax)
          wait(bar_p + x, ph_p);
          ph_p ^= 1;
          if (cleared) { wait(bar_z + x, ph_z); ph_z ^= 1; }
          tc_fence_after();
          const uint32_t v_lo = v_lo0 + st * (C::kTile >> 4);
          umma_ss_lo(tO, p_lo, v_lo, idesc_o, o_begun);
          o_begun = true;
#pragma unroll
          for (int k = 1; k < kBN / 16; ++k)
            umma_ss_lo(tO, p_lo + kmajor_step(k, kTileBlockBytes), v_lo + mnmajor_step(k), idesc_o, 1);
          tc_commit(bar_r + st);
          tc_commit(bar_pv + x);
        };
        scores(0);
        for (int j = 0; j < n_tiles; ++j) {
          if (j + 1 < n_tiles) scores(j + 1);
          values(j);
        }
        if (n_mine > 0) {
          // the last S has no successor that waits for its reading: catch up with that phase
          wait(bar_sl + x, ph_sl);
          ph_sl ^= 1;
        } else {
          if (alt) { wait(bar_q, ph_q); ph_q ^= 1; }   // the other slot's load, for the same reason
          // (at the end, when the producer is past its wait for the segment before)
          mbar_arrive(bar_qe + x);
        }
        at0 += 2 * n_tiles;
      }
      // no arrival may be under way when the CTA ends
      tc_commit(bar_d + x);
      wait(bar_d + x, 0);
    } else if (warp == 3) {
      // ---------------- V rows behind the longest prefix ----------------
      int ph_g[2] = {0, 0}, at0 = 0;
      while (next_segment<true>(sg, tab, s_run[3])) {
        const int n_tiles = sg->j1 - sg->j0;
        const int st = (at0 + v_place(n_tiles - 1, n_tiles)) % NST;
        at0 += 2 * n_tiles;
        if (!ends_inside(sg, p.P)) continue;
        const int r0 = max(sg->len[0], sg->len[1]) - (sg->j1 - 1) * kBN;
        bool asks[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          asks[x] = uses_last(alt, x, n_tiles, slot_tiles(sg, alt, x));
          if (asks[x]) { wait(bar_g + x, ph_g[x]); ph_g[x] ^= 1; }
        }
        for (int i = lane; i < (kBN - r0) * 8 * NB; i += 32) {
          const int ch = i & 7, blk = (i >> 3) % NB, r = r0 + (i >> 3) / NB;
          *reinterpret_cast<uint4*>(sKV + st * C::kTile + blk * kTileBlockBytes + r * 128 + ch * 16) =
              make_uint4(0, 0, 0, 0);
        }
        fence_proxy_async_smem();
#pragma unroll
        for (int x = 0; x < 2; ++x)
          if (asks[x]) mbar_arrive_warp(bar_z + x);
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
    // ---------------- softmax of slot x ----------------
    const int x = (warp >= 8) ? 1 : 0;
    const int r = tid & 127;  // row in the tile = tensor-memory lane
    const uint32_t lane_base = uint32_t((warp & 3) * 32) << 16;
    const uint32_t tS = tmem + lane_base + (x ? C::kS1 : C::kS0);
    const uint32_t tO = tmem + lane_base + (x ? C::kO1 : C::kO0);
    uint8_t* sPx = sP + x * C::kPTile;
    int n_s = 0;              // S tiles taken
    int cut = -1;
    for (int n = 0; next_segment<true>(sg, tab, s_run[3]); ++n) {
      // the row: sequence b, token t, head g of the group
      auto place = [&](int& b, int& t, int& g) {
        if (!alt && sg->len[x] < 0) return false;
        const RowTile rt = row_tile(p, 2 * p.pair_base + s_id[2 * sg->pair + (alt ? 0 : x)]);
        b = rt.b0 + r / (p.gt * p.tt); t = rt.t0 + r / p.gt % p.tt; g = rt.g0 + r % p.gt;
        return r < rows && b < p.B && t < p.T && g < p.G && !(p.seq_len && t >= p.seq_len[b]);
      };
      const int n_mine = slot_tiles(sg, alt, x), n_both = min(n_mine, slot_tiles(sg, alt, x ^ 1));
      int c_hi = sg->len[alt ? 0 : x];   // keys of the next tile, and behind it, that the row sees
      {
        int b, t, g;
        if (place(b, t, g) && p.prefix_len) c_hi = max(0, min(p.P, p.prefix_len[b]));
        c_hi -= (sg->j0 + (alt ? x : 0)) * kBN;
      }
      float m_ref = -INFINITY;  // reference exponent (log2 units), may lag the true row maximum
      float l_sum = 0.f;
      uint32_t sreg[4][32];
      for (int j = 0; j < n_mine; ++j) {
        wait(bar_s + x, n_s++ & 1);
        tc_fence_after();
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_ld32(tS + c * 32, sreg[c]);
        tmem_ld_wait();
        tc_fence_before();
        mbar_arrive_warp(bar_sl + x);   // S_x may be overwritten by the next key tile's scores
        if (c_hi < kBN) {
#pragma unroll
          for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int e = 0; e < 32; ++e) sreg[c][e] = (c * 32 + e < c_hi) ? sreg[c][e] : 0xff800000u;  // -inf
        }
        __syncwarp();
        c_hi -= alt ? 2 * kBN : kBN;
        float mx;
        {
          float mx4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int e = 0; e < 32; e += 8)
#pragma unroll
              for (int k = 0; k < 4; ++k)
                mx4[k] = max3(mx4[k], __uint_as_float(sreg[c][e + k]), __uint_as_float(sreg[c][e + 4 + k]));
          mx = fmaxf(fmaxf(mx4[0], mx4[1]), fmaxf(mx4[2], mx4[3])) * p.scale_log2;
        }
        // the reference moves only when the maximum grew by more than 2^8: fp32 sums and bf16 P have
        // the range for that lag, and O is rarely rescaled
        float corr = 1.f;
        bool rescale = false;
        if (mx > m_ref + 8.f) {
          corr = (m_ref == -INFINITY) ? 0.f : ex2(m_ref - mx);
          m_ref = mx;
          rescale = true;
        }
        // P = 2^(S * scale - m_ref), rounded to bf16 for the second product (its operand type); the
        // row sum takes the unrounded values
        // The slots take turns at this block: side by side they halve each other's rate at the
        // special-function unit (16 a clock and SM), in turn one slot's exponentials run under the
        // other's loads, maxima and stores.  Warps 4 + i and 8 + i share a scheduler and its part of that
        // unit, so the turn passes between these two, over named barriers (mbarriers: 500 cycles a turn).
        if (turn_waits(x, j, n_both)) named_sync(x == 0 ? 7 + (warp & 3) : 3 + (warp & 3), 64);
        const float neg_m = (m_ref == -INFINITY) ? 0.f : -m_ref;
        const unsigned long long scale2 = pack_f32x2(p.scale_log2, p.scale_log2);
        const unsigned long long negm2 = pack_f32x2(neg_m, neg_m);
        unsigned long long ps2[4] = {0ull, 0ull, 0ull, 0ull};
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int e = 0; e < 32; e += 2) {
            const float2 a = unpack_f32x2(fma_f32x2(
                pack_f32x2(__uint_as_float(sreg[c][e]), __uint_as_float(sreg[c][e + 1])), scale2, negm2));
            const float p0 = ex2(a.x), p1 = ex2(a.y);
            ps2[(e >> 1) & 3] = add_f32x2(ps2[(e >> 1) & 3], pack_f32x2(p0, p1));
            sreg[c][e >> 1] = pack_bf16(p0, p1);
          }
        const float2 sm = unpack_f32x2(add_f32x2(add_f32x2(ps2[0], ps2[1]), add_f32x2(ps2[2], ps2[3])));
        if (turn_passes(j, n_both)) named_arrive(x == 0 ? 3 + (warp & 3) : 7 + (warp & 3), 64);
        l_sum = l_sum * corr + (sm.x + sm.y);
        // P V of the slot's previous tile is complete: the buffer of P is free and O_x is at rest
        if (j > 0) {
          wait(bar_pv + x, (n_s - 2) & 1);
          if (__any_sync(0xffffffffu, rescale)) {
            tc_fence_after();
            uint32_t oreg[32];
#pragma unroll
            for (int c = 0; c < D / 32; ++c) {
              tmem_ld32(tO + c * 32, oreg);
              tmem_ld_wait();
#pragma unroll
              for (int e = 0; e < 32; ++e) oreg[e] = __float_as_uint(__uint_as_float(oreg[e]) * corr);
              tmem_st32(tO + c * 32, oreg);
            }
            tmem_st_wait();
            tc_fence_before();
          }
        }
        // row r of P: 16 pieces of 8 keys, piece q in block q / 8 at swizzled place q % 8
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int q = 4 * c + i;
            *reinterpret_cast<uint4*>(sPx + (q >> 3) * kTileBlockBytes + swz128(uint32_t(r), uint32_t(q & 7))) =
                make_uint4(sreg[c][4 * i], sreg[c][4 * i + 1], sreg[c][4 * i + 2], sreg[c][4 * i + 3]);
          }
        fence_proxy_async_smem();
        mbar_arrive_warp(bar_p + x);
      }

      if (n_mine > 0) wait(bar_pv + x, (n_s - 1) & 1);
      tc_fence_after();
      int b, t, g;
      const bool store = place(b, t, g);
      const int unit = sg->hk * p.pairs + sg->pair;
      const bool whole = sg->j0 == 0 && sg->j1 == sg->nt;
      const int part = whole ? 2 * int(gridDim.x) + unit : 2 * int(blockIdx.x) + (n > 0 ? 1 : 0);
      const bool finish = whole && !p.whole_parts;   // nothing to wait for: the row is joined here
      if (finish) {
        wait_for_prior();   // the forward over the rows' own tokens, which this kernel may run beside
        const size_t row = ((size_t(b) * p.Hkv + sg->hk) * p.G + g) * p.T + t;
        // joined with the row's own part (fp32, normalised, with its log-sum-exp) and rounded once
        const float lo = store ? p.own_lse[row] * 1.4426950408889634f : 0.f;
        const float lp = l_sum > 0.f ? m_ref + log2f(l_sum) : -INFINITY;
        const float mm = fmaxf(lo, lp);
        const float wo = ex2(lo - mm), wp = l_sum > 0.f ? ex2(m_ref - mm) : 0.f;
        const float den = wo + l_sum * wp, inv = 1.f / den;
        if (store) p.LSE[row] = (mm + log2f(den)) * 0.6931471805599453f;
        const float4* own = own_row<D>(p, b, sg->hk * p.G + g, t);
        __nv_bfloat16* orow = p.O + row * p.d;
        const float fo = wo * inv, fp = wp * inv;
        // The row's own part comes through this slot's buffer of P, which is free now, 64 columns at a time
        // (a thread's pieces in the places of its row number, neighbours next to each other): sixteen
        // loads under way that take no registers.
        const uint32_t stage = smem_u32(sPx) + r * 16;
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
          if (c % 2 == 0) {
            if (store)
#pragma unroll
              for (int q = 0; q < 16; ++q) cp_async16(stage + q * 2048, own + (c * 8 + q) * 128, 16);
            cp_async_commit();
            cp_async_wait<0>();
          }
          uint32_t oreg[32];
          if (n_mine > 0) { tmem_ld32(tO + c * 32, oreg); tmem_ld_wait(); }
          if (store) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              if (c * 32 + q * 8 >= p.d) continue;
              float v[8];
              *reinterpret_cast<float4*>(v) = reinterpret_cast<const float4*>(sPx)[(c % 2 * 8 + q * 2) * 128 + r];
              *reinterpret_cast<float4*>(v + 4) = reinterpret_cast<const float4*>(sPx)[(c % 2 * 8 + q * 2 + 1) * 128 + r];
#pragma unroll
              for (int e = 0; e < 8; ++e)
                v[e] = v[e] * fo + (n_mine > 0 ? __uint_as_float(oreg[q * 8 + e]) * fp : 0.f);
              *reinterpret_cast<uint4*>(orow + c * 32 + q * 8) =
                  make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]),
                             pack_bf16(v[6], v[7]));
            }
          }
          __syncwarp();
        }
        // the slot's other warps may still read here what this one's next P would overwrite
        named_sync(1 + x, 128);
      } else {
        // a part: a cut unit's go to the CTA's two places (its first segment, its last one), a whole
        // unit's to a place of its own
        const size_t u = (size_t(part) * 2 + x) * 128 + r;
        if (store) *reinterpret_cast<float2*>(p.part_ml + 2 * u) = make_float2(m_ref, l_sum);
        if (n_mine > 0) {
          float4* dst = reinterpret_cast<float4*>(p.part_acc) + (size_t(part) * 2 + x) * (D / 4) * 128 + r;
#pragma unroll
          for (int c = 0; c < D / 32; ++c) {
            uint32_t oreg[32];
            tmem_ld32(tO + c * 32, oreg);
            tmem_ld_wait();
            if (store)
#pragma unroll
              for (int q = 0; q < 8; ++q)
                dst[(c * 8 + q) * 128] =
                    make_float4(__uint_as_float(oreg[4 * q]), __uint_as_float(oreg[4 * q + 1]),
                                __uint_as_float(oreg[4 * q + 2]), __uint_as_float(oreg[4 * q + 3]));
            __syncwarp();
          }
        }
      }
      tc_fence_before();   // O_x is read: the next segment's first product into it waits for P of this thread
      // (slot 1 was through with its last exponentials long ago)
      if (turn_returns(x, n_both)) named_sync(7 + (warp & 3), 64);
      // where the unit's parts are, from the CTA that has its first key tile
      if (sg->j0 == 0 && tid == 128) {
        // number of the unit's last key tile, and the CTA that has it
        const int last = s_run[0] - sg->left - 1 + (sg->nt - sg->j1), run = s_run[1], longer = s_run[2];
        const int c1 = last < longer * (run + 1) ? last / (run + 1) : longer + (last - longer * (run + 1)) / run;
        const int second = sg->len[1] < 0 ? 0xffff : int(s_id[2 * sg->pair + 1]);
        p.unit_parts[unit] = make_int4(finish ? 0 : c1 - int(blockIdx.x) + 1, part, blockIdx.x,
                                       s_id[2 * sg->pair] | second << 16);
        if (!whole) cut = unit;
      }
    }
    // a run starts at most one unit that other CTAs go on with: its last one
    if (tid == 128) p.cut_units[blockIdx.x] = cut;
  }
  wait_for_prior();   // this kernel's end stands for the end of the one it ran beside
  tc_fence_before();
  __syncthreads();
  if (warp == 0) tmem_dealloc(tmem, 512);
}

// Bound by the bytes of the parts (L2 mostly): 36 + 3 parts of 1024 rows, 20 MB, in 5.9 us; the 147
// units of 256 rows that the runs of 148 CTAs cut, 58 MB with the own part, in 20 us.
// Joins the partial results of 32 rows of a row tile: those of the prefix and, of the rows' own keys,
// own_parts of the decode kernel ([row][part][D]) or one normalised result with its log-sum-exp
// (own_lse).  Lane = row; a warp takes CPW times four columns, and SPLIT warps share the parts (each
// a fixed subset in a fixed order).  A part with no key (l = 0) holds no values: what lies there is
// read and dropped.
//   grid (8 * units, column groups): 32 rows of every unit's two slots; CUT: 8 per CTA of the prefix
//   kernel, the unit that it left unfinished (all others are finished already)
constexpr int kJoinThreads = 128;
template <int D, bool CUT, int CPW, int SPLIT>
__global__ void __launch_bounds__(kJoinThreads) prefix_join(const PrefixParams p, const float* own_ml,
                                                            const float* own_acc, int own_parts) {
  wait_for_prior();   // (launched while the kernel before it ends)
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, sp = wid % SPLIT;
  const int col4 = (blockIdx.y * (4 / SPLIT) + wid / SPLIT) * CPW;
  const int unit = CUT ? p.cut_units[blockIdx.x / 8] : int(blockIdx.x) / 8;
  const int x = blockIdx.x / 4 % 2, r = blockIdx.x % 4 * 32 + lane;
  if (unit < 0) return;
  // the row tile: what the prefix kernel says (CUT), or, where no tile drops out, by its number
  const int4 parts = p.unit_parts[unit];
  const int of_pair = CUT ? int(x ? unsigned(parts.w) >> 16 : parts.w & 0xffff) : 2 * (unit % p.pairs) + x;
  const int ti = 2 * p.pair_base + of_pair;
  if (of_pair == 0xffff || ti >= p.m_tiles) return;
  const RowTile rt = row_tile(p, ti);
  const int hk = unit / p.pairs, b = rt.b0 + r / (p.gt * p.tt), t = rt.t0 + r / p.gt % p.tt, g = rt.g0 + r % p.gt;
  const bool here = r < p.gt * p.tt * p.bt && b < p.B && t < p.T && g < p.G && !(p.seq_len && t >= p.seq_len[b]);
  if (SPLIT == 1 && !here) return;
  const size_t row = ((size_t(b) * p.Hkv + hk) * p.G + g) * p.T + t;
  const int sub = p.alternate ? 1 : 0;     // alternate mode: both slots hold the row
  const int n_pfx = here ? parts.x << sub : 0, n_own = here ? own_parts : 0;
  auto place = [&](int i) -> size_t {      // part and slot of the row's i-th prefix part
    const int k = i >> sub, part = k == 0 ? parts.y : 2 * (parts.z + k);
    return size_t(part) * 2 + (sub ? i & 1 : x);
  };
  const float2* pml = reinterpret_cast<const float2*>(p.part_ml) + r;
  const float2* oml = reinterpret_cast<const float2*>(own_ml) + row * own_parts;
  // reference exponent of the warp's parts
  float mm = -INFINITY;
#pragma unroll 8
  for (int i = sp; i < n_pfx; i += SPLIT) {
    const float2 v = pml[place(i) * 128];
    mm = fmaxf(mm, v.y != 0.f ? v.x : -INFINITY);
  }
#pragma unroll 4
  for (int i = sp; i < n_own; i += SPLIT) {
    const float2 v = oml[i];
    mm = fmaxf(mm, v.y != 0.f ? v.x : -INFINITY);
  }
  float lo = -INFINITY;
  if (p.own_lse && here && sp == 0) { lo = p.own_lse[row] * 1.4426950408889634f; mm = fmaxf(mm, lo); }
  float l = 0.f;
  float4 acc[CPW];
#pragma unroll
  for (int c = 0; c < CPW; ++c) acc[c] = make_float4(0.f, 0.f, 0.f, 0.f);
  auto add = [&](float2 ml, const float4* v, size_t step) {
    const bool any = ml.y != 0.f;   // (a NaN is no empty part: it goes through to the output)
    const float w = any ? ex2(ml.x - mm) : 0.f;
    l += any ? ml.y * w : 0.f;
#pragma unroll
    for (int c = 0; c < CPW; ++c) {
      const float4 a = v[c * step];
      acc[c].x += any ? a.x * w : 0.f;
      acc[c].y += any ? a.y * w : 0.f;
      acc[c].z += any ? a.z * w : 0.f;
      acc[c].w += any ? a.w * w : 0.f;
    }
  };
  const float4* pacc = reinterpret_cast<const float4*>(p.part_acc) + size_t(col4) * 128 + r;
  constexpr int kUnroll = CPW == 1 ? 8 : 2;
#pragma unroll kUnroll
  for (int i = sp; i < n_pfx; i += SPLIT) {
    const size_t u = place(i);
    add(pml[u * 128], pacc + u * (D / 4) * 128, 128);
  }
#pragma unroll 2
  for (int i = sp; i < n_own; i += SPLIT)
    add(oml[i], reinterpret_cast<const float4*>(own_acc) + (row * own_parts + i) * (D / 4) + col4, 1);
  if (p.own_lse && here && sp == 0)
    add(make_float2(lo, 1.f), own_row<D>(p, b, hk * p.G + g, t) + col4 * 128, 128);
  if (SPLIT > 1) {
    __shared__ float2 s_ml[kJoinThreads];
    __shared__ float4 s_acc[kJoinThreads * CPW];
    s_ml[threadIdx.x] = make_float2(mm, l);
#pragma unroll
    for (int c = 0; c < CPW; ++c) s_acc[c * kJoinThreads + threadIdx.x] = acc[c];
    __syncthreads();
    if (sp != 0 || !here) return;
    float m = mm;
#pragma unroll
    for (int k = 1; k < SPLIT; ++k) m = fmaxf(m, s_ml[threadIdx.x + 32 * k].x);
    float ls = 0.f;
    float4 sum[CPW];
#pragma unroll
    for (int c = 0; c < CPW; ++c) sum[c] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int k = 0; k < SPLIT; ++k) {
      const float2 ml = s_ml[threadIdx.x + 32 * k];
      if (!(ml.y != 0.f)) continue;
      const float w = ex2(ml.x - m);
      ls += ml.y * w;
#pragma unroll
      for (int c = 0; c < CPW; ++c) {
        const float4 a = s_acc[c * kJoinThreads + threadIdx.x + 32 * k];
        sum[c].x += a.x * w; sum[c].y += a.y * w; sum[c].z += a.z * w; sum[c].w += a.w * w;
      }
    }
    mm = m;
    l = ls;
#pragma unroll
    for (int c = 0; c < CPW; ++c) acc[c] = sum[c];
  }
  const float inv = l != 0.f ? 1.f / l : 0.f;   // a row that sees no key at all: 0, log-sum-exp -inf
#pragma unroll
  for (int c = 0; c < CPW; ++c)
    if ((col4 + c) * 4 < p.d)
      *reinterpret_cast<uint2*>(p.O + row * p.d + (col4 + c) * 4) =
          make_uint2(pack_bf16(acc[c].x * inv, acc[c].y * inv), pack_bf16(acc[c].z * inv, acc[c].w * inv));
  if (p.LSE && col4 == 0) p.LSE[row] = l != 0.f ? (mm + log2f(l)) * 0.6931471805599453f : -INFINITY;
}

template <int D>
cudaError_t launch_join(const PrefixParams& p, int prefix_ctas, const float* own_ml, const float* own_acc, int own_parts,
                 cudaStream_t stream) {
  const unsigned units = unsigned(p.pairs * p.Hkv);
  if (!p.whole_parts)
    return launch_overlapped(prefix_join<D, true, D / 16, 1>, dim3(8 * prefix_ctas), dim3(kJoinThreads), 0, stream, p,
                             own_ml, own_acc, own_parts);
  // Few rows with many parts each: four warps share the parts of a row.  Both measured (us a decode call, four
  // warps / one; heads of 128): 1 unit behind 20 000 entries 27 / 131, 8 behind 8000 24 / 51, 16 behind 4000
  // 34 / 34, 24 behind 4000 29 / 36 (4 sequences) and 51 / 48 (160 sequences), 32 31 / 32, 40 83 / 72, 80
  // 147 / 119; heads of 64: 8 22 / 37, 24 25 / 29 and 34 / 33, 40 55 / 50.
  if (units >= 24)
    return launch_overlapped(prefix_join<D, false, D / 16, 1>, dim3(8 * units), dim3(kJoinThreads), 0, stream, p,
                             own_ml, own_acc, own_parts);
  return launch_overlapped(prefix_join<D, false, 1, 4>, dim3(8 * units, D / 4), dim3(kJoinThreads), 0, stream, p,
                           own_ml, own_acc, own_parts);
}

// bf16 [B][Hkv][G][T][d] as (d, G, T, Hkv, B); box of 64 columns x gt heads x tt tokens x bt sequences.
sepllm_status make_query_map(CUtensorMap* map, const void* base, const PrefixParams& p) {
  EncodeTiledFn enc = get_encode_tiled();
  if (!enc) return SEPLLM_CUDA_ERROR;
  const cuuint64_t row = cuuint64_t(p.d) * 2;
  cuuint64_t dims[5] = {cuuint64_t(p.d), cuuint64_t(p.G), cuuint64_t(p.T), cuuint64_t(p.Hkv), cuuint64_t(p.B)};
  cuuint64_t strides[4] = {row * p.T, row, row * p.T * p.G, row * p.T * p.G * p.Hkv};
  cuuint32_t box[5] = {64, cuuint32_t(p.gt), cuuint32_t(p.tt), 1, cuuint32_t(p.bt)};
  cuuint32_t estr[5] = {1, 1, 1, 1, 1};
  CUresult r = enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<void*>(base), dims, strides, box, estr,
                   CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                   CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? SEPLLM_OK : SEPLLM_CUDA_ERROR;
}

template <int D>
sepllm_status launch_prefix_d(const PrefixParams& p, int grid, const CUtensorMap& mq, const CUtensorMap& mk,
                              const CUtensorMap& mv, cudaStream_t stream) {
  SEPLLM_CUDA_TRY(cudaFuncSetAttribute(prefix_attn<D>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       int(PfxCfg<D>::kRequest)));
  // behind a forward it may start while that ends (a decode's prefix kernel is its call's first)
  if (p.reset_status || p.pair_base > 0)
    prefix_attn<D><<<grid, kPfxThreads, PfxCfg<D>::kRequest, stream>>>(mq, mk, mv, p);
  else
    SEPLLM_CUDA_TRY(launch_overlapped(prefix_attn<D>, dim3(grid), dim3(kPfxThreads), PfxCfg<D>::kRequest, stream, mq,
                                      mk, mv, p));
  SEPLLM_CUDA_TRY(cudaGetLastError());
  return SEPLLM_OK;
}

int all_pairs(const PrefixParams& p) { return (p.m_tiles + 1) / 2; }
// per launch: what the table holds, and a count of key tiles within 31 bits
int launch_pairs(const PrefixParams& p) {
  return int(std::min<int64_t>(std::min(all_pairs(p), kMaxPairs), (int64_t(1) << 30) / (int64_t(p.key_tiles) * p.Hkv)));
}

// CTAs of a launch over `pairs` pairs: one per SM, none without a key tile (two in alternate mode).
int prefix_grid(const PrefixParams& p, int pairs) {
  const int64_t work = int64_t(pairs) * p.Hkv * (p.alternate ? (p.key_tiles + 1) / 2 : p.key_tiles);
  return int(std::min<int64_t>(p.max_ctas, work));
}

// Parts of a launch over `pairs` pairs: two places per CTA, and one per unit where whole units leave parts (decode).
int64_t max_parts(const PrefixParams& p, int pairs) {
  return 2ll * prefix_grid(p, pairs) + (p.whole_parts ? int64_t(pairs) * p.Hkv : 0);
}

size_t part_bytes(const PrefixParams& p, int pairs) {
  const size_t rows = size_t(max_parts(p, pairs)) * 256;
  return align_up(rows * 2 * sizeof(float)) + align_up(rows * kernel_head_dim(p.d) * sizeof(float)) +
         align_up(size_t(pairs) * p.Hkv * sizeof(int4)) + align_up(kSmCount * sizeof(int32_t));
}

}  // namespace

bool plan_prefix(PrefixParams* p, int B, int Hq, int Hkv, int T, int d, int P, bool whole_parts, double own_us) {
  p->B = B;
  p->Hkv = Hkv;
  p->G = Hq / Hkv;
  p->T = T;
  p->d = d;
  p->P = P;
  p->key_tiles = (P + kBN - 1) / kBN;
  p->gt = std::min(p->G, 128);
  p->tt = std::min(T, 128 / p->gt);
  p->bt = p->tt == T && p->gt == p->G ? std::min(B, 128 / (p->gt * p->tt)) : 1;
  p->g_tiles = (p->G + p->gt - 1) / p->gt;
  p->t_tiles = (T + p->tt - 1) / p->tt;
  const int64_t m_tiles = int64_t((B + p->bt - 1) / p->bt) * p->t_tiles * p->g_tiles;
  if (int64_t(B) * Hq * T > 0x7fffffff || m_tiles > 0x3fffffff || Hkv > 65535 || P > (1 << 30) || int64_t(p->key_tiles) * Hkv > (1 << 30)) return false;
  p->m_tiles = int(m_tiles);
  p->alternate = m_tiles == 1 ? 1 : 0;
  p->whole_parts = whole_parts || p->alternate;   // alternate mode: two parts of every row, joined later
  p->max_ctas = kSmCount;
  if (own_us > 0.0) {
    // The own part runs on the SMs that the prefix kernel leaves, and on all of them when it is done.
    // With n CTAs the prefix takes 8 us and 2.1 us for each pair of row tiles and key tile of a CTA
    // (measured); the own part, bound by HBM, loses nothing while it has four fifths of the SMs.
    const double steps = double(launch_pairs(*p)) * Hkv * p->key_tiles * (p->alternate ? 0.5 : 1.0);
    double best = 1e300;
    for (int n = 4; n <= kSmCount; n += 4) {
      const double t = 8.0 + 2.1 * std::ceil(steps / n), rate = std::min(1.0, 1.25 * (kSmCount - n) / kSmCount);
      const double total = rate * t >= own_us ? t : own_us + (1.0 - rate) * t;
      if (total < best) { best = total; p->max_ctas = n; }
    }
    p->est_us = std::max(best, own_us + double(Hkv) * P * d * 4 / 6.2e6);   // not below the bytes of both
    if (p->alternate && p->max_ctas > Hkv) p->max_ctas -= p->max_ctas % Hkv;   // (see n_runs)
  }
  return true;
}

size_t prefix_part_bytes(PrefixParams p) {
  p.max_ctas = kSmCount;
  return part_bytes(p, std::min(all_pairs(p), kMaxPairs));
}

void place_prefix_parts(PrefixParams* p, uint8_t* ws) {
  const size_t rows = size_t(max_parts(*p, launch_pairs(*p))) * 256;
  p->part_ml = reinterpret_cast<float*>(ws);
  ws += align_up(rows * 2 * sizeof(float));
  p->part_acc = reinterpret_cast<float*>(ws);
  ws += align_up(rows * kernel_head_dim(p->d) * sizeof(float));
  p->unit_parts = reinterpret_cast<int4*>(ws);
  p->cut_units = reinterpret_cast<int32_t*>(ws + align_up(size_t(launch_pairs(*p)) * p->Hkv * sizeof(int4)));
}

sepllm_status launch_prefix(PrefixParams p, const void* Q, const void* Kp, const void* Vp, cudaStream_t stream,
                            sepllm_status (*beside)(void*), void* ctx, const float* own_ml, const float* own_acc,
                            int own_parts) {
  CUtensorMap mq, mk, mv;
  sepllm_status st;
  if ((st = make_query_map(&mq, Q, p)) != SEPLLM_OK) return st;
  if ((st = make_tile_map(&mk, Kp, p.d, p.P, p.Hkv, p.d, int64_t(p.P) * p.d, 128)) != SEPLLM_OK) return st;
  if ((st = make_tile_map(&mv, Vp, p.d, p.P, p.Hkv, p.d, int64_t(p.P) * p.d, 128)) != SEPLLM_OK) return st;
  const bool d64 = kernel_head_dim(p.d) == 64;
  for (p.pair_base = 0; p.pair_base < all_pairs(p); p.pair_base += p.pairs) {
    p.pairs = std::min(launch_pairs(p), all_pairs(p) - p.pair_base);
    const int grid = prefix_grid(p, p.pairs);
    p.reset_status = beside && p.pair_base == 0;
    st = d64 ? launch_prefix_d<64>(p, grid, mq, mk, mv, stream) : launch_prefix_d<128>(p, grid, mq, mk, mv, stream);
    if (st != SEPLLM_OK) return st;
    if (beside && p.pair_base == 0 && (st = beside(ctx)) != SEPLLM_OK) return st;
    SEPLLM_CUDA_TRY(d64 ? launch_join<64>(p, grid, own_ml, own_acc, own_parts, stream)
                        : launch_join<128>(p, grid, own_ml, own_acc, own_parts, stream));
  }
  return SEPLLM_OK;
}

}  // namespace sepllm

using namespace sepllm;

namespace {
// How a call is carried out.  direct: the prefix rows are copied in front of every sequence's side rows
// and the forward kernels walk them there; otherwise the forward over the rows' own tokens and the
// prefix kernel, which shares the loads, splits long prefixes and drops padding, with a workspace of
// the forward's own | O32 | LSE of the own part | parts.
struct AttnPrefixLayout {
  size_t off_o, off_lse, off_parts, bytes;
};
bool attn_prefix_direct(const sepllm_attn_desc* d, const sepllm_index_desc* id, const PrefixParams& p) {
  // Microseconds: a wave of forward CTAs (two row tiles each, one CTA per SM) takes 6 and 2 for each key
  // tile; the copy its bytes at 5 TB/s; the prefix kernel 2 for each step of a CTA, and with the join 24
  // (14 where there is a single row tile).  Both measured (us, direct / shared; 32 heads on 8 of 128):
  // 1 sequence x 16 tokens behind 100 entries 17 / 28, behind 1000 32 / 25; 16 x 64 behind 100 37 / 44,
  // behind 1000 80 / 73; 4 x 300 behind 500 54 / 60, behind 2000 107 / 100; 2 x 1024 behind 500 69 / 97,
  // behind 2000 114 / 140, behind 8000 326 / 292; 1 x 8192 behind 500 270 / 317; 12 heads of 64: 8 x 1024
  // behind 1000 116 / 126.  The rule takes the faster form in each of these.  On a grid of 60 points (16 to 8192 tokens, 100 to
  // 8000 entries, 32 heads on 8 of 128 and 12 of 64) it took the slower one in 4: by 2 % (2 x 1024 behind 4000) and 6 % (8 x
  // 1024 behind 2000) at 128, by 6 and 14 % (1 x 16 and 16 x 64 behind 500) at 64, whose steps are shorter
  // than the 2 us taken here.
  const double own_tiles = std::min(d->L, id->n_neighbor) / 128 + 2;
  const double waves = std::ceil(double(d->B) * d->Hq * ((d->L + 127) / 128) / 2 / kSmCount);
  const double copy_us = double(d->B) * d->Hkv * p.P * d->d * 8 / 5e6;
  const double direct_us = 4.0 + copy_us + waves * (6.0 + 2.0 * (own_tiles + p.key_tiles));
  const double steps = double(all_pairs(p)) * d->Hkv * p.key_tiles * (p.alternate ? 0.5 : 1.0);
  const double shared_us = 4.0 + waves * (6.0 + 2.0 * own_tiles) + (p.alternate ? 14.0 : 24.0) +
                           2.0 * std::ceil(steps / kSmCount);
  return direct_us < shared_us && attn_direct_rows(id, p.P) < (1 << 30);
}
AttnPrefixLayout attn_shared_layout(const sepllm_attn_desc* d, const sepllm_index_desc* id, const PrefixParams& p) {
  AttnPrefixLayout a;
  const size_t rows = size_t(d->B) * d->Hq * d->L;
  a.off_o = attn_layout(d, id).fwd_bytes;
  a.off_lse = a.off_o + align_up(size_t(d->B) * d->Hq * ((d->L + 127) / 128 * 128) * kernel_head_dim(d->d) * sizeof(float));
  a.off_parts = a.off_lse + align_up(rows * sizeof(float));
  a.bytes = a.off_parts + prefix_part_bytes(p);
  return a;
}
// Bytes for every prefix of up to p.P rows.  The shared form's grow with the prefix; the direct form's do
// too, but it is not taken for all of them: the longest one that may take it counts (within a key tile
// the rule's direct time grows with the rows, so its first row says whether any takes it).
size_t attn_prefix_bytes(const sepllm_attn_desc* d, const sepllm_index_desc* id, PrefixParams p) {
  const size_t shared = attn_shared_layout(d, id, p).bytes;
  const int P = p.P;
  for (; p.key_tiles > 0; --p.key_tiles) {
    p.P = (p.key_tiles - 1) * kBN + 1;
    if (attn_prefix_direct(d, id, p))
      return std::max(shared, attn_direct_bytes(d, id, std::min(P, p.key_tiles * kBN)));
  }
  return shared;
}
}  // namespace

extern "C" sepllm_status sepllm_attn_prefix_workspace_bytes(const sepllm_attn_desc* desc,
                                                            const sepllm_index_desc* idesc, int32_t P,
                                                            size_t* bytes) {
  sepllm_status st = check_attn(desc, idesc);
  if (st != SEPLLM_OK) return st;
  if (P < 1) return SEPLLM_INVALID_ARG;
  PrefixParams p{};
  if (!plan_prefix(&p, desc->B, desc->Hq, desc->Hkv, desc->L, desc->d, P, false, 0.0)) return SEPLLM_UNSUPPORTED;
  if (bytes) *bytes = attn_prefix_bytes(desc, idesc, p);
  return SEPLLM_OK;
}

extern "C" sepllm_status sepllm_attn_prefix_fwd(const sepllm_attn_desc* desc, const sepllm_index_desc* idesc,
                                                int32_t P, const void* Q, const void* K, const void* V,
                                                const void* index, const void* Kp, const void* Vp,
                                                const int32_t* prefix_len, void* O, float* LSE, void* workspace,
                                                void* stream_) {
  sepllm_status st = check_attn(desc, idesc);
  if (st != SEPLLM_OK) return st;
  if (P < 1 || !Q || !K || !V || !index || !Kp || !Vp || !O || !LSE || !workspace) return SEPLLM_INVALID_ARG;
  if (!aligned(Q, 16) || !aligned(K, 16) || !aligned(V, 16) || !aligned(Kp, 16) || !aligned(Vp, 16) ||
      !aligned(O, 16) || !aligned(LSE, 4) || !aligned(prefix_len, 4) || !aligned(index, kAlign) ||
      !aligned(workspace, kAlign))
    return SEPLLM_INVALID_ARG;
  sepllm_index_header ih;
  if ((st = fill_index_header(idesc, &ih)) != SEPLLM_OK) return st;
  PrefixParams p{};
  if (!plan_prefix(&p, desc->B, desc->Hq, desc->Hkv, desc->L, desc->d, P, false, 0.0)) return SEPLLM_UNSUPPORTED;
  cudaStream_t stream = static_cast<cudaStream_t>(stream_);
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  if (attn_prefix_direct(desc, idesc, p))
    return attn_fwd_direct(desc, idesc, Q, K, V, index, PrefixRows{Kp, Vp, prefix_len, P}, O, LSE, ws, stream);
  const AttnPrefixLayout lay = attn_shared_layout(desc, idesc, p);
  float* own_O = reinterpret_cast<float*>(ws + lay.off_o);
  float* own_lse = reinterpret_cast<float*>(ws + lay.off_lse);
  // the rows' own tokens first (Eq. 2's mask); their result waits in 32 bits so that O is rounded once
  sepllm_attn_desc fresh = *desc;
  fresh.flags &= ~SEPLLM_ATTN_SIDE_READY;   // (the workspace's side rows are the call's own)
  if ((st = attn_fwd_f32(&fresh, idesc, Q, K, V, index, own_O, own_lse, ws, stream)) != SEPLLM_OK) return st;
  place_prefix_parts(&p, ws + lay.off_parts);
  p.prefix_len = prefix_len;
  p.seq_len = reinterpret_cast<const int32_t*>(static_cast<const uint8_t*>(index) + ih.off_seq_len);
  p.own_O = own_O;
  p.own_lse = own_lse;
  p.O = static_cast<__nv_bfloat16*>(O);
  p.LSE = LSE;
  p.status = reinterpret_cast<int32_t*>(ws);
  p.scale_log2 = (desc->scale != 0.f ? desc->scale : 1.0f / sqrtf(float(desc->d))) * 1.4426950408889634f;
  return launch_prefix(p, Q, Kp, Vp, stream, nullptr, nullptr, nullptr, nullptr, 0);
}
