// Attention over a prefix that the whole batch shares.
//
// Every query row (sequence b, head h, token t) attends to the first prefix_len[b] rows of one
// K/V block Kp, Vp [Hkv][P][d] and to keys of its own (the sequence's cache, or the kept tokens of
// its own row).  The two sets are disjoint, so the softmax over both is joined from two partial
// results: with reference exponents m1, m2, sums l1, l2 and unnormalised values a1, a2,
//   O = (a1 2^(m1-M) + a2 2^(m2-M)) / (l1 2^(m1-M) + l2 2^(m2-M)),  M = max(m1, m2).
// This file has the prefix half: all B * G * T rows that read one kv head (G query heads per kv head,
// T tokens) are the rows of one matrix product, 128 to a tile, so the prefix is read once per
// 256 rows instead of once per sequence.
#include <algorithm>

#include "attn_common.cuh"

namespace sepllm {

namespace {

constexpr int kPfxThreads = 384;

template <int D>
struct PfxCfg {
  static constexpr int NB = D / 64;               // 64-column blocks per row
  static constexpr int NST = (D == 128) ? 2 : 4;  // K and V ring depth
  static constexpr uint32_t kTile = NB * kTileBlockBytes;
  static constexpr uint32_t kQ = 0;
  static constexpr uint32_t kK = kQ + 2 * kTile;
  static constexpr uint32_t kV = kK + NST * kTile;
  static constexpr uint32_t kBar = kV + NST * kTile;
  static constexpr uint32_t kTotal = kBar + 512;
  static constexpr uint32_t kRequest = kTotal + 1024;
  static constexpr uint32_t kS0 = 0, kS1 = 128, kO0 = 256, kO1 = 256 + D;  // tensor-memory columns
};
static_assert(PfxCfg<128>::kRequest <= 227 * 1024 && PfxCfg<64>::kRequest > 114 * 1024,
              "one CTA per SM owns all 512 tensor-memory columns");

// One CTA: one kv head, one split of the key tiles, two slots of 128 query rows.
//   pair mode        slot x holds row tile 2 * blockIdx.x + x; both slots walk the same key tiles
//   alternate mode   (one row tile in all) both slots hold that tile and take the key tiles in turn,
//                    so that one slot's softmax runs under the other's loads and products; each
//                    slot leaves a partial result of its own
// Warps as in the forward kernel: 0 TMA, 1 MMA issue, 2 clears V rows behind the prefix, 4-7 and
// 8-11 softmax of slot 0 and 1, one thread per row; P goes back to tensor memory as bf16 over S.
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
  uint8_t* sK = smem + C::kK;
  uint8_t* sV = smem + C::kV;
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::kBar);
  uint64_t* bar_q = bars;          // [2]   Q of slot x landed
  uint64_t* bar_s = bars + 2;      // [2]   S_x complete (and every earlier MMA)
  uint64_t* bar_p = bars + 4;      // [2]   P_x written by the 4 softmax warps of slot x
  uint64_t* bar_o = bars + 6;      //       every MMA of the CTA complete
  uint64_t* bar_z = bars + 7;      //       V rows behind the prefix cleared
  uint64_t* bar_g = bars + 8;      //       V of the last tile landed: clear the rows behind the prefix
  uint64_t* bar_kf = bars + 9;     // [NST] K stage full
  uint64_t* bar_ke = bar_kf + NST; // [NST] K stage free
  uint64_t* bar_vf = bar_ke + NST; // [NST]
  uint64_t* bar_ve = bar_vf + NST; // [NST]
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 9 + 4 * NST);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 2);
  int* s_max = reinterpret_cast<int*>(tmem_slot + 4);  // [2] largest prefix length of slot x

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int hk = blockIdx.y, split = blockIdx.z;
  const int GT = p.G * p.T;
  const bool alt = p.alternate != 0;
  // row tile of slot x: sequences [b0, b0 + bt), rows [r0, r0 + rt) of each
  auto tile_of = [&](int x) { return alt ? 0 : 2 * int(blockIdx.x) + x; };
  auto tile_b0 = [&](int i) { return GT <= 128 ? i * p.bt : i / p.row_tiles; };
  auto tile_r0 = [&](int i) { return GT <= 128 ? 0 : (i % p.row_tiles) * 128; };
  const bool have1 = alt || tile_of(1) < p.m_tiles;

  if (tid == 0) {
    for (int i = 0; i < 2; ++i) { mbar_init(bar_q + i, 1); mbar_init(bar_s + i, 1); mbar_init(bar_p + i, 4); }
    mbar_init(bar_o, 1);
    mbar_init(bar_z, 1);
    mbar_init(bar_g, 1);
    for (int i = 0; i < NST; ++i) {
      mbar_init(bar_kf + i, 1); mbar_init(bar_ke + i, 1); mbar_init(bar_vf + i, 1); mbar_init(bar_ve + i, 1);
    }
    *abort_flag = 0;
    s_max[0] = s_max[1] = 0;
    fence_mbar_init();
    tma_prefetch_desc(&mapQ); tma_prefetch_desc(&mapK); tma_prefetch_desc(&mapV);
  }
  if (warp == 0) {
    __syncwarp();
    tmem_alloc(tmem_slot, 512);
    tmem_relinquish();
  }
  // rows of the tile that no load fills are zero: their scores are finite and nothing is stored
  const int rows = p.rt * p.bt;
  for (int i = tid; i < (128 - rows) * 8 * NB * 2; i += kPfxThreads) {
    const int ch = i & 7, blk = (i >> 3) % (2 * NB), r = rows + (i >> 3) / (2 * NB);
    *reinterpret_cast<uint4*>(sQ + blk * kTileBlockBytes + r * 128 + ch * 16) = make_uint4(0, 0, 0, 0);
  }
  fence_proxy_async_smem();
  __syncthreads();   // s_max is set
  for (int i = tid; i < 2 * p.bt; i += kPfxThreads) {
    const int x = i >= p.bt, ti = tile_of(x), b = tile_b0(ti) + (x ? i - p.bt : i);
    if (ti < p.m_tiles && b < p.B) atomicMax(s_max + x, p.prefix_len ? max(0, min(p.P, p.prefix_len[b])) : p.P);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;

  // key tiles of this split, cut at the longest prefix among the rows
  const int kt0 = int(int64_t(p.key_tiles) * split / p.splits);
  const int kt1 = int(int64_t(p.key_tiles) * (split + 1) / p.splits);
  const int max0 = s_max[0], max1 = s_max[1], max_len = max(max0, max1);
  const int n_tiles = max(0, min(kt1, (max_len + kBN - 1) / kBN) - kt0);
  // slot x works on key tile j of the split
  auto active = [&](int x, int j) {
    return alt ? (j & 1) == x : (kt0 + j) * kBN < (x ? max1 : max0);
  };
  // the last tile holds the end of the longest prefix: V rows behind it may hold anything
  const bool clear_v = n_tiles > 0 && (kt0 + n_tiles) * kBN > max_len;

  bool ok = true;
  auto wait = [&](uint64_t* bar, uint32_t parity) {
    if (!mbar_wait(bar, parity, abort_flag)) {
      if (ok) set_status(p.status, SEPLLM_TIMEOUT);
      ok = false;
    }
  };

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    if (warp == 0 && lane == 0) {
      // ---------------- TMA producer ----------------
      if (n_tiles > 0) {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int ti = tile_of(x);
          if (alt ? x == 1 : !active(x, 0)) continue;   // a slot without work loads (and waits for) nothing
          mbar_expect_tx(bar_q + x, uint32_t(NB * rows) * 128u);
          for (int nb = 0; nb < NB; ++nb)
            tma_load_4d(sQ + x * C::kTile + nb * kTileBlockBytes, &mapQ, bar_q + x, nb * 64, tile_r0(ti), hk,
                        tile_b0(ti));
        }
      }
      for (int j = 0; j < n_tiles; ++j) {
        const int st = j % NST, use = j / NST, y = (kt0 + j) * kBN;
        if (use > 0) wait(bar_ke + st, (use - 1) & 1);
        mbar_expect_tx(bar_kf + st, C::kTile);
        for (int nb = 0; nb < NB; ++nb)
          tma_load_3d(sK + st * C::kTile + nb * kTileBlockBytes, &mapK, bar_kf + st, nb * 64, y, hk);
        if (use > 0) wait(bar_ve + st, (use - 1) & 1);
        mbar_expect_tx(bar_vf + st, C::kTile);
        for (int nb = 0; nb < NB; ++nb)
          tma_load_3d(sV + st * C::kTile + nb * kTileBlockBytes, &mapV, bar_vf + st, nb * 64, y, hk);
      }
    } else if (warp == 1 && lane == 0) {
      // ---------------- MMA issuer ----------------
      constexpr uint32_t idesc_s = make_idesc_bf16(128, 128, 0, 0);
      constexpr uint32_t idesc_o = make_idesc_bf16(128, D, 0, 1);
      const uint32_t q_lo[2] = {desc_lo(smem_u32(sQ), 16), desc_lo(smem_u32(sQ + (alt ? 0 : C::kTile)), 16)};
      const uint32_t k_lo0 = desc_lo(smem_u32(sK), 16);
      const uint32_t v_lo0 = desc_lo(smem_u32(sV), kTileBlockBytes);
      int n_pv[2] = {0, 0};  // PV MMAs issued per slot
      bool q_seen[2] = {false, false};
      bool k_waited, v_waited;
      auto scores = [&](int x, int j) {   // S_x = Q_x K(j)^T
        const int st = j % NST, qx = alt ? 0 : x;
        if (!q_seen[qx]) { wait(bar_q + qx, 0); q_seen[qx] = true; }
        if (!k_waited) { wait(bar_kf + st, (j / NST) & 1); k_waited = true; }
        const uint32_t tS = tmem + (x ? C::kS1 : C::kS0), k_lo = k_lo0 + st * (C::kTile >> 4);
#pragma unroll
        for (int k = 0; k < D / 16; ++k)
          umma_ss_lo(tS, q_lo[x] + kmajor_step(k, kTileBlockBytes), k_lo + kmajor_step(k, kTileBlockBytes),
                     idesc_s, k > 0);
        tc_commit(bar_s + x);
      };
      auto values = [&](int x, int j) {   // O_x += P_x V(j)
        const int st = j % NST;
        wait(bar_p + x, n_pv[x] & 1);
        if (!v_waited) {
          wait(bar_vf + st, (j / NST) & 1);
          if (clear_v && j == n_tiles - 1) { mbar_arrive(bar_g); wait(bar_z, 0); }
          v_waited = true;
        }
        tc_fence_after();
        const uint32_t tS = tmem + (x ? C::kS1 : C::kS0), tO = tmem + (x ? C::kO1 : C::kO0);
        const uint32_t v_lo = v_lo0 + st * (C::kTile >> 4);
        umma_ts_lo(tO, tS, v_lo, idesc_o, n_pv[x] > 0);
#pragma unroll
        for (int k = 1; k < kBN / 16; ++k)
          umma_ts_lo(tO, tS + k * 8, v_lo + mnmajor_step(k), idesc_o, 1);
        ++n_pv[x];
      };
      for (int s = 0; s <= n_tiles; ++s) {
        k_waited = v_waited = false;
        if (alt) {   // the slots never share a step: the next scores go first
          if (s < n_tiles) scores(s & 1, s);
          if (s >= 1) values((s - 1) & 1, s - 1);
        } else {
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            if (s >= 1 && active(x, s - 1)) values(x, s - 1);
            if (s < n_tiles && active(x, s)) scores(x, s);
          }
        }
        if (s < n_tiles) tc_commit(bar_ke + s % NST);
        if (s >= 1) tc_commit(bar_ve + (s - 1) % NST);
      }
      tc_commit(bar_o);
    } else if (warp == 2 && clear_v) {
      // ---------------- V rows behind the longest prefix ----------------
      const int st = (n_tiles - 1) % NST;
      wait(bar_g, 0);
      for (int i = lane; i < (kBN - max_len % kBN) * 8 * NB; i += 32) {
        const int ch = i & 7, blk = (i >> 3) % NB, r = max_len % kBN + (i >> 3) / NB;
        *reinterpret_cast<uint4*>(sV + st * C::kTile + blk * kTileBlockBytes + r * 128 + ch * 16) =
            make_uint4(0, 0, 0, 0);
      }
      fence_proxy_async_smem();
      mbar_arrive_warp(bar_z);
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
    // ---------------- softmax of slot x ----------------
    const int x = (warp >= 8) ? 1 : 0;
    const int r = tid & 127;  // row in the tile = tensor-memory lane
    const uint32_t lane_base = uint32_t((warp & 3) * 32) << 16;
    const uint32_t tS = tmem + lane_base + (x ? C::kS1 : C::kS0);
    const uint32_t tO = tmem + lane_base + (x ? C::kO1 : C::kO0);
    if (x == 0 || have1) {
      const int ti = tile_of(x);
      // the row: sequence b, row rr = head in group * T + token
      int b, rr;
      if (GT <= 128) { b = tile_b0(ti) + r / GT; rr = r % GT; }
      else { b = tile_b0(ti); rr = tile_r0(ti) + r; }
      bool store = r < rows && b < p.B && rr < GT;
      int len = x ? max1 : max0;
      if (store) {
        if (p.prefix_len) len = max(0, min(p.P, p.prefix_len[b]));
        if (p.seq_len && rr % p.T >= p.seq_len[b]) store = false;   // a row of padding
      }
      float m_ref = -INFINITY;  // reference exponent (log2 units), may lag the true row maximum
      float l_sum = 0.f;
      int n_done = 0;
      uint32_t sreg[4][32];
      for (int j = 0; j < n_tiles; ++j) {
        if (!active(x, j)) continue;
        wait(bar_s + x, n_done & 1);
        tc_fence_after();
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_ld32(tS + c * 32, sreg[c]);
        tmem_ld_wait();
        const int c_hi = len - (kt0 + j) * kBN;   // keys of the tile that the row sees
        if (c_hi < kBN) {
#pragma unroll
          for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int e = 0; e < 32; ++e) sreg[c][e] = (c * 32 + e < c_hi) ? sreg[c][e] : 0xff800000u;  // -inf
        }
        __syncwarp();
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
        l_sum = l_sum * corr + (sm.x + sm.y);
        // S_x of this tile complete means P V of the slot's previous tile is: O_x is at rest
        if (n_done > 0 && __any_sync(0xffffffffu, rescale)) {
          uint32_t oreg[32];
#pragma unroll
          for (int c = 0; c < D / 32; ++c) {
            tmem_ld32(tO + c * 32, oreg);
            tmem_ld_wait();
#pragma unroll
            for (int e = 0; e < 32; ++e) oreg[e] = __float_as_uint(__uint_as_float(oreg[e]) * corr);
            tmem_st32(tO + c * 32, oreg);
          }
        }
        // P as packed bf16 over the first 64 columns of S_x: column c holds keys 2c, 2c+1
        {
          uint32_t pk[32];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int e = 0; e < 16; ++e) { pk[e] = sreg[2 * h][e]; pk[16 + e] = sreg[2 * h + 1][e]; }
            tmem_st32(tS + h * 32, pk);
          }
        }
        tmem_st_wait();
        tc_fence_before();
        mbar_arrive_warp(bar_p + x);
        ++n_done;
      }

      if (n_done > 0) wait(bar_o, 0);
      tc_fence_after();
      const size_t row = (size_t(b) * p.Hkv + hk) * GT + rr;
      if (p.merge_O) {
        // joined with the row's own part (fp32, normalised, with its log-sum-exp) and rounded once
        const float lo = store ? p.own_lse[row] * 1.4426950408889634f : 0.f;
        const float lp = l_sum > 0.f ? m_ref + log2f(l_sum) : -INFINITY;
        const float mm = fmaxf(lo, lp);
        const float wo = ex2(lo - mm), wp = l_sum > 0.f ? ex2(m_ref - mm) : 0.f;
        const float den = wo + l_sum * wp, inv = 1.f / den;
        if (store) p.LSE[row] = (mm + log2f(den)) * 0.6931471805599453f;
        const float* own = p.own_O + row * D;
        __nv_bfloat16* orow = p.O + row * p.d;
        const float fo = wo * inv, fp = wp * inv;
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
          uint32_t oreg[32];
          if (n_done > 0) { tmem_ld32(tO + c * 32, oreg); tmem_ld_wait(); }
          if (store) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              if (c * 32 + q * 8 >= p.d) continue;
              float v[8];
              *reinterpret_cast<float4*>(v) = *reinterpret_cast<const float4*>(own + c * 32 + q * 8);
              *reinterpret_cast<float4*>(v + 4) = *reinterpret_cast<const float4*>(own + c * 32 + q * 8 + 4);
#pragma unroll
              for (int e = 0; e < 8; ++e)
                v[e] = v[e] * fo + (n_done > 0 ? __uint_as_float(oreg[q * 8 + e]) * fp : 0.f);
              *reinterpret_cast<uint4*>(orow + c * 32 + q * 8) =
                  make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]),
                             pack_bf16(v[6], v[7]));
            }
          }
        }
      } else {
        const int parts = p.splits << (alt ? 1 : 0);
        const size_t u = row * parts + (alt ? 2 * split + x : split);
        if (store) *reinterpret_cast<float2*>(p.part_ml + 2 * u) = make_float2(m_ref, l_sum);
        if (n_done > 0) {
          float* dst = p.part_acc + u * D;
#pragma unroll
          for (int c = 0; c < D / 32; ++c) {
            uint32_t oreg[32];
            tmem_ld32(tO + c * 32, oreg);
            tmem_ld_wait();
            if (store)
#pragma unroll
              for (int q = 0; q < 8; ++q)
                *reinterpret_cast<uint4*>(dst + c * 32 + q * 4) =
                    make_uint4(oreg[4 * q], oreg[4 * q + 1], oreg[4 * q + 2], oreg[4 * q + 3]);
          }
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 0) tmem_dealloc(tmem, 512);
}

// Joins the partial results of a row: `parts` of the prefix and, of its own keys, own_parts of the
// decode kernel or one normalised result with its log-sum-exp (own_lse).  One warp per row, in a
// fixed order.  A part with no key (l = 0) has no values and is not read.
constexpr int kJoinWarps = 4;
template <int D>
__global__ void __launch_bounds__(kJoinWarps * 32) prefix_join(const PrefixParams p, const float* own_ml,
                                                               const float* own_acc, int own_parts,
                                                               int64_t n_rows) {
  constexpr int E = D / 32;  // elements per lane
  using Vec = typename std::conditional<E == 4, float4, float2>::type;
  const int lane = threadIdx.x & 31;
  const int64_t row = int64_t(blockIdx.x) * kJoinWarps + (threadIdx.x >> 5);
  if (row >= n_rows) return;
  if (p.seq_len && int(row % p.T) >= p.seq_len[row / (int64_t(p.Hkv) * p.G * p.T)]) return;
  const int parts = p.splits << (p.alternate ? 1 : 0);
  const float2* pml = reinterpret_cast<const float2*>(p.part_ml) + row * parts;
  const float2* oml = reinterpret_cast<const float2*>(own_ml) + row * own_parts;
  float mm = -INFINITY;
  for (int s = lane; s < parts; s += 32) mm = fmaxf(mm, pml[s].y > 0.f ? pml[s].x : -INFINITY);
  for (int s = lane; s < own_parts; s += 32) mm = fmaxf(mm, oml[s].y > 0.f ? oml[s].x : -INFINITY);
  float lo = -INFINITY;
  if (p.own_lse) { lo = p.own_lse[row] * 1.4426950408889634f; mm = fmaxf(mm, lo); }
#pragma unroll
  for (int k = 16; k; k >>= 1) mm = fmaxf(mm, __shfl_xor_sync(0xffffffffu, mm, k));
  float l = 0.f, acc[E];
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] = 0.f;
  auto add = [&](const float* a, float w) {
    const Vec v = *reinterpret_cast<const Vec*>(a + lane * E);
    const float* f = reinterpret_cast<const float*>(&v);
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] += f[e] * w;
  };
#pragma unroll 4
  for (int s = 0; s < parts; ++s) {
    const float2 ml = pml[s];
    if (!(ml.y > 0.f)) continue;
    const float w = ex2(ml.x - mm);
    l += ml.y * w;
    add(p.part_acc + (row * parts + s) * D, w);
  }
#pragma unroll 4
  for (int s = 0; s < own_parts; ++s) {
    const float2 ml = oml[s];
    if (!(ml.y > 0.f)) continue;
    const float w = ex2(ml.x - mm);
    l += ml.y * w;
    add(own_acc + (row * own_parts + s) * D, w);
  }
  if (p.own_lse) {
    const float w = ex2(lo - mm);
    l += w;
    add(p.own_O + row * D, w);
  }
  const float inv = l > 0.f ? 1.f / l : 0.f;   // a row that sees no key at all: 0, log-sum-exp -inf
  if (lane * E < p.d) {
    __nv_bfloat16* o = p.O + row * p.d + lane * E;
#pragma unroll
    for (int e = 0; e < E; e += 2)
      *reinterpret_cast<uint32_t*>(o + e) = pack_bf16(acc[e] * inv, acc[e + 1] * inv);
  }
  if (p.LSE && lane == 0) p.LSE[row] = l > 0.f ? (mm + log2f(l)) * 0.6931471805599453f : -INFINITY;
}

// bf16 [B][Hkv][rows][d] as (d, rows, Hkv, B); box of 64 columns x rt rows x bt sequences.
sepllm_status make_query_map(CUtensorMap* map, const void* base, const PrefixParams& p) {
  EncodeTiledFn enc = get_encode_tiled();
  if (!enc) return SEPLLM_CUDA_ERROR;
  const cuuint64_t GT = cuuint64_t(p.G) * p.T, d = cuuint64_t(p.d);
  cuuint64_t dims[4] = {d, GT, cuuint64_t(p.Hkv), cuuint64_t(p.B)};
  cuuint64_t strides[3] = {d * 2, GT * d * 2, GT * d * 2 * p.Hkv};
  cuuint32_t box[4] = {64, cuuint32_t(p.rt), 1, cuuint32_t(p.bt)};
  cuuint32_t estr[4] = {1, 1, 1, 1};
  CUresult r = enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, strides, box, estr,
                   CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                   CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? SEPLLM_OK : SEPLLM_CUDA_ERROR;
}

template <int D>
sepllm_status launch_prefix_d(const PrefixParams& p, const CUtensorMap& mq, const CUtensorMap& mk,
                              const CUtensorMap& mv, cudaStream_t stream) {
  SEPLLM_CUDA_TRY(cudaFuncSetAttribute(prefix_attn<D>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       int(PfxCfg<D>::kRequest)));
  const dim3 grid(p.alternate ? 1 : (p.m_tiles + 1) / 2, p.Hkv, p.splits);
  prefix_attn<D><<<grid, kPfxThreads, PfxCfg<D>::kRequest, stream>>>(mq, mk, mv, p);
  SEPLLM_CUDA_TRY(cudaGetLastError());
  return SEPLLM_OK;
}

}  // namespace

bool plan_prefix(PrefixParams* p, int B, int Hq, int Hkv, int T, int d, int P) {
  p->B = B;
  p->Hkv = Hkv;
  p->G = Hq / Hkv;
  p->T = T;
  p->d = d;
  p->P = P;
  const int64_t GT = int64_t(p->G) * T;
  p->key_tiles = (P + kBN - 1) / kBN;
  p->rt = int(std::min<int64_t>(GT, 128));
  p->bt = GT <= 128 ? std::min(128 / int(GT), B) : 1;
  p->row_tiles = int((GT + 127) / 128);
  const int64_t m_tiles = GT <= 128 ? (B + p->bt - 1) / p->bt : int64_t(B) * p->row_tiles;
  if (GT > 0x7fffffff || m_tiles > 0x7fffffff || Hkv > 65535 || P > (1 << 30)) return false;
  p->m_tiles = int(m_tiles);
  p->alternate = m_tiles == 1 ? 1 : 0;
  // one CTA per SM: split the key tiles until the SMs are full
  const int64_t units = (p->alternate ? 1 : (m_tiles + 1) / 2) * Hkv;
  int64_t s = std::max<int64_t>(1, 148 / units);
  s = std::min<int64_t>(s, p->alternate ? (p->key_tiles + 1) / 2 : p->key_tiles);
  p->splits = int(s);
  return true;
}

size_t prefix_part_bytes(const PrefixParams& p) {
  const size_t units = size_t(p.B) * p.Hkv * p.G * p.T * (size_t(p.splits) << p.alternate);
  return align_up(units * 2 * sizeof(float)) + align_up(units * kernel_head_dim(p.d) * sizeof(float));
}

void place_prefix_parts(PrefixParams* p, uint8_t* ws) {
  const size_t units = size_t(p->B) * p->Hkv * p->G * p->T * (size_t(p->splits) << p->alternate);
  p->part_ml = reinterpret_cast<float*>(ws);
  p->part_acc = reinterpret_cast<float*>(ws + align_up(units * 2 * sizeof(float)));
}

sepllm_status launch_prefix(const PrefixParams& p, const void* Q, const void* Kp, const void* Vp,
                            cudaStream_t stream) {
  CUtensorMap mq, mk, mv;
  sepllm_status st;
  if ((st = make_query_map(&mq, Q, p)) != SEPLLM_OK) return st;
  if ((st = make_tile_map(&mk, Kp, p.d, p.P, p.Hkv, p.d, int64_t(p.P) * p.d, 128)) != SEPLLM_OK) return st;
  if ((st = make_tile_map(&mv, Vp, p.d, p.P, p.Hkv, p.d, int64_t(p.P) * p.d, 128)) != SEPLLM_OK) return st;
  return kernel_head_dim(p.d) == 64 ? launch_prefix_d<64>(p, mq, mk, mv, stream)
                                    : launch_prefix_d<128>(p, mq, mk, mv, stream);
}

sepllm_status launch_prefix_join(const PrefixParams& p, const float* own_ml, const float* own_acc,
                                 int own_parts, cudaStream_t stream) {
  const int64_t rows = int64_t(p.B) * p.Hkv * p.G * p.T;
  const int64_t blocks = (rows + kJoinWarps - 1) / kJoinWarps;
  if (blocks > 0x7fffffff) return SEPLLM_UNSUPPORTED;
  if (kernel_head_dim(p.d) == 64)
    prefix_join<64><<<unsigned(blocks), kJoinWarps * 32, 0, stream>>>(p, own_ml, own_acc, own_parts, rows);
  else
    prefix_join<128><<<unsigned(blocks), kJoinWarps * 32, 0, stream>>>(p, own_ml, own_acc, own_parts, rows);
  SEPLLM_CUDA_TRY(cudaGetLastError());
  return SEPLLM_OK;
}

}  // namespace sepllm

using namespace sepllm;

// Workspace of a forward behind a prefix: the forward's own | O32 | LSE of the own part | parts.
namespace {
struct AttnPrefixLayout {
  size_t off_o, off_lse, off_parts, bytes;
};
AttnPrefixLayout attn_prefix_layout(const sepllm_attn_desc* d, const sepllm_index_desc* id, const PrefixParams& p) {
  AttnPrefixLayout a;
  const size_t rows = size_t(d->B) * d->Hq * d->L;
  a.off_o = attn_layout(d, id).fwd_bytes;
  a.off_lse = a.off_o + align_up(rows * kernel_head_dim(d->d) * sizeof(float));
  a.off_parts = a.off_lse + align_up(rows * sizeof(float));
  a.bytes = a.off_parts + (p.splits > 1 || p.alternate ? prefix_part_bytes(p) : 0);
  return a;
}
}  // namespace

extern "C" sepllm_status sepllm_attn_prefix_workspace_bytes(const sepllm_attn_desc* desc,
                                                            const sepllm_index_desc* idesc, int32_t P,
                                                            size_t* bytes) {
  sepllm_status st = check_attn(desc, idesc);
  if (st != SEPLLM_OK) return st;
  if (P < 1) return SEPLLM_INVALID_ARG;
  PrefixParams p{};
  if (!plan_prefix(&p, desc->B, desc->Hq, desc->Hkv, desc->L, desc->d, P)) return SEPLLM_UNSUPPORTED;
  if (bytes) *bytes = attn_prefix_layout(desc, idesc, p).bytes;
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
  if (!plan_prefix(&p, desc->B, desc->Hq, desc->Hkv, desc->L, desc->d, P)) return SEPLLM_UNSUPPORTED;
  cudaStream_t stream = static_cast<cudaStream_t>(stream_);
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  const AttnPrefixLayout lay = attn_prefix_layout(desc, idesc, p);
  float* own_O = reinterpret_cast<float*>(ws + lay.off_o);
  float* own_lse = reinterpret_cast<float*>(ws + lay.off_lse);
  // the rows' own tokens first (Eq. 2's mask); their result waits in 32 bits so that O is rounded once
  if ((st = attn_fwd_f32(desc, idesc, Q, K, V, index, own_O, own_lse, ws, stream)) != SEPLLM_OK) return st;
  place_prefix_parts(&p, ws + lay.off_parts);
  p.prefix_len = prefix_len;
  p.seq_len = reinterpret_cast<const int32_t*>(static_cast<const uint8_t*>(index) + ih.off_seq_len);
  p.own_O = own_O;
  p.own_lse = own_lse;
  p.merge_O = p.splits == 1 && !p.alternate;
  p.O = static_cast<__nv_bfloat16*>(O);
  p.LSE = LSE;
  p.status = reinterpret_cast<int32_t*>(ws);
  p.scale_log2 = (desc->scale != 0.f ? desc->scale : 1.0f / sqrtf(float(desc->d))) * 1.4426950408889634f;
  if ((st = launch_prefix(p, Q, Kp, Vp, stream)) != SEPLLM_OK) return st;
  return p.merge_O ? SEPLLM_OK : launch_prefix_join(p, nullptr, nullptr, 0, stream);
}
