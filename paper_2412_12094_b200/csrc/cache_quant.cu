// The streaming cache held in 4 bits: update, prompt hand-off, read-back and decode.
//
// Format.  32 neighbouring elements of a row share a step, a bf16 number s = -m / 8 with m their element
// of largest magnitude (the positive one of two equal ones); an element x is held as the whole number
// q in -8 .. 7 nearest to x / s (the even one of two), so m itself is held exactly and the others to
// half a step, except one of the other sign beyond 7.5 steps.  m is a bf16 number, so s = -m / 8 is
// too: nothing is rounded but q, and codes are the same whatever precision they are computed in.
//
// Buffers.  K and V have one each: codes [B][Hkv][slots][d / 2] bytes, then (256-byte aligned) steps
// [B][Hkv][slots][d / 32].  Slots, rings and the state are those of the 16-bit cache.  Inside a row the
// codes q + 8, two to a byte (the low half first), are ordered so that the decode kernel's threads find
// what their matrix operands need in one word: element e of group j stands at place
// ((e / m) * (d / 32) + j) * m + e % m with m = 8 for keys and m = 4 for values.
#include <cuda_fp16.h>

#include "cache_common.cuh"

namespace sepllm {

namespace {

// Every kernel is launched while the one before it ends (it waits for it first), and lets the next one in.  What
// it reads may therefore still be written when it starts: plain loads behind the wait, none that the compiler or the
// cache may take for constant (const __restrict__, __ldg).

constexpr int kGroup = 32;             // elements that share a step
constexpr float kFlush = 0x1p-100f;    // groups whose largest magnitude is below are held as zeros

// One of Kc / Vc.
template <class Byte>
struct QuantRows {
  Byte* codes;
  Byte* steps;
};
inline size_t quant_code_bytes(const sepllm_cache_header& h) {
  return align_up(size_t(h.desc.B) * h.desc.Hkv * h.slots * (h.desc.d / 2));
}
// What the calls take: ring starts and entries are added in 32 bits.
inline sepllm_status check_quant(const sepllm_cache_desc* d, sepllm_cache_header* h) {
  const sepllm_status st = fill_cache_header(d, h);
  if (st != SEPLLM_OK) return st;
  return int64_t(d->c) + d->s > 1 << 30 ? SEPLLM_UNSUPPORTED : SEPLLM_OK;
}
inline QuantRows<uint8_t> quant_rows(const sepllm_cache_header& h, void* buf) {
  uint8_t* p = static_cast<uint8_t*>(buf);
  return {p, p + quant_code_bytes(h)};
}
inline QuantRows<const uint8_t> quant_rows(const sepllm_cache_header& h, const void* buf) {
  const uint8_t* p = static_cast<const uint8_t*>(buf);
  return {p, p + quant_code_bytes(h)};
}

// Blackwell's packed fp32 arithmetic, two numbers to an instruction, and an approximate reciprocal (2^-23).
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 r;
  asm("{.reg .b64 x, y, z; mov.b64 x, {%2, %3}; mov.b64 y, {%4, %5}; mov.b64 z, {%6, %7}; fma.rn.f32x2 x, x, y, z; "
      "mov.b64 {%0, %1}, x;}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return r;
}
__device__ __forceinline__ float2 sum2(float2 a, float2 b) {
  float2 r;
  asm("{.reg .b64 x, y; mov.b64 x, {%2, %3}; mov.b64 y, {%4, %5}; add.rn.f32x2 x, x, y; mov.b64 {%0, %1}, x;}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return r;
}
__device__ __forceinline__ float reciprocal(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// N x 8 neighbouring elements of a group, whose 4 / N lanes are neighbours; all 32 lanes call.  Returns
// their codes, element e of a word at bits 4e .. 4e + 3, and the bits of the group's step.
//
// A code is found from x * (1 / s), within 2^-20 of x / s.  x / s is either half a whole number
// exactly, or at least 2^-10 away from one (x and s have eight significant bits): rounded to a multiple of
// 2^-13 first (the sum with 1536), ties are ties again and nothing else has become one.  The sum with
// 1.5 * 2^23 + 8 - 1536 rounds to whole numbers, even at a tie, and leaves q + 8 in the low bits.
template <int N>
__device__ __forceinline__ uint32_t quantise(const uint4 (&raw)[N], uint32_t (&codes)[N]) {
  const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(raw);
  // largest and smallest element, as (largest, -smallest); a NaN stays one
  __nv_bfloat162 hi = h[0], lo = h[0];
#pragma unroll
  for (int k = 1; k < 4 * N; ++k) {
    hi = __hmax2_nan(hi, h[k]);
    lo = __hmin2_nan(lo, h[k]);
  }
  lo = __hneg2(lo);
  __nv_bfloat162 m2 = __hmax2_nan(__lows2bfloat162(hi, lo), __highs2bfloat162(hi, lo));
#pragma unroll
  for (int o = 1; o < 4 / N; o <<= 1) {
    const uint32_t other = __shfl_xor_sync(0xffffffffu, *reinterpret_cast<uint32_t*>(&m2), o);
    m2 = __hmax2_nan(m2, *reinterpret_cast<const __nv_bfloat162*>(&other));
  }
  const float2 ends = __bfloat1622float2(m2);
  float s = ends.x >= ends.y ? ends.x * -0.125f : ends.y * 0.125f, r = 0.f;
  if (!(fabsf(ends.x) < INFINITY && fabsf(ends.y) < INFINITY))
    s = __int_as_float(0x7fc00000);   // reads back as NaN in every element
  else if (fabsf(s) < kFlush * 0.125f) s = 0.f;
  else r = reciprocal(s);
#pragma unroll
  for (int n = 0; n < N; ++n) {
    uint32_t w = 0, offset = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float2 f = __bfloat1622float2(h[4 * n + k]);
      const float2 t = fma2(f, make_float2(r, r), make_float2(1536.f, 1536.f));
      // (a NaN, of a group whose step is one, goes with it)
      const float2 q = sum2(make_float2(fminf(t.x, 1543.f), fminf(t.y, 1543.f)), make_float2(12581384.f, 12581384.f));
      w += (__float_as_uint(q.x) << (8 * k)) + (__float_as_uint(q.y) << (8 * k + 4));
      offset += (0x4b400000u << (8 * k)) + (0x4b400000u << (8 * k + 4));
    }
    codes[n] = r == 0.f ? 0x88888888u : w - offset;
  }
  return __float_as_uint(s) >> 16;
}

// Stores the codes of elements 8t .. 8t + 7 of group j of a row (and its step from lane t = 0).
template <int D, bool V>
__device__ __forceinline__ void store_codes(uint8_t* codes, uint8_t* steps, int j, int t, uint32_t w, uint32_t step) {
  constexpr int kGroups = D / kGroup;
  if (!V) {
    reinterpret_cast<uint32_t*>(codes)[t * kGroups + j] = w;
  } else {
    uint16_t* c = reinterpret_cast<uint16_t*>(codes);
    c[2 * t * kGroups + j] = uint16_t(w);
    c[(2 * t + 1) * kGroups + j] = uint16_t(w >> 16);
  }
  if (t == 0) reinterpret_cast<uint16_t*>(steps)[j] = uint16_t(step);
}

// grid (B, Hkv).  As the 16-bit cache's update: every CTA moves the rows of its kv head, the one that
// finishes last for a sequence updates the state.  The new rows are quantised by the first warp; rows that
// move keep their codes.  Bound by latency, one round of loads after another: 4 us for 2 small caches, 8 us for 16
// of 1200 slots, some of them at a compaction.
template <int D>
__global__ void __launch_bounds__(kUpdThreads)
quant_update(sepllm_cache_header h, uint8_t* state, QuantRows<uint8_t> Kc, QuantRows<uint8_t> Vc,
             const __nv_bfloat16* k_new, const __nv_bfloat16* v_new, const int32_t* new_token_ids, SepIds sep,
             int max_past) {
  extern __shared__ int16_t flag_s[];   // [max_past] ranks, [max_past] entries that move
  __shared__ int warp_buf[32];
  constexpr int kVec = D / 8, kCode = D / 2, kStep = D / 16;   // 16-byte pieces of a new row; bytes of a held one
  let_dependents_start();
  wait_for_prior();
  const sepllm_cache_desc& d = h.desc;
  const int b = blockIdx.x, hk = blockIdx.y, tid = threadIdx.x;
  const size_t unit = size_t(b) * d.Hkv + hk;
  uint4 raw[1] = {make_uint4(0, 0, 0, 0)};
  const bool mine = tid < 2 * kVec, is_v = tid >= kVec;   // one warp at most
  if (mine)
    raw[0] = reinterpret_cast<const uint4*>(is_v ? v_new : k_new)[unit * kVec + (is_v ? tid - kVec : tid)];
  CacheView v = cache_view(state, h);
  const sepllm_cache_seq q = v.seq[b];
  const UpdatePlan p = plan_update(q, d);
  uint8_t *kc = Kc.codes + unit * h.slots * kCode, *vc = Vc.codes + unit * h.slots * kCode;
  uint8_t *ks = Kc.steps + unit * h.slots * kStep, *vs = Vc.steps + unit * h.slots * kStep;
  if (tid < 32) {
    uint32_t w[1];
    const uint32_t step = quantise(raw, w);
    const int ch = tid % kVec;
    const size_t slot = p.append_slot;
    if (mine && !is_v) store_codes<D, false>(kc + slot * kCode, ks + slot * kStep, ch / 4, ch % 4, w[0], step);
    if (mine && is_v) store_codes<D, true>(vc + slot * kCode, vs + slot * kStep, ch / 4, ch % 4, w[0], step);
  }
  UpdateMoves mv{p.compact && d.s > 0, 0, 0};
  if (mv.any) {
    mv.m = rank_past_separators(v.slot_is_sep + size_t(b) * h.slots, q, d, p.n_past, flag_s, warp_buf);
    mv.drop = max(0, q.size_sep + mv.m - d.s);
    // The entries that move, in order, then all their pieces over all threads: an entry of 16-byte pieces of its
    // codes and its steps.  (Entry by entry, with most entries staying, the copies of a warp waited for one
    // another: 16 sequences, some at a compaction of 690 entries, took 17 us instead of 8.)
    constexpr int kPieces = kCode / 16, kPer = 2 * kPieces + 2;
    int16_t* list = flag_s + max_past;
    const int first = max(0, mv.drop - q.size_sep), n = mv.m - first;   // of the past separators, those kept
    for (int k = tid; k < p.n_past; k += kUpdThreads)
      if (flag_s[k] > first) list[flag_s[k] - 1 - first] = int16_t(k);
    __syncthreads();
    constexpr int kBatch = 4;   // copies of a thread that are on their way at once
    for (int x0 = tid; x0 < n * kPer; x0 += kBatch * kUpdThreads) {
      uint4 v16[kBatch];
      int dst[kBatch], piece[kBatch];
#pragma unroll
      for (int y = 0; y < kBatch; ++y) {
        const int x = x0 + y * kUpdThreads;
        if (x >= n * kPer) break;
        int src;
        past_move(list[x / kPer], flag_s, q, d, mv.drop, &src, &dst[y]);
        piece[y] = x % kPer;
        if (piece[y] < 2 * kPieces) {
          const uint4* c = reinterpret_cast<const uint4*>(piece[y] < kPieces ? kc : vc);
          v16[y] = c[size_t(src) * kPieces + piece[y] % kPieces];
        } else {
          const uint32_t* st = reinterpret_cast<const uint32_t*>(piece[y] == 2 * kPieces ? ks : vs) + size_t(src) * (kStep / 4);
          v16[y].x = st[0];
          if (kStep == 8) v16[y].y = st[1];
        }
      }
#pragma unroll
      for (int y = 0; y < kBatch; ++y) {
        if (x0 + y * kUpdThreads >= n * kPer) break;
        if (piece[y] < 2 * kPieces) {
          uint4* c = reinterpret_cast<uint4*>(piece[y] < kPieces ? kc : vc);
          c[size_t(dst[y]) * kPieces + piece[y] % kPieces] = v16[y];
        } else {
          uint32_t* st = reinterpret_cast<uint32_t*>(piece[y] == 2 * kPieces ? ks : vs) + size_t(dst[y]) * (kStep / 4);
          st[0] = v16[y].x;
          if (kStep == 8) st[1] = v16[y].y;
        }
      }
    }
  }
  __syncthreads();  // this CTA's append and moves are done
  finish_update(v, h, b, q, next_record(q, d, p, mv), p, mv, flag_s, new_token_ids, sep);
}

constexpr int kCopyThreads = 256;
constexpr int kCopyRows = 32;  // slots (or entries) per CTA (64: hand-off 22.5 us, not 21.5; read-back 13, not 12)

// grid (ceil(slots / kCopyRows), Hkv, B), behind the plan of the hand-off.  Quantises the K and V rows of the
// retained positions into their slots, sixteen elements to a lane (eight: 34 us instead of 26).  All loads of a
// thread are under way at once.  Bound by instructions, 15 an element (issue slots 77 % busy), more than by HBM: 21 us for
// 4 caches of 2700 entries (45 MB read), of which the kernel takes 17 behind the plan.
template <int D>
__global__ void __launch_bounds__(kCopyThreads)
quant_prompt(sepllm_cache_header h, const uint8_t* state, const __nv_bfloat16* K, const __nv_bfloat16* V, int L,
             QuantRows<uint8_t> Kc, QuantRows<uint8_t> Vc) {
  constexpr int kHalf = D / 16, kRowsPerPass = kCopyThreads / (2 * kHalf), kPasses = kCopyRows / kRowsPerPass;
  let_dependents_start();
  wait_for_prior();   // (the plan)
  const sepllm_cache_desc& d = h.desc;
  const int b = blockIdx.z, hk = blockIdx.y, tid = threadIdx.x;
  CacheView v = cache_view(const_cast<uint8_t*>(state), h);
  const sepllm_cache_seq q = v.seq[b];
  const int64_t* pos_b = v.slot_pos + size_t(b) * h.slots;
  const size_t unit = size_t(b) * d.Hkv + hk;
  const bool is_v = tid >= kCopyThreads / 2;   // (a warp has rows of one of them: their stores differ)
  const int sub = tid % (kCopyThreads / 2) / kHalf;
  const int ch = tid % kHalf;  // sixteen elements of the row
  const uint4* src = reinterpret_cast<const uint4*>(is_v ? V : K) + unit * size_t(L) * (D / 8) + 2 * ch;
  const int slot0 = blockIdx.x * kCopyRows + sub;
  // (a slot's position is read beside the sizes that say whether there is one)
  int64_t pos[kPasses];
#pragma unroll
  for (int r = 0; r < kPasses; ++r) pos[r] = pos_b[min(slot0 + r * kRowsPerPass, h.slots - 1)];
  uint4 raw[kPasses][2];
  uint32_t used = 0;
#pragma unroll
  for (int r = 0; r < kPasses; ++r) {
    const int slot = slot0 + r * kRowsPerPass;
    const bool u = slot < d.a             ? slot < q.size_init
                   : slot < d.a + d.s     ? slot - d.a < q.size_sep
                   : slot < h.slots       ? slot - d.a - d.s < q.size_win
                                          : false;
    raw[r][0] = raw[r][1] = make_uint4(0, 0, 0, 0);
    if (u) {
      const uint4* row = src + size_t(pos[r]) * (D / 8);
      raw[r][0] = row[0];
      raw[r][1] = row[1];
    }
    used |= uint32_t(u) << r;
  }
  const QuantRows<uint8_t> out = is_v ? Vc : Kc;
#pragma unroll
  for (int r = 0; r < kPasses; ++r) {
    const bool u = used >> r & 1;
    if (!__any_sync(0xffffffffu, u)) continue;
    uint32_t w[2];
    const uint32_t step = quantise(raw[r], w);
    if (!u) continue;
    const size_t row = unit * h.slots + slot0 + r * kRowsPerPass;
    uint8_t *codes = out.codes + row * (D / 2), *steps = out.steps + row * (D / 16);
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      const int j = ch / 2, t = 2 * (ch % 2) + n;
      if (!is_v) store_codes<D, false>(codes, steps, j, t, w[n], step);
      else store_codes<D, true>(codes, steps, j, t, w[n], step);
    }
  }
}

// (w & mask) | bits in one instruction (of the two constants one may be part of it: `bits` is a register).
template <uint32_t MASK>
__device__ __forceinline__ uint32_t and_or(uint32_t w, uint32_t bits) {
  uint32_t r;
  asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(r) : "r"(w), "n"(MASK), "r"(bits));
  return r;
}
// Two bf16 numbers 128 (not a constant to the compiler, which would split and_or()).
__device__ __forceinline__ uint32_t two_128() {
  uint32_t r;
  asm volatile("mov.b32 %0, 0x43004300;" : "=r"(r));
  return r;
}

// The low four bits of w's halves, less 8, as two bf16 numbers: 128 + c by a mask, minus 136 (exact).
__device__ __forceinline__ uint32_t two_codes(uint32_t w, uint32_t k128) {
  const uint32_t n = and_or<0x000f000fu>(w, k128);
  const __nv_bfloat162 q = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&n), __float2bfloat162_rn(136.f));
  return *reinterpret_cast<const uint32_t*>(&q);
}

// Eight codes (element e at bits 4e ..) times their step, rounded to bf16 once (the product has up to
// twelve significant bits, bf16 eight).
__device__ __forceinline__ uint4 values8(uint32_t w, __nv_bfloat16 step, uint32_t k128) {
  uint32_t p[4];   // elements k and k + 4
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const uint32_t q = two_codes(w >> (4 * k), k128);
    const __nv_bfloat162 v = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&q), __bfloat162bfloat162(step));
    p[k] = *reinterpret_cast<const uint32_t*>(&v);
  }
  return make_uint4(__byte_perm(p[0], p[1], 0x5410), __byte_perm(p[2], p[3], 0x5410), __byte_perm(p[0], p[1], 0x7632),
                    __byte_perm(p[2], p[3], 0x7632));
}

// grid (ceil(c / kCopyRows), Hkv, B).  Row v of K and V of sequence b is its retained entry v.  18.6 us for 16 caches
// of 1195 entries (100 MB), 12 us for 4 of 2700, 5 us for the smallest.  Bound by instructions and their latency, not by HBM
// (issue slots 55 and 63 % busy, DRAM 26 and 13 %: most of what it writes is still in L2 when it ends): a lane turns
// eight elements from one word and two half words of codes and two steps.
template <int D>
__global__ void __launch_bounds__(kCopyThreads)
quant_entries(sepllm_cache_header h, const uint8_t* state, QuantRows<const uint8_t> Kc, QuantRows<const uint8_t> Vc,
              int n, __nv_bfloat16* __restrict__ K, __nv_bfloat16* __restrict__ V, int32_t* length) {
  constexpr int kVec = D / 8, kGroups = D / kGroup, kRowsPerPass = kCopyThreads / kVec;
  let_dependents_start();
  wait_for_prior();
  const sepllm_cache_desc& d = h.desc;
  const int b = blockIdx.z, hk = blockIdx.y;
  CacheView cv = cache_view(const_cast<uint8_t*>(state), h);
  const sepllm_cache_seq q = cv.seq[b];
  const int run = min(n, q.size_init + q.size_sep + q.size_win);
  if (length && blockIdx.x == 0 && hk == 0 && threadIdx.x == 0) length[b] = run;
  const int ch = threadIdx.x % kVec, j = ch / 4, t = ch % 4;
  const size_t unit = size_t(b) * d.Hkv + hk;
  const uint32_t k128 = two_128();
#pragma unroll
  for (int r = 0; r < kCopyRows; r += kRowsPerPass) {
    const int v = blockIdx.x * kCopyRows + r + threadIdx.x / kVec;
    if (v >= run) return;
    const size_t row = unit * h.slots + virtual_to_slot(v, q, d);
    const uint32_t wk = reinterpret_cast<const uint32_t*>(Kc.codes + row * (D / 2))[t * kGroups + j];
    const uint16_t* vc = reinterpret_cast<const uint16_t*>(Vc.codes + row * (D / 2));
    const uint32_t wv = vc[2 * t * kGroups + j] | uint32_t(vc[(2 * t + 1) * kGroups + j]) << 16;
    const __nv_bfloat16 sk = reinterpret_cast<const __nv_bfloat16*>(Kc.steps)[row * kGroups + j];
    const __nv_bfloat16 sv = reinterpret_cast<const __nv_bfloat16*>(Vc.steps)[row * kGroups + j];
    const size_t dst = (unit * n + v) * kVec + ch;
    reinterpret_cast<uint4*>(K)[dst] = values8(wk, sk, k128);
    reinterpret_cast<uint4*>(V)[dst] = values8(wv, sv, k128);
  }
}

// ---------------------------------------------------------------------------
// Decode
// ---------------------------------------------------------------------------
constexpr int kDecThreads = 128, kDecWarps = kDecThreads / 32;
constexpr int kTile = 32;                        // entries of a warp's tile
constexpr int kStepRows = kDecWarps * kTile;     // entries of a CTA's step

// D[16 keys x 8 columns] = A[16 x 32] B[32 x 8] + C, e4m3 operands.
__device__ __forceinline__ void mma_e4m3(float (&d)[4], const uint32_t (&a)[4], const uint32_t (&b)[2],
                                         float c0, float c1, float c2, float c3) {
  asm(
      "mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
      "{%8, %9}, {%10, %11, %12, %13};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]), "f"(c0), "f"(c1), "f"(c2), "f"(c3));
}
__device__ __forceinline__ void mma_bf16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                         uint32_t b0, uint32_t b1) {
  asm(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
      "{%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Transposes an 8 x 8 matrix of 16-bit elements held two to a lane.
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
template <int BYTES>
__device__ __forceinline__ void cp_async_small(uint32_t dst, const void* src, uint32_t src_bytes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(dst), "l"(src), "n"(BYTES), "r"(src_bytes)
               : "memory");
}
__device__ __forceinline__ float bf16_low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_high(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
// Two e4m3 numbers, lo in the low byte, and back.
__device__ __forceinline__ uint32_t pack_e4m3(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ float2 unpack_e4m3(uint32_t w) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(uint16_t(w)));
  return __half22float2(*reinterpret_cast<__half2*>(&h));
}

struct QuantDecodeParams {
  sepllm_cache_header h;
  const uint8_t* state;
  const __nv_bfloat16* q;
  QuantRows<const uint8_t> Kc, Vc;
  __nv_bfloat16* o;
  float* lse;
  int4* ends;        // [CTA] b, hk of the unit that began with this CTA and ends with a later one, and that CTA; -1: none
  float2* part_ml;   // [2 * CTA + (0: the former, 1: the latter)][G] reference exponent and sum
  float* part_acc;   // [same][G][D]
  int32_t* status;
  float scale_log2;
  int whole;         // 1: a CTA for every unit, and no parts
};

__device__ __forceinline__ int run_of(const sepllm_cache_seq& s) { return s.size_init + s.size_sep + s.size_win; }
// Steps of a sequence's kv head; one for an empty sequence, whose output has to be written too.
__device__ __forceinline__ int steps_of(const sepllm_cache_seq& s) {
  return max(1, (run_of(s) + kStepRows - 1) / kStepRows);
}
// Slot of entry v, and the first entry behind v whose slot does not follow its predecessor's.
__device__ __forceinline__ int contiguous_from(int v, const sepllm_cache_seq& q, const sepllm_cache_desc& d, int* end) {
  const int i = q.size_init, is = i + q.size_sep;
  *end = i;
  if (v < i) return v;
  const bool sep = v < is;
  const int x = sep ? q.sep_start + v - i : q.win_start + v - is;    // place in the ring, before the turn
  const int ring = sep ? d.s : d.c - d.a, first = sep ? d.a : d.a + d.s;
  *end = sep ? is : 0x7fffffff;
  if (x >= ring) return first + x - ring;
  *end = min(*end, v + ring - x);
  return first + x;
}

// The CTA's share.  The steps of all (sequence, kv head) units, laid end to end, are cut into equal runs,
// one per CTA: sequences of any lengths load the SMs evenly, and a unit is cut at most where a CTA's run
// ends.  All threads call; false: nothing is left for this CTA.
struct Share {
  int b, hk, step;            // where the run starts
  int64_t left;               // its steps
  int64_t total, end;         // all steps, and where the run ends among them
};
// (32-bit divisions wherever the numbers allow)
__device__ __forceinline__ uint64_t quotient(uint64_t a, uint32_t b) {
  return a >> 32 ? a / b : uint32_t(a) / b;
}
__device__ bool share_of(const sepllm_cache_seq* seq, int B, int Hkv, Share* out) {
  __shared__ int64_t s_sum[kDecWarps];
  __shared__ int64_t s_first;
  __shared__ int s_b, s_n;
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  const int n0 = tid < B ? steps_of(seq[tid]) : 0;   // of the first sequences, one to a thread
  int64_t sum = n0;
  for (int b = tid + kDecThreads; b < B; b += kDecThreads) sum += steps_of(seq[b]);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (lane == 0) s_sum[wid] = sum;
  __syncthreads();
  int64_t total = 0;
#pragma unroll
  for (int w = 0; w < kDecWarps; ++w) total += s_sum[w];
  total *= Hkv;
  const uint32_t ctas = uint32_t(min(int64_t(gridDim.x), total));
  if (blockIdx.x >= ctas) return false;
  const int64_t first = quotient(total * blockIdx.x, ctas), last = quotient(total * (blockIdx.x + 1), ctas);
  const int64_t target = quotient(first, Hkv);   // in steps of one kv head
  int64_t before = 0;                            // steps of the sequences before this chunk
  for (int b0 = 0; b0 < B; b0 += kDecThreads) {
    const int b = b0 + tid;
    const int n = b0 == 0 ? n0 : b < B ? steps_of(seq[b]) : 0;
    int64_t incl = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t x = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += x;
    }
    __syncthreads();
    if (lane == 31) s_sum[wid] = incl;
    __syncthreads();
    int64_t chunk = 0;
#pragma unroll
    for (int w = 0; w < kDecWarps; ++w) {
      if (w < wid) incl += s_sum[w];
      chunk += s_sum[w];
    }
    incl += before;
    before += chunk;
    if (n > 0 && incl - n <= target && target < incl) {
      s_b = b;
      s_n = n;
      s_first = incl - n;
    }
    if (target < before) break;   // (the same for all threads)
  }
  __syncthreads();
  out->b = s_b;
  const int n = s_n;
  const int64_t in_seq = first - s_first * Hkv;
  out->hk = int(quotient(in_seq, n));
  out->step = int(in_seq - int64_t(out->hk) * n);
  out->left = last - first;
  out->total = total;
  out->end = last;
  return true;
}

// Shapes of the kernel for groups of up to H query heads per kv head (4, 8 or 16).
template <int D, int H>
struct DecodeShape {
  static constexpr bool kSplit = H == 4;                  // the two parts of q are columns of one product
  static constexpr int NT = H == 16 ? 2 : 1;              // tiles of 8 columns
  static constexpr int kGroups = D / kGroup;
  static constexpr int kCode = D / 2, kStep = D / 16;     // bytes of a row
  static constexpr int kStageB = 2 * kTile * (kCode + kStep);
  // CTAs per SM.  Three: at most 168 registers a thread; four spill (D = 128, H = 4: 61 us instead of 33 for 32
  // caches of 2750 entries).  A fourth stage would take the L1 from what little is spilled (35 us).
  static constexpr int kResident = D == 128 && H == 16 ? 2 : 3;
  static constexpr int kStages = 3;
  // shared memory: the warps' rings, in whose last stages the warps' results stand at a unit's end while the
  // first tiles of the next unit are on their way into the others, and the queries
  static constexpr int kRingB = kDecWarps * kStages * kStageB;
  static constexpr int kEarly = kStages - (H * (D * 4 + 8) + kStageB - 1) / kStageB;   // tiles that may be on their way
  static_assert(kEarly >= 1 && kEarly < kStages, "a warp's results fit into its last stages");
  static constexpr int kQWords = kSplit ? kGroups * 2 * 32 : NT * kGroups * 4 * 32;
  static constexpr int kSmem = kRingB + kQWords * 4 + H * (kGroups + 1) * 4;
};

// 4 warps a CTA; each is a flash-decoding worker over its 32-entry tiles of the CTA's steps, which arrive
// through a ring of cp.async stages.  The products have entries (or elements of V) as the M dimension
// and the G <= H query heads of the kv head as columns.
//
// K q: the e4m3 number with bits 0000cccc is cccc * 2^-9 for every code c, so a word of eight codes becomes
// two operand registers with two masks and a shift.  q is brought near 2^7 by a power of two and split into
// two e4m3 numbers, which hold its eight bits exactly down to 2^-9 of the head's largest element (and
// lose 2^-17 of that below); the products are exact and summed in 32 bits.  The codes' offset 8 is taken
// off by the accumulator's start, -8 times the sum of q over the group, and the key's step multiplies
// the group's 32-bit sum.  Up to four heads: the parts are columns 2h and 2h + 1 of one product.
//
// P V: codes become bf16 128 + c with one mask-and-or (two entries of a word pair to a register), and exact whole
// numbers -8 .. 7 with one packed subtraction.  (The offset 136 could instead be taken off the sums at the end, by a
// product with ones.  But a product's sum is cut off, not rounded, when it is added to an accumulator: with the offset
// in the sums, thirty times a typical code, the output of a CTA that walks 100 000 entries alone was off by
// 3 % where weights are spread out, and no faster: 33.0 and 64.4 us against 32.1 and 62.5 for the two cases below.)
// P times the group's step is rounded to bf16 (2^-8), the only rounding here.
//
// The tensor work is small (16 columns at most; the pipe is a quarter busy), so the products are those whose operands
// come from registers: codes go from the ring through a mask each into an operand, never back to shared memory.
// Measured, H = 4, D = 128: 32 caches of 2750 entries in 31 us, 2 of 112 000 in 62 us (4.1 TB/s; reading those
// bytes cold takes 49 to 53), then the join, 2 us behind it.  ALU pipe 59 % and issue slots 61 % busy, DRAM 49 %: nothing
// is full.  A warp's tile is one chain (copy, scores, softmax, shuffles, values) and 12 warps an SM do not overlap
// the chains fully.  H = 8: 40 and 76 us, H = 16: 59 and 116 us (two score products for each group, transposes, and at D =
// 128, H = 16 two CTAs an SM); D = 64: 20, 24 and 34 us for the 32 caches.
template <int D, int H>
__global__ void __launch_bounds__(kDecThreads, DecodeShape<D, H>::kResident)
decode_quant(const __grid_constant__ QuantDecodeParams p) {
  using S = DecodeShape<D, H>;
  constexpr int kGroups = S::kGroups, kCode = S::kCode, kStep = S::kStep, NT = S::NT, kStages = S::kStages;
  constexpr bool kSplit = S::kSplit;
  constexpr int NE = kSplit ? 1 : 2;   // heads of a lane's scores: t, or 8n + 2t and 8n + 2t + 1
  extern __shared__ __align__(128) uint8_t dec_smem[];
  uint32_t* s_q = reinterpret_cast<uint32_t*>(dec_smem + S::kRingB);
  float* s_start = reinterpret_cast<float*>(s_q + S::kQWords);   // [head][group]
  float* s_factor = s_start + H * kGroups;                        // [head]
  let_dependents_start();
  wait_for_prior();
  const sepllm_cache_desc& d = p.h.desc;
  const int G = d.Hq / d.Hkv;
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  const int g = lane >> 2, t = lane & 3;
  if (tid == 0 && blockIdx.x == 0) *p.status = SEPLLM_OK;
  const sepllm_cache_seq* seqs = cache_view(const_cast<uint8_t*>(p.state), p.h).seq;
  Share sh{};
  if (p.whole) {
    sh.b = blockIdx.x / d.Hkv;
    sh.hk = blockIdx.x - sh.b * d.Hkv;
    sh.left = steps_of(seqs[sh.b]);
  } else if (!share_of(seqs, d.B, d.Hkv, &sh)) {
    if (tid == 0) p.ends[blockIdx.x] = make_int4(-1, -1, -1, -1);
    return;
  }
  const uint32_t k128 = two_128();
  uint8_t* ring = dec_smem + wid * (kStages * S::kStageB);
  const uint32_t ring_u = smem_u32(ring);
  int4 ends = make_int4(-1, -1, -1, -1);

  // The unit at hand: entries v0 to v1 of sequence sh.b's kv head sh.hk are this CTA's.
  constexpr int kPieces = kCode / 16, kRows = 32 / kPieces;   // 16-byte pieces of a row; rows of one copy of the warp
  static_assert(kRows % 8 == 0, "a lane's places in the rows of a stage differ by whole copies");
  constexpr int kPer = D / 8;                                 // threads that load a query head, eight elements each
  constexpr int kQLoads = (H * kPer + kDecThreads - 1) / kDecThreads;
  const int r0 = lane / kPieces, c0 = lane % kPieces;
  sepllm_cache_seq sq;
  int steps, n_steps, v0, v1, my_n;
  uint32_t row0;            // of slot 0 among all rows
  int run_end, run_slot;    // entries up to run_end have slots run_slot + entry
  uint4 q_raw[kQLoads];
  auto begin_unit = [&]() {
    sq = seqs[sh.b];
    steps = steps_of(sq);
    n_steps = int(min(sh.left, int64_t(steps - sh.step)));
    v0 = sh.step * kStepRows;
    v1 = min(run_of(sq), (sh.step + n_steps) * kStepRows);
    const int n_tiles = (v1 - v0 + kTile - 1) / kTile;
    my_n = n_tiles > wid ? (n_tiles - wid + kDecWarps - 1) / kDecWarps : 0;
    row0 = uint32_t((size_t(sh.b) * d.Hkv + sh.hk) * p.h.slots);
    run_end = run_slot = 0;
#pragma unroll
    for (int x = 0; x < kQLoads; ++x) {
      const int c = x * kDecThreads + tid, head = c / kPer;
      q_raw[x] = head < G ? reinterpret_cast<const uint4*>(p.q + (size_t(sh.b) * d.Hq + sh.hk * G + head) * D)[c % kPer]
                          : make_uint4(0, 0, 0, 0);
    }
  };
  // This warp's i-th tile into stage i % kStages: codes of K and V, steps of K and V.  Rows behind v1 are
  // zeros.  The 16-byte pieces of V rows of 64 bytes are turned, so that the threads' reads below meet
  // different banks.
  auto dst_v = [&](int r) {   // place of this lane's piece of V row r in a stage
    const int rv = kSplit ? r : (r & ~7) | (r >> 1 & 3) | (r & 1) << 2;
    return kTile * kCode + rv * kCode + (kPieces == 4 ? c0 ^ (rv & 2) : c0) * 16;
  };
  const uint32_t dst0 = ring_u + r0 * kCode + c0 * 16, dst1 = ring_u + dst_v(r0);
  const uint32_t dst2 = ring_u + 2 * kTile * kCode + lane * kStep;
  auto issue = [&](int i) {
    const int vb = v0 + (wid + i * kDecWarps) * kTile;
    const uint32_t stage = (i % kStages) * S::kStageB;
    if (vb >= run_end) run_slot = contiguous_from(vb, sq, d, &run_end) - vb;
    if (vb + kTile <= min(run_end, v1)) {   // 32 neighbouring slots
      const uint32_t row = row0 + run_slot + vb;
      const uint64_t codes = uint64_t(row) * kCode + lane * 16, steps_at = uint64_t(row + lane) * kStep;
      cp_async_small<kStep>(stage + dst2, p.Kc.steps + steps_at, kStep);
      cp_async_small<kStep>(stage + dst2 + kTile * kStep, p.Vc.steps + steps_at, kStep);
#pragma unroll
      for (int x = 0; x < kTile / kRows; ++x) {
        cp_async16(stage + dst0 + x * kRows * kCode, p.Kc.codes + codes + x * kRows * kCode, 16);
        cp_async16(stage + dst1 + x * kRows * kCode, p.Vc.codes + codes + x * kRows * kCode, 16);
      }
    } else {
      const uint32_t ok = vb + lane < v1;
      const uint32_t row = row0 + virtual_to_slot(min(vb + lane, v1 - 1), sq, d);
      cp_async_small<kStep>(stage + dst2, p.Kc.steps + uint64_t(row) * kStep, ok * kStep);
      cp_async_small<kStep>(stage + dst2 + kTile * kStep, p.Vc.steps + uint64_t(row) * kStep, ok * kStep);
#pragma unroll
      for (int x = 0; x < kTile / kRows; ++x) {
        const int r = x * kRows + r0;
        const uint64_t off = uint64_t(__shfl_sync(0xffffffffu, row, r)) * kCode + c0 * 16;
        const uint32_t bytes = vb + r < v1 ? 16u : 0u;
        cp_async16(stage + dst0 + x * kRows * kCode, p.Kc.codes + off, bytes);
        cp_async16(stage + dst1 + x * kRows * kCode, p.Vc.codes + off, bytes);
      }
    }
  };
  auto issue_tiles = [&](int from, int to) {
    for (int i = from; i < to; ++i) {
      if (i < my_n) issue(i);
      cp_async_commit();
    }
  };

  begin_unit();
  issue_tiles(0, S::kEarly);
  while (true) {
    // The queries as operand words: elements 32j + 8t ..
#pragma unroll
    for (int x0 = 0; x0 < kQLoads; ++x0) {
      const int c = x0 * kDecThreads + tid, head = c / kPer, j = c % kPer / 4;
      if (H * kPer < kDecThreads && c >= H * kPer) break;   // (whole warps)
      const uint4 raw = q_raw[x0];
      const __nv_bfloat162* x = reinterpret_cast<const __nv_bfloat162*>(&raw);
      float2 f[4];
      float most = 0.f;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        f[k] = __bfloat1622float2(x[k]);
        most = fmaxf(most, fmaxf(fabsf(f[k].x), fabsf(f[k].y)));
      }
#pragma unroll
      for (int o = 1; o < kPer; o <<= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
      // 2^e with most * 2^e in [128, 256) (2^e and its inverse stay normal numbers)
      const int e = max(-110, min(110, 134 - int(__float_as_uint(most) >> 23)));
      const float up = __uint_as_float(uint32_t(127 + e) << 23);
      float sum = 0.f;
      uint32_t hi[2] = {0, 0}, lo[2] = {0, 0};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        f[k].x *= up;
        f[k].y *= up;
        // (e4m3 ends at 448: where e is at its end, elements from 1.75 * 2^118 on and infinite ones become NaN)
        if (!(fabsf(f[k].x) < 448.f)) f[k].x = __int_as_float(0x7fc00000);
        if (!(fabsf(f[k].y) < 448.f)) f[k].y = __int_as_float(0x7fc00000);
        const uint32_t a = pack_e4m3(f[k].x, f[k].y);
        const float2 fa = unpack_e4m3(a);
        const uint32_t b = pack_e4m3(f[k].x - fa.x, f[k].y - fa.y);
        const float2 fb = unpack_e4m3(b);
        sum += (fa.x + fb.x) + (fa.y + fb.y);
        hi[0] |= (a & 255) << (8 * k);
        hi[1] |= (a >> 8) << (8 * k);
        lo[0] |= (b & 255) << (8 * k);
        lo[1] |= (b >> 8) << (8 * k);
      }
      sum += __shfl_xor_sync(0xffffffffu, sum, 1);
      sum += __shfl_xor_sync(0xffffffffu, sum, 2);
      const int tt = c % 4;
      if (kSplit) {
        // column 2 head (+ 1): [group][register][lane]
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          s_q[(j * 2 + r) * 32 + head * 8 + tt] = hi[r];
          s_q[(j * 2 + r) * 32 + head * 8 + 4 + tt] = lo[r];
        }
      } else {
        const int n = head / 8;
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          s_q[((n * kGroups + j) * 4 + r) * 32 + (head % 8) * 4 + tt] = hi[r];
          s_q[((n * kGroups + j) * 4 + 2 + r) * 32 + (head % 8) * 4 + tt] = lo[r];
        }
      }
      if (tt == 0) s_start[head * kGroups + j] = sum * (-8.f * 0x1p-9f);
      if (c % kPer == 0) s_factor[head] = p.scale_log2 * __uint_as_float(uint32_t(127 + 9 - e) << 23);
    }
    __syncthreads();   // (and the merge before this unit is over: the last stages are free)
    issue_tiles(S::kEarly, kStages - 1);
    uint32_t q_hi[NT][kGroups][2], q_lo[NT][kGroups][2];   // (kSplit: q_hi alone)
    float start[NT][kGroups][NE], factor[NT][NE];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int j = 0; j < kGroups; ++j) {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          if (kSplit) {
            q_hi[n][j][r] = s_q[(j * 2 + r) * 32 + lane];
          } else {
            q_hi[n][j][r] = s_q[((n * kGroups + j) * 4 + r) * 32 + lane];
            q_lo[n][j][r] = s_q[((n * kGroups + j) * 4 + 2 + r) * 32 + lane];
          }
        }
#pragma unroll
        for (int e = 0; e < NE; ++e) start[n][j][e] = s_start[(kSplit ? t : 8 * n + 2 * t + e) * kGroups + j];
      }
#pragma unroll
      for (int e = 0; e < NE; ++e) factor[n][e] = s_factor[kSplit ? t : 8 * n + 2 * t + e];
    }

    // Sums: rows are elements of V, columns 2t and 2t + 1 the heads 8n + 2t and 8n + 2t + 1 (kSplit: columns 4 to
    // 7 repeat 0 to 3).  m_ref: reference exponent, -inf before the first score; m_use: 0 in its place.
    float oacc[2 * kGroups][NT][4];
    float m_ref[NT][NE], m_use[NT][NE], l_sum[NT][NE];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int j = 0; j < 2 * kGroups; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) oacc[j][n][e] = 0.f;
#pragma unroll
      for (int e = 0; e < NE; ++e) {
        m_ref[n][e] = -INFINITY;
        m_use[n][e] = l_sum[n][e] = 0.f;
      }
    }

    // Scores of the warp's i-th tile: of entries 16x + 8y + g, [2x + y].
    auto scores = [&](int i, float (&sc)[4][NT][NE]) {
      const uint8_t* sK = ring + (i % kStages) * S::kStageB;
      const uint8_t* sks = sK + 2 * kTile * kCode;
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        uint32_t w[2][kGroups], st[2][kGroups / 2];
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const int r = 16 * x + 8 * y + g;
          const uint32_t* src = reinterpret_cast<const uint32_t*>(sK + r * kCode) + t * kGroups;
          const uint32_t* ssrc = reinterpret_cast<const uint32_t*>(sks + r * kStep);
          if constexpr (kGroups == 4) {
            *reinterpret_cast<uint4*>(w[y]) = *reinterpret_cast<const uint4*>(src);
            *reinterpret_cast<uint2*>(st[y]) = *reinterpret_cast<const uint2*>(ssrc);
          } else {
            *reinterpret_cast<uint2*>(w[y]) = *reinterpret_cast<const uint2*>(src);
            st[y][0] = *ssrc;
          }
        }
#pragma unroll
        for (int j = 0; j < kGroups; ++j) {
          const uint32_t a[4] = {w[0][j] & 0x0f0f0f0fu, w[1][j] & 0x0f0f0f0fu, w[0][j] >> 4 & 0x0f0f0f0fu,
                                 w[1][j] >> 4 & 0x0f0f0f0fu};
          const float s0 = j & 1 ? bf16_high(st[0][j / 2]) : bf16_low(st[0][j / 2]);
          const float s1 = j & 1 ? bf16_high(st[1][j / 2]) : bf16_low(st[1][j / 2]);
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            float c[4];
            if constexpr (kSplit) {
              mma_e4m3(c, a, q_hi[n][j], start[n][j][0], 0.f, start[n][j][0], 0.f);
              c[0] += c[1];
              c[1] = c[2] + c[3];
              sc[2 * x][n][0] = j == 0 ? c[0] * s0 : sc[2 * x][n][0] + c[0] * s0;
              sc[2 * x + 1][n][0] = j == 0 ? c[1] * s1 : sc[2 * x + 1][n][0] + c[1] * s1;
            } else {
              mma_e4m3(c, a, q_hi[n][j], start[n][j][0], start[n][j][NE - 1], start[n][j][0], start[n][j][NE - 1]);
              mma_e4m3(c, a, q_lo[n][j], c[0], c[1], c[2], c[3]);
#pragma unroll
              for (int e = 0; e < NE; ++e) {
                sc[2 * x][n][e] = j == 0 ? c[e] * s0 : sc[2 * x][n][e] + c[e] * s0;
                sc[2 * x + 1][n][e] = j == 0 ? c[2 + e] * s1 : sc[2 * x + 1][n][e] + c[2 + e] * s1;
              }
            }
          }
        }
      }
    };
    // Scores to weights, in log2 units; the reference moves up when a score is beyond 2^8 of it.
    auto softmax = [&](int i, float (&sc)[4][NT][NE]) {
      const int vb = v0 + (wid + i * kDecWarps) * kTile;
      bool above = false;
      float top[NT][NE];
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < NE; ++e) {
#pragma unroll
          for (int y = 0; y < 4; ++y) sc[y][n][e] *= factor[n][e];
          if (vb + kTile > v1) {
#pragma unroll
            for (int y = 0; y < 4; ++y)
              if (vb + 8 * y + g >= v1) sc[y][n][e] = -INFINITY;
          }
          top[n][e] = fmaxf(fmaxf(sc[0][n][e], sc[1][n][e]), fmaxf(sc[2][n][e], sc[3][n][e]));
          above |= top[n][e] > m_ref[n][e] + 8.f;
        }
      if (__any_sync(0xffffffffu, above)) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          float corr[2];   // of the columns 2t and 2t + 1
#pragma unroll
          for (int e = 0; e < NE; ++e) {
            float mx = top[n][e];
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
            corr[e] = 1.f;
            if (mx > m_ref[n][e] + 8.f) {
              corr[e] = m_ref[n][e] == -INFINITY ? 0.f : ex2(m_ref[n][e] - mx);
              m_ref[n][e] = m_use[n][e] = mx;
              l_sum[n][e] *= corr[e];
            }
          }
          if (kSplit) {
            const float mine = corr[0];
            corr[0] = __shfl_sync(0xffffffffu, mine, 2 * t & 3);
            corr[1] = __shfl_sync(0xffffffffu, mine, (2 * t + 1) & 3);
          }
#pragma unroll
          for (int e = 0; e < 2; ++e) {
#pragma unroll
            for (int j = 0; j < 2 * kGroups; ++j) {
              oacc[j][n][e] *= corr[e];
              oacc[j][n][e + 2] *= corr[e];
            }
          }
        }
      }
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < NE; ++e) {
#pragma unroll
          for (int y = 0; y < 4; ++y) sc[y][n][e] = ex2(sc[y][n][e] - m_use[n][e]);
          l_sum[n][e] += (sc[0][n][e] + sc[1][n][e]) + (sc[2][n][e] + sc[3][n][e]);
        }

    };
    // The tile's weights times its values.
    auto values = [&](int i, const float (&sc)[4][NT][NE]) {
      const uint8_t* sV = ring + (i % kStages) * S::kStageB + kTile * kCode;
      const uint8_t* svs = sV + kTile * kCode + kTile * kStep;
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        // The four entries of the half tile that a lane's operand registers hold: two of a[0], a[1] and two of
        // a[2], a[3].  kSplit: t and t + 8, t + 4 and t + 12; else 2t and 2t + 1, 2t + 8 and 2t + 9.
        uint32_t w[4][kGroups / 2], st[2][kGroups / 2];
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          const int r = 16 * x + (kSplit ? t + 8 * (y & 1) + 4 * (y >> 1) : 2 * t + (y & 1) + 8 * (y >> 1));
          const int rv = kSplit ? r : (r & ~7) | (r >> 1 & 3) | (r & 1) << 2;
          if constexpr (kGroups == 4) {
            const int piece = (g >> 1) ^ (rv & 2);
            *reinterpret_cast<uint2*>(w[y]) =
                *reinterpret_cast<const uint2*>(sV + rv * kCode + piece * 16 + (g & 1) * 8);
          } else {
            w[y][0] = *reinterpret_cast<const uint32_t*>(sV + rv * kCode + g * 4);
          }
        }
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const uint32_t* ssrc = reinterpret_cast<const uint32_t*>(svs + (16 * x + 8 * y + g) * kStep);
          if constexpr (kGroups == 4) *reinterpret_cast<uint2*>(st[y]) = *reinterpret_cast<const uint2*>(ssrc);
          else st[y][0] = *ssrc;
        }
#pragma unroll
        for (int j = 0; j < kGroups; ++j) {
          const float s0 = j & 1 ? bf16_high(st[0][j / 2]) : bf16_low(st[0][j / 2]);
          const float s1 = j & 1 ? bf16_high(st[1][j / 2]) : bf16_low(st[1][j / 2]);
          uint32_t pb[NT][2];
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            if constexpr (kSplit) {
              // column g is head g % 4; its entries t and t + 8 are with the lane of row t and head g % 4
              const uint32_t u = pack_bf16(sc[2 * x][n][0] * s0, sc[2 * x + 1][n][0] * s1);
              pb[n][0] = __shfl_sync(0xffffffffu, u, 4 * t + (g & 3));
              pb[n][1] = __shfl_sync(0xffffffffu, u, 4 * t + 16 + (g & 3));
            } else {
              pb[n][0] = transpose8(pack_bf16(sc[2 * x][n][0] * s0, sc[2 * x][n][NE - 1] * s0));
              pb[n][1] = transpose8(pack_bf16(sc[2 * x + 1][n][0] * s1, sc[2 * x + 1][n][NE - 1] * s1));
            }
          }
          const uint32_t u = __byte_perm(w[0][j / 2], w[1][j / 2], j & 1 ? 0x7632 : 0x5410);
          const uint32_t z = __byte_perm(w[2][j / 2], w[3][j / 2], j & 1 ? 0x7632 : 0x5410);
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const uint32_t a0 = two_codes(u >> (8 * half), k128), a1 = two_codes(u >> (8 * half + 4), k128);
            const uint32_t a2 = two_codes(z >> (8 * half), k128), a3 = two_codes(z >> (8 * half + 4), k128);
#pragma unroll
            for (int n = 0; n < NT; ++n) mma_bf16(oacc[2 * j + half][n], a0, a1, a2, a3, pb[n][0], pb[n][1]);
          }
        }
      }
    };

    float sc[4][NT][NE];
    for (int i = 0; i < my_n; ++i) {
      cp_async_wait<kStages - 2>();
      __syncwarp();
      if (i + kStages - 1 < my_n) issue(i + kStages - 1);   // (over tile i - 1, which all lanes are done with)
      cp_async_commit();
      scores(i, sc);
      softmax(i, sc);
      values(i, sc);
      __syncwarp();
    }
    cp_async_wait<0>();
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < NE; ++e)
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) l_sum[n][e] += __shfl_xor_sync(0xffffffffu, l_sum[n][e], o);

    // The warps' results, head by head, behind the stages that the next unit's first tiles go to; then merged:
    // the unit's output, or a part of it.
    constexpr int kWarpB = kStages * S::kStageB, kResultB = S::kEarly * S::kStageB;
    auto ml_of = [&](int w) { return reinterpret_cast<float2*>(dec_smem + w * kWarpB + kResultB); };
    auto acc_of = [&](int w) { return reinterpret_cast<float*>(dec_smem + w * kWarpB + kResultB + H * 8); };
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int e = 0; e < NE; ++e)
        if (g == 0) ml_of(wid)[kSplit ? t : 8 * n + 2 * t + e] = make_float2(m_ref[n][e], l_sum[n][e]);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int head = 8 * n + 2 * t + e;
        if (head < G) {
#pragma unroll
          for (int j = 0; j < 2 * kGroups; ++j)
            *reinterpret_cast<float2*>(acc_of(wid) + head * D + (j / 2) * kGroup + 4 * g + 2 * (j & 1)) =
                make_float2(oacc[j][n][e], oacc[j][n][e + 2]);
        }
      }
    }
    const bool head_cut = sh.step > 0, tail_cut = sh.step + n_steps < steps;
    const size_t part = 2 * size_t(blockIdx.x) + (head_cut ? 0 : 1), out0 = size_t(sh.b) * d.Hq + sh.hk * G;
    if (tail_cut && !head_cut) {
      // the CTA that has step e - 1, where e = end + what is left of the unit: the last one that starts before e
      const int64_t e = sh.end + steps - (sh.step + n_steps), ctas = min(int64_t(gridDim.x), sh.total);
      ends = make_int4(sh.b, sh.hk, int((e * ctas + sh.total - 1) / sh.total) - 1, 0);
    }
    sh.left -= n_steps;
    sh.step = 0;
    if (++sh.hk == d.Hkv) { sh.hk = 0; ++sh.b; }
    const bool more = sh.left > 0;
    if (more) {
      begin_unit();
      issue_tiles(0, S::kEarly);
    }
    __syncthreads();
    for (int idx = tid; idx < G * D; idx += kDecThreads) {
      const int hd = idx / D, e = idx % D;
      float mm = -INFINITY;
#pragma unroll
      for (int w = 0; w < kDecWarps; ++w) mm = fmaxf(mm, ml_of(w)[hd].x);
      float ll = 0.f, aa = 0.f;
#pragma unroll
      for (int w = 0; w < kDecWarps; ++w) {
        const float2 ml = ml_of(w)[hd];
        if (ml.y == 0.f) continue;   // a warp without entries (a NaN goes through)
        const float f = ml.x == -INFINITY ? 1.f : ex2(ml.x - mm);
        ll += ml.y * f;
        aa += acc_of(w)[hd * D + e] * f;
      }
      if (head_cut || tail_cut) {
        p.part_acc[(part * G + hd) * D + e] = aa;
        if (e == 0) p.part_ml[part * G + hd] = make_float2(mm, ll);
      } else {
        p.o[(out0 + hd) * D + e] = __float2bfloat16(ll != 0.f ? aa / ll : 0.f);
        if (p.lse && e == 0) p.lse[out0 + hd] = ll != 0.f ? (mm + log2f(ll)) * 0.6931471805599453f : -INFINITY;
      }
    }
    if (!more) break;
  }
  if (tid == 0 && !p.whole) p.ends[blockIdx.x] = ends;
}

// grid (CTAs of decode_quant, G).  Joins the parts of a unit that was cut: the block of the CTA that began it,
// with the parts of the CTAs behind.  LANES threads share an element's parts.
template <int D, int LANES>
__global__ void __launch_bounds__(D* LANES) decode_quant_join(const __grid_constant__ QuantDecodeParams p) {
  constexpr int kLanes = LANES;
  __shared__ float2 s_ml[kLanes];
  __shared__ float s_acc[kLanes][D];
  wait_for_prior();
  const sepllm_cache_desc& d = p.h.desc;
  const int G = d.Hq / d.Hkv, hd = blockIdx.y, e = threadIdx.x % D, y = threadIdx.x / D, i = blockIdx.x;
  const int4 unit = p.ends[i];
  if (unit.x < 0) return;
  float mm = -INFINITY, ll = 0.f, aa = 0.f;
#pragma unroll 4
  for (int k = i + y; k <= unit.z; k += kLanes) {
    const size_t part = (2 * size_t(k) + (k == i)) * G + hd;
    const float2 ml = p.part_ml[part];
    const float acc = p.part_acc[part * D + e];
    const float m = fmaxf(mm, ml.x);
    const float f0 = mm == m ? 1.f : ex2(mm - m), f1 = ml.x == m ? 1.f : ex2(ml.x - m);
    ll = ll * f0 + ml.y * f1;
    aa = aa * f0 + acc * f1;
    mm = m;
  }
  if (e == 0) s_ml[y] = make_float2(mm, ll);
  s_acc[y][e] = aa;
  __syncthreads();
  if (y != 0) return;
#pragma unroll
  for (int k = 1; k < kLanes; ++k) mm = fmaxf(mm, s_ml[k].x);
  ll = aa = 0.f;
#pragma unroll
  for (int k = 0; k < kLanes; ++k) {
    const float2 ml = s_ml[k];
    if (ml.y == 0.f) continue;   // no parts (a NaN goes through)
    const float f = ml.x == mm ? 1.f : ex2(ml.x - mm);
    ll += ml.y * f;
    aa += s_acc[k][e] * f;
  }
  const size_t row = size_t(unit.x) * d.Hq + unit.y * G + hd;
  p.o[row * D + e] = __float2bfloat16(ll != 0.f ? aa / ll : 0.f);
  if (p.lse && e == 0) p.lse[row] = ll != 0.f ? (mm + log2f(ll)) * 0.6931471805599453f : -INFINITY;
}

// f(D, H) for the kernel that serves a descriptor, as integral constants.
template <class F>
auto with_shape(const sepllm_cache_desc& d, F f) {
  const int G = d.Hq / d.Hkv;
  auto heads = [&](auto D) {
    if (G <= 4) return f(D, std::integral_constant<int, 4>{});
    if (G <= 8) return f(D, std::integral_constant<int, 8>{});
    return f(D, std::integral_constant<int, 16>{});
  };
  return d.d == 128 ? heads(std::integral_constant<int, 128>{}) : heads(std::integral_constant<int, 64>{});
}

// Caches of few steps: every unit is one CTA's, and nothing is left to join.
bool decode_quant_whole(const sepllm_cache_desc& d) { return d.c <= 4 * kStepRows; }

// CTAs of a decode: one per unit, or as many as are resident, or one per step of the fullest caches.
int64_t decode_quant_ctas(const sepllm_cache_desc& d) {
  const int64_t units = int64_t(d.B) * d.Hkv, steps = (int64_t(d.c) + kStepRows - 1) / kStepRows;
  if (decode_quant_whole(d)) return units;
  const int resident = with_shape(d, [](auto D, auto H) { return DecodeShape<D(), H()>::kResident; });
  return std::min<int64_t>(resident * kSmCount, units * steps);
}

struct QuantDecodeLayout {
  size_t off_ml, off_acc, bytes;
};
QuantDecodeLayout decode_quant_layout(const sepllm_cache_desc& d) {
  const size_t ctas = decode_quant_whole(d) ? 0 : size_t(decode_quant_ctas(d)), rows = 2 * ctas * (d.Hq / d.Hkv);
  QuantDecodeLayout l;
  l.off_ml = kAlign + align_up(ctas * sizeof(int4));
  l.off_acc = l.off_ml + align_up(rows * sizeof(float2));
  l.bytes = l.off_acc + align_up(rows * d.d * sizeof(float));
  return l;
}

template <int D, int H>
sepllm_status launch_decode_quant(const QuantDecodeParams& p, cudaStream_t stream) {
  constexpr int smem = DecodeShape<D, H>::kSmem;
  const unsigned ctas = unsigned(decode_quant_ctas(p.h.desc));   // (65 535^2 at most, checked by the caller)
  if (smem > 48 * 1024)
    SEPLLM_CUDA_TRY(cudaFuncSetAttribute(decode_quant<D, H>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
  SEPLLM_CUDA_TRY(launch_overlapped(decode_quant<D, H>, dim3(ctas), kDecThreads, smem, stream, p));
  if (p.whole) return SEPLLM_OK;
  const dim3 grid(ctas, p.h.desc.Hq / p.h.desc.Hkv);
  // Few units, cut over many CTAs, are joined by several threads to an element (28 parts: 8 us less than by one);
  // otherwise by one, so that all blocks find room beside decode_quant (1 us less for 256 units in two parts).
  const int64_t units = int64_t(p.h.desc.B) * p.h.desc.Hkv;
  const bool many = ctas > 8 * units;
  auto join = many ? decode_quant_join<D, 512 / D> : decode_quant_join<D, 1>;
  SEPLLM_CUDA_TRY(launch_overlapped(join, grid, many ? 512 : D, 0, stream, p));
  return SEPLLM_OK;
}

}  // namespace

}  // namespace sepllm

using namespace sepllm;

extern "C" sepllm_status sepllm_cache_bytes_quant(const sepllm_cache_desc* desc, size_t* state_bytes,
                                                  size_t* kv_bytes) {
  sepllm_cache_header h;
  const sepllm_status st = check_quant(desc, &h);
  if (st != SEPLLM_OK) return st;
  if (state_bytes) *state_bytes = size_t(h.total_bytes);
  if (kv_bytes)
    *kv_bytes = quant_code_bytes(h) + align_up(size_t(desc->B) * desc->Hkv * h.slots * (desc->d / 16));
  return SEPLLM_OK;
}

extern "C" sepllm_status sepllm_cache_update_quant(const sepllm_cache_desc* desc, void* state, void* Kc, void* Vc,
                                                   const int32_t* new_token_ids, const int32_t* sep_ids,
                                                   int32_t n_sep, const void* k_new, const void* v_new,
                                                   void* stream_) {
  sepllm_cache_header h;
  sepllm_status st = check_quant(desc, &h);
  if (st != SEPLLM_OK) return st;
  if (!state || !Kc || !Vc || !new_token_ids || !k_new || !v_new) return SEPLLM_INVALID_ARG;
  if (!aligned(state, kAlign) || !aligned(Kc, kAlign) || !aligned(Vc, kAlign) || !aligned(k_new, 16) ||
      !aligned(v_new, 16) || !aligned(new_token_ids, 4))
    return SEPLLM_INVALID_ARG;
  SepIds sep;
  int max_past;
  if ((st = update_params(desc, sep_ids, n_sep, &sep, &max_past)) != SEPLLM_OK) return st;
  const size_t smem = size_t(max_past) * 2 * sizeof(int16_t);
  auto kernel = desc->d == 128 ? quant_update<128> : quant_update<64>;
  SEPLLM_CUDA_TRY(allow_update_smem(kernel, smem, 2 * sizeof(int16_t)));
  SEPLLM_CUDA_TRY(launch_overlapped(kernel, dim3(desc->B, desc->Hkv), kUpdThreads, smem, static_cast<cudaStream_t>(stream_),
                                    h, static_cast<uint8_t*>(state), quant_rows(h, Kc), quant_rows(h, Vc),
                                    static_cast<const __nv_bfloat16*>(k_new),
                                    static_cast<const __nv_bfloat16*>(v_new), new_token_ids, sep, max_past));
  return SEPLLM_OK;
}

extern "C" sepllm_status sepllm_cache_from_prompt_quant(const sepllm_cache_desc* desc, const sepllm_index_desc* idesc,
                                                        const void* index, const int32_t* prompt_len, const void* K,
                                                        const void* V, void* state, void* Kc, void* Vc,
                                                        void* stream_) {
  sepllm_cache_header h;
  sepllm_status st = check_quant(desc, &h);
  if (st != SEPLLM_OK) return st;
  sepllm_index_header ih;
  if ((st = fill_index_header(idesc, &ih)) != SEPLLM_OK) return st;
  if (!index || !K || !V || !state || !Kc || !Vc) return SEPLLM_INVALID_ARG;
  if (idesc->B != desc->B || idesc->n_init != desc->a) return SEPLLM_INVALID_ARG;
  if (!aligned(index, kAlign) || !aligned(state, kAlign) || !aligned(K, 16) || !aligned(V, 16) ||
      !aligned(Kc, kAlign) || !aligned(Vc, kAlign) || !aligned(prompt_len, 4))
    return SEPLLM_INVALID_ARG;
  if (desc->B > 65535 || desc->Hkv > 65535) return SEPLLM_UNSUPPORTED;
  cudaStream_t stream = static_cast<cudaStream_t>(stream_);
  if ((st = launch_prompt_plan(h, ih, state, index, prompt_len, stream)) != SEPLLM_OK) return st;
  const dim3 grid((h.slots + kCopyRows - 1) / kCopyRows, desc->Hkv, desc->B);
  auto kernel = desc->d == 128 ? quant_prompt<128> : quant_prompt<64>;
  SEPLLM_CUDA_TRY(launch_overlapped(kernel, grid, kCopyThreads, 0, stream, h, static_cast<const uint8_t*>(state),
                                    static_cast<const __nv_bfloat16*>(K), static_cast<const __nv_bfloat16*>(V),
                                    idesc->L, quant_rows(h, Kc), quant_rows(h, Vc)));
  return SEPLLM_OK;
}

extern "C" sepllm_status sepllm_cache_entries_quant(const sepllm_cache_desc* desc, const void* state, const void* Kc,
                                                    const void* Vc, int32_t n, void* K, void* V, int32_t* length,
                                                    void* stream_) {
  sepllm_cache_header h;
  const sepllm_status st = check_quant(desc, &h);
  if (st != SEPLLM_OK) return st;
  if (n < 1 || !state || !Kc || !Vc || !K || !V) return SEPLLM_INVALID_ARG;
  if (!aligned(state, kAlign) || !aligned(Kc, kAlign) || !aligned(Vc, kAlign) || !aligned(K, 16) || !aligned(V, 16) ||
      !aligned(length, 4))
    return SEPLLM_INVALID_ARG;
  if (n < desc->c) return SEPLLM_BUFFER_TOO_SMALL;
  if (desc->B > 65535 || desc->Hkv > 65535) return SEPLLM_UNSUPPORTED;
  const dim3 grid((desc->c + kCopyRows - 1) / kCopyRows, desc->Hkv, desc->B);   // Size_run never passes c
  auto kernel = desc->d == 128 ? quant_entries<128> : quant_entries<64>;
  SEPLLM_CUDA_TRY(launch_overlapped(kernel, grid, kCopyThreads, 0, static_cast<cudaStream_t>(stream_), h,
                                    static_cast<const uint8_t*>(state), quant_rows(h, Kc), quant_rows(h, Vc), n,
                                    static_cast<__nv_bfloat16*>(K), static_cast<__nv_bfloat16*>(V), length));
  return SEPLLM_OK;
}

extern "C" sepllm_status sepllm_decode_quant_workspace_bytes(const sepllm_cache_desc* desc, size_t* bytes) {
  sepllm_cache_header h;
  const sepllm_status st = fill_cache_header(desc, &h);
  if (st != SEPLLM_OK) return st;
  if (bytes) *bytes = decode_quant_layout(*desc).bytes;
  return SEPLLM_OK;
}

extern "C" sepllm_status sepllm_decode_quant(const sepllm_cache_desc* desc, float scale, const void* q,
                                             const void* state, const void* Kc, const void* Vc, void* o, float* lse,
                                             void* workspace, void* stream_) {
  QuantDecodeParams p{};
  const sepllm_status st = check_quant(desc, &p.h);
  if (st != SEPLLM_OK) return st;
  if (!q || !state || !Kc || !Vc || !o || !workspace) return SEPLLM_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(state, kAlign) || !aligned(Kc, kAlign) || !aligned(Vc, kAlign) || !aligned(o, 2) ||
      !aligned(lse, 4) || !aligned(workspace, kAlign))
    return SEPLLM_INVALID_ARG;
  if (desc->B > 65535 || desc->Hkv > 65535) return SEPLLM_UNSUPPORTED;
  if (size_t(desc->B) * desc->Hkv * p.h.slots > 0xffffffffu) return SEPLLM_UNSUPPORTED;   // rows have 32-bit numbers
  const QuantDecodeLayout l = decode_quant_layout(*desc);
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  p.state = static_cast<const uint8_t*>(state);
  p.q = static_cast<const __nv_bfloat16*>(q);
  p.Kc = quant_rows(p.h, Kc);
  p.Vc = quant_rows(p.h, Vc);
  p.o = static_cast<__nv_bfloat16*>(o);
  p.lse = lse;
  p.status = reinterpret_cast<int32_t*>(ws);
  p.ends = reinterpret_cast<int4*>(ws + kAlign);
  p.part_ml = reinterpret_cast<float2*>(ws + l.off_ml);
  p.part_acc = reinterpret_cast<float*>(ws + l.off_acc);
  p.scale_log2 = (scale != 0.f ? scale : 1.0f / sqrtf(float(desc->d))) * 1.4426950408889634f;
  p.whole = decode_quant_whole(*desc);
  cudaStream_t stream = static_cast<cudaStream_t>(stream_);
  return with_shape(*desc, [&](auto D, auto H) { return launch_decode_quant<D(), H()>(p, stream); });
}
