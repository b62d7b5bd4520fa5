// Norms of every query and key head with the rotary positions in the same pass, and their gradient.
//
// y = x r (offset + w), r = (mean x^2 + eps)^-1/2 over the head, then the rotation.  With g the gradient
// of the outputs rotated back, n = x r and u = g (offset + w): dx = r (u - n mean(n u)), dw = sum g n.
// Bound by HBM like the rotation alone: x (and dy) are read once, the output is written once; the
// gradient computes r anew from x instead of reading it.  Everything is computed in 32 bits (angles as in the
// rotation alone) and rounded once, to the output's type.
#include "rope_common.cuh"

namespace sepllm {

namespace {

constexpr int kWarps = kRopeThreads / 32;
constexpr int kBwdResident = 3;
constexpr int kBwdBlocks = kBwdResident * kSmCount;   // of the gradient, each with a share of the rows and sums of its own

struct NormParams {
  RopeParams r;
  const void* w[2];          // of Q and K, or null
  int w_dtype, half;
  float eps, offset, inv_d;
  // gradient: the forward's inputs, the blocks' sums [block][2][d] and their total
  const void* x[3];          // (V: null, not read)
  int64_t xb[3], xh[3], xl[3];
  float* part;
  float* dw[2];
  int64_t groups;            // of the tokens that a warp takes at once
  int blocks[3];             // that have rows of each tensor (whichever other tensors there are)
  int grid;
};

__device__ __forceinline__ float weight_at(const NormParams& p, int w, int e) {
  if (!p.w[w]) return 1.f;
  return p.offset + (p.w_dtype ? static_cast<const float*>(p.w[w])[e]
                               : __bfloat162float(static_cast<const __nv_bfloat16*>(p.w[w])[e]));
}

// A thread's part of a row in the kernels for 16-byte accesses: as in rope_rows two pieces of eight
// elements, c0 and c1, and whether they turn; d / 16 neighbouring lanes cover a row and a warp has whole
// rows, so that a row's sums are a few shuffles.
struct Pieces {
  int c0, c1;
  bool turn;
};
template <bool HALF>
__device__ __forceinline__ Pieces pieces_of(const RopeParams& p, int t) {
  Pieces s;
  if (HALF) {
    const int pairs = p.rot / 16;
    s.turn = t < pairs;
    s.c0 = 8 * (s.turn ? t : t + pairs);
    s.c1 = s.c0 + (s.turn ? p.rot / 2 : (p.d - p.rot) / 2);
  } else {
    s.c0 = 8 * t;
    s.c1 = s.c0 + p.d / 2;
    s.turn = s.c0 < p.rot;
  }
  return s;
}
// Two neighbouring elements in one register pair: Blackwell's packed fp32 arithmetic does both in one
// instruction (the gradient is bound by its instructions as much as by its loads).
using Pair = unsigned long long;
__device__ __forceinline__ Pair pair_of(float lo, float hi) {
  Pair r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ float2 floats_of(Pair x) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(x));
  return r;
}
__device__ __forceinline__ Pair mul2(Pair a, Pair b) {
  Pair r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) {
  Pair r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ float sum2(Pair x) {
  const float2 f = floats_of(x);
  return f.x + f.y;
}
template <class T>
__device__ __forceinline__ void to_pairs(const Eight<T>& r, Pair (&x)[4]) {
  float f[8];
  to_floats(r, f);
#pragma unroll
  for (int k = 0; k < 4; ++k) x[k] = pair_of(f[2 * k], f[2 * k + 1]);
}
template <class T>
__device__ __forceinline__ void store_pairs(T* s, const Pair (&x)[4]) {
  float f[8];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float2 y = floats_of(x[k]);
    f[2 * k] = y.x;
    f[2 * k + 1] = y.y;
  }
  store8(s, f);
}

template <bool HALF>
__device__ __forceinline__ void angles(const RopeParams& p, const Pieces& s, double pos, float2 (&cs)[8]) {
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int i = HALF ? s.c0 + k : (k < 4 ? s.c0 / 2 + k : s.c1 / 2 + k - 4);
    cs[k] = s.turn && 2 * i < p.rot ? rope_cos_sin(p, pos, i) : make_float2(1.f, 0.f);
  }
}
// (One by one: a packed product has no sign of its own.  Where nothing turns the angle is 0, but the products
// with 0 would spread a NaN.)
template <bool HALF>
__device__ __forceinline__ void rotate(const RopeParams& p, const Pieces& s, const float2 (&cs)[8], Pair (&u)[4],
                                       Pair (&v)[4]) {
  if (HALF) {
    if (!s.turn) return;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float2 a = floats_of(u[k]), b = floats_of(v[k]), c0 = cs[2 * k], c1 = cs[2 * k + 1];
      u[k] = pair_of(a.x * c0.x - b.x * c0.y, a.y * c1.x - b.y * c1.y);
      v[k] = pair_of(b.x * c0.x + a.x * c0.y, b.y * c1.x + a.y * c1.y);
    }
  } else {
    auto turn = [](Pair x, float2 cs) {
      const float2 f = floats_of(x);
      return pair_of(f.x * cs.x - f.y * cs.y, f.y * cs.x + f.x * cs.y);
    };
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (s.c0 + 2 * k < p.rot) u[k] = turn(u[k], cs[k]);
      if (s.c1 + 2 * k < p.rot) v[k] = turn(v[k], cs[4 + k]);
    }
  }
}
// Sum over the row's lanes, in each of them (all 32 lanes call).  PER_ROW: the lanes of a row, 4 or 8 (heads of 64
// and 128), or 0 for any number.
template <int PER_ROW>
__device__ __forceinline__ float row_sum(float x, int per_row, int first) {
  if constexpr (PER_ROW > 0) {
#pragma unroll
    for (int o = 1; o < PER_ROW; o <<= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
  }
  float s = 0.f;
  for (int k = 0; k < per_row; ++k) s += __shfl_sync(0xffffffffu, x, first + k);
  return s;
}

// A thread has sixteen elements of a row, d / 16 lanes a row, and walks the heads of its token with the cos and sin that
// it computed once; the next heads' rows are on their way while one is worked on.  48 heads of 128 on 65 536
// tokens take 252 us: 1.61 GB at 6.4 TB/s, the measured copy rate.  16 384 of them: 75 us (fp32 to bf16 104, bf16 to fp32
// 102, fp32 to fp32 133).  14 heads of 80 on 5997 tokens (27 MB): 12.7 us, where the rotation alone takes 9.9: latency.  A
// warp has 6 such rows at once and one wave of CTAs, in which angles, weights and the first rows come one after the other.
template <class Tin, class Tout, bool HALF, int PER_ROW>
__global__ void __launch_bounds__(kRopeThreads) norm_rows(const __grid_constant__ NormParams np) {
  let_dependents_start();
  wait_for_prior();
  const RopeParams& p = np.r;
  const int per_row = PER_ROW ? PER_ROW : p.d / 16, rows = 32 / per_row;
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  const int rr = lane / per_row;
  const int64_t n = (int64_t(blockIdx.x) * kWarps + wid) * rows + rr;
  const bool here = rr < rows && n < p.tokens;
  const int64_t b = here ? n / p.L : 0;
  const int l = here ? int(n - b * p.L) : 0;
  const Pieces s = pieces_of<HALF>(p, lane - rr * per_row);
  const int h0 = blockIdx.y * p.heads_per_block, h1 = min(p.n_heads, h0 + p.heads_per_block);
  float2 turn[8];
  if (here && h0 < p.t[0].heads + p.t[1].heads) angles<HALF>(p, s, rope_position(p, b, l), turn);
  int first = 0;  // heads of the tensors before this one
#pragma unroll 1
  for (int w = 0; w < 3; ++w) {
    const RopeTensor& x = p.t[w];
    const int a = max(h0 - first, 0), e = min(h1 - first, x.heads);
    first += x.heads;
    if (a >= e) continue;
    const Tin* src = static_cast<const Tin*>(x.in) + b * x.ib + l * x.il + a * x.ih + s.c0;
    Tout* dst = static_cast<Tout*>(x.out) + b * x.ob + l * x.ol + a * x.oh + s.c0;
    const int step = s.c1 - s.c0;
    Pair wu[4], wv[4];
    if (w < 2) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        wu[k] = pair_of(weight_at(np, w, s.c0 + 2 * k), weight_at(np, w, s.c0 + 2 * k + 1));
        wv[k] = pair_of(weight_at(np, w, s.c1 + 2 * k), weight_at(np, w, s.c1 + 2 * k + 1));
      }
    }
    // rows of the next heads are on their way while one is worked on (an output may be its own input, but
    // is no other head's)
    constexpr int kDepth = sizeof(Tin) == 2 ? 4 : 2;
    Eight<Tin> ru[kDepth]{}, rv[kDepth]{};
    auto fetch = [&](int i, int h) {
      if (!here || h >= e) return;
      ru[i] = load8(src);
      rv[i] = load8(src + step);
      src += x.ih;
    };
#pragma unroll
    for (int i = 0; i < kDepth; ++i) fetch(i, a + i);
    for (int h = a; h < e; h += kDepth) {
#pragma unroll
      for (int i = 0; i < kDepth; ++i) {
        if (h + i >= e) break;
        Pair u[4], v[4];
        to_pairs(ru[i], u);
        to_pairs(rv[i], v);
        fetch(i, h + i + kDepth);
        if (w < 2) {
          Pair sum = mul2(u[0], u[0]);
#pragma unroll
          for (int k = 1; k < 4; ++k) sum = fma2(u[k], u[k], sum);
#pragma unroll
          for (int k = 0; k < 4; ++k) sum = fma2(v[k], v[k], sum);
          const float r = rsqrtf(row_sum<PER_ROW>(sum2(sum), per_row, rr * per_row) * np.inv_d + np.eps);
          const Pair r2 = pair_of(r, r);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            u[k] = mul2(u[k], mul2(r2, wu[k]));
            v[k] = mul2(v[k], mul2(r2, wv[k]));
          }
          rotate<HALF>(p, s, turn, u, v);
        }
        if (here) {
          store_pairs(dst, u);
          store_pairs(dst + step, v);
        }
        dst += x.oh;
      }
    }
  }
}

// Any rot_dim, stride and alignment: a warp has one token, a lane up to two pairs of a head and four
// elements that are only scaled.
struct Lane {
  int c0[2], c1[2], e[4];   // -1: none
};
__device__ __forceinline__ Lane lane_elements(const RopeParams& p, bool half, int lane) {
  Lane s;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int i = lane + 32 * k, n = p.rot / 2;
    s.c0[k] = i < n ? (half ? i : 2 * i) : -1;
    s.c1[k] = half ? i + n : 2 * i + 1;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int e = p.rot + lane + 32 * k;
    s.e[k] = e < p.d ? e : -1;
  }
  return s;
}
__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}
// A lane's elements in the order c0[0], c1[0], c0[1], c1[1], e[0..3].
template <class T>
__device__ __forceinline__ void load_lane(const T* row, const Lane& s, float (&x)[8]) {
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    x[2 * k] = s.c0[k] >= 0 ? load1(row + s.c0[k]) : 0.f;
    x[2 * k + 1] = s.c0[k] >= 0 ? load1(row + s.c1[k]) : 0.f;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) x[4 + k] = s.e[k] >= 0 ? load1(row + s.e[k]) : 0.f;
}
template <class T>
__device__ __forceinline__ void store_lane(T* row, const Lane& s, const float (&x)[8]) {
#pragma unroll
  for (int k = 0; k < 2; ++k)
    if (s.c0[k] >= 0) {
      store1(row + s.c0[k], x[2 * k]);
      store1(row + s.c1[k], x[2 * k + 1]);
    }
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (s.e[k] >= 0) store1(row + s.e[k], x[4 + k]);
}
__device__ __forceinline__ void lane_weights(const NormParams& p, int w, const Lane& s, float (&x)[8]) {
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    x[2 * k] = s.c0[k] >= 0 ? weight_at(p, w, s.c0[k]) : 0.f;
    x[2 * k + 1] = s.c0[k] >= 0 ? weight_at(p, w, s.c1[k]) : 0.f;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) x[4 + k] = s.e[k] >= 0 ? weight_at(p, w, s.e[k]) : 0.f;
}
__device__ __forceinline__ void lane_angles(const RopeParams& p, int64_t b, int l, int lane, float2 (&cs)[2]) {
  const double pos = rope_position(p, b, l);
#pragma unroll
  for (int k = 0; k < 2; ++k)
    cs[k] = lane + 32 * k < p.rot / 2 ? rope_cos_sin(p, pos, lane + 32 * k) : make_float2(1.f, 0.f);
}
__device__ __forceinline__ void lane_rotate(const float2 (&cs)[2], float (&x)[8]) {
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const float y = x[2 * k] * cs[k].x - x[2 * k + 1] * cs[k].y;
    x[2 * k + 1] = x[2 * k + 1] * cs[k].x + x[2 * k] * cs[k].y;
    x[2 * k] = y;
  }
}

// Any strides and alignment: a warp per token, its lanes along the head's pairs, element by element and with no row on
// its way ahead.  48 heads of 128 on 16 384 tokens, 118 elements turned in halves: 228 us (norm_rows with all
// 128 turned: 75); 14 heads of 80 on 5997 tokens, 20 turned in halves: 33 us.
template <class Tin, class Tout>
__global__ void __launch_bounds__(kRopeThreads) norm_any(const __grid_constant__ NormParams np) {
  let_dependents_start();
  wait_for_prior();
  const RopeParams& p = np.r;
  const int lane = threadIdx.x & 31;
  const int64_t n = int64_t(blockIdx.x) * kWarps + (threadIdx.x >> 5);
  if (n >= p.tokens) return;
  const int64_t b = n / p.L;
  const int l = int(n - b * p.L);
  const Lane s = lane_elements(p, np.half, lane);
  const int h0 = blockIdx.y * p.heads_per_block, h1 = min(p.n_heads, h0 + p.heads_per_block);
  float2 cs[2];
  lane_angles(p, b, l, lane, cs);
  int first = 0;
#pragma unroll
  for (int w = 0; w < 3; ++w) {
    const RopeTensor& x = p.t[w];
    const int a = max(h0 - first, 0), e = min(h1 - first, x.heads);
    first += x.heads;
    const Tin* src = static_cast<const Tin*>(x.in) + b * x.ib + l * x.il;
    Tout* dst = static_cast<Tout*>(x.out) + b * x.ob + l * x.ol;
    float wt[8];
    if (w < 2 && a < e) lane_weights(np, w, s, wt);
    for (int h = a; h < e; ++h) {
      float y[8];
      load_lane(src + h * x.ih, s, y);
      if (w < 2) {
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < 8; ++k) sum += y[k] * y[k];
        const float r = rsqrtf(warp_sum(sum) * np.inv_d + np.eps);
#pragma unroll
        for (int k = 0; k < 8; ++k) y[k] *= r * wt[k];
        lane_rotate(cs, y);
      }
      store_lane(dst + h * x.oh, s, y);
    }
  }
}

// dx of one row's elements and the row's addition to the weights' gradient.  x, g: inputs and rotated-back
// gradients; w: offset + weights; s1, s2: sums of x^2 and of x g w over the row.
template <int N>
__device__ __forceinline__ void norm_grad(float s1, float s2, const NormParams& p, const float (&w)[N],
                                          const float (&x)[N], float (&g)[N], float (&dw)[N]) {
  const float r = rsqrtf(s1 * p.inv_d + p.eps);
  const float k = r * (r * (s2 * p.inv_d));
#pragma unroll
  for (int e = 0; e < N; ++e) {
    dw[e] += g[e] * (x[e] * r);
    g[e] = r * (g[e] * w[e] - x[e] * k);
  }
}

// A warp's way through the rows of a tensor, head by head and then on to the warp's next tokens (`rows` of
// them, one to a lane's group).
struct RowWalk {
  int64_t b;
  int l, h;
  bool here;   // this lane has a token
};
__device__ __forceinline__ RowWalk walk_from(const RopeParams& p, int64_t group, int h, int rows, int rr) {
  RowWalk k;
  const int64_t n = group * rows + rr;
  k.here = rr < rows && n < p.tokens;
  k.b = n / p.L;
  k.l = int(n - k.b * p.L);
  k.h = h;
  return k;
}
// true: on to the next tokens
__device__ __forceinline__ bool walk_on(const RopeParams& p, RowWalk& k, int heads, int rows, int rr) {
  if (++k.h < heads) return false;
  k.h = 0;
  for (k.l += rows; k.l >= p.L; k.l -= p.L) ++k.b;
  k.here = rr < rows && k.b * p.L + k.l < p.tokens;
  return true;
}

// The rows of a tensor, (tokens of a warp, head), are cut into equal runs, one per warp; the next rows are on
// their way while one is worked on, over the ends of heads and tokens.  The tensors come one after the
// other, so that the sums for one tensor's weights are all that stays in registers.
//
// 48 heads of 128 on 16 384 tokens, fp32 to bf16: 134 us (5.7 TB/s; DRAM 69 % of its cycles); bf16 to bf16 119, bf16 to
// fp32 164, fp32 to fp32 218 (spills 126 to 250 bytes).  36 heads of 64 on 8 x 2048 tokens, bf16: 53 us against 31 of its
// bytes; issue slots 43 %, DRAM 40 %: nothing is full, 12 warps an SM (168 registers: x and dy, their next
// rows, angles and sums, of sixteen elements a lane) wait in turn for loads, the two row sums and the cos and sin of
// a new token (9 %).  Fewer elements to a lane, and so more warps, were not tried.
// Four or two CTAs an SM, rows through shared memory (186 and 58 us) and a longer or shorter register ring were slower.
template <class Tx, class Tg, bool HALF, int PER_ROW>
__global__ void __launch_bounds__(kRopeThreads, kBwdResident) norm_bwd_rows(const __grid_constant__ NormParams np) {
  __shared__ __align__(16) float s_part[2048];   // [row of the block][d]
  __shared__ __align__(16) float s_w[128];
  wait_for_prior();
  const RopeParams& p = np.r;
  const int per_row = PER_ROW ? PER_ROW : p.d / 16, rows = 32 / per_row;
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  const int rr = lane / per_row;
  const Pieces s = pieces_of<HALF>(p, lane - rr * per_row);
  const int step = s.c1 - s.c0;
#pragma unroll 1
  for (int w = 0; w < 3; ++w) {
    const RopeTensor& y = p.t[w];
    Pair acc_u[4], acc_v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) acc_u[k] = acc_v[k] = 0;
    if (w < 2) {
      for (int e = threadIdx.x; e < p.d; e += kRopeThreads) s_w[e] = weight_at(np, w, e);
      __syncthreads();
    }
    const int64_t total = np.groups * y.heads, warps = int64_t(np.blocks[w]) * kWarps;
    const int64_t mine = min(int64_t(blockIdx.x) * kWarps + wid, warps);   // (no rows behind the last of them)
    const int64_t first = total * mine / warps;
    const int n_rows = int(total * min(mine + 1, warps) / warps - first);
    if (n_rows > 0) {
      const int64_t group = first / y.heads;
      RowWalk at = walk_from(p, group, int(first - group * y.heads), rows, rr), ahead = at;
      const Tg* src;
      const Tx* xs;
      Tx* dst;
      auto to_ahead = [&]() {
        src = static_cast<const Tg*>(y.in) + ahead.b * y.ib + ahead.l * y.il + ahead.h * y.ih + s.c0;
        xs = static_cast<const Tx*>(np.x[w]) + ahead.b * np.xb[w] + ahead.l * np.xl[w] + ahead.h * np.xh[w] + s.c0;
      };
      auto to_at = [&]() { dst = static_cast<Tx*>(y.out) + at.b * y.ob + at.l * y.ol + at.h * y.oh + s.c0; };
      constexpr int kDepth = 2;
      Eight<Tg> gu[kDepth]{}, gv[kDepth]{};
      Eight<Tx> xu[kDepth]{}, xv[kDepth]{};
      auto fetch = [&](int i) {
        if (ahead.here) {
          gu[i] = load8(src);
          gv[i] = load8(src + step);
          if (w < 2) {
            xu[i] = load8(xs);
            xv[i] = load8(xs + step);
          }
        }
        src += y.ih;
        xs += np.xh[w];
        if (walk_on(p, ahead, y.heads, rows, rr)) to_ahead();
      };
      to_ahead();
      to_at();
#pragma unroll
      for (int i = 0; i < kDepth; ++i)
        if (i < n_rows) fetch(i);
      float2 turn[8];
      bool moved = true;   // to other tokens, whose angles are not there yet (rows not here add zeros below)
      for (int r = 0; r < n_rows; r += kDepth) {
#pragma unroll
        for (int i = 0; i < kDepth; ++i) {
          if (r + i >= n_rows) break;
          if (moved && w < 2) angles<HALF>(p, s, at.here ? rope_position(p, at.b, at.l) : 0.0, turn);
          Pair fgu[4], fgv[4], fxu[4], fxv[4];
          to_pairs(gu[i], fgu);
          to_pairs(gv[i], fgv);
          to_pairs(xu[i], fxu);
          to_pairs(xv[i], fxv);
          if (!at.here) {
#pragma unroll
            for (int k = 0; k < 4; ++k) fgu[k] = fgv[k] = 0;
          }
          if (r + i + kDepth < n_rows) fetch(i);
          if (w < 2) {
            rotate<HALF>(p, s, turn, fgu, fgv);
            // (the weights stay in shared memory: 16 registers less)
            const Pair* wu = reinterpret_cast<const Pair*>(s_w + s.c0);
            const Pair* wv = reinterpret_cast<const Pair*>(s_w + s.c1);
            Pair s1 = 0, s2 = 0, zu[4], zv[4];   // z = g w
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              zu[k] = mul2(fgu[k], wu[k]);
              zv[k] = mul2(fgv[k], wv[k]);
              s1 = fma2(fxv[k], fxv[k], fma2(fxu[k], fxu[k], s1));
              s2 = fma2(fxv[k], zv[k], fma2(fxu[k], zu[k], s2));
            }
            const float sum1 = row_sum<PER_ROW>(sum2(s1), per_row, rr * per_row);
            const float sum2_ = row_sum<PER_ROW>(sum2(s2), per_row, rr * per_row);
            const float r1 = rsqrtf(sum1 * np.inv_d + np.eps);
            const float k1 = -r1 * (r1 * (sum2_ * np.inv_d));
            const Pair r2 = pair_of(r1, r1), k2 = pair_of(k1, k1);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              acc_u[k] = fma2(fgu[k], mul2(fxu[k], r2), acc_u[k]);
              acc_v[k] = fma2(fgv[k], mul2(fxv[k], r2), acc_v[k]);
              fgu[k] = mul2(r2, fma2(fxu[k], k2, zu[k]));
              fgv[k] = mul2(r2, fma2(fxv[k], k2, zv[k]));
            }
          }
          if (at.here) {
            store_pairs(dst, fgu);
            store_pairs(dst + step, fgv);
          }
          dst += y.oh;
          moved = walk_on(p, at, y.heads, rows, rr);
          if (moved) to_at();
        }
      }
    }
    if (w == 2) break;
    // the block's sums: rows side by side, then added column by column in a fixed order
    __syncthreads();
    if (rr < rows) {
      float* row = s_part + (wid * rows + rr) * p.d;
      store_pairs(row + s.c0, acc_u);
      store_pairs(row + s.c1, acc_v);
    }
    __syncthreads();
    for (int c = threadIdx.x; c < p.d; c += kRopeThreads) {
      float sum = 0.f;
      for (int r = 0; r < kWarps * rows; ++r) sum += s_part[r * p.d + c];
      np.part[(size_t(blockIdx.x) * 2 + w) * p.d + c] = sum;
    }
  }
  let_dependents_start();
}

// The gradient for any strides and alignment, laid out as norm_any.  The two cases named there: 646 and 78 us
// (norm_bwd_rows with all 128 turned: 119).
template <class Tx, class Tg>
__global__ void __launch_bounds__(kRopeThreads) norm_bwd_any(const __grid_constant__ NormParams np) {
  __shared__ float s_part[kWarps][128];
  wait_for_prior();
  const RopeParams& p = np.r;
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  const Lane s = lane_elements(p, np.half, lane);
#pragma unroll 1
  for (int w = 0; w < 3; ++w) {
    const RopeTensor& y = p.t[w];
    float wt[8], acc[8];
    if (w < 2) lane_weights(np, w, s, wt);
#pragma unroll
    for (int k = 0; k < 8; ++k) acc[k] = 0.f;
    const int64_t total = np.groups * y.heads, warps = int64_t(np.blocks[w]) * kWarps;
    const int64_t mine = min(int64_t(blockIdx.x) * kWarps + wid, warps);   // (no rows behind the last of them)
    const int64_t first = total * mine / warps, last = total * min(mine + 1, warps) / warps;
    if (first < last) {
      const int64_t group = first / y.heads;
      RowWalk at = walk_from(p, group, int(first - group * y.heads), 1, 0);
      float2 cs[2];
      bool moved = true;
      for (int64_t r = first; r < last; ++r) {
        if (moved && w < 2) lane_angles(p, at.b, at.l, lane, cs);
        float g[8];
        load_lane(static_cast<const Tg*>(y.in) + at.b * y.ib + at.l * y.il + at.h * y.ih, s, g);
        if (w < 2) {
          float x[8];
          load_lane(static_cast<const Tx*>(np.x[w]) + at.b * np.xb[w] + at.l * np.xl[w] + at.h * np.xh[w], s, x);
          lane_rotate(cs, g);
          float s1 = 0.f, s2 = 0.f;
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            s1 += x[k] * x[k];
            s2 += x[k] * (g[k] * wt[k]);
          }
          norm_grad(warp_sum(s1), warp_sum(s2), np, wt, x, g, acc);
        }
        store_lane(static_cast<Tx*>(y.out) + at.b * y.ob + at.l * y.ol + at.h * y.oh, s, g);
        moved = walk_on(p, at, y.heads, 1, 0);
      }
    }
    if (w == 2) break;
    __syncthreads();
    store_lane(s_part[wid], s, acc);
    __syncthreads();
    for (int c = threadIdx.x; c < p.d; c += kRopeThreads) {
      float sum = 0.f;
#pragma unroll
      for (int r = 0; r < kWarps; ++r) sum += s_part[r][c];
      np.part[(size_t(blockIdx.x) * 2 + w) * p.d + c] = sum;
    }
  }
  let_dependents_start();
}

// grid ceil(2 d / 32): adds the blocks' sums, a column to a lane, in a fixed order.  Latency: 2 us behind the rows.
__global__ void __launch_bounds__(1024) norm_bwd_sum(const __grid_constant__ NormParams np) {
  __shared__ float s_sum[32][33];
  let_dependents_start();
  wait_for_prior();
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, c = blockIdx.x * 32 + lane, d = np.r.d;
  float sum = 0.f;
  for (int i = wid; i < np.grid; i += 32) sum += np.part[size_t(i) * 2 * d + c];   // (2 d: a multiple of 32)
  s_sum[wid][lane] = sum;
  __syncthreads();
  if (wid != 0) return;
  sum = 0.f;
#pragma unroll
  for (int i = 0; i < 32; ++i) sum += s_sum[i][lane];
  float* out = np.dw[c / d];
  if (out) out[c % d] = sum;
}

sepllm_status check_norm(const sepllm_qknorm_desc* n) {
  if (!n || (n->w_dtype != 0 && n->w_dtype != 1)) return SEPLLM_INVALID_ARG;
  if (!finite_positive(n->eps) || !std::isfinite(n->offset)) return SEPLLM_INVALID_ARG;
  const size_t a = n->w_dtype ? 4 : 2;
  return aligned(n->wq, a) && aligned(n->wk, a) ? SEPLLM_OK : SEPLLM_INVALID_ARG;
}

// 16-byte accesses run unless halves end inside a 16-byte piece (these take the kernels for any strides, three to five
// times as long: norm_any).
bool by_rows(const sepllm_rope_desc* d, const RopeParams& p, bool vectors) {
  return vectors && !(d->layout == SEPLLM_ROPE_HALF && p.rot % 16 != 0);
}

void fill_norm(const sepllm_rope_desc* d, const sepllm_qknorm_desc* n, NormParams* p) {
  p->w[0] = n->wq;
  p->w[1] = n->wk;
  p->w_dtype = n->w_dtype;
  p->half = d->layout == SEPLLM_ROPE_HALF;
  p->eps = n->eps;
  p->offset = n->offset;
  p->inv_d = 1.f / float(d->d);
}

// (every kernel is launched while the one before it ends, and waits for it first)
template <class Tin, class Tout>
cudaError_t launch_norm(const NormParams& p, bool rows, dim3 grid, cudaStream_t stream) {
#define SEPLLM_NORM(N) (p.half ? norm_rows<Tin, Tout, true, N> : norm_rows<Tin, Tout, false, N>)
  auto kernel = !rows           ? norm_any<Tin, Tout>
                : p.r.d == 128 ? SEPLLM_NORM(8)
                : p.r.d == 64  ? SEPLLM_NORM(4)
                               : SEPLLM_NORM(0);
#undef SEPLLM_NORM
  return launch_overlapped(kernel, grid, kRopeThreads, 0, stream, p);
}
template <class Tx, class Tg>
cudaError_t launch_norm_bwd(const NormParams& p, bool rows, cudaStream_t stream) {
#define SEPLLM_NORM(N) (p.half ? norm_bwd_rows<Tx, Tg, true, N> : norm_bwd_rows<Tx, Tg, false, N>)
  auto kernel = !rows           ? norm_bwd_any<Tx, Tg>
                : p.r.d == 128 ? SEPLLM_NORM(8)
                : p.r.d == 64  ? SEPLLM_NORM(4)
                               : SEPLLM_NORM(0);
#undef SEPLLM_NORM
  return launch_overlapped(kernel, dim3(unsigned(p.grid)), kRopeThreads, 0, stream, p);
}

}  // namespace

}  // namespace sepllm

using namespace sepllm;

extern "C" sepllm_status sepllm_qknorm_rope_fwd(const sepllm_rope_desc* desc, const sepllm_qknorm_desc* norm,
                                                const int64_t* positions, const sepllm_rope_view* in,
                                                const sepllm_rope_view* out, void* stream_) {
  NormParams p{};
  bool vectors;
  int dt_in, dt_out;
  sepllm_status st = rope_params(desc, positions, in, out, 1.f, &p.r, &vectors, &dt_in, &dt_out);
  if (st != SEPLLM_OK) return st;
  if ((st = check_norm(norm)) != SEPLLM_OK) return st;
  fill_norm(desc, norm, &p);
  const bool rows = by_rows(desc, p.r, vectors);
  const int64_t per_warp = rows ? 32 / (desc->d / 16) : 1;
  const int64_t warps = (p.r.tokens + per_warp - 1) / per_warp, blocks = (warps + kWarps - 1) / kWarps;
  if (blocks > 0x7fffffff) return SEPLLM_UNSUPPORTED;
  p.r.heads_per_block = rope_heads_per_thread(p.r.n_heads, warps * 32);
  const int64_t groups = (p.r.n_heads + p.r.heads_per_block - 1) / p.r.heads_per_block;
  if (groups > 65535) return SEPLLM_UNSUPPORTED;
  const dim3 grid{unsigned(blocks), unsigned(groups)};
  cudaStream_t stream = static_cast<cudaStream_t>(stream_);
  SEPLLM_CUDA_TRY(dt_in == 0 ? (dt_out == 0 ? launch_norm<__nv_bfloat16, __nv_bfloat16>(p, rows, grid, stream)
                                            : launch_norm<__nv_bfloat16, float>(p, rows, grid, stream))
                             : (dt_out == 0 ? launch_norm<float, __nv_bfloat16>(p, rows, grid, stream)
                                            : launch_norm<float, float>(p, rows, grid, stream)));
  return SEPLLM_OK;
}

extern "C" sepllm_status sepllm_qknorm_rope_bwd_workspace_bytes(const sepllm_rope_desc* desc, size_t* bytes) {
  const sepllm_status st = check_rope(desc);
  if (st != SEPLLM_OK) return st;
  if (bytes) *bytes = align_up(size_t(kBwdBlocks) * 2 * desc->d * sizeof(float));
  return SEPLLM_OK;
}

extern "C" sepllm_status sepllm_qknorm_rope_bwd(const sepllm_rope_desc* desc, const sepllm_qknorm_desc* norm,
                                                const int64_t* positions, const sepllm_rope_view* x,
                                                const sepllm_rope_view* in, const sepllm_rope_view* out, float* dwq,
                                                float* dwk, void* workspace, void* stream_) {
  NormParams p{};
  bool vectors;
  int dt_in, dt_out;
  sepllm_status st = rope_params(desc, positions, in, out, -1.f, &p.r, &vectors, &dt_in, &dt_out);
  if (st != SEPLLM_OK) return st;
  if ((st = check_norm(norm)) != SEPLLM_OK) return st;
  if (!x || !workspace || !aligned(workspace, kAlign) || !aligned(dwq, 4) || !aligned(dwk, 4)) return SEPLLM_INVALID_ARG;
  if ((dwq && !norm->wq) || (dwk && !norm->wk)) return SEPLLM_INVALID_ARG;
  for (int w = 0; w < 2; ++w) {
    const sepllm_rope_view &a = x[w], &z = out[w];
    if (!a.data != !z.data) return SEPLLM_INVALID_ARG;
    if (!a.data) continue;
    const int heads = w == 0 ? desc->Hq : desc->Hkv;
    if (a.dtype != dt_out || !aligned(a.data, dt_out ? 4 : 2)) return SEPLLM_INVALID_ARG;
    if (a.stride_b < 0 || a.stride_h < 0 || a.stride_l < 0) return SEPLLM_INVALID_ARG;
    p.x[w] = a.data;
    p.xb[w] = desc->B > 1 ? a.stride_b : 0;
    p.xh[w] = heads > 1 ? a.stride_h : 0;
    p.xl[w] = desc->L > 1 ? a.stride_l : 0;
    const RopeTensor& t = p.r.t[w];
    if (a.data == z.data && (p.xb[w] != t.ob || p.xh[w] != t.oh || p.xl[w] != t.ol)) return SEPLLM_INVALID_ARG;
    vectors = vectors && vector_access(a.data, p.xb[w], p.xh[w], p.xl[w]);
  }
  fill_norm(desc, norm, &p);
  p.dw[0] = dwq;
  p.dw[1] = dwk;
  p.part = static_cast<float*>(workspace);
  const bool rows = by_rows(desc, p.r, vectors);
  const int64_t per_warp = rows ? 32 / (desc->d / 16) : 1;
  p.groups = (p.r.tokens + per_warp - 1) / per_warp;
  p.grid = 1;
  for (int w = 0; w < 3; ++w) {
    p.blocks[w] = int(std::min<int64_t>((p.groups * p.r.t[w].heads + kWarps - 1) / kWarps, kBwdBlocks));
    p.blocks[w] = std::max(p.blocks[w], 1);
    p.grid = std::max(p.grid, p.blocks[w]);
  }
  cudaStream_t stream = static_cast<cudaStream_t>(stream_);
  SEPLLM_CUDA_TRY(dt_out == 0 ? (dt_in == 0 ? launch_norm_bwd<__nv_bfloat16, __nv_bfloat16>(p, rows, stream)
                                            : launch_norm_bwd<__nv_bfloat16, float>(p, rows, stream))
                              : (dt_in == 0 ? launch_norm_bwd<float, __nv_bfloat16>(p, rows, stream)
                                            : launch_norm_bwd<float, float>(p, rows, stream)));
  if (dwq || dwk)
    SEPLLM_CUDA_TRY(launch_overlapped(norm_bwd_sum, dim3(2 * desc->d / 32), 1024, 0, stream, p));
  return SEPLLM_OK;
}
