// Rotary positions of queries and keys, and their gradient.
//
// Pair (x, y) of a head at position p becomes m (x cos a - y sin a), m (y cos a + x sin a) with
// a = p f_i; the gradient is the same map with -a.  Bound by HBM: every element of Q, K (and V,
// which is only laid out) is read once and written once.  cos and sin depend on (token, pair) and
// not on the head, so a thread takes one token and eight pairs, computes their cos and sin once and
// walks the heads with them; there is no table to build, size or read.  Measured: 65 536 tokens of 48
// heads x 128 in bf16, 1.61 GB, in 248 us (6.5 TB/s, the rate of a plain copy; 267 before the loads of
// several heads went out together), fp32 gradients of 16 384 such tokens to bf16 in 93 us (6.5 TB/s).
#include <algorithm>
#include <cmath>

#include "attn_common.cuh"

namespace sepllm {

namespace {

constexpr int kRopeThreads = 128;
constexpr int kMaxPairs = 64;
constexpr double kTwoPi = 6.283185307179586476925286766559;

struct RopeTensor {
  const void* in;
  void* out;
  int64_t ib, ih, il, ob, oh, ol;  // strides in elements
  int heads;
};

struct RopeParams {
  RopeTensor t[3];
  const int64_t* pos;
  int64_t pos_first, pos_stride;
  int64_t tokens;         // B * L
  int L, d, rot, n_heads, heads_per_block;
  float m, sign;          // sign: +1 forward, -1 gradient
  double turns[kMaxPairs];  // f_i / (2 pi)
};

// m cos and m sin of pair i at position p.  The angle is p f_i turns of which only the fraction
// matters: the product and its reduction are 64 bits (p up to 2^31 leaves 2e-7 of a turn), what
// is left is at most half a turn and is rounded to 32 bits.
__device__ __forceinline__ float2 rope_cos_sin(const RopeParams& p, double pos, int i) {
  const double t = pos * p.turns[i];
  float sn, cs;
  sincospif(2.f * float(t - rint(t)), &sn, &cs);
  return make_float2(p.m * cs, p.m * p.sign * sn);
}

__device__ __forceinline__ double rope_position(const RopeParams& p, int64_t b, int l) {
  return double(p.pos ? p.pos[b * p.pos_stride + l] : p.pos_first + l);
}

// Eight elements by 16-byte accesses: as they lie in memory, and as floats.
template <class T>
struct Eight {
  uint4 w[sizeof(T) / 2];
};
template <class T>
__device__ __forceinline__ Eight<T> load8(const T* s) {
  Eight<T> r;
#pragma unroll
  for (int k = 0; k < int(sizeof(T) / 2); ++k) r.w[k] = reinterpret_cast<const uint4*>(s)[k];
  return r;
}
__device__ __forceinline__ void to_floats(const Eight<__nv_bfloat16>& r, float (&x)[8]) {
  const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(r.w);
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float2 f = __bfloat1622float2(h[k]);
    x[2 * k] = f.x;
    x[2 * k + 1] = f.y;
  }
}
__device__ __forceinline__ void to_floats(const Eight<float>& r, float (&x)[8]) {
  const float* f = reinterpret_cast<const float*>(r.w);
#pragma unroll
  for (int k = 0; k < 8; ++k) x[k] = f[k];
}
__device__ __forceinline__ void store8(__nv_bfloat16* s, const float (&x)[8]) {
  *reinterpret_cast<uint4*>(s) = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]),
                                            pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
}
__device__ __forceinline__ void store8(float* s, const float (&x)[8]) {
  reinterpret_cast<float4*>(s)[0] = make_float4(x[0], x[1], x[2], x[3]);
  reinterpret_cast<float4*>(s)[1] = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ __forceinline__ float load1(const __nv_bfloat16* s) { return __bfloat162float(*s); }
__device__ __forceinline__ float load1(const float* s) { return *s; }
__device__ __forceinline__ void store1(__nv_bfloat16* s, float x) { *s = __float2bfloat16(x); }
__device__ __forceinline__ void store1(float* s, float x) { *s = x; }

// A thread owns 16 elements of a row (two 16-byte pieces c0, c1) and walks the heads: eight pairs
// whose halves are the two pieces (HALF), or four pairs in each piece (interleaved), or elements
// that are only copied.  d / 16 neighbouring threads cover a row.
template <class Tin, class Tout, bool HALF>
__global__ void __launch_bounds__(kRopeThreads) rope_rows(const __grid_constant__ RopeParams p) {
  const int per_row = p.d / 16;
  const int64_t id = int64_t(blockIdx.x) * kRopeThreads + threadIdx.x;
  const int64_t n = id / per_row;
  if (n >= p.tokens) return;
  const int t = int(id - n * per_row);
  const int64_t b = n / p.L;
  const int l = int(n - b * p.L);
  int c0, c1;  // first elements of the two pieces
  bool turn0;  // (some of) the thread's elements are rotated (in Q and K)
  // (neighbouring threads take neighbouring pieces, so that an access of a warp is contiguous in a row)
  if (HALF) {
    const int pairs = p.rot / 16;
    turn0 = t < pairs;
    c0 = 8 * (turn0 ? t : t + pairs);
    c1 = c0 + (turn0 ? p.rot / 2 : (p.d - p.rot) / 2);
  } else {
    c0 = 8 * t;
    c1 = c0 + p.d / 2;
    turn0 = c0 < p.rot;
  }
  const int h0 = blockIdx.y * p.heads_per_block, h1 = min(p.n_heads, h0 + p.heads_per_block);
  float2 cs[8];
  if (turn0 && h0 < p.t[0].heads + p.t[1].heads) {
    const double pos = rope_position(p, b, l);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int i = HALF ? c0 + k : (k < 4 ? c0 / 2 + k : c1 / 2 + k - 4);
      cs[k] = 2 * i < p.rot ? rope_cos_sin(p, pos, i) : make_float2(1.f, 0.f);
    }
  }
  int first = 0;  // heads of the tensors before this one
#pragma unroll
  for (int w = 0; w < 3; ++w) {
    const RopeTensor& x = p.t[w];
    const int a = max(h0 - first, 0), e = min(h1 - first, x.heads);
    first += x.heads;
    const Tin* src = static_cast<const Tin*>(x.in) + b * x.ib + l * x.il;
    Tout* dst = static_cast<Tout*>(x.out) + b * x.ob + l * x.ol;
    auto finish = [&](int h, const Eight<Tin>& ru, const Eight<Tin>& rv) {
      float u[8], v[8];
      to_floats(ru, u);
      to_floats(rv, v);
      if (w < 2) {
        if (HALF) {
          if (turn0) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              const float y0 = u[k] * cs[k].x - v[k] * cs[k].y;
              v[k] = v[k] * cs[k].x + u[k] * cs[k].y;
              u[k] = y0;
            }
          }
        } else {
          // (rot may end inside a piece, never inside a pair)
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            if (c0 + 2 * k < p.rot) {
              const float y0 = u[2 * k] * cs[k].x - u[2 * k + 1] * cs[k].y;
              u[2 * k + 1] = u[2 * k + 1] * cs[k].x + u[2 * k] * cs[k].y;
              u[2 * k] = y0;
            }
            if (c1 + 2 * k < p.rot) {
              const float y1 = v[2 * k] * cs[4 + k].x - v[2 * k + 1] * cs[4 + k].y;
              v[2 * k + 1] = v[2 * k + 1] * cs[4 + k].x + v[2 * k] * cs[4 + k].y;
              v[2 * k] = y1;
            }
          }
        }
      }
      store8(dst + h * x.oh + c0, u);
      store8(dst + h * x.oh + c1, v);
    };
    // several heads' loads go out before the first store (the compiler may not move a load over a
    // store: an output may be its input)
    constexpr int kBatch = sizeof(Tin) == 2 ? 4 : 2;   // 32 registers either way
    int h = a;
    for (; h + kBatch <= e; h += kBatch) {
      Eight<Tin> ru[kBatch], rv[kBatch];
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        ru[i] = load8(src + (h + i) * x.ih + c0);
        rv[i] = load8(src + (h + i) * x.ih + c1);
      }
#pragma unroll
      for (int i = 0; i < kBatch; ++i) finish(h + i, ru[i], rv[i]);
    }
    for (; h < e; ++h) finish(h, load8(src + h * x.ih + c0), load8(src + h * x.ih + c1));
  }
}

// Halves whose length is no multiple of a 16-byte piece (16 384 tokens x 48 heads x 128, r = 118: 100 us,
// 4.0 TB/s; element by element 136): a thread owns one piece of a row, a warp whole
// rows, and the other elements of the pairs come from the row in shared memory.
template <class Tin, class Tout>
__global__ void __launch_bounds__(kRopeThreads) rope_halves(const __grid_constant__ RopeParams p) {
  __shared__ __align__(16) float s_rows[kRopeThreads / 32][2][32 * 8];
  const int per_row = p.d / 8, rows = 32 / per_row, half = p.rot / 2;
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  const int rr = lane / per_row, c0 = (lane % per_row) * 8;
  const int64_t n = (int64_t(blockIdx.x) * (kRopeThreads / 32) + wid) * rows + rr;
  const bool here = rr < rows && n < p.tokens;
  const int64_t b = here ? n / p.L : 0;
  const int l = here ? int(n - b * p.L) : 0;
  const int h0 = blockIdx.y * p.heads_per_block, h1 = min(p.n_heads, h0 + p.heads_per_block);
  float2 cs[8];   // of each element: cos, and sin with the sign that its partner takes
  int other[8];   // place of the partner in the warp's rows; an element that is copied is its own
  const double pos = here ? rope_position(p, b, l) : 0.0;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int e = c0 + k;
    other[k] = rr * p.d + (e < half ? e + half : e < p.rot ? e - half : e);
    cs[k] = make_float2(1.f, 0.f);
    if (e < p.rot && h0 < p.t[0].heads + p.t[1].heads) {
      cs[k] = rope_cos_sin(p, pos, e < half ? e : e - half);
      if (e < half) cs[k].y = -cs[k].y;
    }
  }
  int first = 0;
#pragma unroll
  for (int w = 0; w < 3; ++w) {
    const RopeTensor& x = p.t[w];
    const int a = max(h0 - first, 0), z = min(h1 - first, x.heads);
    first += x.heads;
    const Tin* src = static_cast<const Tin*>(x.in) + b * x.ib + l * x.il + c0;
    Tout* dst = static_cast<Tout*>(x.out) + b * x.ob + l * x.ol + c0;
    for (int h = a; h < z; h += 2) {
      float u[2][8];
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (here && h + i < z) to_floats(load8(src + (h + i) * x.ih), u[i]);
      if (w < 2) {
        if (here) {
#pragma unroll
          for (int i = 0; i < 2; ++i)
            if (h + i < z) store8(s_rows[wid][i] + rr * p.d + c0, u[i]);
        }
        __syncwarp();
        if (here) {
#pragma unroll
          for (int i = 0; i < 2; ++i)
            if (h + i < z) {
#pragma unroll
              for (int k = 0; k < 8; ++k)
                if (c0 + k < p.rot) u[i][k] = u[i][k] * cs[k].x + s_rows[wid][i][other[k]] * cs[k].y;
            }
        }
        __syncwarp();
      }
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (here && h + i < z) store8(dst + (h + i) * x.oh, u[i]);
    }
  }
}

// Any rot_dim, stride and alignment: a thread owns one pair or one copied element.
template <class Tin, class Tout, bool HALF>
__global__ void __launch_bounds__(kRopeThreads) rope_elements(const __grid_constant__ RopeParams p) {
  const int half = p.rot / 2, per_row = p.d - half;
  const int64_t id = int64_t(blockIdx.x) * kRopeThreads + threadIdx.x;
  const int64_t n = id / per_row;
  if (n >= p.tokens) return;
  const int t = int(id - n * per_row);
  const int64_t b = n / p.L;
  const int l = int(n - b * p.L);
  const bool pair = t < half;
  const int c0 = pair ? (HALF ? t : 2 * t) : t + half;
  const int c1 = pair ? (HALF ? t + half : 2 * t + 1) : c0;
  const int h0 = blockIdx.y * p.heads_per_block, h1 = min(p.n_heads, h0 + p.heads_per_block);
  float2 cs = make_float2(1.f, 0.f);
  if (pair && h0 < p.t[0].heads + p.t[1].heads) cs = rope_cos_sin(p, rope_position(p, b, l), t);
  int first = 0;
#pragma unroll
  for (int w = 0; w < 3; ++w) {
    const RopeTensor& x = p.t[w];
    const int a = max(h0 - first, 0), e = min(h1 - first, x.heads);
    first += x.heads;
    const Tin* src = static_cast<const Tin*>(x.in) + b * x.ib + l * x.il;
    Tout* dst = static_cast<Tout*>(x.out) + b * x.ob + l * x.ol;
#pragma unroll 4
    for (int h = a; h < e; ++h) {
      float u = load1(src + h * x.ih + c0);
      float v = pair ? load1(src + h * x.ih + c1) : 0.f;
      if (w < 2 && pair) {
        const float y0 = u * cs.x - v * cs.y;
        v = v * cs.x + u * cs.y;
        u = y0;
      }
      store1(dst + h * x.oh + c0, u);
      if (pair) store1(dst + h * x.oh + c1, v);
    }
  }
}

bool finite_positive(double x) { return x > 0.0 && std::isfinite(x); }

sepllm_status check_rope(const sepllm_rope_desc* d) {
  if (!d) return SEPLLM_INVALID_ARG;
  if (d->B <= 0 || d->L <= 0 || d->Hq <= 0 || d->Hkv <= 0) return SEPLLM_INVALID_ARG;
  if (d->d < 64 || d->d > 128 || d->d % 16 != 0) return SEPLLM_UNSUPPORTED;
  const int r = d->rot_dim ? d->rot_dim : d->d;
  if (r < 2 || r > d->d || r % 2 != 0) return SEPLLM_INVALID_ARG;
  if (d->layout != SEPLLM_ROPE_HALF && d->layout != SEPLLM_ROPE_INTERLEAVED) return SEPLLM_INVALID_ARG;
  if (d->scaling < SEPLLM_ROPE_NONE || d->scaling > SEPLLM_ROPE_FACTORS) return SEPLLM_INVALID_ARG;
  if (!(d->base > 1.0) || !std::isfinite(d->base)) return SEPLLM_INVALID_ARG;
  if (d->attn_factor != 0.0 && !finite_positive(d->attn_factor)) return SEPLLM_INVALID_ARG;
  if (d->pos_stride < 0) return SEPLLM_INVALID_ARG;
  if (d->scaling >= SEPLLM_ROPE_LINEAR && d->scaling <= SEPLLM_ROPE_LLAMA3 && !finite_positive(d->factor))
    return SEPLLM_INVALID_ARG;
  if (d->scaling == SEPLLM_ROPE_NTK && r == 2) return SEPLLM_INVALID_ARG;
  if (d->scaling == SEPLLM_ROPE_YARN || d->scaling == SEPLLM_ROPE_LLAMA3)
    if (!finite_positive(d->orig_len) || !finite_positive(d->low) || !finite_positive(d->high) ||
        !(d->low < d->high))
      return SEPLLM_INVALID_ARG;
  if (d->scaling == SEPLLM_ROPE_FACTORS) {
    if (!d->freq_factors) return SEPLLM_INVALID_ARG;
    for (int i = 0; i < r / 2; ++i)
      if (!finite_positive(d->freq_factors[i])) return SEPLLM_INVALID_ARG;
  }
  return SEPLLM_OK;
}

double clamp01(double x) { return x < 0.0 ? 0.0 : (x > 1.0 ? 1.0 : x); }

// f_i, i < r/2, and m of a checked descriptor.
void rope_frequencies(const sepllm_rope_desc* d, double* f, double* m) {
  const int r = d->rot_dim ? d->rot_dim : d->d;
  const double s = d->factor;
  double base = d->base, lo = 0.0, hi = 0.0;
  if (d->scaling == SEPLLM_ROPE_NTK) base *= std::pow(s, double(r) / (r - 2));
  if (d->scaling == SEPLLM_ROPE_YARN) {
    auto pair_of = [&](double turns) {
      return r * std::log(d->orig_len / (kTwoPi * turns)) / (2.0 * std::log(base));
    };
    lo = std::fmax(0.0, std::floor(pair_of(d->high)));
    hi = std::fmin(r - 1.0, std::ceil(pair_of(d->low)));
    // lo behind the last pair (all turn often): the ramp lies behind them; hi before the first one (all
    // turn seldom): in front of them
    if (hi < 0.0) lo = hi - 1.0;
    else if (hi < lo) hi = lo + 1.0;
    else if (hi == lo) hi += 0.001;
  }
  // base^(-2i/r) as base^(-16 (i/8)/r) * base^(-2 (i%8)/r): sixteen powers instead of sixty-four (a
  // call computes them anew), within two roundings
  double small[8], large = 1.0;
  for (int i = 0; i < 8 && i < r / 2; ++i) small[i] = std::pow(base, -2.0 * i / r);
  for (int i = 0; i < r / 2; ++i) {
    if (i % 8 == 0) large = std::pow(base, -2.0 * i / r);
    double v = large * small[i % 8];
    if (d->scaling == SEPLLM_ROPE_LINEAR) v /= s;
    if (d->scaling == SEPLLM_ROPE_FACTORS) v /= d->freq_factors[i];
    if (d->scaling == SEPLLM_ROPE_YARN) {
      const double g = clamp01((i - lo) / (hi - lo));
      v = v * (1.0 - g) + v / s * g;
    }
    if (d->scaling == SEPLLM_ROPE_LLAMA3) {
      const double k = clamp01((d->orig_len * v / kTwoPi - d->low) / (d->high - d->low));
      v = v * k + v / s * (1.0 - k);
    }
    f[i] = v;
  }
  *m = d->attn_factor != 0.0 ? d->attn_factor
       : (d->scaling == SEPLLM_ROPE_YARN && s > 1.0) ? 0.1 * std::log(s) + 1.0
                                                     : 1.0;
}

// No two elements of [B][heads][L][d] share memory.  Sufficient: every stride covers the extent of
// the dimensions with smaller strides.
bool disjoint(const sepllm_rope_view& v, int64_t B, int64_t heads, int64_t L, int64_t d) {
  int64_t size[3] = {B, heads, L}, stride[3] = {v.stride_b, v.stride_h, v.stride_l};
  for (int i = 0; i < 2; ++i)
    for (int j = 0; j < 2 - i; ++j)
      if (stride[j] > stride[j + 1]) {
        const int64_t a = stride[j], c = size[j];
        stride[j] = stride[j + 1]; size[j] = size[j + 1];
        stride[j + 1] = a; size[j + 1] = c;
      }
  int64_t extent = d;  // elements from the first to one past the last of the dimensions so far
  for (int i = 0; i < 3; ++i) {
    if (size[i] == 1) continue;
    if (stride[i] < extent) return false;
    extent += stride[i] * (size[i] - 1);
  }
  return true;
}

bool vector_access(const void* data, int64_t sb, int64_t sh, int64_t sl) {
  return aligned(data, 16) && sb % 8 == 0 && sh % 8 == 0 && sl % 8 == 0;
}

template <class Tin, class Tout>
void launch_rope(const RopeParams& p, bool rows, bool half, dim3 grid, cudaStream_t stream) {
  if (rows && half && p.rot % 16 != 0) {
    rope_halves<Tin, Tout><<<grid, kRopeThreads, 0, stream>>>(p);
  } else if (rows) {
    if (half) rope_rows<Tin, Tout, true><<<grid, kRopeThreads, 0, stream>>>(p);
    else rope_rows<Tin, Tout, false><<<grid, kRopeThreads, 0, stream>>>(p);
  } else {
    if (half) rope_elements<Tin, Tout, true><<<grid, kRopeThreads, 0, stream>>>(p);
    else rope_elements<Tin, Tout, false><<<grid, kRopeThreads, 0, stream>>>(p);
  }
}

sepllm_status rope(const sepllm_rope_desc* d, const int64_t* positions, const sepllm_rope_view* in,
                   const sepllm_rope_view* out, float sign, cudaStream_t stream) {
  sepllm_status st = check_rope(d);
  if (st != SEPLLM_OK) return st;
  if (!in || !out || !aligned(positions, 8)) return SEPLLM_INVALID_ARG;
  RopeParams p{};
  p.rot = d->rot_dim ? d->rot_dim : d->d;
  const bool half = d->layout == SEPLLM_ROPE_HALF;
  bool rows = true;   // 16-byte accesses are possible
  int dt_in = -1, dt_out = -1;
  for (int w = 0; w < 3; ++w) {
    const sepllm_rope_view &a = in[w], &z = out[w];
    if (!a.data && !z.data) continue;
    if (!a.data || !z.data) return SEPLLM_INVALID_ARG;
    if ((a.dtype != 0 && a.dtype != 1) || (z.dtype != 0 && z.dtype != 1)) return SEPLLM_INVALID_ARG;
    if ((dt_in >= 0 && a.dtype != dt_in) || (dt_out >= 0 && z.dtype != dt_out)) return SEPLLM_INVALID_ARG;
    dt_in = a.dtype;
    dt_out = z.dtype;
    if (!aligned(a.data, dt_in ? 4 : 2) || !aligned(z.data, dt_out ? 4 : 2)) return SEPLLM_INVALID_ARG;
    if (a.stride_b < 0 || a.stride_h < 0 || a.stride_l < 0 || z.stride_b < 0 || z.stride_h < 0 ||
        z.stride_l < 0)
      return SEPLLM_INVALID_ARG;
    const int heads = w == 0 ? d->Hq : d->Hkv;
    if (!disjoint(z, d->B, heads, d->L, d->d)) return SEPLLM_INVALID_ARG;
    // strides of dimensions of size 1 are never used
    const int64_t ib = d->B > 1 ? a.stride_b : 0, ih = heads > 1 ? a.stride_h : 0, il = d->L > 1 ? a.stride_l : 0;
    const int64_t ob = d->B > 1 ? z.stride_b : 0, oh = heads > 1 ? z.stride_h : 0, ol = d->L > 1 ? z.stride_l : 0;
    if (a.data == z.data && (a.dtype != z.dtype || ib != ob || ih != oh || il != ol)) return SEPLLM_INVALID_ARG;
    rows = rows && vector_access(a.data, ib, ih, il) && vector_access(z.data, ob, oh, ol);
    p.t[w] = RopeTensor{a.data, z.data, ib, ih, il, ob, oh, ol, heads};
    p.n_heads += heads;
  }
  if (p.n_heads == 0) return SEPLLM_INVALID_ARG;
  double freq[kMaxPairs], m;
  rope_frequencies(d, freq, &m);
  for (int i = 0; i < p.rot / 2; ++i) p.turns[i] = freq[i] / kTwoPi;
  p.m = float(m);
  p.sign = sign;
  p.pos = positions;
  p.pos_first = d->pos_first;
  p.pos_stride = d->pos_stride;
  p.tokens = int64_t(d->B) * d->L;
  p.L = d->L;
  p.d = d->d;
  // threads: 16 elements of a row each (rope_rows), 8 with whole rows to a warp (rope_halves), or one
  // pair or copied element (rope_elements)
  const int64_t warp_rows = 32 / (d->d / 8);
  const int64_t threads = !rows                      ? p.tokens * (d->d - p.rot / 2)
                          : half && p.rot % 16 != 0 ? (p.tokens + warp_rows - 1) / warp_rows * 32
                                                     : p.tokens * (d->d / 16);
  const int64_t blocks = (threads + kRopeThreads - 1) / kRopeThreads;
  if (blocks > 0x7fffffff) return SEPLLM_UNSUPPORTED;
  // Heads are walked by one thread as long as that leaves threads to fill the SMs twice (2 x 2048 each); a
  // thread of its own costs every group of heads another eight sines and cosines.  Whole batches of
  // loads to a group.  Measured (us) with one, two, four times 1024 threads an SM: 36 heads x 64 of 8 x
  // 2048 tokens 29.6 / 28.4 / 28.8, 48 x 128 of 16 384 (fp32 in) 100 / 95 / 93, 14 x 80 of 5997 all 6.6,
  // and 8.5 with groups that do not fill their batches.
  const int64_t want = std::max<int64_t>(1, std::min<int64_t>(p.n_heads, int64_t(kSmCount) * 4096 / threads));
  p.heads_per_block = int((p.n_heads + want - 1) / want + 3) / 4 * 4;
  const int64_t groups = (p.n_heads + p.heads_per_block - 1) / p.heads_per_block;
  if (groups > 65535) return SEPLLM_UNSUPPORTED;
  const dim3 grid{unsigned(blocks), unsigned(groups)};
  if (dt_in == 0 && dt_out == 0) launch_rope<__nv_bfloat16, __nv_bfloat16>(p, rows, half, grid, stream);
  else if (dt_in == 0) launch_rope<__nv_bfloat16, float>(p, rows, half, grid, stream);
  else if (dt_out == 0) launch_rope<float, __nv_bfloat16>(p, rows, half, grid, stream);
  else launch_rope<float, float>(p, rows, half, grid, stream);
  SEPLLM_CUDA_TRY(cudaGetLastError());
  return SEPLLM_OK;
}

}  // namespace

}  // namespace sepllm

using namespace sepllm;

extern "C" sepllm_status sepllm_rope_frequencies(const sepllm_rope_desc* desc, double* freq, double* m) {
  sepllm_status st = check_rope(desc);
  if (st != SEPLLM_OK) return st;
  if (!freq || !m) return SEPLLM_INVALID_ARG;
  rope_frequencies(desc, freq, m);
  return SEPLLM_OK;
}

extern "C" sepllm_status sepllm_rope_fwd(const sepllm_rope_desc* desc, const int64_t* positions,
                                         const sepllm_rope_view* in, const sepllm_rope_view* out,
                                         void* stream_) {
  return rope(desc, positions, in, out, 1.f, static_cast<cudaStream_t>(stream_));
}

extern "C" sepllm_status sepllm_rope_bwd(const sepllm_rope_desc* desc, const int64_t* positions,
                                         const sepllm_rope_view* in, const sepllm_rope_view* out,
                                         void* stream_) {
  return rope(desc, positions, in, out, -1.f, static_cast<cudaStream_t>(stream_));
}
