// What the rotary and the head-norm kernels share: tensors by their strides, angles, 16-byte accesses, and
// the checks of descriptors and views.
#pragma once
#include <algorithm>
#include <cmath>

#include "attn_common.cuh"

namespace sepllm {

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

inline bool finite_positive(double x) { return x > 0.0 && std::isfinite(x); }

inline sepllm_status check_rope(const sepllm_rope_desc* d) {
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

inline double clamp01(double x) { return x < 0.0 ? 0.0 : (x > 1.0 ? 1.0 : x); }

// f_i, i < r/2, and m of a checked descriptor.
inline void rope_frequencies(const sepllm_rope_desc* d, double* f, double* m) {
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
inline bool disjoint(const sepllm_rope_view& v, int64_t B, int64_t heads, int64_t L, int64_t d) {
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

inline bool vector_access(const void* data, int64_t sb, int64_t sh, int64_t sl) {
  return aligned(data, 16) && sb % 8 == 0 && sh % 8 == 0 && sl % 8 == 0;
}

// The views of a call as parameters, checked.  rows: 16-byte accesses are possible; dtypes of the
// inputs and of the outputs (-1: no tensor).
inline sepllm_status rope_params(const sepllm_rope_desc* d, const int64_t* positions, const sepllm_rope_view* in,
                                 const sepllm_rope_view* out, float sign, RopeParams* params, bool* rows_out,
                                 int* dt_in_out, int* dt_out_out) {
  sepllm_status st = check_rope(d);
  if (st != SEPLLM_OK) return st;
  if (!in || !out || !aligned(positions, 8)) return SEPLLM_INVALID_ARG;
  RopeParams& p = *params;
  p = RopeParams{};
  p.rot = d->rot_dim ? d->rot_dim : d->d;
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
  *rows_out = rows;
  *dt_in_out = dt_in;
  *dt_out_out = dt_out;
  return SEPLLM_OK;
}

// Heads walked by one thread of `threads`.  They are walked as long as that leaves threads to fill the SMs
// twice (2 x 2048 each); a thread of its own costs every group of heads another eight sines and cosines.
// Whole batches of loads to a group.  Measured on the rotary kernels (us) with one, two, four times 1024
// threads an SM: 36 heads x 64 of 8 x 2048 tokens 29.6 / 28.4 / 28.8, 48 x 128 of 16 384 (fp32 in) 100 / 95 / 93,
// 14 x 80 of 5997 all 6.6, and 8.5 with groups that do not fill their batches.
inline int rope_heads_per_thread(int n_heads, int64_t threads) {
  const int64_t want = std::max<int64_t>(1, std::min<int64_t>(n_heads, int64_t(kSmCount) * 4096 / threads));
  return int((n_heads + want - 1) / want + 3) / 4 * 4;
}

}  // namespace sepllm
