// Rotary positions of queries and keys, and their gradient.
//
// Pair (x, y) of a head at position p becomes m (x cos a - y sin a), m (y cos a + x sin a) with
// a = p f_i; the gradient is the same map with -a.  Bound by HBM: every element of Q, K (and V,
// which is only laid out) is read once and written once.  cos and sin depend on (token, pair) and
// not on the head, so a thread takes one token and eight pairs, computes their cos and sin once and
// walks the heads with them; there is no table to build, size or read.  Measured: 65 536 tokens of 48
// heads x 128 in bf16, 1.61 GB, in 248 us (6.5 TB/s, the rate of a plain copy; 267 before the loads of
// several heads went out together), fp32 gradients of 16 384 such tokens to bf16 in 93 us (6.5 TB/s).
#include "rope_common.cuh"

namespace sepllm {

namespace {

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
  RopeParams p;
  bool rows;
  int dt_in, dt_out;
  const sepllm_status st = rope_params(d, positions, in, out, sign, &p, &rows, &dt_in, &dt_out);
  if (st != SEPLLM_OK) return st;
  const bool half = d->layout == SEPLLM_ROPE_HALF;
  // threads: 16 elements of a row each (rope_rows), 8 with whole rows to a warp (rope_halves), or one
  // pair or copied element (rope_elements)
  const int64_t warp_rows = 32 / (d->d / 8);
  const int64_t threads = !rows                      ? p.tokens * (d->d - p.rot / 2)
                          : half && p.rot % 16 != 0 ? (p.tokens + warp_rows - 1) / warp_rows * 32
                                                     : p.tokens * (d->d / 16);
  const int64_t blocks = (threads + kRopeThreads - 1) / kRopeThreads;
  if (blocks > 0x7fffffff) return SEPLLM_UNSUPPORTED;
  p.heads_per_block = rope_heads_per_thread(p.n_heads, threads);
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
