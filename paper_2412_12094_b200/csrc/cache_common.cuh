// What the cache calls share whatever the rows are held in: the state's layout, what an update does
// to a sequence, and where its entries are.
#pragma once
#include <algorithm>

#include "attn_common.cuh"

namespace sepllm {

struct CacheView {
  sepllm_cache_header* hdr;
  sepllm_cache_seq* seq;
  int64_t* slot_pos;
  uint8_t* slot_is_sep;
};

__host__ __device__ inline CacheView cache_view(void* state, const sepllm_cache_header& h) {
  uint8_t* p = static_cast<uint8_t*>(state);
  CacheView v;
  v.hdr = reinterpret_cast<sepllm_cache_header*>(p);
  v.seq = reinterpret_cast<sepllm_cache_seq*>(p + h.off_seq);
  v.slot_pos = reinterpret_cast<int64_t*>(p + h.off_slot_pos);
  v.slot_is_sep = p + h.off_slot_is_sep;
  return v;
}

inline sepllm_status fill_cache_header(const sepllm_cache_desc* d, sepllm_cache_header* h) {
  if (!d) return SEPLLM_INVALID_ARG;
  if (d->B <= 0 || d->Hkv <= 0 || d->Hq <= 0 || d->a < 0 || d->s < 0 || d->w < 1 || d->c < 1)
    return SEPLLM_INVALID_ARG;
  if (!(static_cast<int64_t>(d->a) + d->s + d->w < d->c)) return SEPLLM_INVALID_ARG;
  if (d->Hq % d->Hkv != 0) return SEPLLM_INVALID_ARG;
  if (d->d != 64 && d->d != 128) return SEPLLM_UNSUPPORTED;
  if (d->Hq / d->Hkv > 16) return SEPLLM_UNSUPPORTED;
  if (d->flags & ~SEPLLM_CACHE_FIXED_WINDOW) return SEPLLM_INVALID_ARG;
  *h = sepllm_cache_header{};
  h->magic = SEPLLM_CACHE_MAGIC;
  h->version = 1;
  h->slots = d->c + d->s;
  h->desc = *d;
  size_t off = sizeof(sepllm_cache_header);
  h->off_seq = off;
  off = align_up(off + sizeof(sepllm_cache_seq) * size_t(d->B));
  h->off_slot_pos = off;
  off = align_up(off + sizeof(int64_t) * size_t(d->B) * h->slots);
  h->off_slot_is_sep = off;
  off = align_up(off + size_t(d->B) * h->slots);
  h->total_bytes = off;
  return SEPLLM_OK;
}

// What one update does to a sequence, derived from the state before the update.
struct UpdatePlan {
  int append_slot;   // slot that receives the new token's K/V
  bool compact;      // Size_run reaches c with this token
  int n_past;        // Past Window entries examined by the compaction
  int drop;          // oldest Separator Cache entries (old and moved together) that fall out
};

__device__ __forceinline__ UpdatePlan plan_update(const sepllm_cache_seq& q,
                                                  const sepllm_cache_desc& d) {
  UpdatePlan p;
  p.compact = false;
  p.n_past = 0;
  p.drop = 0;
  if (q.size_init < d.a) {
    p.append_slot = q.size_init;
    return p;
  }
  const int ring = d.c - d.a;
  p.append_slot = d.a + d.s + (q.win_start + q.size_win) % ring;
  const int size_win = q.size_win + 1;
  if (d.flags & SEPLLM_CACHE_FIXED_WINDOW) {
    // fundamental design: the run is the w most recent tokens; what is older leaves at once
    if (size_win > d.w) {
      p.compact = true;
      p.n_past = size_win - d.w;
    }
  } else if (q.size_init + q.size_sep + size_win == d.c) {
    p.compact = true;
    p.n_past = size_win - d.w;
  }
  return p;
}

// Ring starts are below the ring size and v is below the region's entry count, so one conditional
// subtraction wraps the index (no integer division on the decode path).
__device__ __forceinline__ int virtual_to_slot(int v, const sepllm_cache_seq& q,
                                               const sepllm_cache_desc& d) {
  if (v < q.size_init) return v;
  v -= q.size_init;
  if (v < q.size_sep) {
    const int x = q.sep_start + v;
    return d.a + (x >= d.s ? x - d.s : x);
  }
  v -= q.size_sep;
  const int ring = d.c - d.a, x = q.win_start + v;
  return d.a + d.s + (x >= ring ? x - ring : x);
}

constexpr int kUpdThreads = 256;

// Exclusive rank of every separator among the Past Window entries, in position order.
// rank_s[k] (k < n_past) = number of separators among past entries [0, k); returns the total.
// n_past <= kMaxPast.
static __device__ int rank_past_separators(const uint8_t* slot_is_sep_b, const sepllm_cache_seq& q,
                                    const sepllm_cache_desc& d, int n_past, int16_t* flag_s,
                                    int* warp_buf) {
  const int ring = d.c - d.a;
  const int base = d.a + d.s;
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  const int per = (n_past + kUpdThreads - 1) / kUpdThreads;
  const int k0 = tid * per, k1 = min(n_past, k0 + per);
  int local = 0;
  for (int k = k0; k < k1; ++k) {
    const int f = slot_is_sep_b[base + (q.win_start + k) % ring];
    flag_s[k] = int16_t(f);
    local += f;
  }
  int incl = local;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int t = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += t;
  }
  if (lane == 31) warp_buf[wid] = incl;
  __syncthreads();
  int woff = 0, total = 0;
  for (int k = 0; k < kUpdThreads / 32; ++k) {
    if (k < wid) woff += warp_buf[k];
    total += warp_buf[k];
  }
  int run = woff + incl - local;
  // flag_s[k] becomes rank+1 for separators, 0 otherwise
  for (int k = k0; k < k1; ++k) {
    if (flag_s[k]) { flag_s[k] = int16_t(run + 1); ++run; }
  }
  __syncthreads();
  return total;
}

constexpr int kMaxPast = 24576;  // int16 ranks in shared memory: 48 KB


// The moves of a compaction: m Past Window separators join the Separator Cache, whose `drop` oldest entries
// (old and joined together) fall out.
struct UpdateMoves {
  bool any;   // the compaction looks at separators at all
  int m, drop;
};

// Where Past Window entry k of a compaction goes (src, dst: slots; flag_s: its rank + 1 among the
// separators, 0 for other tokens); false: it is dropped.
__device__ __forceinline__ bool past_move(int k, const int16_t* flag_s, const sepllm_cache_seq& q,
                                          const sepllm_cache_desc& d, int drop, int* src, int* dst) {
  const int r = flag_s[k];
  if (r == 0) return false;
  const int fifo = q.size_sep + (r - 1);  // place in the queue of old + moved separators
  if (fifo < drop) return false;          // falls out at once
  *src = d.a + d.s + (q.win_start + k) % (d.c - d.a);
  *dst = d.a + (q.sep_start + fifo) % d.s;
  return true;
}

// The sequence's record after an update (every CTA derives the same one).
__device__ __forceinline__ sepllm_cache_seq next_record(const sepllm_cache_seq& q, const sepllm_cache_desc& d,
                                                        const UpdatePlan& p, const UpdateMoves& mv) {
  sepllm_cache_seq nq = q;
  nq.reserved[0] = 0;  // arrival count for the next update
  nq.next_pos = q.next_pos + 1;
  if (q.size_init < d.a) nq.size_init = q.size_init + 1;
  else nq.size_win = q.size_win + 1;
  if (p.compact) {
    if (mv.any) {
      nq.sep_start = (q.sep_start + mv.drop) % d.s;
      nq.size_sep = q.size_sep + mv.m - mv.drop;
    }
    nq.win_start = (q.win_start + p.n_past) % (d.c - d.a);
    nq.size_win = d.w;
    nq.compactions = q.compactions + 1;
  }
  return nq;
}

// The last kv head of the sequence to get here updates the state: per-slot positions and flags, and the
// record.  All threads of the block call it, behind their moves.
static __device__ void finish_update(const CacheView& v, const sepllm_cache_header& h, int b,
                                     const sepllm_cache_seq& q, const sepllm_cache_seq& nq, const UpdatePlan& p,
                                     const UpdateMoves& mv, const int16_t* flag_s, const int32_t* new_token_ids,
                                     const SepIds& sep) {
  __shared__ int s_last;
  const sepllm_cache_desc& d = h.desc;
  const int tid = threadIdx.x;
  if (tid == 0) {
    __threadfence();
    const int prev = atomicAdd(&v.seq[b].reserved[0], 1);
    s_last = (prev == d.Hkv - 1);
  }
  __syncthreads();
  if (!s_last) return;
  __threadfence();
  int64_t* pos_b = v.slot_pos + size_t(b) * h.slots;
  uint8_t* sep_b = v.slot_is_sep + size_t(b) * h.slots;
  if (tid == 0) {
    pos_b[p.append_slot] = q.next_pos;
    sep_b[p.append_slot] = uint8_t(is_separator(new_token_ids[b], sep));
    // a Separator Cache that is not meant to evict did
    if ((d.flags & SEPLLM_CACHE_FIXED_WINDOW) && mv.drop > 0)
      set_status(&v.hdr->status, SEPLLM_CAPACITY_EXCEEDED);
  }
  if (mv.any) {
    for (int k = tid; k < p.n_past; k += kUpdThreads) {
      int src, dst;
      if (!past_move(k, flag_s, q, d, mv.drop, &src, &dst)) continue;
      pos_b[dst] = pos_b[src];
      sep_b[dst] = 1;
    }
  }
  if (tid == 0) v.seq[b] = nq;
}

// Checks and shapes of an update: the separators by value, and the Past Window entries a compaction may
// look at.
inline sepllm_status update_params(const sepllm_cache_desc* desc, const int32_t* sep_ids, int32_t n_sep, SepIds* sep,
                                   int* max_past) {
  if (n_sep < 0 || (n_sep > 0 && !sep_ids)) return SEPLLM_INVALID_ARG;
  if (n_sep > SEPLLM_MAX_SEP_IDS) return SEPLLM_UNSUPPORTED;
  *max_past = (desc->flags & SEPLLM_CACHE_FIXED_WINDOW) ? 1 : desc->c - desc->a - desc->w;
  if (*max_past > kMaxPast || desc->Hkv > 65535) return SEPLLM_UNSUPPORTED;
  sep->n = n_sep;
  for (int k = 0; k < SEPLLM_MAX_SEP_IDS; ++k) sep->id[k] = (k < n_sep) ? sep_ids[k] : -1;
  return SEPLLM_OK;
}

// Lets an update's kernel use `bytes` of shared memory.  The limit is the kernel's, for all calls on the device: it is
// only ever set to what the largest update needs, so that no call takes away another thread's.
template <class Kernel>
cudaError_t allow_update_smem(Kernel kernel, size_t bytes, int bytes_per_entry) {
  if (bytes <= 40 * 1024) return cudaSuccess;   // (48 KB, static memory included, need no leave)
  return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxPast * bytes_per_entry);
}

// The state that a pre-filled prompt leaves (cache.cu): sizes, positions and flags, rings from slot 0.
sepllm_status launch_prompt_plan(const sepllm_cache_header& h, const sepllm_index_header& ih, void* state,
                                 const void* index, const int32_t* prompt_len, cudaStream_t stream);

}  // namespace sepllm
