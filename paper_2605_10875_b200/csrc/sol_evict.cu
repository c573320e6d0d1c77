// Eviction: of every (sequence, kv-head) the budget's tokens of largest accumulated weight stay, and move together in order.
//
//   evict_select_kernel  a CTA per (sequence, kv-head): the row's weights as sortable keys in shared memory, radix select of the
//                        budget's last one (sol_select.cuh), ascending list of the kept tokens
//   evict_move_kernel    rows of keys and values to their new slots, the weights with them.  A key moves from position i to
//                        position j <= i and is rotated by j - i, so that slot t keeps a key at position t, which is where the
//                        decode step will put its queries and the next key.
#include <math.h>

#include "sol_common.cuh"
#include "sol_internal.h"
#include "sol_select.cuh"

namespace sol {

// How many tokens of a sequence stay: the budget, the sinks and the window at least.
struct EvictPlan {
  int T, sinks, window, k;
};
__device__ __forceinline__ EvictPlan evict_plan(const EvictArgs& p, int b) {
  EvictPlan e;
  e.T = min(max(p.kv.seq_lens[b], 0), p.kv.max_pages_per_seq * PAGE);
  e.sinks = min(p.shape.n_sink, e.T);
  e.window = min(p.shape.n_window, e.T - e.sinks);
  e.k = min(e.T, max(p.budgets[b], e.sinks + e.window));
  return e;
}

constexpr int ES_THREADS = 1024;
struct EvictSmem {
  uint32_t hist[SEL_BINS];
  uint32_t rank_key[SEL_RANK_CAP];
  int pick[3];
  int scan[2][SEL_MAX_WARPS];
  int counts[4];
};

__global__ void __launch_bounds__(ES_THREADS) evict_select_kernel(const EvictArgs p) {
  extern __shared__ uint32_t es_keys[];
  __shared__ EvictSmem sm;
  const int kvh = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  pdl_wait();
  pdl_trigger();
  const EvictPlan e = evict_plan(p, b);
  const size_t stride = (size_t)p.kv.max_pages_per_seq * PAGE, row = ((size_t)b * p.shape.n_kv_heads + kvh) * stride;
  int32_t* out = p.kept_idx + row;
  if (e.k >= e.T) {
    for (int i = tid; i < e.T; i += ES_THREADS) out[i] = i;
    return;
  }
  // Forced tokens have the largest key; a weight that is no number counts less than any.
  const int per = ((e.T + ES_THREADS - 1) / ES_THREADS) | 1;  // odd: the threads' runs start in different banks
  for (int i = tid; i < per * ES_THREADS; i += ES_THREADS) {
    uint32_t key = 0;
    if (i < e.T) {
      const float w = p.weights[row + i] + 0.f;  // one zero
      key = w == w ? float_key(w) : 1u;
      if (i < e.sinks || i >= e.T - e.window) key = 0xffffffffu;
    }
    es_keys[i] = key;
  }
  __syncthreads();
  if (e.k <= 0) return;
  int ties = 0;
  const uint32_t kth = select_kth<ES_THREADS, 0>([&](int i) { return es_keys[tid * per + i]; }, e.k, ties, sm, per);
  __syncthreads();
  // kept before this thread's run: those above the k-th, and of its equals the first `ties`
  int above = 0, equal = 0;
  for (int i = 0; i < per; ++i) {
    const uint32_t key = es_keys[tid * per + i];
    above += key > kth;
    equal += key == kth;
  }
  int a = above, q = equal;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, a, o), y = __shfl_up_sync(0xffffffffu, q, o);
    if (lane >= o) {
      a += x;
      q += y;
    }
  }
  if (lane == 31) {
    sm.scan[0][warp] = a;
    sm.scan[1][warp] = q;
  }
  __syncthreads();
  a -= above;
  q -= equal;
  for (int w = 0; w < warp; ++w) {
    a += sm.scan[0][w];
    q += sm.scan[1][w];
  }
  int at = a + min(q, ties);
  for (int i = 0; i < per; ++i) {
    const uint32_t key = es_keys[tid * per + i];
    if (key > kth || (key == kth && q++ < ties)) out[at++] = tid * per + i;
  }
}

// ---- the move ------------------------------------------------------------------------------------
constexpr int EM_THREADS = 256;

// cos and sin of 2 pi (delta * speed), speed in turns per position as a 64-bit fraction: the product wraps at whole turns by
// itself, and what is left is exact to 2^-32 of a turn.
__device__ __forceinline__ float2 turn(int delta, uint64_t speed) {
  const int32_t part = (int32_t)(((uint64_t)(int64_t)delta * speed) >> 32);
  float s, c;
  sincospif((float)part * 0x1p-31f, &s, &c);
  return make_float2(c, s);
}

// A CTA takes four 16-byte pieces of every kept row of a (sequence, kv-head): 64 rows at a time, read, then written, in order.
// In place this is safe: row j goes to slot j and kept_idx[j] >= j, so what a write covers is a row that has been read, and no
// other CTA touches these pieces.  Keys: two pieces and the two half a row on, which are rotated with them.  The last CTA of
// a row moves the weights, a token per thread.
template <int HD>
__global__ void __launch_bounds__(EM_THREADS) evict_move_kernel(const EvictArgs p) {
  constexpr int PPR = HD / 8, SLABS = PPR / 4;
  __shared__ uint64_t speed[16];  // turns per position of the slab's 16 pairs
  const int part = blockIdx.x, kvh = blockIdx.y, b = blockIdx.z, tid = threadIdx.x;
  const int Hkv = p.shape.n_kv_heads, mp = p.kv.max_pages_per_seq;
  const bool keys = part < SLABS, rope = keys && p.shape.rope_theta > 0.f;
  if (rope && tid < 16) {
    const int f = part * 16 + tid;
    const double turns = exp2(-2.0 * f / HD * log2((double)p.shape.rope_theta)) * 0.15915494309189535;  // of one position
    speed[tid] = (uint64_t)((turns - floor(turns)) * 0x1p64);
  }
  pdl_trigger();
  const EvictPlan e = evict_plan(p, b);
  const int32_t *table = p.kv.page_table + (size_t)b * mp, *dst_table = p.dst_table + (size_t)b * mp;
  const size_t row = ((size_t)b * Hkv + kvh) * mp * PAGE;
  pdl_wait();
  if (part == 2 * SLABS) {
    for (int j0 = 0; j0 < e.k; j0 += EM_THREADS) {
      const int j = j0 + tid;
      float w = 0.f;
      if (j < e.k) w = p.weights[row + p.kept_idx[row + j]];
      __syncthreads();
      if (j < e.k) p.dst_weights[row + j] = w;
    }
    if (kvh == 0 && tid == 0) p.dst_lens[b] = e.k;
    return;
  }
  __syncthreads();
  uint4* pool = static_cast<uint4*>(keys ? p.kv.k_pool : p.kv.v_pool);
  const int lane = tid & 3, c = keys ? part * 2 + (lane & 1) + (lane >> 1) * (PPR / 2) : (part - SLABS) * 4 + lane;
  auto at = [&](const int32_t* t, int slot) -> uint4* {
    const int page = t[slot / PAGE];
    if (page < 0 || page >= p.kv.num_pages) {
      atomicOr(p.status + ST_ERR, ERR_BAD_PAGE);
      return nullptr;
    }
    return pool + (((size_t)page * Hkv + kvh) * PAGE + slot % PAGE) * PPR + c;
  };
  for (int j0 = 0; j0 < e.k; j0 += EM_THREADS / 4) {
    const int j = j0 + (tid >> 2);
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    uint4* dst = nullptr;
    int i = j;
    if (j < e.k) {
      i = p.kept_idx[row + j];
      const uint4* src = at(table, i);
      dst = at(dst_table, j);
      if (src && src != dst) v = *src;
      else dst = nullptr;
    }
    if (rope) {  // the partner half of the pairs is in the lane two on
      uint32_t x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const uint32_t y = __shfl_xor_sync(0xffffffffu, x[w], 2);
        float r[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float mine = h ? bf16_hi(x[w]) : bf16_lo(x[w]), other = h ? bf16_hi(y) : bf16_lo(y);
          const float2 cs = turn(j - i, speed[(lane & 1) * 8 + w * 2 + h]);
          r[h] = lane >> 1 ? mine * cs.x + other * cs.y : mine * cs.x - other * cs.y;
        }
        x[w] = i == j ? x[w] : pack_bf16(r[0], r[1]);
      }
      v = make_uint4(x[0], x[1], x[2], x[3]);
    }
    __syncthreads();
    if (dst) *dst = v;
  }
}

void launch_evict(const EvictArgs& a, cudaStream_t st) {
  const int Hkv = a.shape.n_kv_heads, slabs = a.shape.head_dim / 32;
  const int per = ((a.kv.max_pages_per_seq * PAGE + ES_THREADS - 1) / ES_THREADS) | 1;
  const int smem = per * ES_THREADS * 4;
  ensure_dynamic_smem(reinterpret_cast<const void*>(&evict_select_kernel), smem);
  SOL_LAUNCH("evict_select", evict_select_kernel, dim3(Hkv, a.B), dim3(ES_THREADS), smem, st, a);
  const dim3 grid(2 * slabs + 1, Hkv, a.B);
  if (a.shape.head_dim == 64) SOL_LAUNCH("evict_move", evict_move_kernel<64>, grid, dim3(EM_THREADS), 0, st, a);
  else SOL_LAUNCH("evict_move", evict_move_kernel<128>, grid, dim3(EM_THREADS), 0, st, a);
}

}  // namespace sol
