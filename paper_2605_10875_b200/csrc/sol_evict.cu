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

// The sequence with the `place`-th longest cache: the longest first, so that no long one is left over at the end.  By a whole CTA
// (128 threads at least); ends with a barrier.
__device__ __forceinline__ int evict_sequence(const EvictArgs& p, int place) {
  __shared__ int lens[128], found;
  const int tid = threadIdx.x;
  if (tid < 128) lens[tid] = tid < p.B ? p.kv.seq_lens[tid] : 0;
  __syncthreads();
  if (tid < p.B) {
    const int mine = lens[tid];
    int rank = 0;
#pragma unroll 4
    for (int i = 0; i < p.B; ++i) rank += lens[i] > mine || (lens[i] == mine && i < tid);
    if (rank == place) found = tid;
  }
  __syncthreads();
  return found;
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
  const int kvh = blockIdx.x, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  pdl_wait();
  pdl_trigger();
  const int b = evict_sequence(p, blockIdx.y);
  const EvictPlan e = evict_plan(p, b);
  const size_t stride = (size_t)p.kv.max_pages_per_seq * PAGE, row = ((size_t)b * p.shape.n_kv_heads + kvh) * stride;
  int32_t* out = p.kept_idx + row;
  if (e.k >= e.T) {
    for (int i = tid; i < e.T; i += ES_THREADS) out[i] = i;
    return;
  }
  // Forced tokens have the largest key; a weight that is no number counts less than any.
  const int per = ((e.T + ES_THREADS - 1) / ES_THREADS) | 1;  // odd: the threads' runs start in different banks
  constexpr int L = 8;  // loads in flight
#pragma unroll 1
  for (int i0 = tid; i0 < per * ES_THREADS; i0 += L * ES_THREADS) {
    float w[L];
#pragma unroll
    for (int x = 0; x < L; ++x) w[x] = i0 + x * ES_THREADS < e.T ? p.weights[row + i0 + x * ES_THREADS] + 0.f : 0.f;  // one zero
#pragma unroll
    for (int x = 0; x < L; ++x) {
      const int i = i0 + x * ES_THREADS;
      uint32_t key = w[x] == w[x] ? float_key(w[x]) : 1u;
      if (i < e.sinks || i >= e.T - e.window) key = i < e.T ? 0xffffffffu : 0u;
      if (i < per * ES_THREADS) es_keys[i] = key;
    }
  }
  __syncthreads();
  if (e.k <= 0) return;
  int ties = 0;
  const uint32_t kth = select_kth<ES_THREADS, 0, true>([&](int i) { return es_keys[tid * per + i]; }, e.k, ties, sm, per);
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
// cos and sin of -2 pi (back * speed), speed in turns per position as a 64-bit fraction: the product wraps at whole turns by itself,
// and what is left is exact to 2^-32 of a turn.  Of the nearest quarter turn only the rest x is left, |x| <= pi / 4, where the
// Taylor polynomials up to x^9 and x^8 are off by less than 3e-8: a fifth of the instructions of sincospi, which was what bounded
// the move of one long sequence (130 us of 166).
__device__ __forceinline__ float2 turn_back(uint32_t back, uint2 speed) {
  const uint32_t part = 0u - (__umulhi(back, speed.x) + back * speed.y);  // turns * 2^32
  const uint32_t quarter = part + 0x20000000u;
  const float x = (float)(int32_t)(part - (quarter & 0xc0000000u)) * 1.4629180792671596e-9f;  // 2 pi / 2^32
  const float z = x * x;
  const uint64_t zz = f32x2(z, z);  // both polynomials at once: sin x / x, cos x
  uint64_t y = f32x2(2.7557319224e-6f, 2.4801587302e-5f);
  y = fma_f32x2(y, zz, f32x2(-1.9841269841e-4f, -1.3888888889e-3f));
  y = fma_f32x2(y, zz, f32x2(8.3333333333e-3f, 4.1666666667e-2f));
  y = fma_f32x2(y, zz, f32x2(-1.6666666667e-1f, -0.5f));
  y = fma_f32x2(y, zz, f32x2(1.f, 1.f));
  float s, c;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(s), "=f"(c) : "l"(y));
  s *= x;
  const bool odd = quarter & 0x40000000u;
  const float cos_ = odd ? s : c, sin_ = odd ? c : s;
  // quarter turns: 0 (c, s), 1 (-s, c), 2 (-c, -s), 3 (s, -c)
  return make_float2(__uint_as_float(__float_as_uint(cos_) ^ ((quarter ^ (quarter << 1)) & 0x80000000u)),
                     __uint_as_float(__float_as_uint(sin_) ^ (quarter & 0x80000000u)));
}

// A CTA takes `1 / slabs` of the 16-byte pieces of every kept row of a (sequence, kv-head)'s keys or values, a lane per piece and
// U rows per lane at a time: read, then written, in order.  In place this is safe: row j goes to slot j and kept_idx[j] >= j,
// so what a write covers is a row that has been read, and no other CTA touches these pieces.  Keys: the low lanes of a row hold
// pieces of its first half, the high ones the pieces that are rotated with them; each rotates four of the eight pairs.  The last
// CTA of a (sequence, kv-head) moves the weights, a token per thread.
// Bound by memory latency times rows in flight: whole rows where the batch fills the chip, otherwise slabs of 64 bytes, and more
// threads where there are few CTAs.
constexpr int EM_ROWS = 4;  // U
template <int HD>
__global__ void __launch_bounds__(1024) evict_move_kernel(const EvictArgs p, int slabs) {
  constexpr int PPR = HD / 8, U = EM_ROWS;
  __shared__ uint2 speeds[HD / 2];  // turns per position: low, high word
  const int kvh = blockIdx.y, tid = threadIdx.x, threads = blockDim.x;
  const int Hkv = p.shape.n_kv_heads, mp = p.kv.max_pages_per_seq;
  const bool keys = blockIdx.x < slabs, rope = keys && p.shape.rope_theta > 0.f;
  if (rope && tid < HD / 2) {
    const double turns = exp2(-2.0 * tid / HD * log2((double)p.shape.rope_theta)) * 0.15915494309189535;  // of one position
    const uint64_t fraction = (uint64_t)((turns - floor(turns)) * 0x1p64);
    speeds[tid] = make_uint2((uint32_t)fraction, (uint32_t)(fraction >> 32));
  }
  pdl_trigger();
  const int b = evict_sequence(p, blockIdx.z);  // its barriers are the speeds' too
  const EvictPlan e = evict_plan(p, b);
  const int32_t *table = p.kv.page_table + (size_t)b * mp, *dst_table = p.dst_table + (size_t)b * mp;
  const size_t row = ((size_t)b * Hkv + kvh) * mp * PAGE;
  const int32_t* kept = p.kept_idx + row;
  pdl_wait();
  if (blockIdx.x == 2 * slabs) {
#pragma unroll 1
    for (int j0 = 0; j0 < e.k; j0 += U * threads) {
      float w[U];
#pragma unroll
      for (int x = 0; x < U; ++x) {
        const int j = j0 + x * threads + tid;
        w[x] = j < e.k ? p.weights[row + kept[j]] : 0.f;
      }
      __syncthreads();
#pragma unroll
      for (int x = 0; x < U; ++x) {
        const int j = j0 + x * threads + tid;
        if (j < e.k) p.dst_weights[row + j] = w[x];
      }
    }
    if (kvh == 0 && tid == 0) p.dst_lens[b] = e.k;
    return;
  }
  uint4* pool = static_cast<uint4*>(keys ? p.kv.k_pool : p.kv.v_pool);
  const int lanes = PPR / slabs, half = lanes / 2, lane = tid % lanes, slab = keys ? blockIdx.x : blockIdx.x - slabs;
  const bool high = lane >= half;
  const int c = keys ? slab * half + (high ? lane - half + PPR / 2 : lane) : slab * lanes + lane;
  uint2 speed[4] = {};
  if (rope) {
#pragma unroll
    for (int i = 0; i < 4; ++i) speed[i] = speeds[(c % (PPR / 2)) * 8 + (high ? 4 : 0) + i];
  }
  auto at = [&](const int32_t* t, int slot) -> uint4* {
    const int page = t[slot / PAGE];
    if ((unsigned)page >= (unsigned)p.kv.num_pages) {
      atomicOr(p.status + ST_ERR, ERR_BAD_PAGE);
      return nullptr;
    }
    return pool + (((size_t)page * Hkv + kvh) * PAGE + slot % PAGE) * PPR + c;
  };
  const int step = threads / lanes, mine = tid / lanes;  // rows that the CTA takes side by side
  int next[U];
#pragma unroll
  for (int x = 0; x < U; ++x) next[x] = mine + x * step < e.k ? kept[mine + x * step] : -1;
#pragma unroll 1
  for (int j0 = mine; j0 - mine < e.k; j0 += U * step) {  // the same number of turns for every thread
    uint4 v[U];
    uint4* dst[U];
    int from[U];
#pragma unroll
    for (int x = 0; x < U; ++x) {
      from[x] = next[x];
      dst[x] = nullptr;
      v[x] = make_uint4(0u, 0u, 0u, 0u);
      if (from[x] >= 0) {
        const uint4* src = at(table, from[x]);
        uint4* to = at(dst_table, j0 + x * step);
        if (src && to && src != to) {
          v[x] = *src;
          dst[x] = to;
        }
      }
    }
#pragma unroll
    for (int x = 0; x < U; ++x) {
      const int j = j0 + (U + x) * step;
      next[x] = j < e.k ? kept[j] : -1;
    }
    if (rope) {
#pragma unroll
      for (int x = 0; x < U; ++x) {
        const uint32_t back = (uint32_t)(from[x] - (j0 + x * step));
        // the four pairs of this lane: its own elements, and the partner's
        const uint32_t give0 = high ? v[x].x : v[x].z, give1 = high ? v[x].y : v[x].w;
        const uint32_t got0 = __shfl_xor_sync(0xffffffffu, give0, half), got1 = __shfl_xor_sync(0xffffffffu, give1, half);
        const uint32_t lo[2] = {high ? got0 : v[x].x, high ? got1 : v[x].y}, hi[2] = {high ? v[x].z : got0, high ? v[x].w : got1};
        uint32_t new_lo[2], new_hi[2];
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          const float2 a = turn_back(back, speed[2 * w]), b2 = turn_back(back, speed[2 * w + 1]);
          new_lo[w] = pack_bf16(bf16_lo(lo[w]) * a.x - bf16_lo(hi[w]) * a.y, bf16_hi(lo[w]) * b2.x - bf16_hi(hi[w]) * b2.y);
          new_hi[w] = pack_bf16(bf16_lo(hi[w]) * a.x + bf16_lo(lo[w]) * a.y, bf16_hi(hi[w]) * b2.x + bf16_hi(lo[w]) * b2.y);
        }
        const uint32_t back0 = __shfl_xor_sync(0xffffffffu, high ? new_lo[0] : new_hi[0], half);
        const uint32_t back1 = __shfl_xor_sync(0xffffffffu, high ? new_lo[1] : new_hi[1], half);
        if (back) v[x] = high ? make_uint4(back0, back1, new_hi[0], new_hi[1]) : make_uint4(new_lo[0], new_lo[1], back0, back1);
      }
    }
    __syncthreads();
#pragma unroll
    for (int x = 0; x < U; ++x)
      if (dst[x]) *dst[x] = v[x];
  }
}

template <int HD>
static void launch_move(const EvictArgs& a, cudaStream_t st) {
  const int Hkv = a.shape.n_kv_heads, rows = 2 * a.B * Hkv;
  const int slabs = rows >= 4 * sm_count() ? 1 : HD / 32, ctas = rows * slabs;
  const int threads = ctas <= sm_count() ? 1024 : ctas <= 2 * sm_count() ? 512 : 256;
  SOL_LAUNCH("evict_move", evict_move_kernel<HD>, dim3(2 * slabs + 1, Hkv, a.B), dim3(threads), 0, st, a, slabs);
}

void launch_evict(const EvictArgs& a, cudaStream_t st) {
  const int per = ((a.kv.max_pages_per_seq * PAGE + ES_THREADS - 1) / ES_THREADS) | 1;
  const int smem = per * ES_THREADS * 4;
  ensure_dynamic_smem(reinterpret_cast<const void*>(&evict_select_kernel), smem);
  SOL_LAUNCH("evict_select", evict_select_kernel, dim3(a.shape.n_kv_heads, a.B), dim3(ES_THREADS), smem, st, a);
  if (a.shape.head_dim == 64) launch_move<64>(a, st);
  else launch_move<128>(a, st);
}

}  // namespace sol
