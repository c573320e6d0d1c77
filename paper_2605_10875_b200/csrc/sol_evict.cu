// Eviction: of every (sequence, kv-head) the budget's tokens of largest accumulated weight stay, and move together in order.
//
//   evict_select_kernel  a CTA per (sequence, kv-head): the row's weights in shared memory, radix select of the budget's last one
//                        (sol_select.cuh), ascending list of the kept tokens, their weights moved together
//   evict_move_kernel    rows of keys and values to their new slots.  A key moves from position i to position j <= i and is
//                        rotated by j - i, so that slot t keeps a key at position t, which is where the decode step will put
//                        its queries and the next key.
//   evict_moved_kernel   with tracked origins: how far every kept key has been moved in all
//
// A key that is rotated where it lies is rounded to bf16 each time, and the roundings of many small turns do not cancel: a pair that
// turns by less than half a step stays where it was.  (Keys off by 0.0017 after one move; 200 moves of one position 0.032, 1000 0.44.)
// With tracked origins a key is rotated from what it was before its first move, by the whole distance, and rounded once.  That writes
// every moved key twice and leaves its angles to the polynomials where neighbours have moved unequally far (half of 24 caches of 9000
// 216 us, tracked 276; one token of 16 caches of 4097, head_dim 64, 69 us, tracked 92).
#include <math.h>

#include <algorithm>

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

// Order of the kept: forced tokens, then by weight; a weight that is no number counts less than any, and there is one zero.
__device__ __forceinline__ uint32_t evict_key(const EvictPlan& e, int i, float w) {
  const uint32_t key = w == w ? float_key(w + 0.f) : 1u;
  return i < e.sinks || i >= e.T - e.window ? 0xffffffffu : key;
}

__global__ void __launch_bounds__(ES_THREADS) evict_select_kernel(const EvictArgs p) {
  extern __shared__ __align__(16) float es_w[];  // the row's weights: in place, too, they are all read before one is written
  __shared__ EvictSmem sm;
  const int kvh = blockIdx.x, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  pdl_wait();
  pdl_trigger();
  const int b = evict_sequence(p, blockIdx.y);
  const EvictPlan e = evict_plan(p, b);
  const size_t stride = (size_t)p.kv.max_pages_per_seq * PAGE, row = ((size_t)b * p.shape.n_kv_heads + kvh) * stride;
  int32_t* out = p.kept_idx + row;
  if (kvh == 0 && tid == 0) p.dst_lens[b] = e.k;
  constexpr int L = 8;  // loads in flight
#pragma unroll 1
  for (int i0 = tid; i0 < e.T; i0 += L * ES_THREADS) {
    float w[L];
#pragma unroll
    for (int x = 0; x < L; ++x) w[x] = i0 + x * ES_THREADS < e.T ? p.weights[row + i0 + x * ES_THREADS] : 0.f;
#pragma unroll
    for (int x = 0; x < L; ++x) {
      const int i = i0 + x * ES_THREADS;
      if (i >= e.T) break;
      es_w[i] = w[x];
      if (e.k >= e.T) {  // all stay
        out[i] = i;
        p.dst_weights[row + i] = w[x];
      }
    }
  }
  if (e.k >= e.T || e.k <= 0) return;
  __syncthreads();
  const int per = ((e.T + ES_THREADS - 1) / ES_THREADS) | 1;  // odd: the threads' runs start in different banks
  int ties = 0;
  const uint32_t kth = select_kth<ES_THREADS, 0, true>(
      [&](int x) {
        const int i = tid * per + x;
        return i < e.T ? evict_key(e, i, es_w[i]) : 0u;
      },
      e.k, ties, sm, per);
  __syncthreads();
  // A warp lists a run of tokens, 128 side by side, four a lane: those above the k-th, and of its equals the first `ties`.  (A run per
  // thread writes every entry to a sector of its own, 18 us of 37 for a row of 32000; one token a lane takes twice the instructions:
  // evictions of 16 sequences of 4096 33 us instead of 30, though 109 instead of 111 for one of 30000, whose entries it writes denser.)
  const int run = (e.T + ES_THREADS * 4 - 1) / (ES_THREADS * 4) * 128, i0 = warp * run, i1 = min(e.T, i0 + run);
  const auto read4 = [&](int i, float (&w)[4], uint32_t (&key)[4]) {  // behind the row: key 0, which no kth is
    const float4 v = i < i1 ? *reinterpret_cast<const float4*>(es_w + i) : make_float4(0.f, 0.f, 0.f, 0.f);
    w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
#pragma unroll
    for (int x = 0; x < 4; ++x) key[x] = i + x < i1 ? evict_key(e, i + x, w[x]) : 0u;
  };
  int both = 0;  // equal << 16 | above, of at most 49152 / 32 tokens
#pragma unroll 2
  for (int c = i0; c < i1; c += 128) {
    float w[4];
    uint32_t key[4];
    read4(c + 4 * lane, w, key);
#pragma unroll
    for (int x = 0; x < 4; ++x) both += (key[x] > kth) + ((key[x] == kth) << 16);
  }
  both = __reduce_add_sync(0xffffffffu, both);
  if (lane == 0) {
    sm.scan[0][warp] = both & 0xffff;
    sm.scan[1][warp] = both >> 16;
  }
  __syncthreads();
  int above = __reduce_add_sync(0xffffffffu, lane < warp ? sm.scan[0][lane] : 0);
  int same = __reduce_add_sync(0xffffffffu, lane < warp ? sm.scan[1][lane] : 0);
#pragma unroll 1
  for (int c = i0; c < i1; c += 128) {
    const int i = c + 4 * lane;
    float w[4];
    uint32_t key[4];
    read4(i, w, key);
    int mine = 0;
#pragma unroll
    for (int x = 0; x < 4; ++x) mine += (key[x] > kth) + ((key[x] == kth) << 16);
    int upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += v;
    }
    int at = above + ((upto - mine) & 0xffff), eq = same + ((upto - mine) >> 16);  // tokens above and equal ahead of this lane's
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      if (key[x] > kth || (key[x] == kth && eq < ties)) {
        const int j = at + min(eq, ties);
        out[j] = i + x;
        p.dst_weights[row + j] = w[x];
      }
      at += key[x] > kth;
      eq += key[x] == kth;
    }
    const int all = __shfl_sync(0xffffffffu, upto, 31);
    above += all & 0xffff;
    same += all >> 16;
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

// A CTA moves `1 / slabs` of every kept row of a (sequence, kv-head)'s keys or values, chunks of 32 rows through a ring in shared
// memory: half of its warps request chunks in turn, 16 bytes a lane, half write them out in turn, and one says how many have
// arrived.  In place this is safe: row j goes to slot j and kept_idx[j] >= j, so what the write of a chunk covers is a row of that
// chunk or an earlier one, and a warp writes a chunk only when that chunk and all before it have arrived; what is requested later
// lies behind every slot written so far; and no other CTA touches these pieces.
// Keys: a slab of a row is a piece of its first half and the piece that is rotated with it, eight pairs per lane.  How far a row
// moves back never falls from one row to the next and hardly changes within a chunk, so its angle is put together from two tables
// in shared memory, of 0 .. 63 positions and of the chunk's few multiples of 64 (an angle from the polynomials for every pair takes
// three times the instructions); chunks that span more have their angles from the polynomials.
// Bound by HBM and the time from a chunk's request to its write for batches (half of 24 ragged caches, 1.1 GB: 214 us, and 199 where
// nothing is rotated), by that time and the chunks of the longest sequence otherwise (half of 30000 tokens: 82 us; a quarter of 16
// sequences of 4096: 27, 22 without rotation; by events around the kernel, which are some 3 us of each).  Dropped: rows read into
// registers, between barriers, 4 us a round, 317 us for the first; bulk copies of single rows, 25 to 40 ns each, 1447 us; every
// writer asking for every chunk itself, 250 ns a chunk, 33 us for the third; seven readers for a CTA that has an SM to itself, 121 us
// for the second; rotated keys' pieces without their swap, 218 us for the first.
constexpr int EM_FEW = 7, EM_MANY = 15;  // warps that read: where two CTAs share an SM, where one has it to itself
constexpr uint32_t EM_POLLS = 1u << 22;  // some tenths of a second
constexpr int EM_FAR = 4;          // multiples of 64 positions in a chunk's table
constexpr int EM_MAX_STAGES = 30;  // a warp's lanes ask for as many at once

struct MoveShape {
  int slabs, key_stages, value_stages;
  uint2 speeds[64];  // turns per position of a head's pairs, as 64-bit fractions: low, high word
};
// Shared memory of a stage: the rows, where each comes from, goes to and how far it moves; keys: angles of EM_FAR multiples of 64.
__host__ __device__ constexpr int em_far_bytes(int hd, int slabs) { return EM_FAR * 2 * (hd / 2 / slabs) * 4; }
__host__ __device__ constexpr int em_stage_bytes(int hd, int slabs, bool keys) {
  return 32 * (hd * 2 / slabs + 8 + 8 + 4) + (keys ? em_far_bytes(hd, slabs) : 0);
}
__host__ __device__ constexpr int em_near_bytes(int hd, int slabs) { return 64 * 2 * (hd / 2 / slabs) * 4; }

__device__ __forceinline__ void em_copy16(uint32_t dst_smem, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst_smem), "l"(src) : "memory");
}

// TRACK: with tracked origins.  A key that has been moved before comes from its row of first_keys, and every key that moves leaves
// there what it was, in the same order as the rows themselves: what is read later lies behind every slot written so far, in either pool.
template <int HD, int READERS, bool TRACK>
__global__ void __launch_bounds__((2 * READERS + 2) * 32) evict_move_kernel(const EvictArgs p, const MoveShape sh) {
  constexpr int WRITERS = READERS + 1, ORDER = WRITERS + READERS, THREADS = (ORDER + 1) * 32;
  constexpr int ROW = HD * 2;      // bytes of a row
  extern __shared__ __align__(128) unsigned char em_smem[];
  __shared__ uint64_t full[EM_MAX_STAGES], empty[EM_MAX_STAGES];
  __shared__ int arrived;            // chunks from the first on, without a gap
  __shared__ uint2 speeds[HD / 2];   // of the slab
  __shared__ int far0[EM_MAX_STAGES];  // first multiple of 64 in the stage's table; -1: its angles are in no table
  const int slabs = sh.slabs, bytes = ROW / slabs, F = HD / 2 / slabs, chunk = 32 * bytes;
  const int kvh = blockIdx.y, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int Hkv = p.shape.n_kv_heads, mp = p.kv.max_pages_per_seq;
  const bool keys = blockIdx.x < slabs, rope = keys && p.shape.rope_theta > 0.f;
  const ptrdiff_t to_first = TRACK ? static_cast<unsigned char*>(p.first_keys) - static_cast<unsigned char*>(p.kv.k_pool) : 0;
  const int stages = keys ? sh.key_stages : sh.value_stages;
  const int slab = keys ? blockIdx.x : blockIdx.x - slabs;
  float* near = reinterpret_cast<float*>(em_smem);  // [64][2][F] cosines, sines
  unsigned char* stage0 = em_smem + (keys ? em_near_bytes(HD, slabs) : 0);
  const int stage_bytes = em_stage_bytes(HD, slabs, keys);
  struct Stage {
    unsigned char* data;
    unsigned char **src, **dst;  // nullptr: nothing to move
    int* back;
    float* far;
  };
  auto stage = [&](int st) {
    Stage s;
    s.data = stage0 + (size_t)st * stage_bytes;
    s.far = reinterpret_cast<float*>(s.data + chunk);
    s.src = reinterpret_cast<unsigned char**>(s.data + chunk + (keys ? em_far_bytes(HD, slabs) : 0));
    s.dst = s.src + 32;
    s.back = reinterpret_cast<int*>(s.dst + 32);
    return s;
  };
  if (rope && tid < F) speeds[tid] = sh.speeds[slab * F + tid];
  if (tid == 0) {
    for (int i = 0; i < stages; ++i) {
      mbar_init(&full[i], 64);  // every lane of the reader, once for what it wrote and once for its copies
      mbar_init(&empty[i], 1);
    }
    arrived = 0;
    fence_mbar_init();
  }
  pdl_trigger();
  const int b = evict_sequence(p, blockIdx.z);  // its barriers are the speeds' too
  const EvictPlan e = evict_plan(p, b);
  const size_t row = ((size_t)b * Hkv + kvh) * mp * PAGE;
  const int32_t* kept = p.kept_idx + row;
  // an entry's F angles: the first four speeds of every lane of a row side by side, then the other four
  auto enter = [&](float* entry, int f, int back) {
    const float2 a = turn_back((uint32_t)back, speeds[f]);
    const int at = (f >> 2 & 1) * (F / 2) + (f >> 3) * 4 + (f & 3);
    entry[at] = a.x;
    entry[F + at] = a.y;
  };
  if (rope)
    for (int i = tid; i < 64 * F; i += THREADS) enter(near + i / F * 2 * F, i % F, i / F);
  __syncthreads();
  pdl_wait();
  const int chunks = (e.k + 31) / 32;
  const int pieces = bytes / 16, half = keys ? pieces / 2 : pieces;  // of a row's slab; those of its first half
  // A lane copies piece `q` of every (32 / pieces)-th row from row r0 on
  const int q = lane & (pieces - 1), r0 = lane / pieces, r_step = 32 / pieces, at_q = q < half ? q * 16 : ROW / 2 + (q - half) * 16;
  const int f_shift = 31 - __clz(F);
  // Where rotated keys' pieces lie: the halves of rows that a warp reads at once change places, so that they lie in different banks
  auto swap = [&](int r) { return rope ? (r * half >> 2 & 1) * half : 0; };
  bool alive = true;
  auto wait = [&](uint64_t* bar, uint32_t parity) { alive = alive && __all_sync(0xffffffffu, mbar_wait(bar, parity, p.status)); };

  auto wait_arrived = [&](int n) {
    const volatile int* a = &arrived;
#pragma unroll 1
    for (uint32_t i = 0; alive && *a < n; ++i)
      if (i == EM_POLLS) {
        alive = false;
        atomicOr(p.status + ST_ERR, ERR_TIMEOUT);
      }
    __threadfence_block();
    alive = __all_sync(0xffffffffu, alive);
  };

  if (warp == ORDER) {  // ---- a lane per chunk of the next ones asks whether it has arrived ----
    int st = lane, phase = 0, n = 0;  // of the lane's chunk, n + lane; the phase before this one is over: chunk n + lane - stages was seen
#pragma unroll 1
    for (uint32_t i = 0; n < chunks && i < EM_POLLS; ++i) {
      const bool got = lane < stages && n + lane < chunks && mbar_test_wait_at(smem_u32(&full[st]), phase);
      const int more = __ffs((int)~__ballot_sync(0xffffffffu, got)) - 1;  // at most the stages: fewer than 32
      if (more == 0) continue;
      i = 0;
      n += more;
      st += more;
      if (st >= stages) {
        st -= stages;
        phase ^= 1;
      }
      __threadfence_block();
      if (lane == 0) *const_cast<volatile int*>(&arrived) = n;
    }
    if (n < chunks && lane == 0) atomicOr(p.status + ST_ERR, ERR_TIMEOUT);
    return;
  }

  if (warp >= WRITERS) {  // ---- requests ----
    const int32_t *table = p.kv.page_table + (size_t)b * mp, *dst_table = p.dst_table + (size_t)b * mp;
    unsigned char* pool = static_cast<unsigned char*>(keys ? p.kv.k_pool : p.kv.v_pool);
    const int first = slab * half * 16;
    int next;  // kept token of this lane's row
    auto look = [&](int c) {
      const int j = c * 32 + lane;
      next = j < e.k ? kept[j] : -1;
    };
    const int to_q = lane ^ swap(r0);
    int c = warp - WRITERS, st = c, phase = 1;  // phase: of the stage's `empty`; the first use waits for none
    look(c);
#pragma unroll 1
    for (; c < chunks; c += READERS) {
      const Stage s = stage(st);
      unsigned char *src = nullptr, *dst = nullptr;
      const int i = next, j = c * 32 + lane, before = TRACK && keys && i >= 0 ? p.moved[row + i] : 0;
      const int back = i < 0 ? 0 : i - j + before;
      if (i >= 0) {
        const int from = table[i / PAGE], to = dst_table[j / PAGE];
        if ((unsigned)from >= (unsigned)p.kv.num_pages || (unsigned)to >= (unsigned)p.kv.num_pages) {
          atomicOr(p.status + ST_ERR, ERR_BAD_PAGE);
        } else {
          src = pool + (((size_t)from * Hkv + kvh) * PAGE + i % PAGE) * ROW + first;
          dst = pool + (((size_t)to * Hkv + kvh) * PAGE + j % PAGE) * ROW + first;
          if (src == dst) src = dst = nullptr;  // it stays where it is
          else if (TRACK && before) src += to_first;
        }
      }
      look(c + READERS);
      if (c >= stages) {
        wait_arrived(c - stages + 1);  // so the stage has been left once less than is asked for next, and no phase is mistaken
        wait(&empty[st], phase);
      }
      if (!alive) break;
      s.src[lane] = src;
      s.dst[lane] = dst;
      s.back[lane] = back;
      __syncwarp();
      const uint32_t data = smem_u32(s.data);
#pragma unroll 4
      for (int x = 0; x < pieces; ++x) {
        const unsigned char* from = s.src[r0 + x * r_step];
        if (from) em_copy16(data + (to_q + 32 * x) * 16, from + at_q);
      }
      if (rope) {
        const int low = __reduce_min_sync(0xffffffffu, i < 0 ? 0x7fffffff : back >> 6), top = __reduce_max_sync(0xffffffffu, back >> 6);
        const bool fits = top - low < EM_FAR;
        if (fits)
          for (int x = lane; x < (top - low + 1) << f_shift; x += 32)
            enter(s.far + (x >> f_shift) * 2 * F, x & (F - 1), (low + (x >> f_shift)) * 64);
        if (lane == 0) far0[st] = fits ? low : -1;
      }
      asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(&full[st])) : "memory");
      mbar_arrive(&full[st]);
      st += READERS;
      if (st >= stages) {
        st -= stages;
        phase ^= 1;
      }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");  // also where a wait gave up: nothing is in flight when the CTA ends
    return;
  }

  // ---- a warp writes a chunk when it and all before it have arrived; of rotated keys a lane has piece f0 and the one half a row on ----
  int st = warp, phase = 0;
  const int f0 = lane & (half - 1), f_r0 = lane / half, f_step = 32 / half, f_at = (f_r0 * pieces + f0) ^ swap(f_r0);
#pragma unroll 1
  for (int c = warp; c < chunks; c += WRITERS) {
    wait_arrived(c + 1);
    wait(&full[st], phase);  // (it has; now this warp has seen it)
    if (!alive) break;
    const Stage s = stage(st);
    const uint4* data = reinterpret_cast<const uint4*>(s.data);
    if (!rope) {
#pragma unroll 4
      for (int x = 0; x < pieces; ++x) {
        unsigned char* to = s.dst[r0 + x * r_step];
        if (to) *reinterpret_cast<uint4*>(to + at_q) = data[lane + 32 * x];
      }
    } else {
      const int low = far0[st];
#pragma unroll 2
      for (int r = f_r0; r < 32; r += f_step) {
        uint4* dst = reinterpret_cast<uint4*>(s.dst[r]);
        if (dst == nullptr) continue;
        const int back = s.back[r];
        const int at = f_at + (r - f_r0) * pieces;
        const uint4 lo = data[at], hi = data[at ^ half];
        const uint32_t l[4] = {lo.x, lo.y, lo.z, lo.w}, h[4] = {hi.x, hi.y, hi.z, hi.w};
        uint32_t new_l[4], new_h[4];
        const float *a = near + (back & 63) * 2 * F + f0 * 4, *w = s.far + ((back >> 6) - max(low, 0)) * 2 * F + f0 * 4;
#pragma unroll
        for (int q = 0; q < 2; ++q) {  // four pairs at a time
          float cs[4], sn[4];
          if (low >= 0) {
            const float4 ac = *reinterpret_cast<const float4*>(a + q * F / 2), as = *reinterpret_cast<const float4*>(a + F + q * F / 2);
            const float4 wc = *reinterpret_cast<const float4*>(w + q * F / 2), ws = *reinterpret_cast<const float4*>(w + F + q * F / 2);
            cs[0] = wc.x * ac.x - ws.x * as.x; sn[0] = ws.x * ac.x + wc.x * as.x;
            cs[1] = wc.y * ac.y - ws.y * as.y; sn[1] = ws.y * ac.y + wc.y * as.y;
            cs[2] = wc.z * ac.z - ws.z * as.z; sn[2] = ws.z * ac.z + wc.z * as.z;
            cs[3] = wc.w * ac.w - ws.w * as.w; sn[3] = ws.w * ac.w + wc.w * as.w;
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float2 t = turn_back((uint32_t)back, speeds[f0 * 8 + q * 4 + i]);
              cs[i] = t.x;
              sn[i] = t.y;
            }
          }
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const float l0 = bf16_lo(l[2 * q + i]), l1 = bf16_hi(l[2 * q + i]), h0 = bf16_lo(h[2 * q + i]), h1 = bf16_hi(h[2 * q + i]);
            new_l[2 * q + i] = cvt_bf16x2(l0 * cs[2 * i] - h0 * sn[2 * i], l1 * cs[2 * i + 1] - h1 * sn[2 * i + 1]);
            new_h[2 * q + i] = cvt_bf16x2(h0 * cs[2 * i] + l0 * sn[2 * i], h1 * cs[2 * i + 1] + l1 * sn[2 * i + 1]);
          }
        }
        dst[f0] = back ? make_uint4(new_l[0], new_l[1], new_l[2], new_l[3]) : lo;
        dst[f0 + ROW / 32] = back ? make_uint4(new_h[0], new_h[1], new_h[2], new_h[3]) : hi;
        if (TRACK) {
          uint4* first = reinterpret_cast<uint4*>(reinterpret_cast<unsigned char*>(dst) + to_first);
          first[f0] = lo;
          first[f0 + ROW / 32] = hi;
        }
      }
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(&empty[st]);
    st += WRITERS;
    if (st >= stages) {
      st -= stages;
      phase ^= 1;
    }
  }
}

// How far the kept keys have been moved in all; none of what lies behind them has.  A CTA per (sequence, kv-head): in place the entries
// of a chunk are read before any is written, and those of later chunks lie behind them (kept_idx[j] >= j).
__global__ void __launch_bounds__(ES_THREADS) evict_moved_kernel(const EvictArgs p) {
  pdl_trigger();
  const int b = blockIdx.y, n = p.kv.max_pages_per_seq * PAGE, k = evict_plan(p, b).k;
  const size_t row = ((size_t)b * p.shape.n_kv_heads + blockIdx.x) * n;
  pdl_wait();
#pragma unroll 1
  for (int j0 = 0; j0 < n; j0 += ES_THREADS) {
    const int j = j0 + threadIdx.x;
    int far = 0;
    if (j < k) {
      const int i = p.kept_idx[row + j];
      far = p.moved[row + i] + i - j;
    }
    __syncthreads();
    if (j < n) p.dst_moved[row + j] = far;
  }
}

template <int HD, bool TRACK>
static void launch_move(const EvictArgs& a, cudaStream_t st) {
  const int Hkv = a.shape.n_kv_heads, rows = 2 * a.B * Hkv;
  MoveShape sh;
  // Pieces of 64 bytes of a key, or of 32 where every CTA then still has an SM to itself (four sequences of 8000: 41 us with pieces
  // of 64 and an SM each, 56 with pieces of 32 and two CTAs an SM)
  sh.slabs = rows * (HD / 32) > sm_count() ? HD / 64 : HD / 32;
  for (int f = 0; f < 64; ++f) sh.speeds[f] = make_uint2(0, 0);
  if (a.shape.rope_theta > 0.f)
    for (int f = 0; f < HD / 2; ++f) {
      const double turns = exp2(-2.0 * f / HD * log2((double)a.shape.rope_theta)) * 0.15915494309189535;
      const uint64_t fraction = (uint64_t)((turns - floor(turns)) * 0x1p64);
      sh.speeds[f] = make_uint2((uint32_t)fraction, (uint32_t)(fraction >> 32));
    }
  const bool two = rows * sh.slabs > sm_count();  // CTAs per SM
  const int near = em_near_bytes(HD, sh.slabs), room = (two ? 108 : 216) * 1024;
  sh.key_stages = std::min(EM_MAX_STAGES, (room - near) / em_stage_bytes(HD, sh.slabs, true));  // at least as many as readers, writers
  sh.value_stages = std::min(EM_MAX_STAGES, room / em_stage_bytes(HD, sh.slabs, false));
  const int smem = std::max(near + sh.key_stages * em_stage_bytes(HD, sh.slabs, true), sh.value_stages * em_stage_bytes(HD, sh.slabs, false));
  const auto kernel = two ? evict_move_kernel<HD, EM_FEW, TRACK> : evict_move_kernel<HD, EM_MANY, TRACK>;
  ensure_dynamic_smem(reinterpret_cast<const void*>(kernel), smem);
  SOL_LAUNCH("evict_move", kernel, dim3(2 * sh.slabs, Hkv, a.B), dim3((2 * (two ? EM_FEW : EM_MANY) + 2) * 32), smem, st, a, sh);
}

void launch_evict(const EvictArgs& a, cudaStream_t st) {
  const int per = ((a.kv.max_pages_per_seq * PAGE + ES_THREADS - 1) / ES_THREADS) | 1;
  const int smem = per * ES_THREADS * 4;
  ensure_dynamic_smem(reinterpret_cast<const void*>(&evict_select_kernel), smem);
  SOL_LAUNCH("evict_select", evict_select_kernel, dim3(a.shape.n_kv_heads, a.B), dim3(ES_THREADS), smem, st, a);
  if (a.first_keys) {
    if (a.shape.head_dim == 64) launch_move<64, true>(a, st);
    else launch_move<128, true>(a, st);
    SOL_LAUNCH("evict_moved", evict_moved_kernel, dim3(a.shape.n_kv_heads, a.B), dim3(ES_THREADS), 0, st, a);
  } else {
    if (a.shape.head_dim == 64) launch_move<64, false>(a, st);
    else launch_move<128, false>(a, st);
  }
}

}  // namespace sol
