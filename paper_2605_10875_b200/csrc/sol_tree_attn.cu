// Attention of a tree of drafted tokens over the paged cache on the tensor cores' 5th generation: a (sequence, kv-head) has
// G n query rows (G heads, n nodes), up to 512, for which its keys and values are streamed once.
//
//   o_r = sum_t p_rt v_t,  p_rt = 2^(s_rt - m_r) / l_r,  s_rt = (q_r . k_t) log2(e) / sqrt(head_dim)  where row r sees token t
//
// One CTA per SM takes its run of tiles (sol_chain.cuh; a tile is two cache pages, 128 tokens), cut chains are merged by
// chain_merge_kernel.  Two units of 128 rows work on it, each with scores (128 columns) and sums (head_dim columns) in tensor
// memory: blocks of more than 128 rows give each unit its own rows and both read every tile; smaller ones give both units the
// same rows and every second tile, and the units' results are merged at the end of the chain.  So one unit's products run
// while the other's softmax does.
//
//   warps 0-3, 4-7   the units' softmax, a row per thread: scores from tensor memory, running maximum (moved only where it
//                    grows by more than 2^8: then the sums are rescaled), weights as bf16 back to where the scores were
//   warp 8           TMA of keys and values into a ring of 128-token operand tiles (128-byte swizzle)
//   warp 9           tcgen05.mma: S = Q K^T (both from shared memory), O += P V (P from tensor memory)
//   warps 10, 11     clear rows of a tile that no weight may meet: behind the sequence, of a page out of range, and of drafted
//                    tokens with values that are not finite, which the softmax threads add in float32 for the rows that see them
#include <cuda.h>
#include <math.h>

#include <algorithm>

#include "sol_chain.cuh"
#include "sol_umma.cuh"

namespace sol {

constexpr int TA_ROWS = 128;            // rows of a unit
constexpr int TA_BLOCK = 2 * TA_ROWS;   // rows of a chain
constexpr int TA_TILE = 2 * PAGE;       // tokens of a tile
constexpr int TA_MIN_TILES = 2;
constexpr int TA_THREADS = 12 * 32;
constexpr float TA_SLACK = 8.f;         // weights reach 2^8 before the maximum moves
enum : int { TAW_LOAD = 8, TAW_MMA = 9, TAW_CLEAR = 10 };

template <int HD>
struct TaSize {
  static constexpr int CHUNKS = HD / 64;
  static constexpr int CHUNK = 128 * 128;         // a 64-wide chunk of an operand: [128 rows][128 B]
  static constexpr int OPER = CHUNKS * CHUNK;     // queries of a unit, keys or values of a tile
  static constexpr int SLOTS = HD == 64 ? 12 : 5;
  static constexpr int SMEM = 1024 + (2 + SLOTS) * OPER;
  static constexpr int UNIT = TA_TILE + HD;       // tensor-memory columns of a unit
};

struct TreeDev {
  ChainShape c;
  int Hq;
  float scale_log2;
  const uint64_t* mask;
  const uint16_t* q;
  uint16_t* out;
  ChainParts part;
  int* status;
};

struct TreeClearJob {  // from the MMA warp to the clearing warps
  int slot, base, C, T, pages, units, quit;
};

template <int HD>
struct TreeShared {
  ChainPlan plan;
  uint64_t full[TaSize<HD>::SLOTS], empty[TaSize<HD>::SLOTS];
  uint64_t q_ready[2], s_full[2], p_ready[2], o_done[2], go, clean;
  unsigned long long dirty[2];  // per unit: drafted tokens whose values were taken out
  TreeClearJob job;
  uint32_t tmem;
  unsigned char pages[TaSize<HD>::SLOTS];  // bit i: page i of the tile is there
};

__device__ __forceinline__ uint32_t ta_piece(uint32_t oper, int r, int c) {  // address of 16-byte piece c of row r of an operand
  return oper + (uint32_t)((c >> 3) * (128 * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4));
}
__device__ __forceinline__ float ta_exp2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// What a piece of a chain means to every role.
struct TreePiece : ChainPiece {
  int rows, steps, C;  // query rows of the block, tiles of the piece, tokens of the committed context
  bool both;           // both units read every tile
};
__device__ __forceinline__ TreePiece tree_piece(const ChainShape& c, const ChainPlan& plan, int u, int end) {
  TreePiece r;
  static_cast<ChainPiece&>(r) = chain_piece(c, plan, u, end);
  r.rows = min(TA_BLOCK, r.seq.n * c.G - r.block * TA_BLOCK);
  r.steps = r.tile1 - r.tile0;
  r.C = r.seq.T - r.seq.n;
  r.both = r.rows > TA_ROWS;
  return r;
}

// ---- TMA ----
template <int HD>
__device__ void tree_load(const TreeDev& p, TreeShared<HD>& sh, unsigned char* ring, const CUtensorMap* kmap, const CUtensorMap* vmap,
                          int u0, int u1) {
  using Z = TaSize<HD>;
  const int lane = threadIdx.x & 31;
  bool alive = true;
  int n = 0;  // tiles requested so far
  for (int u = u0; u < u1;) {
    const TreePiece c = tree_piece(p.c, sh.plan, u, u1);
    const int32_t* table = p.c.kv.page_table + (size_t)c.b * p.c.kv.max_pages_per_seq;
    const int pages = (c.seq.T + PAGE - 1) / PAGE;
    // page numbers of 16 steps at a time, the next 16 requested two steps after the last ones came into use (values come one
    // step after keys, so both sets are in use for a while)
    int win[2];
    auto fetch = [&](int w) {
      const int i = 2 * (c.tile0 + 16 * w) + lane;
      return i < pages && i < 2 * c.tile1 ? table[i] : -1;
    };
    win[0] = fetch(0);
    win[1] = c.steps > 16 ? fetch(1) : -1;
    auto push = [&](const CUtensorMap* map, int step) {
      const int w = win[(step >> 4) & 1], at = 2 * (step & 15);
      const int page0 = __shfl_sync(0xffffffffu, w, at), page1 = __shfl_sync(0xffffffffu, w, at + 1);
      const int slot = n % Z::SLOTS, use = n / Z::SLOTS;
      if (alive && use > 0) alive = __all_sync(0xffffffffu, mbar_wait(&sh.empty[slot], (use - 1) & 1, p.status));
      if (!alive) return;
      ++n;
      if (lane == 0) {
        const int tile = c.tile0 + step;
        const int ids[2] = {page0, page1};
        int there = 0;
        for (int x = 0; x < 2; ++x) {
          if (2 * tile + x >= pages) continue;
          if (ids[x] >= 0 && ids[x] < p.c.kv.num_pages) there |= 1 << x;
          else atomicOr(p.status + ST_ERR, ERR_BAD_PAGE);
        }
        sh.pages[slot] = (unsigned char)there;
        const int parts = (there & 1) + (there >> 1);
        if (parts == 0) {
          mbar_arrive(&sh.full[slot]);
        } else {
          mbar_expect_tx(&sh.full[slot], (uint32_t)parts * (Z::OPER / 2));
          for (int x = 0; x < 2; ++x) {
            if (!((there >> x) & 1)) continue;
            const int row = (ids[x] * p.c.Hkv + c.kvh) * PAGE;
#pragma unroll
            for (int h = 0; h < Z::CHUNKS; ++h)
              tma_load_2d(ring + (size_t)slot * Z::OPER + h * Z::CHUNK + x * (PAGE * 128), map, h * 64, row, &sh.full[slot]);
          }
        }
      }
      __syncwarp();
    };
    auto turn = [&](int step) {  // keys of `step` have been pushed
      if ((step & 15) == 2 && step > 16) win[((step >> 4) + 1) & 1] = fetch((step >> 4) + 1);
    };
    if (c.both) {
      for (int j = 0; j < c.steps; ++j) {
        push(kmap, j);
        push(vmap, j);
        turn(j);
      }
    } else {
      push(kmap, 0);
      for (int j = 0; j < c.steps; ++j) {
        if (j + 1 < c.steps) {
          push(kmap, j + 1);
          turn(j + 1);
        }
        push(vmap, j);
      }
    }
    u += c.steps;
  }
  if (!alive)  // a wait gave up: what has been requested still arrives before the CTA ends
    for (int i = max(0, n - Z::SLOTS); i < n; ++i) mbar_wait(&sh.full[i % Z::SLOTS], (i / Z::SLOTS) & 1, p.status);
}

// ---- tensor cores ----
template <int HD>
__device__ void tree_mma(const TreeDev& p, TreeShared<HD>& sh, uint32_t q_oper, uint32_t ring, int u0, int u1) {
  using Z = TaSize<HD>;
  constexpr uint32_t S_IDESC = umma_idesc_bf16_m128(TA_TILE, 0, 0), O_IDESC = umma_idesc_bf16_m128(HD, 0, 1);
  const uint32_t tmem = sh.tmem;
  bool alive = true;
  auto wait = [&](uint64_t* bar, uint32_t parity) {  // after one that gave up, the others return at once
    alive = alive && mbar_wait(bar, parity, p.status);
    __syncwarp();
  };
  int n = 0, piece = 0, jobs = 0;
  int done[2] = {0, 0};  // steps whose weights have been waited for
  for (int u = u0; u < u1; ++piece) {
    const TreePiece c = tree_piece(p.c, sh.plan, u, u1);
    wait(&sh.q_ready[0], piece & 1);
    wait(&sh.q_ready[1], piece & 1);
    tc_fence_after();
    auto slot_full = [&]() {  // the next tile of the ring
      const int slot = n % Z::SLOTS;
      wait(&sh.full[slot], (n / Z::SLOTS) & 1);
      ++n;
      return slot;
    };
    auto scores = [&](int slot, int unit, bool last) {
      tc_fence_after();
      if (elect_one()) {
        const uint32_t a = q_oper + (c.both && unit ? Z::OPER : 0), b = ring + slot * Z::OPER;
#pragma unroll
        for (int k = 0; k < HD / 16; ++k) {
          const uint32_t off = (k >> 2) * Z::CHUNK + (k & 3) * 32;
          umma_bf16(tmem + unit * Z::UNIT, umma_smem_desc(a + off, 16, 1024), umma_smem_desc(b + off, 16, 1024), S_IDESC, k > 0);
        }
        umma_commit(&sh.s_full[unit]);
        if (last) umma_commit(&sh.empty[slot]);
      }
      __syncwarp();
    };
    auto values_ready = [&](int slot, int step) {  // where rows have to be cleared first, that is asked for
      const int base = (c.tile0 + step) * TA_TILE, there = sh.pages[slot];
      if (base + TA_TILE <= c.C && there == 3) return;
      if ((threadIdx.x & 31) == 0) {
        TreeClearJob j;
        j.slot = slot; j.base = base; j.C = c.C; j.T = c.seq.T; j.pages = there;
        j.units = c.both ? 3 : 1 << (step & 1);
        j.quit = 0;
        sh.job = j;
        mbar_arrive(&sh.go);
      }
      __syncwarp();
      wait(&sh.clean, jobs & 1);
      ++jobs;
    };
    auto values = [&](int slot, int unit, bool fresh, bool last, bool end) {
      wait(&sh.p_ready[unit], done[unit] & 1);
      ++done[unit];
      tc_fence_after();
      if (elect_one()) {
        const uint32_t pa = tmem + unit * Z::UNIT, b = ring + slot * Z::OPER;
#pragma unroll
        for (int k = 0; k < TA_TILE / 16; ++k)
          umma_bf16_ts(pa + TA_TILE, pa + k * 8, umma_smem_desc(b + k * 2048, Z::CHUNK, 1024), O_IDESC, !fresh || k > 0);
        if (last) umma_commit(&sh.empty[slot]);
        if (end) {
          umma_commit(&sh.o_done[unit]);
          mbar_arrive(&sh.o_done[unit]);  // what this warp has seen, the unit sees: the clearing warps' finds among it
        }
      }
      __syncwarp();
    };
    if (c.both) {
      int slot = slot_full();
      scores(slot, 0, false);
      scores(slot, 1, true);
      for (int j = 0; j < c.steps; ++j) {
        const bool more = j + 1 < c.steps;
        const int vs = slot_full();
        values_ready(vs, j);
        values(vs, 0, j == 0, false, !more);
        if (more) {
          slot = slot_full();
          scores(slot, 0, false);
        }
        values(vs, 1, j == 0, true, !more);
        if (more) scores(slot, 1, true);
      }
    } else {
      scores(slot_full(), 0, true);
      for (int j = 0; j < c.steps; ++j) {
        if (j + 1 < c.steps) scores(slot_full(), (j + 1) & 1, true);
        const int vs = slot_full();
        values_ready(vs, j);
        values(vs, j & 1, j < 2, true, j + 2 >= c.steps);
      }
    }
    u += c.steps;
  }
  if ((threadIdx.x & 31) == 0) {
    sh.job.quit = 1;
    mbar_arrive(&sh.go);
  }
}

// ---- rows that no weight may meet ----
template <int HD>
__device__ void tree_clear(const TreeDev& p, TreeShared<HD>& sh, uint32_t ring) {
  using Z = TaSize<HD>;
  const int tid = threadIdx.x - TAW_CLEAR * 32;  // 0 .. 63
  for (int n = 0;; ++n) {
    // the MMA warp asks seldom: wait for as long as it lives (its own waits are limited, and its last word is `quit`)
    bool got = false;
    for (int i = 0; i < 64 && !got; ++i)
      for (uint32_t x = 0; x < WAIT_LIMIT && !got; ++x) got = mbar_try_wait(&sh.go, n & 1);
    if (!__all_sync(0xffffffffu, got)) {
      atomicOr(p.status + ST_ERR, ERR_TIMEOUT);
      return;
    }
    const TreeClearJob j = sh.job;
    if (j.quit) return;
    const uint32_t tile = ring + j.slot * Z::OPER;
#pragma unroll 1
    for (int r = tid; r < TA_TILE; r += 64) {
      const int tok = j.base + r;
      bool drop = tok >= j.T || !((j.pages >> (r / PAGE)) & 1);
      if (!drop && tok >= j.C) {
        for (int c = 0; c < HD / 8; ++c) {
          const uint4 v = lds128(ta_piece(tile, r, c));
          const uint32_t x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) drop = drop || (x[e] & 0x7f80u) == 0x7f80u || (x[e] & 0x7f800000u) == 0x7f800000u;
        }
        if (drop)
          for (int w = 0; w < 2; ++w)
            if ((j.units >> w) & 1) atomicOr(&sh.dirty[w], 1ull << (tok - j.C));
      }
      if (drop)
        for (int c = 0; c < HD / 8; ++c)
          asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(ta_piece(tile, r, c)), "r"(0u) : "memory");
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    mbar_arrive(&sh.clean);
  }
}

// ---- softmax, a row per thread ----
__device__ __forceinline__ void tree_units_sync() {
  __syncwarp();
  asm volatile("bar.sync 1, 256;" ::: "memory");
}

// Bits of the 32 tokens from `base` on that a row sees: the context, and its mask's nodes.
__device__ __forceinline__ uint32_t tree_seen(int base, int C, uint64_t nodes) {
  const int ctx = C - base;
  if (ctx >= 32) return 0xffffffffu;
  if (ctx > 0) return ((1u << ctx) - 1) | (uint32_t)(nodes << ctx);
  return -ctx < 64 ? (uint32_t)(nodes >> -ctx) : 0u;
}

template <int HD>
__device__ void tree_softmax(const TreeDev& p, TreeShared<HD>& sh, unsigned char* q_smem, int u0, int u1) {
  using Z = TaSize<HD>;
  constexpr int EX = HD / 2;  // columns that unit 1 hands over at a time
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, unit = warp >> 2, quad = warp & 3, row_in_unit = quad * 32 + lane;
  const int G = p.c.G;
  const uint32_t lanes = (uint32_t)(quad * 32) << 16;
  const uint32_t tm_s = sh.tmem + unit * Z::UNIT + lanes, tm_o = tm_s + TA_TILE;
  float* ex = reinterpret_cast<float*>(q_smem + Z::OPER);       // [EX][128] sums of unit 1
  float2* ex_ml = reinterpret_cast<float2*>(q_smem);            // [2][128], once the scores are done
  bool alive = true;
  auto wait = [&](uint64_t* bar, uint32_t parity) {  // after one that gave up, the others return at once
    alive = alive && mbar_wait(bar, parity, p.status);
    __syncwarp();
  };
  int done = 0, ends = 0;
  for (int u = u0; u < u1;) {
    const TreePiece c = tree_piece(p.c, sh.plan, u, u1);
    const int T = c.seq.T, n = c.seq.n;
    tree_units_sync();  // both units are done with the queries of the piece before, and with what lay in their place
    if ((threadIdx.x & 127) == 0) sh.dirty[unit] = 0;
    // ---- queries into their operand tiles ----
    const int block0 = c.block * TA_BLOCK, my_row = (c.both ? unit * TA_ROWS : 0) + row_in_unit;
    const bool real = my_row < c.rows;
    {
      // a 16-lane (HD 128) or 8-lane group per row; where both units share their rows, each brings half of them
      constexpr int PPR = HD / 8;
      const int t = threadIdx.x & 127, per = c.both ? TA_ROWS : TA_ROWS / 2, r0 = c.both ? 0 : unit * per;
      const uint32_t oper = smem_u32(q_smem) + (c.both ? unit * Z::OPER : 0);
#pragma unroll 4
      for (int i = t; i < per * PPR; i += 128) {
        const int r = r0 + i / PPR, piece = i % PPR, row = block0 + (c.both ? unit * TA_ROWS : 0) + r, node = row / G;
        uint4 v = make_uint4(0u, 0u, 0u, 0u);
        if (row < block0 + c.rows)
          v = *reinterpret_cast<const uint4*>(
              p.q + (((size_t)c.b * p.c.max_nodes + node) * p.Hq + c.kvh * G + (row - node * G)) * HD + piece * 8);
        asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(ta_piece(oper, r, piece)), "r"(v.x), "r"(v.y), "r"(v.z),
                     "r"(v.w)
                     : "memory");
      }
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    tc_fence_before();
    mbar_arrive(&sh.q_ready[unit]);
    const int node = (block0 + my_row) / G;
    uint64_t nodes = 0;
    if (real) nodes = p.mask[(size_t)c.b * p.c.max_nodes + node] & (n < 64 ? (1ull << n) - 1 : ~0ull);
    const size_t base_row = (((size_t)c.b * p.c.max_nodes + node) * p.Hq + c.kvh * G + (block0 + my_row - node * G)) * HD;
    const bool warp_real = (c.both ? unit * TA_ROWS : 0) + quad * 32 < c.rows;

    const int32_t* table = p.c.kv.page_table + (size_t)c.b * p.c.kv.max_pages_per_seq;
    const int pages = (T + PAGE - 1) / PAGE, stride = c.both ? 1 : 2, from = c.both ? 0 : unit;
    auto page_bits = [&](int step) {
      int bits = 0;
      for (int x = 0; x < 2; ++x) {
        const int i = 2 * (c.tile0 + step) + x;
        if (step < c.steps && i < pages) {
          const int id = table[i];
          bits |= (id >= 0 && id < p.c.kv.num_pages) << x;
        }
      }
      return bits;
    };
    float m = -INFINITY, l = 0.f;
    int there = page_bits(from);
#pragma unroll 1
    for (int j = from; j < c.steps; j += stride) {
      const int base = (c.tile0 + j) * TA_TILE, there_next = page_bits(j + stride);
      wait(&sh.s_full[unit], done & 1);
      ++done;
      tc_fence_after();
      if (warp_real) {
        uint32_t s[TA_TILE];
#pragma unroll
        for (int x = 0; x < 4; ++x) tmem_ld32_issue(tm_s + x * 32, s + x * 32);
#pragma unroll
        for (int x = 0; x < 4; ++x) tmem_ld32_wait(s + x * 32);
        if (base + TA_TILE > c.C || there != 3) {
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const uint32_t seen = (there >> (x >> 1)) & 1 ? tree_seen(base + 32 * x, c.C, nodes) : 0u;
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (!((seen >> i) & 1)) s[x * 32 + i] = 0xff800000u;  // minus infinity
          }
        }
        float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int i = 0; i < TA_TILE; ++i) mx[i & 3] = fmaxf(mx[i & 3], __uint_as_float(s[i]));
        const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * p.scale_log2;
        if (__any_sync(0xffffffffu, top > m + TA_SLACK)) {
          const float m_new = fmaxf(m, top), f = m_new == -INFINITY ? 1.f : ta_exp2(m - m_new);
          m = m_new;
          l *= f;
          if (j != from) {  // this unit's products so far were done before these scores
#pragma unroll 1
            for (int x = 0; x < HD / 32; ++x) {
              uint32_t o[32];
              tmem_ld32_issue(tm_o + x * 32, o);
              tmem_ld32_wait(o);
#pragma unroll
              for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
              tmem_st32(tm_o + x * 32, o);
            }
          }
        }
        const float shift = m == -INFINITY ? 0.f : -m;
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          uint32_t w[32];
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            const float a = ta_exp2(fmaf(__uint_as_float(s[x * 64 + 2 * i]), p.scale_log2, shift));
            const float b = ta_exp2(fmaf(__uint_as_float(s[x * 64 + 2 * i + 1]), p.scale_log2, shift));
            sum[(2 * i) & 3] += a;
            sum[(2 * i + 1) & 3] += b;
            w[i] = pack_bf16(a, b);
          }
          tmem_st32(tm_s + x * 32, w);
        }
        l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
        tmem_st_wait();
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh.p_ready[unit]);
      there = there_next;
    }

    // ---- the end of the piece ----
    const bool worked = from < c.steps, pair = !c.both && c.steps > 1;
    if (worked) {
      wait(&sh.o_done[unit], ends & 1);
      ++ends;
    }
    tc_fence_after();
    const uint64_t dirty = worked && real && c.tile1 * TA_TILE > c.C ? sh.dirty[unit] & nodes : 0ull;
    float f = 1.f;
    if (pair) {  // both units' rows are the same: with the larger maximum from here on
      ex_ml[unit * 128 + row_in_unit] = make_float2(m, l);
      tree_units_sync();
      const float2 other = ex_ml[(unit ^ 1) * 128 + row_in_unit];
      const float m_new = fmaxf(m, other.x);
      f = m_new == -INFINITY ? 1.f : exp2f(m - m_new);
      l = l * f + other.y * (m_new == -INFINITY ? 1.f : exp2f(other.x - m_new));
      if (dirty == 0) m = m_new;
    }
    const float m_own = m;  // what this unit's sums are relative to, where dirty tokens are added
    if (pair && dirty) m = fmaxf(m, ex_ml[(unit ^ 1) * 128 + row_in_unit].x);
    const bool whole = c.whole(), writes = real && (c.both || unit == 0);
    const float inv = whole ? (l == 0.f ? 0.f : 1.0f / l) : 1.f;
    const size_t part = (size_t)(2 * blockIdx.x + (u > u0)) * p.part.rows + my_row;
#pragma unroll 1
    for (int x = 0; x < HD / 32; ++x) {
      uint32_t o[32];
      float v[32];
      __syncwarp();
      if (warp_real && worked) {
        tmem_ld32_issue(tm_o + x * 32, o);
        tmem_ld32_wait(o);
      }
#pragma unroll
      for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(o[i]);
      if (dirty) {
        for (uint64_t left = dirty; left; left &= left - 1) {
          const int slot = c.C + __ffsll((long long)left) - 1, id = table[slot / PAGE];
          const size_t at = (((size_t)id * p.c.Hkv + c.kvh) * PAGE + slot % PAGE) * HD;
          const uint16_t *kr = static_cast<const uint16_t*>(p.c.kv.k_pool) + at, *vr = static_cast<const uint16_t*>(p.c.kv.v_pool) + at;
          float dot = 0.f;
          for (int d = 0; d < HD; ++d) dot += bf2f(p.q[base_row + d]) * bf2f(kr[d]);
          const float w = ta_exp2(fmaf(dot, p.scale_log2, m_own == -INFINITY ? 0.f : -m_own));
#pragma unroll
          for (int i = 0; i < 32; ++i) v[i] += w * bf2f(vr[x * 32 + i]);
        }
      }
#pragma unroll
      for (int i = 0; i < 32; ++i) v[i] *= f;
      if (pair) {
        // unit 1's columns 0 .. EX - 1, then the others, by way of shared memory
        const int half = x * 32 / EX;
        if (unit == 1)
#pragma unroll
          for (int i = 0; i < 32; ++i) ex[(x * 32 - half * EX + i) * 128 + row_in_unit] = v[i];
        tree_units_sync();
        if (unit == 0)
#pragma unroll
          for (int i = 0; i < 32; ++i) v[i] += ex[(x * 32 - half * EX + i) * 128 + row_in_unit];
        if ((x + 1) * 32 == EX) tree_units_sync();  // the first half's space is used again
      }
      if (writes) {
        if (whole) {
          uint4* dst = reinterpret_cast<uint4*>(p.out + base_row + x * 32);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            dst[i] = make_uint4(pack_bf16(v[8 * i] * inv, v[8 * i + 1] * inv), pack_bf16(v[8 * i + 2] * inv, v[8 * i + 3] * inv),
                                pack_bf16(v[8 * i + 4] * inv, v[8 * i + 5] * inv), pack_bf16(v[8 * i + 6] * inv, v[8 * i + 7] * inv));
        } else {
          float4* dst = reinterpret_cast<float4*>(p.part.sums + part * HD + x * 32);
#pragma unroll
          for (int i = 0; i < 8; ++i) dst[i] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
        }
      }
    }
    if (writes && !whole) p.part.ml[part] = make_float2(m, l);
    u += c.steps;
  }
}

template <int HD>
__global__ void __launch_bounds__(TA_THREADS, 1) tree_attn_kernel(const __grid_constant__ CUtensorMap kmap,
                                                                  const __grid_constant__ CUtensorMap vmap, const TreeDev p) {
  using Z = TaSize<HD>;
  extern __shared__ unsigned char ta_smem[];
  __shared__ TreeShared<HD> sh;
  unsigned char* q_smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(ta_smem) + 1023) & ~(uintptr_t)1023);
  unsigned char* ring = q_smem + 2 * Z::OPER;
  const int tid = threadIdx.x, warp = tid >> 5;
  if (tid == 0) {
    for (int s = 0; s < Z::SLOTS; ++s) {
      mbar_init(&sh.full[s], 1);
      mbar_init(&sh.empty[s], 1);
    }
    for (int x = 0; x < 2; ++x) {
      mbar_init(&sh.q_ready[x], TA_ROWS);
      mbar_init(&sh.s_full[x], 1);
      mbar_init(&sh.p_ready[x], 4);
      mbar_init(&sh.o_done[x], 2);
    }
    mbar_init(&sh.go, 1);
    mbar_init(&sh.clean, 64);
    fence_mbar_init();
    tma_prefetch_map(&kmap);
    tma_prefetch_map(&vmap);
  }
  pdl_wait();
  pdl_trigger();
  if (warp == TAW_MMA) tmem_alloc(&sh.tmem, 512);  // not ahead of the wait: a kernel before this one may need it
  tc_fence_before();
  chain_plan(p.c, sh.plan, blockIdx.x == 0 ? p.status : nullptr);
  tc_fence_after();
  const int run = chain_run(p.c, sh.plan, gridDim.x), total = sh.plan.cum[p.c.B];
  const int u0 = (int)min((long long)blockIdx.x * run, (long long)total), u1 = min(total, u0 + run);
  if (warp < 8) tree_softmax<HD>(p, sh, q_smem, u0, u1);
  else if (warp == TAW_LOAD) tree_load<HD>(p, sh, ring, &kmap, &vmap, u0, u1);
  else if (warp == TAW_MMA) tree_mma<HD>(p, sh, smem_u32(q_smem), smem_u32(ring), u0, u1);
  else tree_clear<HD>(p, sh, smem_u32(ring));
  tc_fence_before();
  __syncthreads();
  if (warp == TAW_MMA) tmem_dealloc(sh.tmem, 512);
}

static int tree_rows(const sol_shape_t& sh, int max_nodes) { return std::min(TA_BLOCK, max_nodes * (sh.n_q_heads / sh.n_kv_heads)); }
size_t tree_part_bytes(const sol_shape_t& sh, int max_nodes) { return chain_part_bytes(sm_count(), tree_rows(sh, max_nodes), sh.head_dim); }

template <int HD>
static void launch_tree(const TreeDev& d, const CUtensorMap& kmap, const CUtensorMap& vmap, int ctas, cudaStream_t st) {
  ensure_dynamic_smem(reinterpret_cast<const void*>(&tree_attn_kernel<HD>), TaSize<HD>::SMEM);
  SOL_LAUNCH("tree_attn", tree_attn_kernel<HD>, dim3(ctas), dim3(TA_THREADS), TaSize<HD>::SMEM, st, kmap, vmap, d);
  launch_chain_merge(d.c, d.part, d.Hq, HD, ctas, d.out, st);
}

void launch_tree_attention(const RowsArgs& a, cudaStream_t st) {
  const sol_shape_t& sh = a.shape;
  CUtensorMap kmap, vmap;
  if (!encode_pool_map(&kmap, a.kv.k_pool, sh, a.kv.num_pages, PAGE) || !encode_pool_map(&vmap, a.kv.v_pool, sh, a.kv.num_pages, PAGE))
    return;
  const int ctas = sm_count();
  TreeDev d;
  d.c = chain_shape(a, TA_BLOCK, TA_TILE, TA_MIN_TILES);
  d.Hq = sh.n_q_heads;
  d.scale_log2 = 1.4426950408889634f / sqrtf((float)sh.head_dim);
  d.mask = a.mask;
  d.q = static_cast<const uint16_t*>(a.q);
  d.out = static_cast<uint16_t*>(a.out);
  d.part = chain_parts(a.part, ctas, tree_rows(sh, a.max_nodes), sh.head_dim);
  d.status = a.status;
  if (sh.head_dim == 64) launch_tree<64>(d, kmap, vmap, ctas, st);
  else launch_tree<128>(d, kmap, vmap, ctas, st);
}

}  // namespace sol
