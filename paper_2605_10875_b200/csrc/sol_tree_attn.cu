// Attention of a tree of drafted tokens over the paged cache on the tensor cores' 5th generation: a (sequence, kv-head) has
// G n query rows (G heads, n nodes), up to 512, for which its keys and values are streamed once.
//
//   o_r = sum_t p_rt v_t,  p_rt = 2^(s_rt - m_r) / l_r,  s_rt = (q_r . k_t) log2(e) / sqrt(head_dim)  where row r sees token t
//
// One CTA per SM takes its run of tiles (sol_chain.cuh; a tile is two cache pages of one kv-head, 128 tokens), cut chains are
// merged by chain_merge_kernel.  Two units of 128 tensor-memory lanes work on it, each with scores (128 columns) and sums
// (head_dim columns): while one unit's softmax runs, the other's products do.  Blocks of more than 128 query rows give each unit
// its own rows, and both read every tile; smaller ones give both units the same rows and every second tile.  Up to 64 (32) rows
// are there twice (four times) in a unit's lanes, so that each copy weighs only half (a quarter) of a tile's tokens and the
// softmax uses all four of the SM's quarters.  What the units and the copies have is added up at the end of a piece.
//
//   warps 0-3, 4-7   the units' softmax, a lane per thread: scores from tensor memory, running maximum (moved only where it
//                    grows by more than 2^8: then the sums are rescaled), weights as bf16 (LOW: in two parts) back to where the
//                    scores were
//   warps 8, 9       TMA of keys, of values into a ring each of 128-token operand tiles (128-byte swizzle)
//   warp 10          tcgen05.mma: S = Q K^T (both from shared memory), O += P V (P from tensor memory)
//   warp 11          clears rows of values that no weight may meet: behind the sequence, and of drafted tokens that are not finite,
//                    which the softmax threads add in float32 for the rows that see them
//
// Code that runs once a piece is kept short (rolled loops, rare work in functions of their own): fetched cold, it took longer
// than the piece's end does.
#include <cuda.h>
#include <math.h>

#include <algorithm>

#include "sol_chain.cuh"
#include "sol_umma.cuh"

namespace sol {

constexpr int TA_ROWS = 128;            // lanes of a unit
constexpr int TA_BLOCK = 2 * TA_ROWS;   // rows of a chain
constexpr int TA_TILE = 2 * PAGE;       // tokens of a tile
constexpr int TA_MIN_TILES = 2;
constexpr int ta_piece_cost(int hd) { return hd == 64 ? 8 : 4; }
constexpr int TA_THREADS = 12 * 32;
constexpr uint32_t POLL_LIMIT = 1u << 24;  // polls of the products' warp: some tenths of a second
constexpr float TA_SLACK = 8.f;         // weights reach 2^8 before the maximum moves
constexpr int TA_LOW = TA_TILE / 2;     // columns from weights' high parts to their low parts, over the tile's scores
constexpr int TA_EX = 32;               // columns handed over at a time at the end of a piece
enum : int { TAW_KEYS = 8, TAW_VALUES = 9, TAW_MMA = 10, TAW_CLEAR = 11 };

template <int HD>
struct TaSize {
  static constexpr int CHUNKS = HD / 64;
  static constexpr int CHUNK = 128 * 128;        // a 64-wide chunk of an operand: [128 rows][128 B]
  static constexpr int OPER = CHUNKS * CHUNK;    // a unit's queries, a tile's keys or values
  static constexpr int K_SLOTS = HD == 64 ? 5 : 2, V_SLOTS = HD == 64 ? 6 : 3;
  static constexpr int RINGS = (K_SLOTS + V_SLOTS) * OPER;
  static constexpr int EX = HD == 64 ? 0 : OPER;                        // where columns of sums are handed over: [TA_EX][256]
  static constexpr int ML = HD == 64 ? 2 * OPER + RINGS : 0;            // ... maxima and sums of weights: [256]
  static constexpr int SMEM = 1024 + 2 * OPER + RINGS + (HD == 64 ? 256 * 8 : 0);
  static constexpr int UNIT = TA_TILE + HD;      // columns of a unit: scores, sums
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

constexpr int TA_JOBS = 8;  // two of a piece that ends, and as many as there are slots for values
struct TreeClearJob {       // from the values' warp to the clearing warp
  int slot, phase, base, C, T;  // slot < 0: that was all
};

template <int HD>
struct TreeShared {
  ChainPlan plan;
  uint64_t k_full[TaSize<HD>::K_SLOTS], k_empty[TaSize<HD>::K_SLOTS];
  uint64_t v_full[TaSize<HD>::V_SLOTS], v_empty[TaSize<HD>::V_SLOTS], v_clean[TaSize<HD>::V_SLOTS];
  uint64_t q_ready, s_full[2], p_half[2], p_ready[2], o_end[2];
  TreeClearJob jobs[TA_JOBS];
  unsigned long long dirty[TA_JOBS];  // per job: drafted tokens whose values were taken out
  int posted;                         // jobs so far
  uint32_t tmem;
};

// Address of 16-byte piece c of row r of an operand.
__device__ __forceinline__ uint32_t ta_piece(uint32_t oper, int r, int c) {
  return oper + (uint32_t)((c >> 3) * (128 * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4));
}
__device__ __forceinline__ float ta_exp2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ float ta_max3(float a, float b, float c) {  // of numbers: NaN loses
  float y;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}
__device__ __forceinline__ uint64_t ta_add2(uint64_t a, uint64_t b) {
  uint64_t y;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(y) : "l"(a), "l"(b));
  return y;
}
__device__ __forceinline__ float2 ta_unpack2(uint64_t a) {
  float2 y;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(y.x), "=f"(y.y) : "l"(a));
  return y;
}

// What a piece of a chain means to every role.
struct TreePiece : ChainPiece {
  int rows, steps, C;  // query rows of the block, tiles of the piece, tokens of the committed context
  bool both;           // both units read every tile
  int lanes;           // lanes of a copy of the rows
  __device__ __forceinline__ int first_mixed() const { return max(tile0, C / TA_TILE); }  // from here on: drafted tokens, the end
};
__device__ __forceinline__ TreePiece tree_piece(const ChainShape& c, const ChainPlan& plan, int u, int end) {
  TreePiece r;
  static_cast<ChainPiece&>(r) = chain_piece(c, plan, u, end);
  r.rows = min(TA_BLOCK, r.seq.n * c.G - r.block * TA_BLOCK);
  r.steps = r.tile1 - r.tile0;
  r.C = r.seq.T - r.seq.n;
  r.both = r.rows > TA_ROWS;
  r.lanes = r.rows > 64 ? 128 : r.rows > 32 ? 64 : 32;
  return r;
}

// ---- TMA, a warp for the keys and one for the values ----
// A page out of range is reported and not read: no row sees its tokens, and its values are zeros.  Tiles of values that need it are
// handed to the clearing warp as soon as they are on their way.
template <int HD, bool VALUES>
__device__ void tree_load(const TreeDev& p, TreeShared<HD>& sh, unsigned char* ring, const CUtensorMap* map, int u0, int u1) {
  using Z = TaSize<HD>;
  constexpr int SLOTS = VALUES ? Z::V_SLOTS : Z::K_SLOTS;
  uint64_t *full = VALUES ? sh.v_full : sh.k_full, *empty = VALUES ? sh.v_empty : sh.k_empty;
  const int lane = threadIdx.x & 31;
  bool alive = true;
  int slot = 0, n = 0, jobs = 0;  // slot of the next tile; tiles, jobs so far
  uint32_t phase = 1;             // of the slot's `empty`: a fresh barrier counts as having completed the phase before its first
  for (int u = u0; u < u1;) {
    const TreePiece c = tree_piece(p.c, sh.plan, u, u1);
    const int pages = (c.seq.T + PAGE - 1) / PAGE - 2 * c.tile0;  // of the sequence, from the piece's first on
    const int32_t* table = p.c.kv.page_table + (size_t)c.b * p.c.kv.max_pages_per_seq + 2 * c.tile0;
    const int last = min(pages, 2 * c.steps);
    int now = 0, next = lane < last ? table[lane] : -1;  // page numbers, 32 at a time
#pragma unroll 1
    for (int j = 0; j < c.steps; ++j) {
      if ((j & 15) == 0) {
        now = next;
        next = 2 * j + 32 + lane < last ? table[2 * j + 32 + lane] : -1;
      }
      const int id0 = __shfl_sync(0xffffffffu, now, 2 * j & 31), id1 = __shfl_sync(0xffffffffu, now, 2 * j + 1 & 31);
      alive = alive && __all_sync(0xffffffffu, mbar_wait(&empty[slot], phase, p.status));
      if (!alive) continue;
      unsigned char* dst = ring + (size_t)slot * Z::OPER;
      const bool two = 2 * j + 1 < pages, good0 = id0 >= 0 && id0 < p.c.kv.num_pages, good1 = two && id1 >= 0 && id1 < p.c.kv.num_pages;
      if (!good0 || (two && !good1)) {
        for (int i = lane; i < Z::OPER / 16; i += 32) {
          const bool second = (i >> 9) & 1;  // 16-byte pieces: the second page's half of a chunk
          if (second ? two && !good1 : !good0) reinterpret_cast<uint4*>(dst)[i] = make_uint4(0u, 0u, 0u, 0u);
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        if (lane == 0) atomicOr(p.status + ST_ERR, ERR_BAD_PAGE);
        __syncwarp();
      }
      if (lane == 0) {
        uint64_t* bar = &full[slot];
        const int bytes = ((int)good0 + (int)good1) * (Z::OPER / 2);
        if (bytes) mbar_expect_tx(bar, bytes);
        else mbar_arrive(bar);
#pragma unroll
        for (int h = 0; h < Z::CHUNKS; ++h) {
          if (good0) tma_load_2d(dst + h * Z::CHUNK, map, h * 64, (id0 * p.c.Hkv + c.kvh) * PAGE, bar);
          if (good1) tma_load_2d(dst + h * Z::CHUNK + Z::CHUNK / 2, map, h * 64, (id1 * p.c.Hkv + c.kvh) * PAGE, bar);
        }
        if (VALUES && c.tile0 + j >= c.first_mixed()) {
          TreeClearJob job;
          job.slot = slot; job.phase = phase ^ 1; job.base = (c.tile0 + j) * TA_TILE; job.C = c.C; job.T = c.seq.T;
          sh.jobs[jobs % TA_JOBS] = job;
          __threadfence_block();
          *const_cast<volatile int*>(&sh.posted) = ++jobs;
        }
      }
      __syncwarp();
      ++n;
      if (++slot == SLOTS) {
        slot = 0;
        phase ^= 1;
      }
    }
    u = c.next;
  }
  if (!alive)  // a wait gave up: what has been requested still arrives before the CTA ends
    for (int i = max(0, n - SLOTS); i < n; ++i) mbar_wait(&full[i % SLOTS], (i / SLOTS) & 1, p.status);
  if (VALUES && lane == 0) {
    sh.jobs[jobs % TA_JOBS].slot = -1;
    __threadfence_block();
    *const_cast<volatile int*>(&sh.posted) = ++jobs;
  }
}

// ---- rows that no weight may meet ----
template <int HD>
__device__ void tree_clear(const TreeDev& p, TreeShared<HD>& sh, uint32_t v_ring) {
  using Z = TaSize<HD>;
  const int lane = threadIdx.x & 31;
#pragma unroll 1
  for (int n = 0;; ++n) {
    // there is seldom anything to do: asked for as long as the values' warp lives (its own waits are limited, and it always ends)
    bool got = false;
#pragma unroll 1
    for (uint32_t i = 0; i < 4 * WAIT_LIMIT && !got; ++i) {
      got = *const_cast<volatile int*>(&sh.posted) > n;
      if (!got) __nanosleep(64);
    }
    if (!__all_sync(0xffffffffu, got)) {
      atomicOr(p.status + ST_ERR, ERR_TIMEOUT);
      return;
    }
    __threadfence_block();
    const TreeClearJob j = sh.jobs[n % TA_JOBS];
    if (j.slot < 0) return;
    __all_sync(0xffffffffu, mbar_wait(&sh.v_full[j.slot], j.phase, p.status));
    const uint32_t tile = v_ring + j.slot * Z::OPER;
    uint32_t lo = 0, hi = 0;
#pragma unroll 1
    for (int r = lane; r < TA_TILE; r += 32) {
      const int tok = j.base + r;
      bool drop = tok >= j.T;
      if (!drop && tok >= j.C) {
#pragma unroll 4
        for (int c = 0; c < HD / 8; ++c) {
          const uint4 v = lds128(ta_piece(tile, r, c));
          const uint32_t x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) drop = drop || (x[e] & 0x7f80u) == 0x7f80u || (x[e] & 0x7f800000u) == 0x7f800000u;
        }
        if (drop) {
          if (tok - j.C < 32) lo |= 1u << (tok - j.C);
          else hi |= 1u << (tok - j.C - 32);
        }
      }
      if (drop)
        for (int c = 0; c < HD / 8; ++c)
          asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(ta_piece(tile, r, c)), "r"(0u) : "memory");
    }
    lo = __reduce_or_sync(0xffffffffu, lo);
    hi = __reduce_or_sync(0xffffffffu, hi);
    if (lane == 0) sh.dirty[n % TA_JOBS] = (uint64_t)lo | ((uint64_t)hi << 32);
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    mbar_arrive(&sh.v_clean[j.slot]);
  }
}

// ---- tensor cores ----
// This warp's pace is the kernel's.  It waits without naps (mbar_test_wait_at) for all that a step needs at once, a barrier per
// lane, and issues a step's products and commits in one elected block on operands that are the same in all lanes: 32 to 62 cycles
// a product, where predicated ones took 80 and blocks on lanes' own values more than that.
template <int HD, bool LOW>
__device__ void tree_mma(const TreeDev& p, TreeShared<HD>& sh, uint32_t q_oper, uint32_t k_ring, uint32_t v_ring, int u0, int u1) {
  using Z = TaSize<HD>;
  constexpr uint32_t S_IDESC = umma_idesc_bf16_m128(TA_TILE, 0, 0), O_IDESC = umma_idesc_bf16_m128(HD, 0, 1);
  const int lane = threadIdx.x & 31;
  const uint32_t tmem = __shfl_sync(0xffffffffu, sh.tmem, 0);
  const uint64_t q_desc = umma_smem_desc(q_oper, 16, 1024);
  const uint64_t k_desc = umma_smem_desc(k_ring, 16, 1024), v_desc = umma_smem_desc(v_ring, Z::CHUNK, 1024);
  const uint32_t k_full = smem_u32(sh.k_full), v_full = smem_u32(sh.v_full), v_clean = smem_u32(sh.v_clean);
  const uint32_t p_half = smem_u32(sh.p_half), p_ready = smem_u32(sh.p_ready);
  bool alive = true;
  auto wait = [&](uint32_t bar, uint32_t parity) {  // bar, parity: this lane's.  After one that gave up, the others return at once
    if (!alive) return;
#pragma unroll 1
    for (uint32_t i = 0; i < POLL_LIMIT; ++i)
      if (__all_sync(0xffffffffu, mbar_test_wait_at(bar, parity))) return;
    alive = false;
    if (lane == 0) atomicOr(p.status + ST_ERR, ERR_TIMEOUT);
  };
  int k_slot = 0, v_slot = 0;  // of the next tiles
  uint32_t k_phase = 0, v_phase = 0, clean_phases = 0, p_phases = 0;  // clean_phases, p_phases: a bit per slot, per unit
  auto k_step = [&]() {
    if (++k_slot == Z::K_SLOTS) {
      k_slot = 0;
      k_phase ^= 1;
    }
  };
  auto v_step = [&]() {
    if (++v_slot == Z::V_SLOTS) {
      v_slot = 0;
      v_phase ^= 1;
    }
  };
  // by the elected lane: a tile's scores, over the unit's last weights, whose product was asked for before
  auto scores = [&](int unit, uint64_t queries, bool last) {
    const uint64_t keys = k_desc + (uint64_t)(k_slot * (Z::OPER >> 4));
#pragma unroll
    for (int k = 0; k < HD / 16; ++k) {
      const uint64_t off = ((k >> 2) * Z::CHUNK + (k & 3) * 32) >> 4;
      umma_bf16(tmem + unit * Z::UNIT, queries + off, keys + off, S_IDESC, k > 0);
    }
    umma_commit(&sh.s_full[unit]);
    if (last) umma_commit(&sh.k_empty[k_slot]);
  };
  // ... and the product of the unit's weights with the values: of the tile's first half, of its second
  auto values = [&](int unit, int half, bool fresh) {
    const uint32_t base = tmem + unit * Z::UNIT;
    const uint64_t b = v_desc + (uint64_t)(v_slot * (Z::OPER >> 4));
#pragma unroll
    for (int k = half * 4; k < half * 4 + 4; ++k) {
      const uint64_t v = b + (uint64_t)(k * 2048 >> 4);
      umma_bf16_ts(base + TA_TILE, base + k * 8, v, O_IDESC, !fresh || k > 0);
      if (LOW) umma_bf16_ts(base + TA_TILE, base + TA_LOW + k * 8, v, O_IDESC, true);
    }
  };
  auto values_end = [&](int unit, bool last, bool end) {
    if (last) umma_commit(&sh.v_empty[v_slot]);
    if (end) {
      umma_commit(&sh.o_end[unit]);
      mbar_arrive(&sh.o_end[unit]);  // what this warp has seen, the unit sees: the clearing warp's finds among it
    }
  };
  uint32_t piece = 0;
  for (int u = u0; u < u1; ++piece) {
    const TreePiece c = tree_piece(p.c, sh.plan, u, u1);
    const int steps = c.steps, mixed = c.first_mixed() - c.tile0;
    wait(smem_u32(&sh.q_ready), piece & 1);
    // A unit's turn, as its weights come, half a tile at a time: their product with the values (cleared, where that is needed),
    // then, if there are `keys`, the next scores
    auto turn = [&](int unit, int j, bool fresh, bool last, bool keys, uint64_t queries) {
      const bool mix = j >= mixed;
      const uint32_t mine = (p_phases >> unit) & 1;
      wait(lane == 0 ? p_half + unit * 8 : (mix ? v_clean : v_full) + v_slot * 8,
           lane == 0 ? mine : mix ? (clean_phases >> v_slot) & 1 : v_phase);
      tc_fence_after();
      if (elect_one()) values(unit, 0, fresh);
      __syncwarp();
      wait(lane == 0 || !keys ? p_ready + unit * 8 : k_full + k_slot * 8, lane == 0 || !keys ? mine : k_phase);
      p_phases ^= 1u << unit;
      tc_fence_after();
      if (elect_one()) {
        values(unit, 1, false);
        values_end(unit, last, !keys);
        if (keys) scores(unit, queries, last);
      }
      __syncwarp();
    };
    auto values_used = [&](int j) {
      if (j >= mixed) clean_phases ^= 1u << v_slot;
      v_step();
    };
    if (c.both) {
      const uint64_t q1_desc = q_desc + (uint64_t)(Z::OPER >> 4);
      wait(k_full + k_slot * 8, k_phase);
      tc_fence_after();
      if (elect_one()) {
        scores(0, q_desc, false);
        scores(1, q1_desc, true);
      }
      __syncwarp();
      k_step();
#pragma unroll 1
      for (int j = 0; j < steps; ++j) {
        const bool more = j + 1 < steps;
        turn(0, j, j == 0, false, more, q_desc);
        turn(1, j, j == 0, true, more, q1_desc);
        values_used(j);
        if (more) k_step();
      }
    } else {
      for (int j = 0; j < min(2, steps); ++j) {
        wait(k_full + k_slot * 8, k_phase);
        tc_fence_after();
        if (elect_one()) scores(j, q_desc, true);
        __syncwarp();
        k_step();
      }
#pragma unroll 1
      for (int j = 0; j < steps; ++j) {
        const bool more = j + 2 < steps;
        turn(j & 1, j, j < 2, true, more, q_desc);
        values_used(j);
        if (more) k_step();
      }
    }
    u = c.next;
  }
}

// ---- softmax, a lane per thread ----
__device__ __forceinline__ void tree_units_sync() {
  __syncwarp();
  asm volatile("bar.sync 1, 256;" ::: "memory");
}

// ... and whether any thread says so
__device__ __forceinline__ bool tree_units_any(bool mine) {
  uint32_t y;
  __syncwarp();
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 p, %1, 0;\n\t"
      "bar.red.or.pred q, 1, 256, p;\n\t"
      "selp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(y)
      : "r"((uint32_t)mine)
      : "memory");
  return y != 0;
}

// Bits of the 32 tokens from `base` on that a row sees: the context, and its mask's nodes.
__device__ __forceinline__ uint32_t tree_seen(int base, int C, uint64_t nodes) {
  const int ctx = C - base;
  if (ctx >= 32) return 0xffffffffu;
  if (ctx > 0) return ((1u << ctx) - 1) | (uint32_t)(nodes << ctx);
  return -ctx < 64 ? (uint32_t)(nodes >> -ctx) : 0u;
}

// A unit's sums times f, seldom.
template <int HD>
__device__ __noinline__ void tree_rescale(uint32_t tm_o, float f) {
#pragma unroll 1
  for (int x = 0; x < HD; x += 16) {
    uint32_t o[16];
    tmem_ld16_issue(tm_o + x, o);
    tmem_ld16_wait(o);
#pragma unroll
    for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
    tmem_st16(tm_o + x, o);
  }
}

// A tile's W tokens from column `seg` W of the scores on: weights to the front of the scores' columns (the other tokens' are zero).
// base: the first of these tokens; m, l: running maximum (base 2) and sum; fresh: the unit has no sums yet.  (Its products so far
// are over: these scores were asked for after them.)  A whole tile's weights are handed over in two halves: the first is multiplied
// while the second is computed (in runs too short for the power cap: 256 rows of the 8B shape 295 -> 280 us, 48 ragged sequences 169 ->
// 151; in long ones the second takes 318 to 338 and 158 to 168).  A quarter of the powers as a cubic on the FMA pipes instead of the
// special-function unit was slower (289 -> 299, 151 -> 177).
// The weights are rounded to bf16 for their product, which puts an output off by 0.0023 in all where its own rounding alone makes 0.0017;
// LOW, the caller's choice, multiplies what the rounding took as well.  It is not the rule because the products then bound even what HBM
// did: 16 trees of 64 rows 40 -> 47 us, 48 ragged ones 168 -> 229, 256 rows of the 8B shape 338 -> 443, one of 100 rows 47.4 -> 48.4.
template <int HD, int W, bool LOW>
__device__ __forceinline__ void tree_step(const TreeDev& p, uint32_t tm_s, int seg, int base, int C, uint64_t nodes, int there,
                                          bool fresh, float& m, float& l, uint64_t* first_half) {
  uint32_t s[W];
#pragma unroll
  for (int x = 0; x < W; x += 32) tmem_ld32_issue(tm_s + seg * W + x, s + x);
#pragma unroll
  for (int x = 0; x < W; x += 32) tmem_ld32_wait(s + x);
  if (base + W > C || there != 3) {
#pragma unroll
    for (int x = 0; x < W; x += 32) {
      const uint32_t seen = (there >> ((base + x) / PAGE & 1)) & 1 ? tree_seen(base + x, C, nodes) : 0u;
#pragma unroll
      for (int i = 0; i < 32; ++i)
        if (!((seen >> i) & 1)) s[x + i] = 0xff800000u;  // minus infinity
    }
  }
  float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
  for (int i = 0; i < W; i += 2) mx[(i >> 1) & 3] = ta_max3(mx[(i >> 1) & 3], __uint_as_float(s[i]), __uint_as_float(s[i + 1]));
  const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * p.scale_log2;
  if (__any_sync(0xffffffffu, top > m + TA_SLACK)) {
    const float m_new = fmaxf(m, top), f = m_new == -INFINITY ? 1.f : ta_exp2(m - m_new);
    m = m_new;
    l *= f;
    if (!fresh) tree_rescale<HD>(tm_s + TA_TILE, f);
  }
  const float shift = m == -INFINITY ? 0.f : -m;
  const uint64_t scale2 = f32x2(p.scale_log2, p.scale_log2), shift2 = f32x2(shift, shift);
  uint64_t sum[2] = {0, 0};
  constexpr int N = LOW ? 16 : 32;  // words of a whole tile that are stored at a time
  uint32_t hi[W / 2], lo[LOW ? W / 2 : 1];
#pragma unroll
  for (int i = 0; i < W / 2; ++i) {
    const float2 e = ta_unpack2(fma_f32x2(f32x2(__uint_as_float(s[2 * i]), __uint_as_float(s[2 * i + 1])), scale2, shift2));
    const float a = ta_exp2(e.x), b = ta_exp2(e.y);
    sum[i & 1] = ta_add2(sum[i & 1], f32x2(a, b));
    hi[i] = cvt_bf16x2(a, b);
    if constexpr (LOW) lo[i] = cvt_bf16x2(a - bf16_lo(hi[i]), b - bf16_hi(hi[i]));
    if (W == TA_TILE && i % N == N - 1) {
      if constexpr (LOW) {
        tmem_st16(tm_s + i - (N - 1), hi + i - (N - 1));
        tmem_st16(tm_s + TA_LOW + i - (N - 1), lo + i - (N - 1));
      } else {
        tmem_st32(tm_s + i - (N - 1), hi + i - (N - 1));
      }
    }
    if (W == TA_TILE && i == 35) {  // the first half is stored by now
      tmem_st_wait();
      tc_fence_before();
      __syncwarp();
      if (threadIdx.x % 32 == 0) mbar_arrive(first_half);
    }
  }
  if constexpr (W != TA_TILE) {  // seg W / 2 words of zeros, the weights, zeros
    uint32_t z[32];
#pragma unroll
    for (int half = 0; half < (LOW ? 4 : 2); ++half) {
#pragma unroll
      for (int i = 0; i < 32; ++i)
        z[i] = seg == ((half & 1) * 32 + i) / (W / 2) ? (LOW && half > 1 ? lo : hi)[i % (W / 2)] : 0u;
      tmem_st32(tm_s + (half >> 1) * TA_LOW + (half & 1) * 32, z);
    }
  }
  const float2 both = ta_unpack2(ta_add2(sum[0], sum[1]));
  l += both.x + both.y;
  tmem_st_wait();
}

// Drafted tokens whose values were taken out, for a row that sees them: this lane's share of the tokens, columns x .. x + 31.  Rare:
// kept out of the way of the code that always runs.
template <int HD>
__device__ __noinline__ void tree_add_dirty(const TreeDev& p, int b, int kvh, int C, int lanes, uint64_t left, int seg, size_t q_at,
                                            float m, float f, int x, float* ex, int me) {
  const uint16_t* q = p.q + q_at;
  for (; left; left &= left - 1) {
    const int slot = C + __ffsll((long long)left) - 1;
    if (slot % TA_TILE / lanes != seg) continue;
    const int id = p.c.kv.page_table[(size_t)b * p.c.kv.max_pages_per_seq + slot / PAGE];
    const size_t row = (((size_t)id * p.c.Hkv + kvh) * PAGE + slot % PAGE) * HD;
    const uint16_t *k = static_cast<const uint16_t*>(p.c.kv.k_pool) + row, *v = static_cast<const uint16_t*>(p.c.kv.v_pool) + row + x;
    float dot = 0.f;
    for (int d = 0; d < HD; ++d) dot += bf2f(q[d]) * bf2f(k[d]);
    const float w = ta_exp2(fmaf(dot, p.scale_log2, m == -INFINITY ? 0.f : -m)) * f;
    for (int i = 0; i < TA_EX; ++i) ex[i * 256 + (me ^ (i >> 3 << 3))] += w * bf2f(v[i]);
  }
}

// Are a row's weights numbers?  (pad: lanes from one of its shares to the next)
__device__ __forceinline__ bool tree_weights_ok(const float2* ml, int row, int pad) {
  bool ok = true;
  for (int i = row; i < 256; i += pad) ok = ok && ml[i].y < INFINITY;  // NaN is not
  return ok;
}

// A piece with sums that are no numbers, by the units' 256 threads: each takes the elements that it has stored, eight a time.
template <int HD>
__device__ __noinline__ void tree_redo(const TreeDev& p, const TreePiece c, int pad, const float2* ml, int* flags, float* part) {
  const int tid = threadIdx.x, G = p.c.G, t0 = c.tile0 * TA_TILE, t1 = min(c.seq.T, c.tile1 * TA_TILE);
  const ValueRows v = value_rows(p.c.kv, p.c.Hkv, c.b, c.kvh);
  if (tid < HD) flags[tid] = 0;
  tree_units_sync();
  value_flags<HD>(v, t0, min(t1, c.C), tid, 256, flags);
  tree_units_sync();
#pragma unroll 1
  for (int x = 0; x < HD; x += TA_EX)
#pragma unroll 1
    for (int t = tid; t < pad * 4; t += 256) {
      const int r = t >> 2;
      if (r >= c.rows) break;
      if (!tree_weights_ok(ml, r, pad)) continue;
      const int row = c.block * TA_BLOCK + r, node = row / G;
      uint64_t nodes = p.mask[(size_t)c.b * p.c.max_nodes + node];
      if (c.seq.n < 64) nodes &= (1ull << c.seq.n) - 1;
      uint16_t* out = p.out + (((size_t)c.b * p.c.max_nodes + node) * p.Hq + c.kvh * G + (row - node * G)) * HD;
#pragma unroll 1
      for (int d = x + (t & 3) * 8; d < x + (t & 3) * 8 + 8; ++d) {
        const float was = part ? part[(size_t)r * HD + d] : bf2f(out[d]);
        if (fabsf(was) < INFINITY) continue;
        const float now = flagged_sum(flags[d] | node_flags<HD>(v, t0, t1, c.C, nodes, d), was);
        if (part) part[(size_t)r * HD + d] = now;
        else out[d] = f2bf(now);
      }
    }
  tree_units_sync();
}

template <int HD, bool LOW>
__device__ void tree_softmax(const TreeDev& p, TreeShared<HD>& sh, unsigned char* q_smem, int u0, int u1) {
  using Z = TaSize<HD>;
  constexpr int PPR = HD / 8, STEP = 256 / PPR;  // 16-byte pieces of a row; rows that 256 threads bring at once
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, unit = warp >> 2, quad = warp & 3, at = quad * 32 + lane;
  const int G = p.c.G, g_inv = 65536 / G + 1;  // r * g_inv >> 16 is r / G, exact for rows below 512 and groups up to 8
  const uint32_t tm_s = sh.tmem + unit * Z::UNIT + ((uint32_t)(quad * 32) << 16), tm_o = tm_s + TA_TILE;
  float* ex = reinterpret_cast<float*>(q_smem + Z::EX);      // [TA_EX][256]: columns of both units' lanes
  float2* ex_ml = reinterpret_cast<float2*>(q_smem + Z::ML);  // [256]
  bool alive = true;
  auto wait = [&](uint64_t* bar, uint32_t parity) {
    alive = alive && mbar_wait(bar, parity, p.status);
    __syncwarp();
  };
  // element of q and of the output where row r of the piece's sequence begins
  auto q_at = [&](const TreePiece& c, int r) {
    const int node = (r * g_inv) >> 16;
    return (((size_t)c.b * p.c.max_nodes + node) * p.Hq + c.kvh * G + (r - node * G)) * HD;
  };
  auto row_of = [&](const TreePiece& c) { return (c.both ? unit * TA_ROWS : 0) + (at & (c.lanes - 1)); };  // this lane's, of the block
  if (u0 >= u1) return;
  TreePiece c = tree_piece(p.c, sh.plan, u0, u1);
  uint32_t done = 0, ends = 0, jobs = 0;  // tiles weighed, pieces ended, tiles that were cleared
#pragma unroll 1
  for (int u = u0;;) {
    const int block0 = c.block * TA_BLOCK, my_row = row_of(c), seg = at / c.lanes;
    const bool real = my_row < c.rows, warp_real = my_row - lane < c.rows;
    uint64_t nodes = 0;
    if (real) nodes = p.mask[(size_t)c.b * p.c.max_nodes + (((block0 + my_row) * g_inv) >> 16)];
    // ---- the queries into their operand tiles, every row once, with its copies; lanes beyond the rows hold zeros ----
    {
      const int rows = c.both ? TA_BLOCK : c.lanes;
#pragma unroll 1
      for (int r0 = tid / PPR; r0 < rows; r0 += 8 * STEP) {
        uint4 q[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int r = r0 + i * STEP;
          q[i] = make_uint4(0u, 0u, 0u, 0u);
          if (r < c.rows) q[i] = *reinterpret_cast<const uint4*>(p.q + q_at(c, block0 + r) + tid % PPR * 8);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int r = r0 + i * STEP;
          const uint32_t dst = smem_u32(q_smem) + (r >= TA_ROWS ? Z::OPER : 0);
          if (r >= rows) break;
#pragma unroll 1
          for (int to = r & (TA_ROWS - 1); to < TA_ROWS; to += c.lanes)
            asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(ta_piece(dst, to, tid % PPR)), "r"(q[i].x), "r"(q[i].y),
                         "r"(q[i].z), "r"(q[i].w)
                         : "memory");
        }
      }
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    tc_fence_before();
    mbar_arrive(&sh.q_ready);
    if (c.seq.n < 64) nodes &= (1ull << c.seq.n) - 1;
    const int stride = c.both ? 1 : 2, from = c.both ? 0 : unit;
    const int32_t* table = p.c.kv.page_table + (size_t)c.b * p.c.kv.max_pages_per_seq + 2 * c.tile0;
    const int pages = min((c.seq.T + PAGE - 1) / PAGE - 2 * c.tile0, 2 * c.steps);  // of the piece
    bool bad = false;
#pragma unroll 4
    for (int i = lane; i < pages; i += 32) bad |= (unsigned)table[i] >= (unsigned)p.c.kv.num_pages;
    bad = __any_sync(0xffffffffu, bad);  // a page is out of range: each tile's pages are looked up
    float m = -INFINITY, l = 0.f;
#pragma unroll 1
    for (int j = from; j < c.steps; j += stride, ++done) {
      const int base = (c.tile0 + j) * TA_TILE;
      int there = 3;
      if (bad)
        there = (int)((unsigned)table[2 * j] < (unsigned)p.c.kv.num_pages) |
                (int)(2 * j + 1 < pages && (unsigned)table[2 * j + 1] < (unsigned)p.c.kv.num_pages) << 1;
      wait(&sh.s_full[unit], done & 1);
      tc_fence_after();
      if (warp_real) {
        if (c.lanes == 128) tree_step<HD, 128, LOW>(p, tm_s, 0, base, c.C, nodes, there, j == from, m, l, &sh.p_half[unit]);
        else if (c.lanes == 64) tree_step<HD, 64, LOW>(p, tm_s, seg, base + seg * 64, c.C, nodes, there, j == from, m, l, &sh.p_half[unit]);
        else tree_step<HD, 32, LOW>(p, tm_s, seg, base + seg * 32, c.C, nodes, there, j == from, m, l, &sh.p_half[unit]);
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        if (!warp_real || c.lanes < TA_TILE) mbar_arrive(&sh.p_half[unit]);
        mbar_arrive(&sh.p_ready[unit]);
      }
    }
    const int u_next = c.next;
    TreePiece next = c;
    if (u_next < u1) {  // the next queries on their way to L2 while this piece ends
      next = tree_piece(p.c, sh.plan, u_next, u1);
      for (int r = tid; r < next.rows; r += 256)
        asm volatile("prefetch.global.L2 [%0];" ::"l"(p.q + q_at(next, next.block * TA_BLOCK + r)));
    }

    // ---- the end of the piece: what the units, and the copies of a row, have is added up ----
    const bool worked = from < c.steps, whole = c.whole();
    if (worked) {
      wait(&sh.o_end[unit], ends & 1);
      ++ends;
    }
    tc_fence_after();
    tree_units_sync();  // nobody reads the queries any more
    const int pad = c.both ? 256 : c.lanes, me = unit * 128 + at, first = me & (pad - 1);
    const size_t part = (size_t)(2 * blockIdx.x + (u > u0)) * p.part.rows;
    ex_ml[me] = make_float2(m, l);
    tree_units_sync();
    float f;  // what this lane's sums count
    {
      float2 ml[8];  // a row's shares: one, two, four or eight
      float top = -INFINITY, sum = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) ml[i] = first + i * pad < 256 ? ex_ml[first + i * pad] : make_float2(-INFINITY, 0.f);
#pragma unroll
      for (int i = 0; i < 8; ++i) top = fmaxf(top, ml[i].x);
      const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += ml[i].y * ta_exp2(ml[i].x - base);
      f = ta_exp2(m - base);
      if (whole) f = sum == 0.f ? 0.f : f / sum;
      else if (me < pad && real) p.part.ml[part + my_row] = make_float2(top, sum);
    }
    uint64_t dirty = 0;  // drafted tokens whose values were taken out, of this unit's tiles
    for (int t = c.first_mixed(); t < c.tile1; ++t, ++jobs)
      if (c.both || ((t - c.tile0) & 1) == unit) dirty |= sh.dirty[jobs % TA_JOBS];
    dirty = worked && real ? dirty & nodes : 0ull;
    bool redo = false;  // any sums that are no numbers
    // 32 columns at a time: every lane leaves its own, then a thread adds up eight columns of a row (the places are turned by the
    // columns' group, so that the four threads of a row read from different banks)
#pragma unroll 1
    for (int x = 0; x < HD; x += TA_EX) {
      uint32_t o[TA_EX];
#pragma unroll
      for (int i = 0; i < TA_EX; ++i) o[i] = 0u;
      if (warp_real && worked) {
        tmem_ld32_issue(tm_o + x, o);
        tmem_ld32_wait(o);
      }
#pragma unroll
      for (int i = 0; i < TA_EX; ++i) ex[i * 256 + (me ^ (i >> 3 << 3))] = __uint_as_float(o[i]) * f;
      if (dirty) tree_add_dirty<HD>(p, c.b, c.kvh, c.C, c.lanes, dirty, seg, q_at(c, block0 + my_row), m, f, x, ex, me);
      tree_units_sync();
#pragma unroll 1
      for (int t = tid; t < pad * 4; t += 256) {
        const int r = t >> 2, col = (t & 3) * 8;
        if (r >= c.rows) break;
        float a[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
        for (int i = r; i < 256; i += pad)
#pragma unroll
          for (int e = 0; e < 8; ++e) a[e] += ex[(col + e) * 256 + (i ^ col)];
        float none = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) none = fmaf(a[e], 0.f, none);
        if (none != 0.f) redo = redo || tree_weights_ok(ex_ml, r, pad);
        if (whole) {
          *reinterpret_cast<uint4*>(p.out + q_at(c, block0 + r) + x + col) =
              make_uint4(cvt_bf16x2(a[0], a[1]), cvt_bf16x2(a[2], a[3]), cvt_bf16x2(a[4], a[5]), cvt_bf16x2(a[6], a[7]));
        } else {
          float4* dst = reinterpret_cast<float4*>(p.part.sums + (part + r) * HD + x + col);
          dst[0] = make_float4(a[0], a[1], a[2], a[3]);
          dst[1] = make_float4(a[4], a[5], a[6], a[7]);
        }
      }
      redo = tree_units_any(redo);
    }
    if (redo) tree_redo<HD>(p, c, pad, ex_ml, reinterpret_cast<int*>(ex), whole ? nullptr : p.part.sums + part * HD);
    if (u_next >= u1) break;
    c = next;
    u = u_next;
  }
}

template <int HD, bool LOW>
__global__ void __launch_bounds__(TA_THREADS, 1) tree_attn_kernel(const __grid_constant__ CUtensorMap kmap,
                                                                  const __grid_constant__ CUtensorMap vmap, const __grid_constant__ TreeDev p) {
  using Z = TaSize<HD>;
  extern __shared__ unsigned char ta_smem[];
  __shared__ TreeShared<HD> sh;
  unsigned char* q_smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(ta_smem) + 1023) & ~(uintptr_t)1023);
  unsigned char *k_ring = q_smem + 2 * Z::OPER, *v_ring = k_ring + Z::K_SLOTS * Z::OPER;
  const int tid = threadIdx.x, warp = tid >> 5;
  if (tid == 0) {
    for (int i = 0; i < Z::K_SLOTS; ++i) {
      mbar_init(&sh.k_full[i], 1);
      mbar_init(&sh.k_empty[i], 1);
    }
    for (int i = 0; i < Z::V_SLOTS; ++i) {
      mbar_init(&sh.v_full[i], 1);
      mbar_init(&sh.v_empty[i], 1);
      mbar_init(&sh.v_clean[i], 32);
    }
    mbar_init(&sh.q_ready, 256);
    for (int x = 0; x < 2; ++x) {
      mbar_init(&sh.s_full[x], 1);
      mbar_init(&sh.p_half[x], 4);
      mbar_init(&sh.p_ready[x], 4);
      mbar_init(&sh.o_end[x], 2);
    }
    sh.posted = 0;
    fence_mbar_init();
    tma_prefetch_map(&kmap);
    tma_prefetch_map(&vmap);
  }
  pdl_wait();
  pdl_trigger();
  if (warp == TAW_MMA) tmem_alloc(&sh.tmem, 512);  // not ahead of the wait: a kernel before this one may need it
  tc_fence_before();
  chain_plan(p.c, sh.plan, gridDim.x, blockIdx.x == 0 ? p.status : nullptr);
  tc_fence_after();
  const int2 range = chain_range(p.c, sh.plan, blockIdx.x);
  const int u0 = range.x, u1 = range.y;
  if (warp >= 8) asm volatile("setmaxnreg.dec.sync.aligned.u32 104;");  // 168 a thread at launch: 128 threads give 64 each,
  else asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");            // 256 take 32 each
  if (warp < 8) tree_softmax<HD, LOW>(p, sh, q_smem, u0, u1);
  else if (warp == TAW_KEYS) tree_load<HD, false>(p, sh, k_ring, &kmap, u0, u1);
  else if (warp == TAW_VALUES) tree_load<HD, true>(p, sh, v_ring, &vmap, u0, u1);
  else if (warp == TAW_MMA) tree_mma<HD, LOW>(p, sh, smem_u32(q_smem), smem_u32(k_ring), smem_u32(v_ring), u0, u1);
  else {
    if (tid == TAW_CLEAR * 32) chain_describe(p.c, sh.plan, blockIdx.x, u0, u1, p.part.desc);
    __syncwarp();
    tree_clear<HD>(p, sh, smem_u32(v_ring));
  }
  tc_fence_before();
  __syncthreads();
  if (warp == TAW_MMA) tmem_dealloc(sh.tmem, 512);
}

static int tree_rows(const sol_shape_t& sh, int max_nodes) { return std::min(TA_BLOCK, max_nodes * (sh.n_q_heads / sh.n_kv_heads)); }
size_t tree_part_bytes(const sol_shape_t& sh, int max_nodes) { return chain_part_bytes(sm_count(), tree_rows(sh, max_nodes), sh.head_dim); }

template <int HD, bool LOW>
static void launch_tree(const TreeDev& d, const CUtensorMap& kmap, const CUtensorMap& vmap, int ctas, cudaStream_t st) {
  ensure_dynamic_smem(reinterpret_cast<const void*>(&tree_attn_kernel<HD, LOW>), TaSize<HD>::SMEM);
  SOL_LAUNCH("tree_attn", (tree_attn_kernel<HD, LOW>), dim3(ctas), dim3(TA_THREADS), TaSize<HD>::SMEM, st, kmap, vmap, d);
  launch_chain_merge(d.c, d.part, d.Hq, HD, ctas, d.out, st);
}

void launch_tree_attention(const RowsArgs& a, cudaStream_t st) {
  const sol_shape_t& sh = a.shape;
  CUtensorMap kmap, vmap;
  if (!encode_pool_map(&kmap, a.kv.k_pool, sh, a.kv.num_pages) || !encode_pool_map(&vmap, a.kv.v_pool, sh, a.kv.num_pages))
    return;
  const int ctas = sm_count();
  TreeDev d;
  d.c = chain_shape(a, TA_BLOCK, TA_TILE, TA_MIN_TILES, ta_piece_cost(sh.head_dim));
  d.Hq = sh.n_q_heads;
  d.scale_log2 = 1.4426950408889634f / sqrtf((float)sh.head_dim);
  d.mask = a.mask;
  d.q = static_cast<const uint16_t*>(a.q);
  d.out = static_cast<uint16_t*>(a.out);
  d.part = chain_parts(a.part, ctas, tree_rows(sh, a.max_nodes), sh.head_dim);
  d.status = a.status;
  if (sh.head_dim == 64) {
    if (a.low_parts) launch_tree<64, true>(d, kmap, vmap, ctas, st);
    else launch_tree<64, false>(d, kmap, vmap, ctas, st);
  } else {
    if (a.low_parts) launch_tree<128, true>(d, kmap, vmap, ctas, st);
    else launch_tree<128, false>(d, kmap, vmap, ctas, st);
  }
}

}  // namespace sol
