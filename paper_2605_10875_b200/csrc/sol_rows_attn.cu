// Dense attention of few query rows over the paged cache: the decode step that keeps the attention weights
// (sol_weighted_decode_attn) and small trees of drafted tokens (sol_tree_attn).
//
//   o_r = sum_t p_rt v_t,  p_rt = 2^(s_rt - m_r) / l_r,  s_rt = (q_r . k_t) log2(e) / sqrt(head_dim)  where row r sees token t
//
//   rows_attn_kernel   one CTA per SM takes its run of tiles (sol_chain.cuh; a tile is a 64-token page of one kv-head).  A
//                      producer warp brings a tile's keys and values by TMA (128-byte swizzle) at a time, 16 or 32 KB,
//                      which the other warps take in turn, each into its own ring of stages.  Tokens (then head_dim) are the M side of
//                      mma.sync m16n8k16 and the query rows the N side, 16, 8 or 4 of them (S^T = K Q^T, O^T = V^T P^T);
//                      online softmax in registers, weights as bf16 high and low parts, of four rows in one product.  At
//                      the end of a chain the warps' results are merged through shared memory.
//   chain_merge_kernel merges the chains that were cut between CTAs.
//   weight_kernel      the same for decode steps, and then the weights: w_t <- decay w_t + sum_g 2^(s_gt - lse_g) from the
//                      logits that the first kernel left.
#include <cuda.h>
#include <math.h>

#include <algorithm>

#include "sol_chain.cuh"
#include "sol_umma.cuh"

namespace sol {

constexpr int RA_MAX_ROWS = 16;  // query rows of a chain at most
constexpr int RA_MIN_TILES = 4;
constexpr int ra_piece_cost(int hd) { return hd == 64 ? 8 : 4; }

struct RowsDev {
  ChainShape c;
  int Hq;
  float scale_log2;      // log2(e) / sqrt(head_dim)
  const uint64_t* mask;  // [B][max_nodes]; nullptr: a decode step
  const uint16_t* q;     // [B][max_nodes][Hq][HD]
  uint16_t* out;
  ChainParts part;       // 2 slots per CTA
  float* logits;         // decode steps with weights: [B][Hkv][G][Tmax] base-2 logits, else nullptr
  float* lse;            // ... [B][Hq] base-2 log of the weights' sum (infinite where no token counts), of chains that were not cut
  int* status;
};

// ROWS query rows per chain: 16, 8 or 4.
// Bound by HBM: one query token of 64 sequences of 8000 of the 8B shape takes 316 us (2.1 GB, 6.6 TB/s; steps of half a tile, in
// 4 KB boxes, took 403), with 16 rows 32 sequences take 171 us of which the bytes need 161; at head_dim 64 64 sequences take 175
// of 161 with up to 8 rows, 204 with 16, where the products of two blocks of rows fill the warps' time.
template <int HD, int ROWS>
struct RaSize {
  static constexpr int HALF = PAGE * 128;      // a 64-wide half of the keys: [64 tokens][128 B]
  static constexpr int TILE = HALF * (HD / 64);
  // Consumer warps, stages of a warp's ring: one warp per quarter of the SM (the producer in the fourth) keeps up and has the
  // deeper ring (128 ragged decode steps 336 us, with four warps 356, with six 352).  Only 16 rows at head_dim 64 keep three warps busy
  // (16 sequences of 4000: 41 us, with six 37).
  static constexpr int STAGES = 192 * 1024 / (2 * TILE), WARPS = HD == 64 && ROWS == 16 ? 6 : 3, DEPTH = STAGES / WARPS;
  static constexpr int THREADS = (WARPS + 1) * 32;
  static constexpr int NB = ROWS == 16 ? 2 : 1;         // blocks of eight rows
  static constexpr int REGS = (HD / 16 * 4 + 4) * NB;   // sums, two maxima, two sums of weights
  static constexpr int MERGE = 2 * REGS * 32 * 4;
  static constexpr int SMEM = 1024 + STAGES * 2 * TILE + MERGE;
};

// Shared-memory address of 16-byte piece c of token r of a step.
template <int HALF>
__device__ __forceinline__ uint32_t ra_piece(uint32_t base, int r, int c) {
  return base + (uint32_t)((c >> 3) * HALF + r * 128 + (((c & 7) ^ (r & 7)) << 4));
}
template <int THREADS>
__device__ __forceinline__ void ra_consumer_sync() {
  __syncwarp();
  asm volatile("bar.sync 1, %0;" ::"n"(THREADS) : "memory");
}

// Rows of a piece with sums that are no numbers (`redo`: a bit per lane's row), by the warp that has stored them: bf16 to the output
// or float32 to the partial results.
template <int HD, int ROWS>
__device__ __noinline__ void ra_redo(const ValueRows v, const uint64_t* mask, int G, int C, int t0, int t1, int row0, int redo, int* flags,
                                     uint16_t* out, int Hq, float* part) {
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  for (int d = lane; d < HD; d += 32) flags[d] = 0;
  __syncwarp();
  value_flags<HD>(v, t0, min(t1, C), lane, 32, flags);
  __syncwarp();
#pragma unroll 1
  for (int i = 0; i < 4; ++i) {
    if (!((redo >> i) & 1)) continue;
    const int r = (i >> 1) * 8 + 2 * t + (i & 1), node = (row0 + r) / G;
    const uint64_t nodes = mask ? mask[node] : 1ull;  // (nodes that are not there lie behind t1)
#pragma unroll 1
    for (int d = g; d < HD; d += 8) {
      uint16_t* o = out + ((size_t)node * Hq + (row0 + r - node * G)) * HD + d;
      const float was = part ? part[r * HD + d] : bf2f(*o);
      if (fabsf(was) < INFINITY) continue;
      const float now = flagged_sum(flags[d] | node_flags<HD>(v, t0, t1, C, nodes, d), was);
      if (part) part[r * HD + d] = now;
      else *o = f2bf(now);
    }
  }
  __syncwarp();
}

template <int HD, int ROWS>
__global__ void __launch_bounds__(RaSize<HD, ROWS>::THREADS, 1)
    rows_attn_kernel(const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap, const RowsDev p) {
  using Z = RaSize<HD, ROWS>;
  static_assert(Z::THREADS >= CHAIN_MAX_BATCH, "chain_plan");
  constexpr int KS = HD / 16, MT = PAGE / 16, NB = Z::NB;  // steps of head_dim, of tokens; blocks of eight rows
  constexpr bool PACK = ROWS == 4;  // rows 4 .. 7 of the block are rows 0 .. 3 again: their weights' low parts
  extern __shared__ unsigned char ra_smem[];
  __shared__ ChainPlan plan;
  __shared__ uint64_t full[Z::STAGES], empty[Z::STAGES];
  __shared__ int page_ok[Z::STAGES];
  __shared__ int flags[HD];
  unsigned char* ring = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(ra_smem) + 1023) & ~(uintptr_t)1023);
  float* merge = reinterpret_cast<float*>(ring + Z::STAGES * 2 * Z::TILE);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int s = 0; s < Z::STAGES; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    fence_mbar_init();
    tma_prefetch_map(&kmap);
    tma_prefetch_map(&vmap);
  }
  pdl_wait();
  pdl_trigger();
  chain_plan(p.c, plan, gridDim.x, blockIdx.x == 0 ? p.status : nullptr);
  const int2 range = chain_range(p.c, plan, blockIdx.x);
  const int u0 = range.x, u1 = range.y;

  if (tid == 0) chain_describe(p.c, plan, blockIdx.x, u0, u1, p.part.desc);
  if (warp == Z::WARPS) {  // ---- the producer ----
    int it = 0;
    for (int u = u0; u < u1;) {
      const ChainPiece c = chain_piece(p.c, plan, u, u1);
      const int32_t* table = p.c.kv.page_table + (size_t)c.b * p.c.kv.max_pages_per_seq;
      for (int g0 = c.tile0; g0 < c.tile1; g0 += 32) {
        int mine = 0;
        if (g0 + lane < c.tile1 && c.seq.T > 0) mine = table[g0 + lane];
        const int cnt = min(32, c.tile1 - g0);
        for (int x = 0; x < cnt; ++x, ++it) {
          int page = __shfl_sync(0xffffffffu, mine, x);
          // step `it` goes to warp it % Z::WARPS, whose use number `use` of its ring it is
          const int use = it / Z::WARPS, st = it % Z::WARPS * Z::DEPTH + use % Z::DEPTH;
          if (use >= Z::DEPTH && !__all_sync(0xffffffffu, mbar_wait(&empty[st], (use / Z::DEPTH - 1) & 1, p.status))) {
            // the consumers give up too; what has been requested still arrives before the CTA ends
            for (int i = max(0, it - Z::STAGES); i < it; ++i)
              mbar_wait(&full[i % Z::WARPS * Z::DEPTH + i / Z::WARPS % Z::DEPTH], (i / Z::WARPS / Z::DEPTH) & 1, p.status);
            return;
          }
          if (lane == 0) {
            const bool ok = page >= 0 && page < p.c.kv.num_pages;
            if (!ok) {
              atomicOr(p.status + ST_ERR, ERR_BAD_PAGE);
              page = 0;  // some memory of the pool; none of its tokens is seen
            }
            page_ok[st] = ok;
            unsigned char* dst = ring + (size_t)st * 2 * Z::TILE;
            mbar_expect_tx(&full[st], 2 * Z::TILE);
            const int row = (page * p.c.Hkv + c.kvh) * PAGE;
#pragma unroll
            for (int h = 0; h < HD / 64; ++h) {
              tma_load_2d(dst + h * Z::HALF, &kmap, h * 64, row, &full[st]);
              tma_load_2d(dst + Z::TILE + h * Z::HALF, &vmap, h * 64, row, &full[st]);
            }
          }
          __syncwarp();
        }
      }
      u = c.next;
    }
    return;
  }

  // ---- the consumers ----
  // a lane's share: tokens (or elements of the head) g and g + 8 of every 16, rows 2 t and 2 t + 1 of every block of eight
  const int g = lane >> 2, t = lane & 3, G = p.c.G;
  int it = 0;
  bool alive = true;
  for (int u = u0; u < u1;) {
    const ChainPiece c = chain_piece(p.c, plan, u, u1);
    const int C = c.seq.T - c.seq.n, T = c.seq.T, rows = c.seq.n * G, row0 = c.block * ROWS;
    auto row_at = [&](int r) {  // element of q and of the output where row r of the chain begins
      const int node = (row0 + r) / G;
      return (((size_t)c.b * p.c.max_nodes + node) * p.Hq + c.kvh * G + (row0 + r - node * G)) * HD;
    };
    uint32_t q[NB][KS][2];
    uint64_t seen[NB][2];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const int r = nb * 8 + (PACK ? g & 3 : g);
      const bool real = row0 + r < rows;
      const uint16_t* src = p.q + (real ? row_at(r) : 0);
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        q[nb][k][0] = real ? *reinterpret_cast<const uint32_t*>(src + k * 16 + 2 * t) : 0u;
        q[nb][k][1] = real ? *reinterpret_cast<const uint32_t*>(src + k * 16 + 8 + 2 * t) : 0u;
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int col = nb * 8 + (PACK ? (2 * t + e) & 3 : 2 * t + e);
        seen[nb][e] = row0 + col < rows ? (p.mask ? p.mask[(size_t)c.b * p.c.max_nodes + (row0 + col) / G] : ~0ull) : 0ull;
      }
    }
    float m[NB][2], l[NB][2], o[NB][KS][4];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      m[nb][0] = m[nb][1] = -INFINITY;
      l[nb][0] = l[nb][1] = 0.f;
#pragma unroll
      for (int k = 0; k < KS; ++k) o[nb][k][0] = o[nb][k][1] = o[nb][k][2] = o[nb][k][3] = 0.f;
    }

    const int len = c.tile1 - c.tile0;
#pragma unroll 1
    for (int x = (warp - it % Z::WARPS + Z::WARPS) % Z::WARPS; x < len; x += Z::WARPS) {
      const int use = (it + x) / Z::WARPS, st = warp * Z::DEPTH + use % Z::DEPTH;
      const int tok0 = (c.tile0 + x) * PAGE;  // first token of the step
      alive = alive && __all_sync(0xffffffffu, mbar_wait(&full[st], (use / Z::DEPTH) & 1, p.status));
      if (!alive) break;
      const uint32_t kb = smem_u32(ring + (size_t)st * 2 * Z::TILE), vb = kb + Z::TILE;
      const bool ok = page_ok[st] != 0;
      float sc[NB][MT][4];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int i = 0; i < MT; ++i) sc[nb][i][0] = sc[nb][i][1] = sc[nb][i][2] = sc[nb][i][3] = 0.f;
#pragma unroll
      for (int k = 0; k < KS; ++k)
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          uint32_t a[4];
          ldsm_x4(a, ra_piece<Z::HALF>(kb, i * 16 + (lane & 15), k * 2 + (lane >> 4)));
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) mma_bf16(sc[nb][i], a[0], a[1], a[2], a[3], q[nb][k][0], q[nb][k][1]);
        }
      // ---- which tokens are seen; a step inside the context is seen whole by every row ----
      uint64_t bad = 0;  // drafted tokens of the step with values that are not finite
      if (ok && tok0 + PAGE <= C) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) sc[nb][i][e] *= p.scale_log2;
      } else {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int tok = tok0 + i * 16 + g + (e >> 1) * 8;
              const bool s = ok && (tok < C || (tok < T && ((seen[nb][e & 1] >> (tok - C)) & 1)));
              sc[nb][i][e] = s ? sc[nb][i][e] * p.scale_log2 : -INFINITY;
            }
        // A weight of zero must not meet a value that is not finite.  Rows of the page behind the sequence are cleared, and so
        // are drafted tokens' rows with such values, which are added below for the query rows that see them.
#pragma unroll 1
        for (int w = 0; w < PAGE / 32; ++w) {
          const int r = lane + 32 * w, tok = tok0 + r;
          bool drop = tok >= T || !ok;
          if (!drop && tok >= C) {
            for (int cc = 0; cc < HD / 8; ++cc) {
              const uint4 v = lds128(ra_piece<Z::HALF>(vb, r, cc));
              const uint32_t x4[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
              for (int e = 0; e < 4; ++e)
                drop = drop || (x4[e] & 0x7f80u) == 0x7f80u || (x4[e] & 0x7f800000u) == 0x7f800000u;
            }
          }
          if (drop)
            for (int cc = 0; cc < HD / 8; ++cc)
              asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(ra_piece<Z::HALF>(vb, r, cc)), "r"(0u) : "memory");
          const uint32_t votes = __ballot_sync(0xffffffffu, drop && ok && tok >= C && tok < T);
          bad |= (uint64_t)votes << (32 * w);
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // ahead of the TMA write that takes the stage next
        __syncwarp();
      }
      if (p.logits) {  // decode steps: the G heads are the first rows
        const size_t stride = (size_t)p.c.kv.max_pages_per_seq * PAGE;
        float* dst = p.logits + ((size_t)c.b * p.c.Hkv + c.kvh) * G * stride + tok0 + g;
#pragma unroll
        for (int e = 0; e < 2; ++e)
          if (2 * t + e < G) {
#pragma unroll
            for (int i = 0; i < MT; ++i) {
              dst[(2 * t + e) * stride + i * 16] = sc[0][i][e];
              dst[(2 * t + e) * stride + i * 16 + 8] = sc[0][i][2 + e];
            }
          }
      }
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        float f[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float top = -INFINITY;
#pragma unroll
          for (int i = 0; i < MT; ++i) top = fmaxf(top, fmaxf(sc[nb][i][e], sc[nb][i][2 + e]));
#pragma unroll
          for (int off = 4; off <= 16; off <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
          const float now = fmaxf(m[nb][e], top), base = now == -INFINITY ? 0.f : now;  // a row that has seen nothing yet
          f[e] = exp2f(m[nb][e] - base);
          m[nb][e] = now;
          l[nb][e] *= f[e];
#pragma unroll
          for (int i = 0; i < MT; ++i) {
            sc[nb][i][e] = exp2f(sc[nb][i][e] - base);
            sc[nb][i][2 + e] = exp2f(sc[nb][i][2 + e] - base);
            l[nb][e] += sc[nb][i][e] + sc[nb][i][2 + e];
          }
        }
        if (__any_sync(0xffffffffu, f[0] != 1.f || f[1] != 1.f)) {
#pragma unroll
          for (int k = 0; k < KS; ++k) {
            o[nb][k][0] *= f[0];
            o[nb][k][1] *= f[1];
            o[nb][k][2] *= f[0];
            o[nb][k][3] *= f[1];
          }
        }
      }
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        uint32_t hi[NB][2], lo[NB][2];  // the weights of 16 tokens, transposed
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const float v0 = sc[nb][i][2 * h], v1 = sc[nb][i][2 * h + 1];
            const uint32_t w = pack_bf16(v0, v1), r = pack_bf16(v0 - bf16_lo(w), v1 - bf16_hi(w));
            if (PACK) {
              hi[nb][h] = movm_trans(t < 2 ? w : r);
            } else {
              hi[nb][h] = movm_trans(w);
              lo[nb][h] = movm_trans(r);
            }
          }
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          uint32_t a[4];
          ldsm_x4_trans(a, ra_piece<Z::HALF>(vb, i * 16 + (lane & 7) + (lane >> 4) * 8, k * 2 + ((lane >> 3) & 1)));
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            mma_bf16(o[nb][k], a[0], a[1], a[2], a[3], hi[nb][0], hi[nb][1]);
            if (!PACK) mma_bf16(o[nb][k], a[0], a[1], a[2], a[3], lo[nb][0], lo[nb][1]);
          }
        }
      }
      if (bad) {  // p v in float32 for the rows that see such a token, from the cache
        const int page = p.c.kv.page_table[(size_t)c.b * p.c.kv.max_pages_per_seq + tok0 / PAGE];
        const uint16_t* v =
            static_cast<const uint16_t*>(p.c.kv.v_pool) + (((size_t)page * p.c.Hkv + c.kvh) * PAGE + tok0 % PAGE) * HD;
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll 1
          for (int j = 0; j < 16; ++j) {
            const int tok = i * 16 + j;
            if (!((bad >> tok) & 1)) continue;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const float w = __shfl_sync(0xffffffffu, j < 8 ? sc[nb][i][e] : sc[nb][i][2 + e], (j & 7) * 4 + t);
                if (!((seen[nb][e] >> (tok0 + tok - C)) & 1) || (PACK && t >= 2)) continue;
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                  o[nb][k][e] += w * bf2f(v[tok * HD + k * 16 + g]);
                  o[nb][k][2 + e] += w * bf2f(v[tok * HD + k * 16 + 8 + g]);
                }
              }
          }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&empty[st]);
    }
    it += len;

    // ---- merge the warps (six: 4 and 5 into 0 and 1), then 2 and 3, then 1; a lane holds the same elements in every warp ----
#pragma unroll 1
    for (int half = Z::WARPS > 4 ? 4 : 2; half; half >>= 1) {
      float* slot = merge + (size_t)(warp & 1 & (half - 1)) * Z::REGS * 32 + lane;
      const bool gives = warp >= half && warp < min(2 * half, Z::WARPS), takes = warp + half < min(2 * half, Z::WARPS);
      if (gives) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          float* s = slot + nb * (KS * 4 + 4) * 32;
#pragma unroll
          for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[(k * 4 + e) * 32] = o[nb][k][e];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            s[(KS * 4 + e) * 32] = m[nb][e];
            s[(KS * 4 + 2 + e) * 32] = l[nb][e];
          }
        }
      }
      ra_consumer_sync<Z::WARPS * 32>();
      if (takes) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          const float* s = slot + nb * (KS * 4 + 4) * 32;
          float f[2], h[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float y = s[(KS * 4 + e) * 32], now = fmaxf(m[nb][e], y), base = now == -INFINITY ? 0.f : now;
            f[e] = exp2f(m[nb][e] - base);
            h[e] = exp2f(y - base);
            m[nb][e] = now;
            l[nb][e] = l[nb][e] * f[e] + s[(KS * 4 + 2 + e) * 32] * h[e];
          }
#pragma unroll
          for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[nb][k][e] = o[nb][k][e] * f[e & 1] + s[(k * 4 + e) * 32] * h[e & 1];
        }
      }
      ra_consumer_sync<Z::WARPS * 32>();
    }
    if (warp == 0) {
      const bool whole = c.whole();
      const size_t part = (size_t)(2 * blockIdx.x + (u > u0)) * p.part.rows;
      int redo = 0;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        if (PACK) {  // high and low parts
#pragma unroll
          for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[nb][k][e] += __shfl_xor_sync(0xffffffffu, o[nb][k][e], 2);
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float sum = l[nb][e];
#pragma unroll
          for (int off = 4; off <= 16; off <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
          const int r = nb * 8 + 2 * t + e;
          if (row0 + r >= rows || (PACK && t >= 2)) continue;
          if (whole) {
            const float inv = sum == 0.f ? 0.f : 1.0f / sum;
            uint16_t* dst = p.out + row_at(r) + g;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
              dst[k * 16] = f2bf(o[nb][k][e] * inv);
              dst[k * 16 + 8] = f2bf(o[nb][k][2 + e] * inv);
            }
            if (p.lse && g == 0) p.lse[(size_t)c.b * p.Hq + c.kvh * G + r] = sum == 0.f ? INFINITY : m[nb][e] + log2f(sum);
          } else {
            float* dst = p.part.sums + (part + r) * HD + g;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
              dst[k * 16] = o[nb][k][e];
              dst[k * 16 + 8] = o[nb][k][2 + e];
            }
            if (g == 0) p.part.ml[part + r] = make_float2(m[nb][e], sum);
          }
          float none = 0.f;
#pragma unroll
          for (int k = 0; k < KS; ++k) none = fmaf(o[nb][k][e], 0.f, fmaf(o[nb][k][2 + e], 0.f, none));
          if (none != 0.f && sum < INFINITY) redo |= 1 << (nb * 2 + e);  // (NaN differs from 0, and is not below infinity)
        }
      }
      if (__any_sync(0xffffffffu, redo))
        ra_redo<HD, ROWS>(value_rows(p.c.kv, p.c.Hkv, c.b, c.kvh), p.mask ? p.mask + (size_t)c.b * p.c.max_nodes : nullptr, G, C,
                          c.tile0 * PAGE, min(T, c.tile1 * PAGE), row0, redo, flags,
                          p.out + ((size_t)c.b * p.c.max_nodes * p.Hq + c.kvh * G) * HD, p.Hq, whole ? nullptr : p.part.sums + part * HD);
    }
    u = c.next;
  }
}

// ---- merge of the chains that were cut -----------------------------------------------------------
constexpr int RM_THREADS = 256;
constexpr int RM_ROWS = RM_THREADS / 16;  // rows of a CTA, 16 lanes each

// A CTA per (CTA of the attention kernel, 16 rows): the chain that begins in that CTA's run and goes on in the next.  The
// attention kernel has written down which one that is: finding it again from the lengths took longer than the merge.
template <int HD>
__global__ void __launch_bounds__(RM_THREADS) chain_merge_kernel(const ChainParts part, int G, int max_nodes, int Hq, int block_rows,
                                                                 uint16_t* __restrict__ out) {
  pdl_trigger();
  pdl_wait();
  const ChainDesc d = part.desc[blockIdx.x];
  if (blockIdx.y * RM_ROWS >= d.rows || d.pieces == 0) return;
  ChainCut cut;
  cut.first = blockIdx.x;
  cut.last = blockIdx.x + d.pieces - 1;
  cut.first_slot = d.first_slot;
  const int row = blockIdx.y * RM_ROWS + (threadIdx.x >> 4);
  const float2 ml = chain_merged_ml(part, cut, min(row, d.rows - 1));  // whole warps take part in the reductions
  if (row >= d.rows) return;
  const int r = d.block * block_rows + row, node = r / G;
  chain_merged_row<HD>(part, cut, row, ml, out + (((size_t)d.b * max_nodes + node) * Hq + d.kvh * G + (r - node * G)) * HD);
}

// After an attention kernel of `ctas` CTAs that left its cut chains in `part`.
void launch_chain_merge(const ChainShape& c, const ChainParts& part, int Hq, int hd, int ctas, uint16_t* out, cudaStream_t st) {
  const dim3 grid(ctas, (part.rows + RM_ROWS - 1) / RM_ROWS);
  if (hd == 64)
    SOL_LAUNCH("chain_merge", chain_merge_kernel<64>, grid, dim3(RM_THREADS), 0, st, part, c.G, c.max_nodes, Hq, c.block_rows, out);
  else
    SOL_LAUNCH("chain_merge", chain_merge_kernel<128>, grid, dim3(RM_THREADS), 0, st, part, c.G, c.max_nodes, Hq, c.block_rows, out);
}

// ---- the weights of a decode step ----------------------------------------------------------------
constexpr int WK_V = 2;                          // four tokens at a time, so many times per thread
constexpr int WK_TOKENS = RM_THREADS * 4 * WK_V;  // tokens of a unit

// A CTA takes (sequence, kv-head, WK_TOKENS tokens) units in turn.  Its threads request logits and weights first and find the
// heads' sums of weights (of chains that were cut: from the pieces) while those travel: one after the other, the waits for
// memory were what the kernel consisted of (62 us for 160 MB).
template <int HD>
__global__ void __launch_bounds__(RM_THREADS, 3) weight_kernel(const RowsDev p, int ctas, float decay, float* __restrict__ weights) {
  __shared__ ChainPlan plan;
  __shared__ float lse[RM_ROWS];
  __shared__ int units[CHAIN_MAX_BATCH + 1];
  const int tid = threadIdx.x;
  pdl_trigger();
  chain_plan(p.c, plan, ctas, nullptr);
  const int G = p.c.G;
  if (tid < 32) {  // units before each sequence
    int n = 0;
    for (int b0 = 0; b0 < CHAIN_MAX_BATCH; b0 += 32) {
      const int b = b0 + tid;
      int v = b < p.c.B ? max(1, (plan.at(b).T + WK_TOKENS - 1) / WK_TOKENS) * p.c.Hkv : 0;
      const int mine = v;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, v, o);
        if (tid >= o) v += x;
      }
      units[b] = n + v - mine;
      n += __shfl_sync(0xffffffffu, v, 31);
    }
    if (tid == 0) units[CHAIN_MAX_BATCH] = n;
  }
  __syncthreads();
  pdl_wait();
  const size_t stride = (size_t)p.c.kv.max_pages_per_seq * PAGE;
#pragma unroll 1
  for (int u = blockIdx.x; u < units[CHAIN_MAX_BATCH]; u += gridDim.x) {
    int lo = 0, hi = p.c.B - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (units[mid] <= u) lo = mid;
      else hi = mid - 1;
    }
    const int b = lo, T = plan.at(b).T, per = max(1, (T + WK_TOKENS - 1) / WK_TOKENS);
    const int kvh = (u - units[b]) / per, chunk = (u - units[b]) - kvh * per, tok0 = chunk * WK_TOKENS + tid * 4;
    const size_t bk = (size_t)b * p.c.Hkv + kvh;
    float* dst = weights + bk * stride;
    float4 s[4][WK_V], w[WK_V], sum[WK_V];
    auto request = [&](int g0) {
#pragma unroll
      for (int g = 0; g < 4; ++g)
#pragma unroll
        for (int v = 0; v < WK_V; ++v) {
          const int tok = tok0 + v * RM_THREADS * 4;
          s[g][v] = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
          if (g0 + g < G && tok < T) s[g][v] = *reinterpret_cast<const float4*>(p.logits + (bk * G + g0 + g) * stride + tok);
        }
    };
    request(0);
#pragma unroll
    for (int v = 0; v < WK_V; ++v) {
      const int tok = tok0 + v * RM_THREADS * 4;
      sum[v] = make_float4(0.f, 0.f, 0.f, 0.f);
      w[v] = tok < T ? *reinterpret_cast<const float4*>(dst + tok) : sum[v];
    }
    const ChainCut cut = chain_cut(p.c, plan, b, kvh);
    __syncthreads();  // the sums of the unit before have been read
    if (cut.cut()) {
      const int g = tid >> 4;
      if (g < (G + 1) / 2 * 2) {  // whole warps
        const float2 ml = chain_merged_ml(p.part, cut, min(g, G - 1));
        if (g < G && chunk == 0) chain_merged_row<HD>(p.part, cut, g, ml, p.out + ((size_t)b * p.Hq + kvh * G + g) * HD);
        if (g < G && (tid & 15) == 0) lse[g] = ml.y == 0.f ? INFINITY : ml.x + log2f(ml.y);
      }
    } else if (tid < G) {
      lse[tid] = p.lse[(size_t)b * p.Hq + kvh * G + tid];
    }
    __syncthreads();
#pragma unroll 1
    for (int g0 = 0; g0 < G; g0 += 4) {
      if (g0) request(g0);
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const float z = g0 + g < G ? lse[g0 + g] : INFINITY;
#pragma unroll
        for (int v = 0; v < WK_V; ++v) {
          sum[v].x += exp2f(s[g][v].x - z);
          sum[v].y += exp2f(s[g][v].y - z);
          sum[v].z += exp2f(s[g][v].z - z);
          sum[v].w += exp2f(s[g][v].w - z);
        }
      }
    }
#pragma unroll
    for (int v = 0; v < WK_V; ++v) {
      const int tok = tok0 + v * RM_THREADS * 4;
      if (tok >= T) continue;
      const float old[4] = {w[v].x, w[v].y, w[v].z, w[v].w}, got[4] = {sum[v].x, sum[v].y, sum[v].z, sum[v].w};
      float now[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) now[i] = tok + i < T - 1 ? decay * old[i] + got[i] : tok + i == T - 1 ? got[i] : old[i];
      *reinterpret_cast<float4*>(dst + tok) = make_float4(now[0], now[1], now[2], now[3]);
    }
  }
}

// ---- host ----------------------------------------------------------------------------------------
static int rows_of_chain(int rows) { return rows <= 4 ? 4 : rows <= 8 ? 8 : 16; }
size_t rows_part_bytes(const sol_shape_t& sh) { return chain_part_bytes(sm_count(), RA_MAX_ROWS, sh.head_dim); }

template <int HD, int ROWS>
static void launch_rows(RowsDev d, const RowsArgs& a, cudaStream_t st) {
  using Z = RaSize<HD, ROWS>;
  CUtensorMap kmap, vmap;
  if (!encode_pool_map(&kmap, a.kv.k_pool, a.shape, a.kv.num_pages) ||
      !encode_pool_map(&vmap, a.kv.v_pool, a.shape, a.kv.num_pages))
    return;
  // fewer CTAs where the caller's space for partial results is short
  const int rows = std::min(ROWS, d.c.max_nodes * d.c.G);
  const int ctas = (int)std::min<size_t>(sm_count(), a.part_bytes / chain_part_bytes(1, rows, HD));
  d.part = chain_parts(a.part, ctas, rows, HD);
  ensure_dynamic_smem(reinterpret_cast<const void*>(&rows_attn_kernel<HD, ROWS>), Z::SMEM);
  SOL_LAUNCH("rows_attn", (rows_attn_kernel<HD, ROWS>), dim3(ctas), dim3(Z::THREADS), Z::SMEM, st, kmap, vmap, d);
  if (a.weights) SOL_LAUNCH("attn_weights", weight_kernel<HD>, dim3(3 * sm_count()), dim3(RM_THREADS), 0, st, d, ctas, a.decay, a.weights);
  else launch_chain_merge(d.c, d.part, d.Hq, HD, ctas, d.out, st);
}

void launch_rows_attention(const RowsArgs& a, cudaStream_t st) {
  const sol_shape_t& sh = a.shape;
  const int rows = rows_of_chain(a.max_nodes * (sh.n_q_heads / sh.n_kv_heads));
  RowsDev d;
  memset(&d, 0, sizeof(d));
  d.c = chain_shape(a, rows, PAGE, RA_MIN_TILES, ra_piece_cost(sh.head_dim));
  d.Hq = sh.n_q_heads;
  d.scale_log2 = 1.4426950408889634f / sqrtf((float)sh.head_dim);
  d.mask = a.mask;
  d.q = static_cast<const uint16_t*>(a.q);
  d.out = static_cast<uint16_t*>(a.out);
  d.logits = a.weights ? a.logits : nullptr;
  d.lse = a.weights ? a.lse : nullptr;
  d.status = a.status;
  if (sh.head_dim == 64) {
    if (rows == 4) launch_rows<64, 4>(d, a, st);
    else if (rows == 8) launch_rows<64, 8>(d, a, st);
    else launch_rows<64, 16>(d, a, st);
  } else {
    if (rows == 4) launch_rows<128, 4>(d, a, st);
    else if (rows == 8) launch_rows<128, 8>(d, a, st);
    else launch_rows<128, 16>(d, a, st);
  }
}

}  // namespace sol
