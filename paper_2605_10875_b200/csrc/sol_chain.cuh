// Work sharing of the dense attention kernels over the paged cache (trees of drafted tokens, decode steps that keep the
// attention weights).
//
// A chain is what one softmax runs along: a (sequence, kv-head, block of query rows) over the sequence's tokens, a tile of one
// or two cache pages at a time.  The tiles of all chains, one chain after the other, form one line, of which every CTA takes a
// run.  A run that ends inside a chain leaves a partial result; a second kernel merges the pieces of chains that were cut.
// A chain has piece_cost places on the line ahead of its tiles, as many tiles as beginning and ending a piece is worth, so that
// runs of many short chains are not the longest (the attention of 128 ragged decode steps, as it then was: 394 us without, 330
// with).  Two ways to cut, of which every CTA works out for itself, from the lengths (at most 128), which one is the better:
//   equal runs       whatever the lengths are.  A run covers the end of one chain, some whole chains and the beginning of another
//   CTAs per chain   in proportion to its tiles, one at least: every CTA has one piece.  Taken if none is much longer than an equal
//                    run, where a CTA has the end of one chain and the beginning of another
#pragma once
#include "sol_common.cuh"
#include "sol_internal.h"

namespace sol {

constexpr int CHAIN_MAX_BATCH = 128;

// What the kernels know of a sequence: T tokens in the cache, the last n of them drafted.
struct ChainSeq {
  int T, n;
};
// n_nodes == nullptr: a decode step, one query token per sequence, which is the newest token (an empty sequence has it too: its
// output is zero).
__device__ __forceinline__ ChainSeq chain_seq(const sol_kv_t& kv, const int32_t* n_nodes, int max_nodes, int b, int* status) {
  ChainSeq s;
  const int len = kv.seq_lens[b], room = kv.max_pages_per_seq * PAGE;
  s.T = min(max(len, 0), room);
  s.n = 1;
  if (n_nodes) {
    const int n = n_nodes[b];
    s.n = min(min(max(n, 0), max_nodes), s.T);
    if (status && (s.n != n || s.T != len)) atomicOr(status + ST_ERR, ERR_BAD_ACTION);
  }
  return s;
}

struct ChainShape {
  sol_kv_t kv;
  int B, Hkv, G, max_nodes;
  const int32_t* n_nodes;  // nullptr: decode steps
  int block_rows;          // query rows of a chain
  int tile;                // tokens of a tile: PAGE or 2 PAGE
  int min_tiles;           // tiles of a CTA's run at least
  int piece_cost;          // tiles that beginning and ending a piece is worth
};

// The line of tiles.
struct ChainPlan {
  int cum[CHAIN_MAX_BATCH + 1];    // places of the sequences before b
  int first[CHAIN_MAX_BATCH + 1];  // CTAs per chain: CTAs of the sequences before b
  uint32_t seq[CHAIN_MAX_BATCH];   // T << 8 | n
  int wsum[8];
  int run;                         // equal runs: places of each; 0: CTAs per chain
  __device__ __forceinline__ ChainSeq at(int b) const {
    ChainSeq s;
    s.T = (int)(seq[b] >> 8);
    s.n = (int)(seq[b] & 255u);
    return s;
  }
};

inline ChainShape chain_shape(const RowsArgs& a, int block_rows, int tile, int min_tiles, int piece_cost) {
  ChainShape c;
  c.kv = a.kv;
  c.B = a.B;
  c.Hkv = a.shape.n_kv_heads;
  c.G = a.shape.n_q_heads / a.shape.n_kv_heads;
  c.max_nodes = a.max_nodes;
  c.n_nodes = a.n_nodes;
  c.block_rows = block_rows;
  c.tile = tile;
  c.min_tiles = min_tiles;
  c.piece_cost = piece_cost;
  return c;
}

__device__ __forceinline__ int chain_tiles(const ChainShape& c, const ChainSeq& s) {
  return max(1, (s.T + c.tile - 1) / (c.tile == PAGE ? PAGE : 2 * PAGE));
}
__device__ __forceinline__ int chain_blocks(const ChainShape& c, const ChainSeq& s) { return (s.n * c.G + c.block_rows - 1) / c.block_rows; }

// For a kernel of `ctas` CTAs, by a whole CTA (128 threads at least); ends with a barrier.
__device__ __forceinline__ void chain_plan(const ChainShape& c, ChainPlan& p, int ctas, int* status) {
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  auto scan = [&](int v, int* out) {  // out[b + 1] = v of sequences 0 .. b
    if (tid < CHAIN_MAX_BATCH) {
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += x;
      }
      if (lane == 31) p.wsum[warp] = v;
    }
    __syncthreads();
    if (tid < CHAIN_MAX_BATCH) {
      for (int w = 0; w < warp; ++w) v += p.wsum[w];
      out[tid + 1] = v;
      if (tid == 0) out[0] = 0;
    }
    __syncthreads();
  };
  ChainSeq s;
  s.T = s.n = 0;
  if (tid < c.B) s = chain_seq(c.kv, c.n_nodes, c.max_nodes, tid, status);
  if (tid < CHAIN_MAX_BATCH) p.seq[tid] = (uint32_t)s.T << 8 | (uint32_t)s.n;
  const int chains = s.n > 0 ? chain_blocks(c, s) * c.Hkv : 0, tiles = chain_tiles(c, s);
  const int places = tiles + c.piece_cost;
  scan(places * chains, p.cum);
  const int total = p.cum[c.B], run = max(c.min_tiles, (total + ctas - 1) / ctas);
  const int share = max(1, (int)((long long)places * ctas / max(total, 1)));  // CTAs of each of the sequence's chains
  const int give = min(share, max(1, tiles / c.min_tiles));
  scan(give * chains, p.first);
  const int worst = __syncthreads_or(chains > 0 && (tiles + give - 1) / give > run + c.piece_cost / 2);
  if (tid == 0) p.run = worst || p.first[c.B] > ctas ? run : 0;
  __syncthreads();
}

// The sequence that holds place u of the line.
__device__ __forceinline__ int chain_find(const ChainShape& c, const ChainPlan& p, int u) {
  int lo = 0, hi = c.B - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (p.cum[mid] <= u) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// The run [u0, u1) of a CTA, empty or with a tile at its end.
__device__ __forceinline__ int2 chain_range(const ChainShape& c, const ChainPlan& p, int cta) {
  const int total = p.cum[c.B];
  if (p.run) {
    const int u0 = (int)min((long long)cta * p.run, (long long)total);
    int u1 = min(total, u0 + p.run);
    if (u0 < u1) {  // what it holds of a chain's places ahead of the tiles, at its end, is nothing
      const int b = chain_find(c, p, u1 - 1), places = chain_tiles(c, p.at(b)) + c.piece_cost, at = (u1 - p.cum[b]) % places;
      if (at && at <= c.piece_cost) u1 -= at;
    }
    return make_int2(u0, max(u0, u1));
  }
  if (cta >= p.first[c.B]) return make_int2(total, total);
  int lo = 0, hi = c.B - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (p.first[mid] <= cta) lo = mid;
    else hi = mid - 1;
  }
  const ChainSeq s = p.at(lo);
  const int tiles = chain_tiles(c, s), each = (p.first[lo + 1] - p.first[lo]) / (chain_blocks(c, s) * c.Hkv);
  const int local = cta - p.first[lo], chain = local / each, i = local - chain * each;
  const int base = p.cum[lo] + chain * (tiles + c.piece_cost) + c.piece_cost;
  return make_int2(base + (int)((long long)tiles * i / each), base + (int)((long long)tiles * (i + 1) / each));
}

// A run's next piece: tiles [tile0, tile1) of a chain.
struct ChainPiece {
  int b, kvh, block;
  int tile0, tile1, tiles;  // tiles: of the whole chain
  int next;                 // place where the run goes on
  ChainSeq seq;
  __device__ __forceinline__ bool whole() const { return tile0 == 0 && tile1 == tiles; }
};
__device__ __forceinline__ ChainPiece chain_piece(const ChainShape& c, const ChainPlan& p, int u, int end) {
  ChainPiece r;
  r.b = chain_find(c, p, u);
  r.seq = p.at(r.b);
  r.tiles = chain_tiles(c, r.seq);
  const int places = r.tiles + c.piece_cost, local = u - p.cum[r.b], chain = local / places, blocks = chain_blocks(c, r.seq);
  const int at = local - chain * places, to = min(places, at + end - u);
  r.tile0 = max(0, at - c.piece_cost);
  r.tile1 = to - c.piece_cost;
  r.next = u + to - at;
  r.kvh = chain / blocks;
  r.block = chain - r.kvh * blocks;
  return r;
}

// Where the pieces of a cut chain lie: CTAs first .. last, of which the first one's piece is in its slot 1 unless the chain
// begins with its run; the others' are in slot 0.
struct ChainCut {
  int first, last, first_slot;  // CTAs, and the first piece's slot
  __device__ __forceinline__ bool cut() const { return last > first; }
  __device__ __forceinline__ int slot(int i) const { return i == 0 ? first_slot : 2 * (first + i); }  // of piece i
  __device__ __forceinline__ int pieces() const { return last - first + 1; }
};
__device__ __forceinline__ ChainCut chain_cut(const ChainShape& c, const ChainPlan& p, int b, int chain) {
  const ChainSeq s = p.at(b);
  ChainCut r;
  if (p.run) {
    const int tiles = chain_tiles(c, s), base = p.cum[b] + chain * (tiles + c.piece_cost), u0 = base + c.piece_cost;
    r.first = u0 / p.run;
    r.last = (u0 + tiles - 1) / p.run;
    r.first_slot = 2 * r.first + (base > r.first * p.run ? 1 : 0);
  } else {
    const int each = (p.first[b + 1] - p.first[b]) / (chain_blocks(c, s) * c.Hkv);
    r.first = p.first[b] + chain * each;
    r.last = r.first + each - 1;
    r.first_slot = 2 * r.first;
  }
  return r;
}

// ---- partial results of cut chains ----
// A chain that begins in a CTA's run and goes on in the next: for the kernel that merges its pieces.
struct ChainDesc {
  int pieces;  // 0: there is none
  int b, kvh, block, rows, first_slot;
};
// Per slot and row of a chain: HD weighted sums, and (maximum in the base-2 domain, sum of the weights).
struct ChainParts {
  float* sums;      // [slots][rows][HD]
  float2* ml;       // [slots][rows]
  ChainDesc* desc;  // [ctas]
  int rows;
};
inline size_t chain_part_bytes(int ctas, int rows, int hd) {
  return (size_t)2 * ctas * rows * (hd * 4 + 8) + ctas * sizeof(ChainDesc);
}
inline ChainParts chain_parts(void* base, int ctas, int rows, int hd) {
  ChainParts p;
  p.sums = static_cast<float*>(base);
  p.ml = reinterpret_cast<float2*>(p.sums + (size_t)2 * ctas * rows * hd);
  p.desc = reinterpret_cast<ChainDesc*>(p.ml + (size_t)2 * ctas * rows);
  p.rows = rows;
  return p;
}

// What CTA `cta` with run [u0, u1) of the line leaves to be merged, by one thread.
__device__ __forceinline__ void chain_describe(const ChainShape& c, const ChainPlan& p, int cta, int u0, int u1, ChainDesc* out) {
  ChainDesc d;
  d.pieces = d.b = d.kvh = d.block = d.rows = d.first_slot = 0;
  if (u0 < u1) {
    const ChainPiece last = chain_piece(c, p, u1 - 1, u1);
    const int start = u1 - 1 - last.tile0;
    if (last.tile0 + 1 < last.tiles && start >= u0) {
      const ChainCut cut = chain_cut(c, p, last.b, last.kvh * chain_blocks(c, last.seq) + last.block);
      d.pieces = cut.pieces();
      d.first_slot = cut.first_slot;
      d.b = last.b;
      d.kvh = last.kvh;
      d.block = last.block;
      d.rows = min(c.block_rows, last.seq.n * c.G - last.block * c.block_rows);
    }
  }
  out[cta] = d;
}

// ---- sums that are no numbers ----
// The value of a token that is infinite makes its column of every row that sees it infinite, or NaN where it meets NaN or the other
// infinity.  The products do not keep to that: a weight that is zero in one of its parts, or in a copy of the row that leaves the
// token to another copy, makes NaN of it.  So where a sum of numbers' weights is no number, the column is made out again from what the
// values are.  Nothing but such sums pays for it.
enum : int { VALUE_PLUS = 1, VALUE_MINUS = 2, VALUE_NAN = 4 };
__device__ __forceinline__ int value_flag(uint32_t bf16) {
  return (bf16 & 0x7f80u) != 0x7f80u ? 0 : bf16 & 0x7fu ? VALUE_NAN : bf16 & 0x8000u ? VALUE_MINUS : VALUE_PLUS;
}
__device__ __forceinline__ float flagged_sum(int flags, float was) {
  return flags == 0 ? was : flags == VALUE_PLUS ? INFINITY : flags == VALUE_MINUS ? -INFINITY : NAN;
}
struct ValueRows {  // a (sequence, kv-head)'s
  const uint16_t* pool;
  const int32_t* table;
  int num_pages, Hkv, kvh;
  template <int HD>
  __device__ __forceinline__ const uint16_t* row(int tok) const {  // nullptr: its page is out of range
    const int page = table[tok / PAGE];
    return (unsigned)page < (unsigned)num_pages ? pool + (((size_t)page * Hkv + kvh) * PAGE + tok % PAGE) * HD : nullptr;
  }
};
__device__ __forceinline__ ValueRows value_rows(const sol_kv_t& kv, int Hkv, int b, int kvh) {
  ValueRows v;
  v.pool = static_cast<const uint16_t*>(kv.v_pool);
  v.table = kv.page_table + (size_t)b * kv.max_pages_per_seq;
  v.num_pages = kv.num_pages;
  v.Hkv = Hkv;
  v.kvh = kvh;
  return v;
}
// What tokens [t0, t1) hold: a word of flags per column, cleared before, by thread `i` of n (a multiple of HD / 8).
template <int HD>
__device__ __noinline__ void value_flags(const ValueRows v, int t0, int t1, int i, int n, int* flags) {
  constexpr int PPR = HD / 8;
  uint32_t found = 0;  // three bits per column
#pragma unroll 4
  for (int t = t0 + i / PPR; t < t1; t += n / PPR) {
    const uint16_t* row = v.row<HD>(t);
    if (row == nullptr) continue;
    const uint4 x = *reinterpret_cast<const uint4*>(row + i % PPR * 8);
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int e = 0; e < 8; ++e) found |= (uint32_t)value_flag(e & 1 ? w[e >> 1] >> 16 : w[e >> 1] & 0xffffu) << (3 * e);
  }
  for (int e = 0; e < 8; ++e)
    if ((found >> (3 * e)) & 7u) atomicOr(flags + i % PPR * 8 + e, (int)((found >> (3 * e)) & 7u));
}
// ... and of the nodes among [t0, t1) that a row sees, in one column.  C: slot of node 0.
template <int HD>
__device__ __forceinline__ int node_flags(const ValueRows& v, int t0, int t1, int C, uint64_t nodes, int col) {
  int f = 0;
  for (; nodes; nodes &= nodes - 1) {
    const int t = C + __ffsll((long long)nodes) - 1;
    const uint16_t* row = t >= t0 && t < t1 ? v.row<HD>(t) : nullptr;
    if (row) f |= value_flag(row[col]);
  }
  return f;
}

// A row's merged maximum and 1 / (sum of the weights) (0 for a row that sees nothing), by the 16 lanes of half a warp.
__device__ __forceinline__ float2 chain_merged_ml(const ChainParts& p, const ChainCut& cut, int row) {
  const int sub = threadIdx.x & 15, np = cut.pieces();
  float m = -INFINITY;
  for (int i = sub; i < np; i += 16) m = fmaxf(m, p.ml[(size_t)cut.slot(i) * p.rows + row].x);
#pragma unroll
  for (int o = 8; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  const float base = m == -INFINITY ? 0.f : m;
  float l = 0.f;
  for (int i = sub; i < np; i += 16) {
    const float2 v = p.ml[(size_t)cut.slot(i) * p.rows + row];
    l += v.y * exp2f(v.x - base);
  }
#pragma unroll
  for (int o = 8; o; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
  return make_float2(base, l);
}

// The merged row, HD / 16 of its columns per lane, as bf16 to dst (the row's first element).
template <int HD>
__device__ __forceinline__ void chain_merged_row(const ChainParts& p, const ChainCut& cut, int row, float2 ml, uint16_t* dst) {
  constexpr int V = HD / 64;  // float4 per lane
  const int sub = threadIdx.x & 15, np = cut.pieces();
  const float inv = ml.y == 0.f ? 0.f : 1.0f / ml.y;
  float4 a[V];
#pragma unroll
  for (int x = 0; x < V; ++x) a[x] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int i = 0; i < np; ++i) {
    const size_t at = (size_t)cut.slot(i) * p.rows + row;
    const float f = fmaxf(exp2f(p.ml[at].x - ml.x), 1e-37f) * inv;  // above 0: sums may be infinite
#pragma unroll
    for (int x = 0; x < V; ++x) {
      const float4 v = *reinterpret_cast<const float4*>(p.sums + at * HD + x * 64 + sub * 4);
      a[x].x += f * v.x;
      a[x].y += f * v.y;
      a[x].z += f * v.z;
      a[x].w += f * v.w;
    }
  }
#pragma unroll
  for (int x = 0; x < V; ++x)
    *reinterpret_cast<uint2*>(dst + x * 64 + sub * 4) = make_uint2(pack_bf16(a[x].x, a[x].y), pack_bf16(a[x].z, a[x].w));
}

// Merges the cut chains of an attention kernel of `ctas` CTAs (sol_rows_attn.cu).
void launch_chain_merge(const ChainShape& c, const ChainParts& part, int Hq, int hd, int ctas, uint16_t* out, cudaStream_t st);

}  // namespace sol
