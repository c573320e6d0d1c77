// The bookkeeping of a speculative step: ancestor masks and depths of drafted trees, the path that the model's own tokens
// accept, and the move of its keys and values to the end of the committed context.
//
// All of it is a few KB per sequence, so latency is what counts: a warp per sequence with two nodes per lane (a tree has at
// most 64 nodes, so a set of nodes is one 64-bit word), and one launch for the rows of up to 64 layers.
#include <cuda_runtime.h>
#include <stdint.h>

#include "sol_common.cuh"
#include "sol_internal.h"

namespace sol {

constexpr int TB_WARPS = 4;  // sequences per CTA

// A node's parent as a node before it, or -1: anything else is a root.
__device__ __forceinline__ int tree_parent(const int32_t* parents, int i, int n) {
  const int p = i < n ? parents[i] : -1;
  return p >= 0 && p < i ? p : -1;
}

// mask_i = {i} + mask of its parent, by pointer jumping: after round r a node's word holds its nearest 2^r ancestors (itself
// among them) and `up` the next one beyond, so six rounds reach 64 steps.
__global__ void __launch_bounds__(TB_WARPS * 32) tree_build_kernel(int B, int max_nodes, const int32_t* __restrict__ n_nodes,
                                                                    const int32_t* __restrict__ parents, uint64_t* __restrict__ mask,
                                                                    int32_t* __restrict__ depth) {
  pdl_wait();
  pdl_trigger();
  const int b = blockIdx.x * TB_WARPS + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (b >= B) return;
  const int n = min(max(n_nodes[b], 0), max_nodes);
  const size_t row = (size_t)b * max_nodes;
  uint64_t m[2];
  int up[2];
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const int i = lane + 32 * x;
    up[x] = tree_parent(parents + row, i, n);
    m[x] = 1ull << i;
  }
#pragma unroll
  for (int r = 0; r < 6; ++r) {
    uint64_t add[2];
    int next[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int from = up[x] & 31;
      const uint64_t m0 = __shfl_sync(0xffffffffu, m[0], from), m1 = __shfl_sync(0xffffffffu, m[1], from);
      const int u0 = __shfl_sync(0xffffffffu, up[0], from), u1 = __shfl_sync(0xffffffffu, up[1], from);
      add[x] = up[x] < 0 ? 0ull : up[x] < 32 ? m0 : m1;
      next[x] = up[x] < 0 ? -1 : up[x] < 32 ? u0 : u1;
    }
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      m[x] |= add[x];
      up[x] = next[x];
    }
  }
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const int i = lane + 32 * x;
    if (i >= n) continue;
    mask[row + i] = m[x];
    if (depth) depth[row + i] = __popcll(m[x]) - 1;
  }
}

// From node 0 on: the first child whose drafted token is the one the model puts after the current node, until there is none.
__global__ void __launch_bounds__(TB_WARPS * 32) tree_accept_kernel(int B, int max_nodes, const int32_t* __restrict__ n_nodes,
                                                                     const int32_t* __restrict__ parents,
                                                                     const int32_t* __restrict__ draft,
                                                                     const int32_t* __restrict__ target, int32_t* __restrict__ path,
                                                                     int32_t* __restrict__ path_len, int32_t* __restrict__ next_token) {
  pdl_wait();
  pdl_trigger();
  const int b = blockIdx.x * TB_WARPS + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (b >= B) return;
  const int n = min(max(n_nodes[b], 0), max_nodes);
  const size_t row = (size_t)b * max_nodes;
  int up[2], tok[2], want[2];
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const int i = lane + 32 * x;
    up[x] = tree_parent(parents + row, i, n);
    tok[x] = i < n ? draft[row + i] : 0;
    want[x] = i < n ? target[row + i] : 0;
  }
  int count = 0, cur = 0, next = -1;
#pragma unroll 1
  while (count < n) {  // a node comes after its parent, so every turn goes to a later node
    if (lane == 0) path[row + count] = cur;
    ++count;
    const int w0 = __shfl_sync(0xffffffffu, want[0], cur & 31), w1 = __shfl_sync(0xffffffffu, want[1], cur & 31);
    next = cur < 32 ? w0 : w1;
    const uint32_t lo = __ballot_sync(0xffffffffu, up[0] == cur && tok[0] == next);
    const uint32_t hi = __ballot_sync(0xffffffffu, up[1] == cur && tok[1] == next);
    if (!(lo | hi)) break;
    cur = lo ? __ffs(lo) - 1 : 31 + __ffs(hi);
  }
  if (lane == 0) {
    path_len[b] = count;
    if (next_token) next_token[b] = next;
  }
}

// ---- commit -------------------------------------------------------------------------------------
struct CommitDev {
  sol_kv_t kv[COMMIT_LAYERS];
  int Hkv, hd, max_nodes;
  int quest;  // tokens of a Quest page; 0: no extrema
  const int32_t* n_nodes;
  const int32_t* path;
  const int32_t* path_len;
  int32_t* new_lens;  // optional; lengths by the first layer
  int* status;
};

// A CTA moves the accepted rows of a (layer, sequence, group of heads): thread = (head, K or V, 16-byte piece of a row), which
// takes its piece of every row in the path's order, eight in flight.  In place: row j of the path goes to slot j, the path
// ascends, so slot j is no later row's source (path[j'] >= j' > j), and no other thread touches the piece.  With Quest pages the
// thread then takes its eight dimensions' extrema of every block that drafted tokens lay in, over the tokens that are left: what
// a decode step renews is the newest token's block alone.  (16 layers of 64 sequences,
// 8 of 64 nodes accepted: 16 us; with blocks of 4 tokens 20.)
constexpr int COMMIT_THREADS = 128;
__global__ void __launch_bounds__(COMMIT_THREADS) tree_commit_kernel(const CommitDev p) {
  __shared__ int s_path[64], s_count;
  const int layer = blockIdx.z, b = blockIdx.y, tid = threadIdx.x;
  const sol_kv_t& kv = p.kv[layer];
  pdl_wait();
  pdl_trigger();
  // counts out of range count as the nearest in range, as they do in the attention
  const int room = kv.max_pages_per_seq * PAGE;
  const int len = kv.seq_lens[b], nodes = p.n_nodes[b], steps = p.path_len[b];
  const int T = min(max(len, 0), room), n = min(min(max(nodes, 0), p.max_nodes), T);
  int count = min(max(steps, 0), n);
  const bool fits = T == len && n == nodes && count == steps;
  if (tid < 32) {  // the path as far as it ascends within the tree
    bool ok[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int j = tid + 32 * x;
      const int at = j < count ? p.path[(size_t)b * p.max_nodes + j] : 0;
      const int before = j < count && j > 0 ? p.path[(size_t)b * p.max_nodes + j - 1] : -1;
      ok[x] = j < count && at > before && at >= 0 && at < n;
      s_path[j] = at;
    }
    const uint32_t lo = __ballot_sync(0xffffffffu, ok[0]), hi = __ballot_sync(0xffffffffu, ok[1]);
    const uint64_t good = (uint64_t)lo | ((uint64_t)hi << 32);
    if (tid == 0) {
      const int run = ~good ? __ffsll((long long)~good) - 1 : 64;
      if (!fits || run < count) atomicOr(p.status + ST_ERR, ERR_BAD_ACTION);
      s_count = min(run, count);
      if (layer == 0 && blockIdx.x == 0 && p.new_lens) p.new_lens[b] = T - n + s_count;
    }
  }
  __syncthreads();
  count = s_count;
  const int ppr = p.hd / 8, first = T - n;
  const int i = blockIdx.x * COMMIT_THREADS + tid;
  if (i >= p.Hkv * 2 * ppr) return;
  const int piece = i % ppr, kvh = i / ppr % p.Hkv;
  uint4* pool = static_cast<uint4*>(i / (ppr * p.Hkv) ? kv.v_pool : kv.k_pool);
  const int32_t* table = kv.page_table + (size_t)b * kv.max_pages_per_seq;
  auto row = [&](int slot) -> uint4* {
    const int page = table[slot / PAGE];
    if (page < 0 || page >= kv.num_pages) {
      atomicOr(p.status + ST_ERR, ERR_BAD_PAGE);
      return nullptr;
    }
    return pool + (((size_t)page * p.Hkv + kvh) * PAGE + slot % PAGE) * ppr + piece;
  };
#pragma unroll 1
  for (int j0 = 0; j0 < count; j0 += 8) {
    uint4 v[8];
    uint4* dst[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int j = j0 + u;
      dst[u] = nullptr;
      if (j >= count || s_path[j] == j) continue;  // already there
      const uint4* src = row(first + s_path[j]);
      uint4* to = row(first + j);
      if (src && to) {
        v[u] = *src;
        dst[u] = to;
      }
    }
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (dst[u]) *dst[u] = v[u];
  }
  if (p.quest == 0 || kv.quest_meta == nullptr || n == 0 || i >= p.Hkv * ppr) return;
  const int end = first + count;
#pragma unroll 1
  for (int t0 = first / p.quest * p.quest; t0 < end; t0 += p.quest) {
    const uint4* rows = row(t0);
    if (rows == nullptr) continue;
    float top[8], low[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      top[e] = -INFINITY;
      low[e] = INFINITY;
    }
#pragma unroll 4
    for (int j = 0; j < min(p.quest, end - t0); ++j) {
      const uint4 v = rows[(size_t)j * ppr];
      const uint32_t x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float k = e & 1 ? bf16_hi(x[e >> 1]) : bf16_lo(x[e >> 1]);
        top[e] = fmaxf(top[e], k);
        low[e] = fminf(low[e], k);
      }
    }
    const int page = table[t0 / PAGE];
    uint32_t* meta = static_cast<uint32_t*>(kv.quest_meta) +
                     ((((size_t)page * p.Hkv + kvh) * (PAGE / p.quest)) + t0 % PAGE / p.quest) * p.hd + piece * 4;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      meta[e] = pack_bf16(top[2 * e], top[2 * e + 1]);
      meta[p.hd / 2 + e] = pack_bf16(-low[2 * e], -low[2 * e + 1]);
    }
  }
}

void launch_tree_build(int B, int max_nodes, const int32_t* n_nodes, const int32_t* parents, uint64_t* mask, int32_t* depth,
                       cudaStream_t st) {
  SOL_LAUNCH("tree_build", tree_build_kernel, dim3((B + TB_WARPS - 1) / TB_WARPS), dim3(TB_WARPS * 32), 0, st, B, max_nodes,
             n_nodes, parents, mask, depth);
}

void launch_tree_accept(int B, int max_nodes, const int32_t* n_nodes, const int32_t* parents, const int32_t* draft,
                        const int32_t* target, int32_t* path, int32_t* path_len, int32_t* next_token, cudaStream_t st) {
  SOL_LAUNCH("tree_accept", tree_accept_kernel, dim3((B + TB_WARPS - 1) / TB_WARPS), dim3(TB_WARPS * 32), 0, st, B, max_nodes,
             n_nodes, parents, draft, target, path, path_len, next_token);
}

void launch_tree_commit(const sol_shape_t& sh, int n_layers, const sol_kv_t* kvs, const sol_tree_t& tree, int B,
                        const int32_t* path, const int32_t* path_len, int32_t* new_lens, int* status, cudaStream_t st) {
  const int pieces = sh.n_kv_heads * 2 * (sh.head_dim / 8);
  for (int l0 = 0; l0 < n_layers; l0 += COMMIT_LAYERS) {
    const int nl = n_layers - l0 < COMMIT_LAYERS ? n_layers - l0 : COMMIT_LAYERS;
    CommitDev d;
    memset(&d, 0, sizeof(d));
    for (int l = 0; l < nl; ++l) d.kv[l] = kvs[l0 + l];
    d.Hkv = sh.n_kv_heads;
    d.hd = sh.head_dim;
    d.max_nodes = tree.max_nodes;
    d.quest = sh.token_select == SOL_SELECT_QUEST_PAGES ? sh.quest_page_size : 0;
    d.n_nodes = tree.n_nodes;
    d.path = path;
    d.path_len = path_len;
    d.new_lens = l0 == 0 ? new_lens : nullptr;
    d.status = status;
    SOL_LAUNCH("tree_commit", tree_commit_kernel, dim3((pieces + COMMIT_THREADS - 1) / COMMIT_THREADS, B, nl), dim3(COMMIT_THREADS),
               0, st, d);
  }
}

}  // namespace sol
