"""Plain fp64 oracle of what a serving loop does around the decode step: attention of drafted trees, the bookkeeping of a
speculative step, decode attention that keeps its weights, and eviction by them.

TEST INFRASTRUCTURE (same status as sol_oracle.py): literal NumPy, one sequence and one head at a time, no code shared with the
CUDA path.  bf16 tensors are uint16 bit patterns; caches are sol_oracle.PagedKV.
"""
from __future__ import annotations

import numpy as np

from oracle import sol_oracle as O


def _rows(pool, table_row, T, kvh):
    """Tokens 0..T-1 of one kv-head of one sequence, float64 [T][hd]."""
    return O.cache_rows(pool, table_row, T, kvh) if T else np.zeros((0, pool.shape[3]))


def ancestor_masks(parents):
    """Per node the set of its ancestors and itself, as an int with bit j for node j; depth of a root is 0."""
    masks, depths = [], []
    for i, p in enumerate(parents):
        p = int(p) if 0 <= int(p) < i else -1
        masks.append((1 << i) | (masks[p] if p >= 0 else 0))
        depths.append(depths[p] + 1 if p >= 0 else 0)
    return masks, depths


def seen_by_node(T: int, n: int, mask: int) -> np.ndarray:
    """Which of the T cached tokens a node attends to: the context before the n nodes, and the nodes of its mask."""
    return np.array([t < T - n or bool((mask >> (t - (T - n))) & 1) for t in range(T)], bool)


def _attend(q, K, V, seen):
    """Output, softmax weights, and sum of p |v| (what errors of the weights are multiplied with) of one query."""
    out, p, mass = np.zeros(K.shape[1]), np.zeros(len(K)), np.zeros(K.shape[1])
    at = np.flatnonzero(seen)
    if len(at):
        s = K[at] @ q / np.sqrt(K.shape[1])
        e = np.exp(s - s.max())
        p[at] = e / e.sum()
        out, mass = p[at] @ V[at], p[at] @ np.abs(V[at])
    return out, p, mass


def score_error(q, K, seen):
    """Bound of a float32 tensor-core score's error: 16 u sum |q_d k_d| / sqrt(hd), and two roundings of the scaling."""
    at = np.flatnonzero(seen)
    if not len(at):
        return 0.0
    return float((np.abs(K[at]) @ np.abs(q)).max() / np.sqrt(K.shape[1])) * 20 * 2.0 ** -24


def tree_attn(shape: O.Shape, q_bf16, kv: O.PagedKV, n_nodes, masks):
    """q [B][N][Hq][hd].  Returns (out, mass, dscore): outputs, sum of p |v|, bound of the scores' error; zero rows behind a tree."""
    q = O.bf16_to_f64(q_bf16)
    out, mass, err = np.zeros(q.shape), np.zeros(q.shape), np.zeros(q.shape[:3])
    G = shape.n_q_heads // shape.n_kv_heads
    for b, n in enumerate(n_nodes):
        T = int(kv.seq_lens[b])
        for kvh in range(shape.n_kv_heads):
            K = _rows(kv.k_pool, kv.page_table[b], T, kvh)
            V = _rows(kv.v_pool, kv.page_table[b], T, kvh)
            for i in range(int(n)):
                seen = seen_by_node(T, int(n), int(masks[b][i]))
                for h in range(kvh * G, kvh * G + G):
                    out[b, i, h], _, mass[b, i, h] = _attend(q[b, i, h], K, V, seen)
                    err[b, i, h] = score_error(q[b, i, h], K, seen)
    return out, mass, err


def tree_accept(parents, draft, target):
    """The accepted path of one tree (lists of its nodes), and the token after it."""
    n, path = len(parents), []
    if not n:
        return path, -1
    cur = 0
    while True:
        path.append(cur)
        hits = [i for i in range(cur + 1, n) if parents[i] == cur and draft[i] == target[cur]]
        if not hits:
            return path, int(target[cur])
        cur = hits[0]


def tree_commit(kv: O.PagedKV, n_nodes, paths):
    """Moves the rows of every path in place; returns the new lengths."""
    lens = []
    for b, (n, path) in enumerate(zip(n_nodes, paths)):
        first = int(kv.seq_lens[b]) - int(n)
        for pool in (kv.k_pool, kv.v_pool):
            rows = [pool[kv.page_table[b][(first + i) // 64], :, (first + i) % 64].copy() for i in path]
            for j, r in enumerate(rows):
                pool[kv.page_table[b][(first + j) // 64], :, (first + j) % 64] = r
        lens.append(first + len(path))
    return lens


def weighted_decode_attn(shape: O.Shape, q_bf16, kv: O.PagedKV, decay: float, weights):
    """q [B][Hq][hd]; weights [B][Hkv][stride] float64.  Returns (out, mass, dscore, new weights, this step's sums)."""
    q, new = O.bf16_to_f64(q_bf16), np.array(weights, np.float64)
    got = np.zeros_like(new)
    out, mass, err = np.zeros(q.shape), np.zeros(q.shape), np.zeros(q.shape[:2])
    G = shape.n_q_heads // shape.n_kv_heads
    for b in range(len(q)):
        T = int(kv.seq_lens[b])
        for kvh in range(shape.n_kv_heads):
            K = _rows(kv.k_pool, kv.page_table[b], T, kvh)
            V = _rows(kv.v_pool, kv.page_table[b], T, kvh)
            for h in range(kvh * G, kvh * G + G):
                out[b, h], p, mass[b, h] = _attend(q[b, h], K, V, np.ones(T, bool))
                err[b, h] = score_error(q[b, h], K, np.ones(T, bool))
                got[b, kvh, :T] += p
            if T:
                new[b, kvh, :T] *= decay
                new[b, kvh, T - 1] = 0.0
                new[b, kvh, :T] += got[b, kvh, :T]
    return out, mass, err, new, got


def evict_keep(weights_row, T: int, budget: int, n_sink: int, n_window: int) -> np.ndarray:
    """Old slots that stay, ascending: forced ones, then the largest weights, ties to the lower index, NaN below everything."""
    sinks = min(n_sink, T)
    window = min(n_window, T - sinks)
    k = min(T, max(int(budget), sinks + window))
    forced = set(range(sinks)) | set(range(T - window, T))

    def rank(i):
        w = float(weights_row[i])
        return (0, 0.0, i) if i in forced else (2, 0.0, i) if w != w else (1, -w, i)

    return np.array(sorted(sorted(range(T), key=rank)[:k]), np.int64)


def kv_evict(shape: O.Shape, kv: O.PagedKV, budgets, weights, n_sink: int, n_window: int):
    """Per sequence and head the kept slots, and the rotated keys and the values (float64) that follow them."""
    kept, keys, values = [], [], []
    for b in range(len(budgets)):
        T = int(kv.seq_lens[b])
        kept.append([]), keys.append([]), values.append([])
        for kvh in range(shape.n_kv_heads):
            idx = evict_keep(weights[b][kvh], T, budgets[b], n_sink, n_window)
            K = _rows(kv.k_pool, kv.page_table[b], T, kvh)
            V = _rows(kv.v_pool, kv.page_table[b], T, kvh)
            moved = [O.rope_rotate(K[i], j - int(i), shape.rope_theta) if shape.rope_theta else K[i] for j, i in enumerate(idx)]
            kept[-1].append(idx)
            keys[-1].append(np.array(moved).reshape(len(idx), kv.k_pool.shape[3]))
            values[-1].append(V[idx])
    return kept, keys, values
