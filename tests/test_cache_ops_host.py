"""The tree and cache-budget calls without a GPU: refusals before any launch, and pins of their oracle."""
import itertools

import numpy as np
import pytest
import torch

from oracle import cache_ops as OC
from oracle import sol_oracle as O
from paper_2605_10875_b200 import binding as sol
from paper_2605_10875_b200 import synth

FAKE = 0x1000  # a non-null address that must never be dereferenced on these paths
BIG = 1 << 40


def _shape(**over):
    kw = dict(d_model=256, n_q_heads=4, n_kv_heads=2, head_dim=64, d_ff=1024)
    kw.update(over)
    return sol.make_shape(**kw)


def _kv(**over):
    kw = dict(k_pool=FAKE, v_pool=FAKE, page_table=FAKE, seq_lens=FAKE, max_pages_per_seq=8, num_pages=32)
    kw.update(over)
    return sol.make_kv(**kw)


BAD_SHAPES = [dict(head_dim=96), dict(n_q_heads=18, n_kv_heads=2, head_dim=128), dict(d_model=300), dict(n_sink=-1)]


def _refusals(call, ok=sol.SOL_OK):
    before = sol.launch_count()
    for want, kw in call:
        assert kw() == want
    assert sol.launch_count() == before


def test_tree_build_and_accept_refuse():
    b = lambda B=2, N=4, n=FAKE, p=FAKE, m=FAKE: (lambda: sol.tree_build(B, N, n, p, m, None, check=False))  # noqa: E731
    a = lambda B=2, N=4, x=FAKE, y=FAKE, z=FAKE: (lambda: sol.tree_accept(B, N, FAKE, FAKE, x, y, z, FAKE, None, check=False))  # noqa: E731
    I, U = sol.SOL_ERR_INVALID_ARG, sol.SOL_ERR_UNSUPPORTED
    _refusals([(I, b(B=-1)), (I, b(N=0)), (U, b(N=65)), (I, b(n=None)), (I, b(p=None)), (I, b(m=None)), (sol.SOL_OK, b(B=0)),
               (I, a(B=-1)), (I, a(N=0)), (U, a(N=65)), (I, a(x=None)), (I, a(y=None)), (I, a(z=None)), (sol.SOL_OK, a(B=0))])


def test_tree_attn_refuses():
    def call(shape=None, q=FAKE, kv=None, N=8, n=FAKE, m=FAKE, B=2, out=FAKE, ws=FAKE, size=BIG):
        return lambda: sol.tree_attn(shape or _shape(), q, kv or _kv(), sol.make_tree(N, n, m), B, out, ws, size, check=False)

    I, U = sol.SOL_ERR_INVALID_ARG, sol.SOL_ERR_UNSUPPORTED
    need = sol.tree_workspace_bytes(_shape(), 2, 8, 8)
    assert need > 256
    _refusals([(I, call(q=None)), (I, call(n=None)), (I, call(m=None)), (I, call(out=None)), (I, call(ws=None)), (I, call(B=-1)),
               (I, call(N=0)), (U, call(N=65)), (U, call(B=129)), (I, call(kv=_kv(k_pool=None))), (I, call(kv=_kv(num_pages=0))),
               (I, call(q=FAKE + 2)), (I, call(out=FAKE + 8)), (I, call(kv=_kv(v_pool=FAKE + 8))), (I, call(ws=FAKE + 4)),
               (U, call(kv=_kv(max_pages_per_seq=769))), (U, call(kv=_kv(num_pages=1 << 25))),
               (U, call(shape=_shape(n_q_heads=512, n_kv_heads=512))),
               (sol.SOL_ERR_WORKSPACE_TOO_SMALL, call(size=need - 1)), (sol.SOL_OK, call(B=0))]
              + [(U, call(shape=_shape(**s))) for s in BAD_SHAPES])


def test_tree_workspace_sizes():
    s = _shape()
    assert sol.tree_workspace_bytes(s, 128, 768, 64) > 0
    for bad in ((0, 8, 8), (129, 8, 8), (1, 0, 8), (1, 769, 8), (1, 8, 0), (1, 8, 65)):
        assert sol.tree_workspace_bytes(s, *bad) == 0
    assert all(sol.tree_workspace_bytes(_shape(**b), 1, 8, 8) == 0 for b in BAD_SHAPES)


def test_tree_commit_refuses():
    def call(kvs=None, N=8, n=FAKE, B=2, path=FAKE, count=FAKE, ws=FAKE, shape=None):
        return lambda: sol.tree_commit(shape or _shape(), [_kv()] if kvs is None else kvs, sol.make_tree(N, n), B, path, count, None,
                                       ws, check=False)

    I, U = sol.SOL_ERR_INVALID_ARG, sol.SOL_ERR_UNSUPPORTED
    _refusals([(I, call(kvs=[])), (I, call(n=None)), (I, call(path=None)), (I, call(count=None)), (I, call(ws=None)), (I, call(B=-1)),
               (I, call(N=0)), (U, call(N=65)), (U, call(B=129)), (I, call(kvs=[_kv(), _kv(page_table=None)])),
               (U, call(kvs=[_kv(), _kv(max_pages_per_seq=769)])), (I, call(kvs=[_kv(k_pool=FAKE + 2)])), (sol.SOL_OK, call(B=0))]
              + [(U, call(shape=_shape(**s))) for s in BAD_SHAPES])


def test_weighted_decode_attn_refuses():
    def call(shape=None, q=FAKE, kv=None, B=2, decay=1.0, w=FAKE, out=FAKE, ws=FAKE, size=BIG):
        return lambda: sol.weighted_decode_attn(shape or _shape(), q, kv or _kv(), B, decay, w, out, ws, size, check=False)

    I, U = sol.SOL_ERR_INVALID_ARG, sol.SOL_ERR_UNSUPPORTED
    need = sol.workspace_bytes(_shape(), 2, 8)
    _refusals([(I, call(q=None)), (I, call(w=None)), (I, call(out=None)), (I, call(ws=None)), (I, call(B=-1)), (U, call(B=129)),
               (I, call(decay=-0.1)), (I, call(decay=1.5)), (I, call(decay=float("nan"))), (I, call(w=FAKE + 4)),
               (I, call(kv=_kv(seq_lens=None))), (U, call(kv=_kv(max_pages_per_seq=769))),
               (sol.SOL_ERR_WORKSPACE_TOO_SMALL, call(size=need - 1)), (sol.SOL_OK, call(B=0))]
              + [(U, call(shape=_shape(**s))) for s in BAD_SHAPES])


def test_kv_evict_refuses():
    OTHER = 0x2000

    def call(shape=None, kv=None, B=2, budgets=FAKE, w=FAKE, table=FAKE, dst_w=FAKE, lens=OTHER, ws=FAKE, size=BIG):
        return lambda: sol.kv_evict(shape or _shape(), kv or _kv(), B, budgets, w, table, dst_w, lens, None, ws, size, check=False)

    I, U = sol.SOL_ERR_INVALID_ARG, sol.SOL_ERR_UNSUPPORTED
    need = sol.workspace_bytes(_shape(), 2, 8)
    _refusals([(I, call(budgets=None)), (I, call(w=None)), (I, call(table=None)), (I, call(dst_w=None)), (I, call(lens=None)),
               (I, call(lens=FAKE)), (I, call(ws=None)), (I, call(B=-1)), (U, call(B=129)), (I, call(kv=_kv(v_pool=FAKE + 2))),
               (U, call(kv=_kv(max_pages_per_seq=769))), (sol.SOL_ERR_WORKSPACE_TOO_SMALL, call(size=need - 1)),
               (sol.SOL_OK, call(B=0))] + [(U, call(shape=_shape(**s))) for s in BAD_SHAPES])


def test_outputs_that_share_an_input_and_misaligned_words_are_refused():
    I = sol.SOL_ERR_INVALID_ARG

    def commit(lens, n=0x3000, count=0x4000, kvs=None, ws=FAKE):
        return lambda: sol.tree_commit(_shape(), kvs or [_kv(seq_lens=0x2000)], sol.make_tree(8, n), 4, FAKE, count, lens, ws,
                                       check=False)

    def evict(lens):
        return lambda: sol.kv_evict(_shape(), _kv(seq_lens=0x2000), 4, 0x3000, FAKE, FAKE, FAKE, lens, None, FAKE, BIG, check=False)

    _refusals([(I, commit(0x2000)), (I, commit(0x200C)), (I, commit(0x1FF4)), (I, commit(0x3000)), (I, commit(0x400C)),
               (I, commit(0x5000, kvs=[_kv(seq_lens=0x2000), _kv(seq_lens=0x5004)])), (I, commit(0x5000, ws=FAKE + 4)),
               (I, evict(0x2004)), (I, evict(0x1FF4)), (I, evict(0x3008)),
               (I, lambda: sol.tree_build(2, 4, FAKE, FAKE, FAKE + 4, None, check=False)),
               (I, lambda: sol.tree_attn(_shape(), FAKE, _kv(), sol.make_tree(8, FAKE, FAKE + 4), 2, FAKE, FAKE, BIG, check=False))])


def test_new_lengths_over_the_path_are_refused():
    """Every layer's CTAs read the path while the first layer's write the lengths."""
    def commit(lens, path=0x5000, B=4, N=8):
        kv = _kv(seq_lens=0x2000)
        return lambda: sol.tree_commit(_shape(), [kv], sol.make_tree(N, 0x3000), B, path, 0x4000, lens, FAKE, check=False)

    I = sol.SOL_ERR_INVALID_ARG
    _refusals([(I, commit(0x5000)), (I, commit(0x5000 + 31 * 4)), (I, commit(0x5000 - 12)), (I, commit(0x5040, B=1, N=64)),
               (sol.SOL_OK, commit(0x5000, B=0))])


def test_weight_parts_are_one_or_two():
    def call(parts, size=0):
        return lambda: sol.tree_attn(_shape(), FAKE, _kv(), sol.make_tree(8, FAKE, FAKE, parts), 2, FAKE, FAKE, size, check=False)

    _refusals([(sol.SOL_ERR_INVALID_ARG, call(3)), (sol.SOL_ERR_INVALID_ARG, call(-1))]
              + [(sol.SOL_ERR_WORKSPACE_TOO_SMALL, call(p)) for p in (0, 1, 2)])


def test_tracked_eviction_refuses():
    """What sol_kv_evict refuses, an origin that is not whole, keys without rotation, pools and arrays that overlap."""
    POOL = 32 * 2 * 64 * 64 * 2  # bytes of the cache's keys
    ROWS = 2 * 2 * 8 * 64 * 4    # ... of `moved`
    FAR = 1 << 30

    def call(pool=FAR, moved=FAKE, dst=None, shape=None, kv=None, B=2, lens=0x2000, size=BIG):
        origin = sol.make_key_origin(pool, moved, dst)
        kv = kv or _kv(k_pool=0x100000, v_pool=0x100000 + POOL)
        return lambda: sol.kv_evict(shape or _shape(rope_theta=10000.0), kv, B, FAKE, FAKE, FAKE, FAKE, lens, None, FAKE, size,
                                    check=False, origin=origin)

    I, U, Z = sol.SOL_ERR_INVALID_ARG, sol.SOL_ERR_UNSUPPORTED, sol.SOL_ERR_WORKSPACE_TOO_SMALL
    _refusals([(I, call(pool=None)), (I, call(moved=None, dst=FAKE)), (I, call(pool=FAR + 8)), (I, call(shape=_shape())),
               (I, call(pool=0x100000)), (I, call(pool=0x100000 + POOL - 16)), (I, call(pool=0x100000 - POOL + 16)),
               (I, call(pool=0x100000 + 2 * POOL - 16)), (Z, call(pool=0x100000 + 2 * POOL, size=0)),
               (I, call(dst=FAKE + ROWS - 4)), (Z, call(dst=FAKE + ROWS, size=0)), (Z, call(dst=FAKE, size=0)),
               (I, call(lens=FAKE)), (I, call(B=-1)), (U, call(B=129)), (U, call(kv=_kv(max_pages_per_seq=769))), (sol.SOL_OK, call(B=0))]
              + [(U, call(shape=_shape(rope_theta=10000.0, **s))) for s in BAD_SHAPES])


# ---- pins of the oracle --------------------------------------------------------------------------
def _cache(lens, seed=0, theta=0.0):
    cfg = dict(synth.WORKLOADS["tiny"], shuffle_pages=True)
    table, n = synth.make_page_table(np.asarray(lens), True, seed)
    k, v = synth.make_kv_pool(cfg, n, seed)
    return O.Shape(256, 4, 2, 64, 1024, rope_theta=theta), O.PagedKV(k, v, table, np.asarray(lens, np.int32))


def _dense(pool, table, T):
    return torch.from_numpy(np.concatenate([O.bf16_to_f64(pool[p]) for p in table[: -(-T // 64)]], 1)[:, :T])


def test_tree_attention_of_a_chain_is_causal_attention():
    shape, kv = _cache([90, 40])
    n = 10
    rng = np.random.default_rng(0)
    q = synth.normal_bf16(rng, (2, n, 4, 64), 0.0, 1.0)
    out, mass, _ = OC.tree_attn(shape, q, kv, [n, n], [[(2 << i) - 1 for i in range(n)]] * 2)
    for b, T in enumerate((90, 40)):
        K, V = (_dense(x, kv.page_table[b], T).repeat_interleave(2, 0) for x in (kv.k_pool, kv.v_pool))
        full = torch.zeros(4, T, 64, dtype=torch.float64)
        full[:, T - n:] = torch.from_numpy(O.bf16_to_f64(q[b])).transpose(0, 1)
        want = torch.nn.functional.scaled_dot_product_attention(full, K, V, is_causal=True)[:, T - n:]
        assert np.allclose(out[b], want.transpose(0, 1).numpy(), atol=1e-12)
        assert np.all(mass[b] >= np.abs(out[b]) - 1e-12)


def test_masks_by_walking_up():
    rng = np.random.default_rng(1)
    parents = [-1] + [int(rng.integers(-1, i)) for i in range(1, 64)]
    masks, depths = OC.ancestor_masks(parents)
    for i in range(64):
        up, at = set(), i
        while at >= 0:
            up.add(at)
            at = parents[at]
        assert masks[i] == sum(1 << j for j in up) and depths[i] == len(up) - 1


def test_accept_is_the_longest_right_chain_by_brute_force():
    rng = np.random.default_rng(2)
    for _ in range(200):
        n = int(rng.integers(1, 9))
        parents = [-1] + [int(rng.integers(0, i)) for i in range(1, n)]
        draft, target = rng.permutation(20)[:n], rng.integers(0, 20, n)
        for i in range(1, n):
            if rng.random() < 0.6:
                target[parents[i]] = draft[i]
        best = max((c for r in range(n) for c in itertools.combinations(range(1, n), r)
                    if all(parents[x] == y and draft[x] == target[y] for x, y in zip(c, (0,) + c))), key=len)
        path, token = OC.tree_accept(parents, draft, target)
        assert path == [0, *best] and token == target[path[-1]]


def test_commit_by_hand():
    _, kv = _cache([70])
    row = lambda pool, t: pool[kv.page_table[0][t // 64], :, t % 64].copy()  # noqa: E731
    want = [row(kv.k_pool, t) for t in (62, 64, 69)]
    assert OC.tree_commit(kv, [8], [[0, 2, 7]]) == [65]
    for t, w in zip((62, 63, 64), want):
        assert np.array_equal(row(kv.k_pool, t), w)


def test_weights_are_the_softmax_rows_summed():
    shape, kv = _cache([100, 1])
    q = synth.normal_bf16(np.random.default_rng(3), (2, 4, 64), 0.0, 1.0)
    old = np.random.default_rng(4).random((2, 2, kv.page_table.shape[1] * 64))
    out, _, _, new, got = OC.weighted_decode_attn(shape, q, kv, 0.5, old)
    for b, T in enumerate((100, 1)):
        K, V = _dense(kv.k_pool, kv.page_table[b], T), _dense(kv.v_pool, kv.page_table[b], T)
        qq = torch.from_numpy(O.bf16_to_f64(q[b])).view(2, 2, 64)
        p = torch.softmax(qq @ K.transpose(1, 2) / 8.0, -1)
        assert np.allclose(got[b, :, :T], p.sum(1).numpy(), atol=1e-13)
        assert np.allclose(out[b].reshape(2, 2, 64), (p @ V).numpy(), atol=1e-12)
        assert np.allclose(new[b, :, : T - 1], 0.5 * old[b, :, : T - 1] + got[b, :, : T - 1])
        assert np.allclose(new[b, :, T - 1], got[b, :, T - 1]) and np.array_equal(new[b, :, T:], old[b, :, T:])


@pytest.mark.parametrize("budget", [0, 1, 3, 5, 6, 7, 50])
def test_eviction_keeps_what_brute_force_keeps(budget):
    rng = np.random.default_rng(budget)
    for _ in range(30):
        T, sink, window = 7, int(rng.integers(0, 3)), int(rng.integers(0, 3))
        w = rng.integers(0, 3, T).astype(np.float64)
        forced = set(range(sink)) | set(range(T - window, T))
        k = min(T, max(budget, len(forced)))
        best = max((c for c in itertools.combinations(range(T), k) if forced <= set(c)),
                   key=lambda c: (sum(w[i] for i in c), [-i for i in c]))
        assert tuple(OC.evict_keep(w, T, budget, sink, window)) == best


def test_evicted_keys_sit_at_their_new_positions():
    """A cache whose keys are one vector rotated to its slots stays one after any eviction, and scores depend on distance alone."""
    theta, T = 10000.0, 60
    shape, kv = _cache([T], theta=theta)
    base = np.random.default_rng(5).standard_normal(64)
    exact = np.array([O.rope_rotate(base, t, theta) for t in range(T)])
    idx = OC.evict_keep(np.random.default_rng(6).random(T), T, 20, 1, 2)
    for j, i in enumerate(idx):
        assert np.allclose(O.rope_rotate(exact[i], j - int(i), theta), O.rope_rotate(base, j, theta), atol=1e-9)
    kept, keys, values = OC.kv_evict(shape, kv, [20], np.random.default_rng(6).random((1, 2, 64)), 1, 2)
    assert keys[0][0].shape == values[0][1].shape == (20, 64)
