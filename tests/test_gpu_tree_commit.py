"""sol_tree_commit beyond the ordinary path: counts and lengths out of range, and the Quest extrema of what was committed."""
import numpy as np
import pytest
import torch

from oracle import cache_ops as OC
from oracle import checker
from oracle import sol_oracle as O
from paper_2605_10875_b200 import binding as sol
from paper_2605_10875_b200 import synth
from tests import cache_cases as CC
from tests import harness as H

pytestmark = pytest.mark.gpu

BAD_ACTION = 4


def _commit(shape, kvs, counts, paths, lens, N):
    ws = torch.zeros(256, dtype=torch.uint8, device=H.DEV)
    new = H.dev_i32([-99] * len(counts))
    n_nodes, path = H.dev_i32(counts), H.dev_i32(paths)
    sol.tree_commit(shape, [kv.struct() for kv in kvs], sol.make_tree(N, n_nodes), len(counts), path, H.dev_i32(lens), new, ws)
    return list(new.cpu().numpy()), sol.read_device_status(ws)[0]


# (length, nodes, path length) as the call is told them, and what they count as with 8 nodes at most and two pages
COUNTS = {
    "more nodes than the arrays hold": ((80, 9, 3), (80, 8, 3)),
    "many more nodes": ((80, 2**31 - 1, 8), (80, 8, 8)),
    "more nodes than tokens": ((5, 8, 4), (5, 5, 4)),
    "nodes below zero": ((80, -1, 2), (80, 0, 0)),
    "nodes far below zero": ((80, -2**31, 2), (80, 0, 0)),
    "a path longer than the tree": ((80, 4, 7), (80, 4, 3)),
    "a path far longer": ((80, 4, 2**31 - 1), (80, 4, 3)),
    "a path of length below zero": ((80, 8, -1), (80, 8, 0)),
    "a length beyond the pages": ((200, 8, 3), (128, 8, 3)),
    "a length far beyond": ((2**31 - 1, 8, 3), (128, 8, 3)),
    "a length below zero": ((-4, 8, 3), (0, 0, 0)),
}


@pytest.mark.parametrize("what", sorted(COUNTS))
def test_commit_clamps_counts_as_the_attention_does(what):
    """A count out of range counts as the nearest in range and raises the bit; the path stays valid as far as it ascends in the
    tree, and the drafted rows that it leaves out are no part of the sequence any more."""
    told, means = COUNTS[what]
    cfg = CC.config("g2")
    shape, _ = H.make_shapes(cfg)
    path = np.tile(np.array([0, 1, 2, 3, 4, 5, 6, 7], np.int32), (3, 1))
    path[1] = [1, 3, 4, 5, 6, 7, 0, 0]
    # sequence 1 is the one; its neighbours are in order
    paths, counts, lens = path, [8, told[1], 8], [3, told[2], 1]
    if what == "many more nodes":
        path[1] = np.arange(8)
    elif means[1] == 5:
        path[1] = [0, 1, 2, 4, 0, 0, 0, 0]
    elif means[1] == 4:
        path[1] = [0, 2, 3, 5, 6, 7, 0, 0]  # ends where the tree does
    kv, _ = CC.make_cache(cfg, [80, 128, 70])
    old = kv.to_oracle()
    kv.seq_lens.copy_(torch.tensor([80, told[0], 70], dtype=torch.int32))
    new, status = _commit(shape, [kv], counts, paths, lens, 8)
    want = O.PagedKV(old.k_pool.copy(), old.v_pool.copy(), old.page_table, np.array([80, means[0], 70], np.int32))
    took = [[int(x) for x in p[:n]] for p, n in zip(path, (3, means[2], 1))]
    assert new == OC.tree_commit(want, [8, means[1], 8], took)
    assert status == BAD_ACTION
    assert np.array_equal(H.host_u16(kv.k_pool), want.k_pool) and np.array_equal(H.host_u16(kv.v_pool), want.v_pool)


# ---- Quest extrema -------------------------------------------------------------------------------
def _extrema(kv, shape):
    S = shape.quest_page_size
    return H.host_u16(kv.quest_meta).reshape(kv.num_pages, shape.n_kv_heads, 64 // S, 2, shape.head_dim)


def _built(kv, shape, lens):
    """The extrema of the cache as it is, for these lengths; blocks that hold no token: zeros."""
    fresh = H.DeviceKV(kv.k_pool, kv.v_pool, kv.page_table, H.dev_i32(lens), kv.max_pages, kv.num_pages)
    fresh.build_quest_meta(shape, len(lens))
    return _extrema(fresh, shape)


def _same_where_tokens_are(kv, got, want, lens, S):
    table = kv.page_table.cpu().numpy()
    for b, T in enumerate(lens):
        for t in range(0, T, S):
            at = (table[b, t // 64], slice(None), t % 64 // S)
            assert np.array_equal(got[at], want[at]), (b, t)


@pytest.mark.parametrize("heads,S", [("g2", 4), ("g2", 16), ("g8", 8), ("g4", 64), ("g3", 32)])
@pytest.mark.parametrize("drafted_too", [False, True])
def test_commit_renews_the_quest_extrema(heads, S, drafted_too):
    """In every layer, for every block the drafted tokens lie in: whether the extrema were those of the context or those of all
    tokens before, they are afterwards what sol_quest_build_meta finds; the other blocks are left alone."""
    cfg = CC.config(heads)
    shape, _ = H.make_shapes(cfg, token_select=sol.SELECT_QUEST_PAGES, quest_page_size=S)
    rng = np.random.default_rng(S)
    N, layers = 64, 66  # more layers than one launch takes
    counts = [64, 5, 20, 7, 0, 12, 64]
    paths = [list(range(0, 64, 3)), [0, 2, 4], [0], [], [], list(range(12)), list(range(64))]
    contexts = [63, 0, 127, 61, 30, 64, 200]
    lens = [c + n for c, n in zip(contexts, counts)]
    kvs = [CC.make_cache(cfg, lens, seed=l)[0] for l in range(2)]
    for kv in kvs:
        kv.seq_lens = H.dev_i32(lens if drafted_too else contexts)
        kv.build_quest_meta(shape, len(lens))
        kv.seq_lens = H.dev_i32(lens)
        for b, T in enumerate(lens):  # keys that stand out, so that no rejected one stays unnoticed
            for t in range(contexts[b], T):
                CC.poke(kv.k_pool, kv.page_table.cpu().numpy(), b, t, int(rng.choice([0x4120, 0xC120])) + int(rng.integers(0, 64)))
        if drafted_too:
            kv.build_quest_meta(shape, len(lens))
    path = np.zeros((len(lens), N), np.int32)
    for b, p in enumerate(paths):
        path[b, : len(p)] = p
    before = [_extrema(kv, shape) for kv in kvs]
    bare = CC.make_cache(cfg, lens, seed=9)[0]  # a layer without extrema among them
    new, status = _commit(shape, [kvs[0]] + [bare] * (layers - 2) + [kvs[1]], counts, path, [len(p) for p in paths], N)
    want_lens = [c + len(p) for c, p in zip(contexts, paths)]
    assert new == want_lens and status == 0
    for kv, old in zip(kvs, before):
        got = _extrema(kv, shape)
        _same_where_tokens_are(kv, got, _built(kv, shape, want_lens), want_lens, S)
        changed = np.zeros(got.shape[:3], bool)
        table = kv.page_table.cpu().numpy()
        for b, (c, T) in enumerate(zip(contexts, want_lens)):
            for t in range(c // S * S, T, S):
                changed[table[b, t // 64], :, t % 64 // S] = True
        assert np.array_equal(got[~changed], old[~changed])


def test_a_quest_decode_step_after_a_commit():
    """A path over several blocks of four, then the decode layer, which renews the newest token's block alone."""
    cfg, S = CC.config("g2"), 4
    shape, oshape = H.make_shapes(cfg, token_select=sol.SELECT_QUEST_PAGES, quest_page_size=S)
    contexts, counts = [118, 63, 5], [10, 16, 9]
    lens = [c + n for c, n in zip(contexts, counts)]
    kv, _ = CC.make_cache(cfg, [n + 1 for n in lens], seed=3)
    kv.seq_lens = H.dev_i32(contexts)
    kv.build_quest_meta(shape, 3)
    kv.seq_lens = H.dev_i32(lens)
    path = np.zeros((3, 16), np.int32)
    paths = [[0, 1, 3, 4, 5, 8, 9], [0, 2, 4, 6, 8, 10, 12, 14, 15], [0, 8]]
    for b, p in enumerate(paths):
        path[b, : len(p)] = p
    new, status = _commit(shape, [kv], counts, path, [len(p) for p in paths], 16)
    assert status == 0
    now = [n + 1 for n in new]
    kv.seq_lens = H.dev_i32(now)
    rng = np.random.default_rng(4)
    h_in = synth.normal_bf16(rng, (3, cfg["d_model"]), 0.0, 1.0)
    lw = synth.make_layer_weights(cfg, 1)
    r, p, bits = [150, 150, 500], [0, 0, 0], [16, 16, 16]
    okv = kv.to_oracle()
    got, _, st = H.gpu_layer(shape, H.device_weights(lw, shape), kv, h_in, r, p, bits, trace=False)
    want, _ = O.decode_layer(oshape, H.oracle_weights(lw), okv, O.bf16_to_f64(h_in), r, p, bits,
                             token_select=O.SELECT_QUEST_PAGES, quest_page_size=S)
    rel = checker.output_errors(want, got)[1]
    assert st[0] == 0 and rel <= checker.OUT_REL_L2, rel
    _same_where_tokens_are(kv, _extrema(kv, shape), _built(kv, shape, now), now, S)
