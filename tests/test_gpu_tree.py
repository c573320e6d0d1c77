"""Trees of drafted tokens over the paged cache (sol_tree_build, sol_tree_attn, sol_tree_accept, sol_tree_commit) against the
fp64 oracle: head layouts, lengths from one token on, masks that leave rows empty, values that are no numbers where nobody
looks, pages out of range, streams and graphs."""
import numpy as np
import pytest
import torch

from oracle import cache_ops as OC
from oracle import sol_oracle as O
from paper_2605_10875_b200 import binding as sol
from paper_2605_10875_b200 import synth
from tests import cache_cases as CC
from tests import harness as H

pytestmark = pytest.mark.gpu

FILL = 0x4123  # what rows behind a tree hold before a call


class Case:
    def __init__(self, heads, contexts, counts, N, seed=0, masks=None):
        self.cfg = CC.config(heads)
        self.shape, self.oshape = H.make_shapes(self.cfg)
        self.counts, self.N, self.B = list(counts), N, len(counts)
        self.kv, _ = CC.make_cache(self.cfg, [c + n for c, n in zip(contexts, counts)], seed)
        rng = np.random.default_rng(seed + 77)
        self.parents = CC.random_trees(rng, self.counts, N)
        self.masks = masks or [OC.ancestor_masks(p[:n])[0] for p, n in zip(self.parents, self.counts)]
        self.q = synth.normal_bf16(rng, (self.B, N, self.cfg["n_q_heads"], self.cfg["head_dim"]), 0.0, 1.0)
        self.ws = CC.TreeWorkspace(self.shape, self.B, self.kv.max_pages, N)
        self.n_nodes, self.dmask, self.dq = H.dev_i32(self.counts), CC.dev_masks(self.masks, N), H.dev_bf16(self.q)
        self.out = H.dev_bf16(np.full(self.q.shape, FILL, np.uint16))

    def launch(self, out=None, stream=None):
        sol.tree_attn(self.shape, self.dq, self.kv.struct(), sol.make_tree(self.N, self.n_nodes, self.dmask), self.B,
                      self.out if out is None else out, self.ws.buf, self.ws.bytes, stream)

    def check(self, what, status=0):
        self.launch()
        got = H.host_u16(self.out)
        assert self.ws.status()[0] == status, what
        out, mass, err = OC.tree_attn(self.oshape, self.q, self.kv.to_oracle(), self.counts, self.masks)
        for b, n in enumerate(self.counts):
            assert np.all(got[b, n:] == FILL), what
            CC.assert_attention(got[b, :n], out[b, :n], mass[b, :n], err[b, :n], (what, b))
        return got


@pytest.mark.parametrize("heads", sorted(CC.HEADS))
def test_head_layouts(heads):
    """Groups of 1 to 8, both head sizes; contexts around page ends, ragged trees of odd sizes."""
    Case(heads, [0, 1, 63, 64, 65, 200], [1, 9, 13, 64, 33, 7], 64, seed=1).check(heads)


@pytest.mark.parametrize("N", [1, 2, 3, 4, 5, 8, 16, 17, 31, 32, 63, 64])
def test_tree_sizes(N):
    """Row counts on both sides of every block size (four query heads a group)."""
    Case("g4", [130, 0, 62], [N, N, max(1, N - 1)], N, seed=N).check(N)


@pytest.mark.parametrize("heads,context,n", [("g4", 5000, 5), ("g2", 9000, 1), ("g4", 3000, 40), ("g8", 2100, 64), ("g1", 4097, 64)])
def test_long_contexts_are_split_and_merged(heads, context, n):
    Case(heads, [context], [n], n, seed=5).check((heads, context, n))


def test_many_sequences_of_very_different_lengths():
    rng = np.random.default_rng(8)
    Case("g2", [int(x) for x in np.exp(rng.uniform(0, 6.5, 128))], [int(x) for x in rng.integers(0, 12, 128)], 12, seed=8).check("128")


def test_mask_shapes():
    """A chain, nodes without themselves, nodes that see nothing but the context, and bits of nodes that are not there."""
    n = 20
    chain = [(2 << i) - 1 for i in range(n)]
    later = [0xFFFFFFFFFFFFFFFF ^ ((1 << i) - 1) for i in range(n)]
    Case("g4", [100, 0, 70, 5], [n] * 4, 24, seed=2, masks=[chain, chain, [0] * n, later]).check("shapes")


def test_rows_that_see_nothing_are_zero():
    """No context and an empty mask."""
    c = Case("g2", [0, 0], [3, 40], 40, masks=[[0, 1, 0], [0] * 39 + [1 << 39]])
    got = c.check("empty")
    assert not got[0, 0].any() and not got[0, 2].any() and not got[1, :39].any()


@pytest.mark.parametrize("n", [6, 40])
@pytest.mark.parametrize("bits", [0x7FC0, 0x7F80, 0xFF80])
def test_masked_nodes_may_hold_anything(n, bits):
    """NaN and infinities in the key and value of a node reach the rows that see it, and no others."""
    masks = [[(1 << i) | (4 if i in (2, 5) else 0) for i in range(n)], [1 << i for i in range(n)]]
    c = Case("g4", [100, 60], [n, n], n, seed=3, masks=masks)
    table = c.kv.page_table.cpu().numpy()
    CC.poke(c.kv.v_pool, table, 0, 102, bits)
    CC.poke(c.kv.k_pool, table, 1, 60 + 4, bits)
    CC.poke(c.kv.v_pool, table, 1, 60 + 4, 0x7FC0)
    c.launch()
    got = O.bf16_to_f64(H.host_u16(c.out))
    with np.errstate(all="ignore"):
        out, mass, err = OC.tree_attn(c.oshape, c.q, c.kv.to_oracle(), c.counts, c.masks)
    for i in range(n):  # sequence 0: rows 2 and 5 see node 2
        if i in (2, 5):
            want = np.full(out[0, i].shape, np.nan if bits == 0x7FC0 else np.inf if bits == 0x7F80 else -np.inf)
            assert np.array_equal(got[0, i], want, equal_nan=True), i
        else:
            CC.assert_attention(H.host_u16(c.out)[0, i], out[0, i], mass[0, i], err[0, i], i)
        if i == 4:
            assert np.isnan(got[1, i]).all()
        else:
            CC.assert_attention(H.host_u16(c.out)[1, i], out[1, i], mass[1, i], err[1, i], i)


@pytest.mark.parametrize("n", [4, 50])
def test_a_context_value_that_is_no_number_reaches_every_row(n):
    c = Case("g2", [200], [n], n, seed=4)
    CC.poke(c.kv.v_pool, c.kv.page_table.cpu().numpy(), 0, 70, 0x7FC0)
    c.launch()
    assert np.isnan(O.bf16_to_f64(H.host_u16(c.out))).all()


@pytest.mark.parametrize("n", [3, 60])
def test_large_scores(n):
    """Scores of some thousands, far apart: one token takes everything, and nothing overflows."""
    c = Case("g4", [150], [n], n, seed=6)
    c.q = synth.to_bf16(O.bf16_to_f64(c.q).astype(np.float32) * 300)
    c.dq = H.dev_bf16(c.q)
    c.check("large")


@pytest.mark.parametrize("n", [5, 64])
def test_pages_out_of_range_are_skipped(n):
    c = Case("g4", [300, 100], [n, n], n, seed=9)
    table = c.kv.page_table.clone()
    table[0, 1], table[0, 2] = -1, c.kv.num_pages
    want = Case("g4", [300 - 128, 100], [n, n], n, seed=9)  # the same without those 128 tokens
    good = c.kv.page_table.cpu().numpy()
    keep = [0] + list(range(3, good.shape[1]))
    want.kv = H.DeviceKV(c.kv.k_pool, c.kv.v_pool, H.dev_i32(np.ascontiguousarray(good[:, keep])),
                         H.dev_i32([300 - 128 + n, 100 + n]), len(keep), c.kv.num_pages)
    want.kv.page_table[1, :] = c.kv.page_table[1, : len(keep)]
    want.q, want.dq = c.q, c.dq
    want.masks, want.dmask = c.masks, c.dmask
    c.kv.page_table = table
    c.launch()
    assert c.ws.status()[0] == 2
    got = H.host_u16(c.out)
    out, mass, err = OC.tree_attn(want.oshape, want.q, want.kv.to_oracle(), want.counts, want.masks)
    CC.assert_attention(got, out, mass, err, "skipped")


def test_counts_out_of_range_are_clamped_and_reported():
    c = Case("g2", [10, 20, 30], [4, 4, 4], 4)
    c.n_nodes = H.dev_i32([5, -1, 4])
    c.launch()
    assert c.ws.status()[0] == 4
    got = H.host_u16(c.out)
    out, mass, err = OC.tree_attn(c.oshape, c.q, c.kv.to_oracle(), c.counts, c.masks)
    for b in (0, 2):
        CC.assert_attention(got[b], out[b], mass[b], err[b], b)
    assert np.all(got[1] == FILL)


def test_cache_beyond_four_gigabytes():
    """Pages whose offsets pass 32 bits."""
    cfg = CC.config("g8")
    pages = (5 << 30) // (2 * 64 * 128 * 2)
    for n in (2, 40):
        small = Case("g8", [150], [n], n, seed=11)
        small.check("small")
        k, v = (torch.empty((pages, 2, 64, 128), dtype=torch.bfloat16, device=H.DEV) for _ in range(2))
        m = small.kv.max_pages
        table = [pages - 1 - 3 * i for i in range(m)]
        for i, page in enumerate(table):
            src = int(small.kv.page_table[0, i])
            k[page], v[page] = small.kv.k_pool[src], small.kv.v_pool[src]
        want = H.host_u16(small.out)
        small.kv = H.DeviceKV(k, v, H.dev_i32([table]), small.kv.seq_lens, m, pages)
        small.launch()
        assert np.array_equal(H.host_u16(small.out), want)
    assert cfg["head_dim"] == 128


def test_repeated_calls_streams_and_a_shared_workspace_give_the_same_bits():
    a, b = Case("g4", [700, 33, 2500], [40, 3, 21], 40, seed=12), Case("g4", [64, 900, 5], [7, 40, 40], 40, seed=13)
    b.ws = a.ws
    first = [a.check("a"), b.check("b")]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        for c in (a, b):
            c.out.fill_(0)
            torch.cuda.synchronize()
            c.launch(stream=s)
        s.synchronize()
        for c, want in zip((a, b), first):
            got = H.host_u16(c.out)
            assert all(np.array_equal(got[i, :n], want[i, :n]) for i, n in enumerate(c.counts))


def test_captured_and_replayed_with_other_lengths():
    c = Case("g4", [500, 100], [20, 8], 20, seed=14)
    s = torch.cuda.Stream()
    c.launch(stream=s)
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        c.launch(stream=torch.cuda.current_stream())
    for lens, counts in (([520, 108], [20, 8]), ([300, 70], [3, 20]), ([20, 1], [20, 1])):
        c.kv.seq_lens.copy_(H.dev_i32(lens))
        c.counts = counts
        c.n_nodes.copy_(H.dev_i32(counts))
        c.parents = CC.random_trees(np.random.default_rng(lens[0]), counts, 20)
        c.masks = [OC.ancestor_masks(p[:n])[0] for p, n in zip(c.parents, counts)]
        c.dmask.copy_(CC.dev_masks(c.masks, 20))
        c.out.copy_(H.dev_bf16(np.full(c.q.shape, FILL, np.uint16)))
        g.replay()
        torch.cuda.synchronize()
        got = H.host_u16(c.out)
        out, mass, err = OC.tree_attn(c.oshape, c.q, c.kv.to_oracle(), counts, c.masks)
        for b, n in enumerate(counts):
            CC.assert_attention(got[b, :n], out[b, :n], mass[b, :n], err[b, :n], (lens, b))
            assert np.all(got[b, n:] == FILL)


def test_the_longest_context_and_the_largest_batch():
    Case("g2", [768 * 64 - 64], [64], 64, seed=15).check("long")
    Case("g4", [768 * 64 - 3], [3], 3, seed=16).check("long, few rows")
    Case("g6", [(29 * b) % 150 for b in range(128)], [(7 * b) % 65 if b % 5 else 0 for b in range(128)], 64, seed=17).check("wide")


def test_two_streams_at_once_with_workspaces_of_their_own():
    make = lambda: [Case("g8", [900, 40], [33, 64], 64, seed=18), Case("g2", [2000, 7, 300], [5, 8, 1], 8, seed=19)]  # noqa: E731
    alone, both = make(), make()
    for c in alone:
        c.launch()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in both]
    for _ in range(3):
        for c, s in zip(both, streams):
            c.launch(stream=s)
    torch.cuda.synchronize()
    for a, b in zip(alone, both):
        assert np.array_equal(H.host_u16(a.out), H.host_u16(b.out)) and b.ws.status()[0] == 0


# ---- bookkeeping ---------------------------------------------------------------------------------
@pytest.mark.parametrize("N,near", [(1, 1), (2, 1), (33, 5), (64, 1), (64, 8), (64, 64)])
def test_build_matches_the_walk_up(N, near):
    rng = np.random.default_rng(N + near)
    counts = [int(x) for x in rng.integers(0, N + 1, 37)] + [N]
    parents = CC.random_trees(rng, counts, N, near)
    parents[rng.random(parents.shape) < 0.05] = -1
    parents[3, N // 2:] = 70  # no node: a root
    parents[4, 0] = 0
    mask = torch.full((38, N), -7, dtype=torch.int64, device=H.DEV)
    depth = torch.full((38, N), -7, dtype=torch.int32, device=H.DEV)
    sol.tree_build(38, N, H.dev_i32(counts), H.dev_i32(parents), mask, depth)
    got_m, got_d = mask.cpu().numpy().view(np.uint64), depth.cpu().numpy()
    for b, n in enumerate(counts):
        m, d = OC.ancestor_masks(parents[b, :n])
        assert [int(x) for x in got_m[b, :n]] == m and list(got_d[b, :n]) == d, b
        assert np.all(got_m[b, n:].view(np.int64) == -7) and np.all(got_d[b, n:] == -7)
    only = torch.zeros_like(mask)
    sol.tree_build(38, N, H.dev_i32(counts), H.dev_i32(parents), only)
    assert all(torch.equal(only[b, :n], mask[b, :n]) for b, n in enumerate(counts))


@pytest.mark.parametrize("N", [1, 5, 32, 33, 64])
def test_accept_takes_the_first_matching_child(N):
    """Few token values, so that several children match and paths go deep."""
    rng = np.random.default_rng(N)
    B = 61
    counts = [int(x) for x in rng.integers(0, N + 1, B - 1)] + [N]
    parents = CC.random_trees(rng, counts, N, 3)
    draft, target = rng.integers(0, 3, (B, N)).astype(np.int32), rng.integers(0, 3, (B, N)).astype(np.int32)
    draft[B - 1] = target[B - 1] = 7  # every node is right
    path = torch.full((B, N), -9, dtype=torch.int32, device=H.DEV)
    count, token = H.dev_i32([-9] * B), H.dev_i32([-9] * B)
    sol.tree_accept(B, N, H.dev_i32(counts), H.dev_i32(parents), H.dev_i32(draft), H.dev_i32(target), path, count, token)
    path, count, token = path.cpu().numpy(), count.cpu().numpy(), token.cpu().numpy()
    for b, n in enumerate(counts):
        want, last = OC.tree_accept(parents[b, :n], draft[b], target[b])
        assert list(path[b, : len(want)]) == want and count[b] == len(want) and token[b] == last, b
        assert np.all(path[b, len(want):] == -9)


@pytest.mark.parametrize("heads", ["g2", "g8"])
def test_commit_moves_the_path_in_every_layer(heads):
    cfg = CC.config(heads)
    shape, oshape = H.make_shapes(cfg)
    rng = np.random.default_rng(3)
    N, B, layers = 64, 9, 67  # more layers than one launch takes
    counts = [64, 1, 20, 40, 64, 0, 17, 33, 5]
    paths = [sorted([0] + [int(x) for x in rng.choice(np.arange(1, n), k, replace=False)]) if n else []
             for n, k in zip(counts, [30, 0, 3, 12, 63, 0, 16, 1, 2])]
    lens = [n + int(c) for n, c in zip(counts, rng.integers(0, 200, B))]
    kvs, olds = [], []
    for l in range(layers):
        kv, _ = CC.make_cache(cfg, lens, seed=l % 3)
        kvs.append(kv)
        olds.append(kv.to_oracle())
    path = np.full((B, N), -5, np.int32)
    for b, p in enumerate(paths):
        path[b, : len(p)] = p
    ws = torch.zeros(256, dtype=torch.uint8, device=H.DEV)
    new, n_nodes = H.dev_i32([-1] * B), H.dev_i32(counts)
    sol.tree_commit(shape, [k.struct() for k in kvs], sol.make_tree(N, n_nodes), B, H.dev_i32(path),
                    H.dev_i32([len(p) for p in paths]), new, ws)
    assert sol.read_device_status(ws)[0] == 0
    for kv, old in zip(kvs, olds):
        old = O.PagedKV(old.k_pool.copy(), old.v_pool.copy(), old.page_table, old.seq_lens)
        want = OC.tree_commit(old, counts, paths)
        assert np.array_equal(H.host_u16(kv.k_pool), old.k_pool) and np.array_equal(H.host_u16(kv.v_pool), old.v_pool)
    assert list(new.cpu().numpy()) == want


def test_commit_reports_paths_that_do_not_ascend_and_bad_pages():
    cfg = CC.config("g2")
    shape, _ = H.make_shapes(cfg)
    counts, lens = [8, 8, 8, 8], [80, 80, 80, 80]
    path = np.array([[0, 3, 2, 5, 0, 0, 0, 0], [0, 2, 9, 0, 0, 0, 0, 0], [-1, 0, 0, 0, 0, 0, 0, 0], [0, 4, 6, 0, 0, 0, 0, 0]], np.int32)
    kv, _ = CC.make_cache(cfg, lens)
    old = kv.to_oracle()
    ws = torch.zeros(256, dtype=torch.uint8, device=H.DEV)
    new, n_nodes = H.dev_i32([-1] * 4), H.dev_i32(counts)
    tree = sol.make_tree(8, n_nodes)
    sol.tree_commit(shape, [kv.struct()], tree, 4, H.dev_i32(path), H.dev_i32([4, 3, 2, 3]), new, ws)
    assert sol.read_device_status(ws)[0] == 4
    assert list(new.cpu().numpy()) == [74, 74, 72, 75]
    want = O.PagedKV(old.k_pool.copy(), old.v_pool.copy(), old.page_table, old.seq_lens)
    OC.tree_commit(want, counts, [[0, 3], [0, 2], [], [0, 4, 6]])
    assert np.array_equal(H.host_u16(kv.k_pool), want.k_pool) and np.array_equal(H.host_u16(kv.v_pool), want.v_pool)
    kv.page_table[0, 1] = -1
    sol.workspace_init(ws, 256)
    sol.tree_commit(shape, [kv.struct()], tree, 4, H.dev_i32(path), H.dev_i32([2, 1, 1, 1]), None, ws)
    assert sol.read_device_status(ws)[0] & 2


def test_a_whole_step_captured_and_replayed():
    """Masks, attention, acceptance and commit as one graph, replayed on other trees, against the calls one by one."""
    B, N = 3, 20
    rng = np.random.default_rng(5)
    c = Case("g4", [90, 200, 64], [20, 7, 13], N, seed=20)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device=H.DEV)  # noqa: E731
    parents, draft, target, path, count, token, new = i32(B, N), i32(B, N), i32(B, N), i32(B, N), i32(B), i32(B), i32(B)

    def step(stream):
        tree = sol.make_tree(N, c.n_nodes, c.dmask)
        sol.tree_build(B, N, c.n_nodes, parents, c.dmask, stream=stream)
        c.launch(stream=stream)
        sol.tree_accept(B, N, c.n_nodes, parents, draft, target, path, count, token, stream=stream)
        sol.tree_commit(c.shape, [c.kv.struct()], tree, B, path, count, new, c.ws.buf, stream)

    pools = c.kv.k_pool.clone(), c.kv.v_pool.clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        step(torch.cuda.current_stream())
    for counts in ([20, 7, 13], [1, 20, 0]):
        c.n_nodes.copy_(H.dev_i32(counts))
        parents.copy_(H.dev_i32(CC.random_trees(rng, counts, N, 3)))
        for x in (draft, target):
            x.copy_(H.dev_i32(rng.integers(0, 2, (B, N)).astype(np.int32)))
        results = []
        for go in (lambda: step(None), g.replay):
            c.kv.k_pool.copy_(pools[0])
            c.kv.v_pool.copy_(pools[1])
            for x in (path, count, token, new):
                x.fill_(-1)
            c.out.zero_()
            torch.cuda.synchronize()
            go()
            torch.cuda.synchronize()
            assert c.ws.status()[0] == 0
            results.append([x.clone() for x in (path, count, token, new, c.out.view(torch.int16), c.kv.k_pool.view(torch.int16),
                                                c.kv.v_pool.view(torch.int16))])
        assert all(torch.equal(a, b) for a, b in zip(*results))
        assert all(min(1, n) <= int(k) <= n for k, n in zip(results[0][1], counts))
