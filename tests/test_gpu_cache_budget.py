"""The bounded cache: decode attention that keeps its weights (sol_weighted_decode_attn) and eviction by them (sol_kv_evict)
against the fp64 oracle, and a run of all the cache calls together with the decode layer."""
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

MAX_PAGES = 768  # of a sequence


class Weighted:
    def __init__(self, heads, lens, seed=0, decay=1.0, pages=None):
        self.cfg = CC.config(heads)
        self.shape, self.oshape = H.make_shapes(self.cfg)
        self.kv, _ = CC.make_cache(self.cfg, lens, seed)
        if pages:  # a wider page table than the lengths need
            wide = torch.full((len(lens), pages), -1, dtype=torch.int32, device=H.DEV)
            wide[:, : self.kv.max_pages] = self.kv.page_table
            self.kv.page_table, self.kv.max_pages = wide, pages
        self.B, self.decay = len(lens), decay
        rng = np.random.default_rng(seed + 5)
        self.q = synth.normal_bf16(rng, (self.B, self.cfg["n_q_heads"], self.cfg["head_dim"]), 0.0, 1.0)
        self.dq = H.dev_bf16(self.q)
        self.old = rng.exponential(1.0, (self.B, self.cfg["n_kv_heads"], self.kv.max_pages * 64)).astype(np.float32)
        for b, T in enumerate(lens):  # what a slot held before its token came does not count
            if T:
                self.old[b, :, T - 1] = np.nan
        self.weights = torch.from_numpy(self.old).to(H.DEV)
        self.out = torch.zeros(self.q.shape, dtype=torch.bfloat16, device=H.DEV)
        self.ws = H.Workspace(self.shape, self.B, self.kv.max_pages)

    def launch(self, stream=None):
        sol.weighted_decode_attn(self.shape, self.dq, self.kv.struct(), self.B, self.decay, self.weights, self.out, self.ws.buf,
                                 self.ws.bytes, stream)

    def check(self, what):
        self.launch()
        assert self.ws.status()[0] == 0
        out, mass, err, new, got = OC.weighted_decode_attn(self.oshape, self.q, self.kv.to_oracle(), self.decay, self.old)
        # weights of the products with V are carried to 2^-16 here (two bf16 parts)
        CC.assert_attention(H.host_u16(self.out), out, mass, err, what, 2.0 ** -16)
        w = self.weights.cpu().numpy().astype(np.float64)
        G = self.cfg["n_q_heads"] // self.cfg["n_kv_heads"]
        for b, T in enumerate(self.kv.seq_lens.cpu().numpy()):
            assert np.array_equal(w[b, :, T:], self.old[b, :, T:].astype(np.float64)), what  # entries behind are left alone
            # a softmax weight is off by its score's error, twice (its own and the sum's), and 2^-17 for the base-2 exponential and
            # logarithm of numbers up to 64 in float32; the decay's product and the sums round to 2^-24 of each term
            d = 2.1 * err[b].reshape(-1, G).max(1)[:, None] + 2.0 ** -17
            tol = got[b, :, :T] * d + (got[b, :, :T] + np.nan_to_num(np.abs(self.old[b, :, :T]))) * 2.0 ** -22 + 1e-37
            diff = np.abs(w[b, :, :T] - new[b, :, :T])
            assert np.all(diff <= tol), (what, b, float((diff / tol).max()))


@pytest.mark.parametrize("heads", sorted(CC.HEADS))
def test_weighted_head_layouts(heads):
    Weighted(heads, [1, 2, 63, 64, 65, 128, 300], seed=1).check(heads)


@pytest.mark.parametrize("heads,lens,decay", [("g4", [7001], 1.0), ("g2", [5000, 3, 900], 0.5), ("g8", [2500], 0.0), ("g1", [4096], 0.9)])
def test_weighted_long_contexts(heads, lens, decay):
    Weighted(heads, lens, seed=2, decay=decay).check((heads, lens))


def test_weighted_empty_sequences_and_many_of_them():
    rng = np.random.default_rng(4)
    lens = [int(x) for x in np.exp(rng.uniform(0, 6.2, 128))]
    lens[3] = lens[77] = 0
    c = Weighted("g2", lens, seed=4, pages=13)
    c.check("128")
    assert not H.host_u16(c.out)[3].any()


def test_weighted_wide_page_table():
    Weighted("g4", [40, 200], pages=300).check("wide")


def test_weights_add_up_over_steps_and_replays():
    c = Weighted("g4", [200, 70], seed=6, decay=0.75)
    c.check("first")
    want = c.weights.double().cpu().numpy()
    step = OC.weighted_decode_attn(c.oshape, c.q, c.kv.to_oracle(), 0.0, c.old)[4]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        c.launch(torch.cuda.current_stream())
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    for _ in range(3):
        for b, T in enumerate((200, 70)):
            want[b, :, :T] *= 0.75
            want[b, :, T - 1] = 0.0
            want[b, :, :T] += step[b, :, :T]
    got = c.weights.cpu().numpy()
    for b, T in enumerate((200, 70)):
        assert np.allclose(got[b, :, :T], want[b, :, :T], rtol=1e-4, atol=1e-7)


def test_weighted_bad_page_counts_for_nothing():
    c = Weighted("g2", [200], seed=7)
    before = c.weights.clone()
    c.kv.page_table[0, 1] = c.kv.num_pages
    c.launch()
    assert c.ws.status()[0] == 2
    got = c.weights.cpu().numpy()
    assert np.array_equal(got[0, :, 64:128], before[0, :, 64:128].cpu().numpy())
    G = 2
    added = got[0, :, :199] - before[0, :, :199].cpu().numpy()
    assert np.allclose(added.sum(-1) + got[0, :, 199], G, atol=1e-4)
    assert np.isfinite(O.bf16_to_f64(H.host_u16(c.out))).all()


# ---- eviction ------------------------------------------------------------------------------------
class Evict:
    def __init__(self, heads, lens, budgets, theta=10000.0, sink=2, window=3, seed=0, in_place=False, weights=None):
        self.cfg = CC.config(heads, theta)
        self.shape, self.oshape = H.make_shapes(self.cfg, n_sink=sink, n_window=window)
        self.lens, self.budgets, self.sink, self.window, self.in_place = list(lens), list(budgets), sink, window, in_place
        self.B = len(lens)
        pages = [-(-max(T, 1) // 64) for T in lens]
        self.kv, used = CC.make_cache(self.cfg, lens, seed, 0 if in_place else sum(pages))
        self.old = self.kv.to_oracle()
        self.mp = self.kv.max_pages
        rng = np.random.default_rng(seed + 9)
        w = rng.exponential(1.0, (self.B, self.cfg["n_kv_heads"], self.mp * 64)).astype(np.float32) if weights is None else weights
        self.old_w = w.astype(np.float32)
        self.weights = torch.from_numpy(self.old_w.copy()).to(H.DEV)
        if in_place:
            self.dst_table, self.dst_w = self.kv.page_table, self.weights
        else:
            order = used + rng.permutation(sum(pages))
            t = np.full((self.B, self.mp), -1, np.int32)
            at = 0
            for b, n in enumerate(pages):
                t[b, :n] = order[at:at + n]
                at += n
            self.dst_table, self.dst_w = H.dev_i32(t), torch.full_like(self.weights, -3.0)
        self.dst_lens = H.dev_i32([-1] * self.B)
        self.kept = torch.full(self.weights.shape, -1, dtype=torch.int32, device=H.DEV)
        self.dev_budgets = H.dev_i32(self.budgets)
        self.ws = H.Workspace(self.shape, self.B, self.mp)

    def launch(self, stream=None, kept=True):
        sol.kv_evict(self.shape, self.kv.struct(), self.B, self.dev_budgets, self.weights, self.dst_table, self.dst_w,
                     self.dst_lens, self.kept if kept else None, self.ws.buf, self.ws.bytes, stream)

    def check(self, what):
        self.launch()
        assert self.ws.status()[0] == 0
        kept, keys, values = OC.kv_evict(self.oshape, self.old, self.budgets, self.old_w, self.sink, self.window)
        got_k, got_v = O.bf16_to_f64(H.host_u16(self.kv.k_pool)), O.bf16_to_f64(H.host_u16(self.kv.v_pool))
        idx, lens, w = self.kept.cpu().numpy(), self.dst_lens.cpu().numpy(), self.dst_w.cpu().numpy()
        table = self.dst_table.cpu().numpy()
        written = np.zeros(got_k.shape[:3], bool)
        for b in range(self.B):
            assert lens[b] == len(kept[b][0]), what
            for h, want in enumerate(kept[b]):
                n = len(want)
                assert np.array_equal(idx[b, h, :n], want) and np.all(idx[b, h, n:] == -1), (what, b, h)
                assert np.array_equal(w[b, h, :n], self.old_w[b, h, want], equal_nan=True), (what, b, h)
                j = np.arange(n)
                page, slot = table[b][j // 64], j % 64
                written[page, h, slot] = True
                assert np.array_equal(got_v[page, h, slot], values[b][h]), (what, b, h)
                # bf16 rounds to 2^-8 of a value; sine, cosine and products in float32, of the pair's length
                x = keys[b][h]
                pair = np.hypot(x, np.roll(x, x.shape[1] // 2, 1))
                assert np.all(np.abs(got_k[page, h, slot] - x) <= np.abs(x) * 2.0 ** -8 + pair * 2.0 ** -20), (what, b, h)
                still = j == want
                if still.any():  # a key that does not move is not touched
                    src = O.bf16_to_f64(self.old.k_pool)[self.old.page_table[b][want // 64], h, want % 64]
                    assert np.array_equal(got_k[page, h, slot][still], src[still])
        for got, old in ((H.host_u16(self.kv.k_pool), self.old.k_pool), (H.host_u16(self.kv.v_pool), self.old.v_pool)):
            assert np.array_equal(got[~written], old[~written]), what  # nothing else was written
        if self.in_place:
            for b, n in enumerate(lens):
                assert np.array_equal(w[b, :, n:], self.old_w[b, :, n:], equal_nan=True)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("heads", ["g2", "g3", "g4", "g8"])
def test_evict_head_layouts(heads, in_place):
    Evict(heads, [1, 5, 64, 65, 200, 333], [1, 3, 20, 64, 100, 400], in_place=in_place, seed=1).check((heads, in_place))


@pytest.mark.parametrize("theta", [0.0, 10000.0, 500000.0])
@pytest.mark.parametrize("in_place", [False, True])
def test_evict_long_rows(theta, in_place):
    Evict("g4", [3000, 1500], [700, 1499], theta=theta, in_place=in_place, seed=2, sink=4, window=16).check((theta, in_place))


@pytest.mark.parametrize("sink,window", [(0, 0), (0, 1), (100, 0), (3, 500), (64, 64)])
def test_evict_forced_tokens(sink, window):
    """Budgets below, at and above what the sinks and the window hold, and of zero."""
    Evict("g2", [150, 150, 150, 150, 0, 70], [0, 1, 101, 130, 5, -3], sink=sink, window=window, seed=3).check((sink, window))


def test_evict_ties_zeros_and_odd_weights():
    """Equal weights stay by the lower index; zeros of either sign are equal; infinities rank as numbers, NaN last."""
    B, T = 5, 700
    w = np.ones((B, 2, 704), np.float32)
    rng = np.random.default_rng(5)
    w[1] = rng.choice([0.0, -0.0, 1.0], (2, 704))
    w[2] = rng.choice([np.inf, -np.inf, np.nan, 0.5], (2, 704))
    w[3] = np.nan
    w[4] = rng.integers(0, 4, (2, 704)) * 1e-41  # below the normal range
    for budget in (1, 100, 350, 699):
        Evict("g2", [T] * B, [budget] * B, weights=w, seed=4).check(budget)


def test_evict_far_moves_keep_their_angle():
    """Keys that move by tens of thousands of positions."""
    T = 40000
    w = np.zeros((1, 2, 40000), np.float32)
    w[0, :, 39000:] = 1.0
    c = Evict("g2", [T], [1000], theta=500000.0, weights=w, sink=1, window=1, seed=6)
    c.check("far")


def test_evict_without_list_and_on_a_stream():
    a, b = Evict("g4", [500, 90], [200, 90], seed=7), Evict("g4", [500, 90], [200, 90], seed=7)
    a.check("a")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    b.launch(s, kept=False)
    s.synchronize()
    assert torch.equal(a.kv.k_pool.view(torch.int16), b.kv.k_pool.view(torch.int16))
    assert torch.equal(a.kv.v_pool.view(torch.int16), b.kv.v_pool.view(torch.int16)) and torch.equal(a.dst_w, b.dst_w)
    assert np.all(b.kept.cpu().numpy() == -1)


def test_evict_reports_bad_pages():
    c = Evict("g2", [200], [100], seed=8)
    c.dst_table[0, 1] = c.kv.num_pages
    c.launch()
    assert c.ws.status()[0] == 2 and int(c.dst_lens[0]) == 100


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("heads,B", [("g1", 19), ("g3", 128), ("g4", 19), ("g8", 40), ("g4", 18)])
def test_evict_many_rows(heads, B, in_place):
    """Batches on both sides of where two CTAs share an SM, up to the largest."""
    lens = [(37 * b * b + 5 * b) % 300 for b in range(B)]
    Evict(heads, lens, [(b * 53) % 250 for b in range(B)], in_place=in_place, seed=10).check((heads, B, in_place))


@pytest.mark.parametrize("heads", ["g2", "g4"])
def test_evict_the_longest_row(heads):
    """A full page table of the largest size, next to an empty sequence and one of a single token."""
    T = MAX_PAGES * 64
    Evict(heads, [T, 0, 1], [20000, 5, 1], theta=500000.0, in_place=True, seed=11, sink=4, window=100).check("long")


def test_weighted_the_longest_row_and_the_largest_batch():
    Weighted("g2", [MAX_PAGES * 64], decay=0.5).check("long")
    Weighted("g6", [(31 * b) % 200 for b in range(128)], seed=3, decay=0.5).check("wide")


def test_two_streams_at_once_with_workspaces_of_their_own():
    """Runs on two streams at the same time give what each gives alone."""
    def run(c, e, stream):
        c.launch(stream)
        e.launch(stream)

    alone = [(Weighted("g4", [900, 40, 3000], seed=s, decay=0.5), Evict("g4", [2500, 700], [1000, 300], seed=s)) for s in (20, 21)]
    both = [(Weighted("g4", [900, 40, 3000], seed=s, decay=0.5), Evict("g4", [2500, 700], [1000, 300], seed=s)) for s in (20, 21)]
    for c, e in alone:
        run(c, e, None)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in both]
    for (c, e), s in zip(both, streams):
        run(c, e, s)
    torch.cuda.synchronize()
    for (c, e), (c2, e2) in zip(alone, both):
        assert torch.equal(c.out.view(torch.int16), c2.out.view(torch.int16))
        assert torch.equal(c.weights.view(torch.int32), c2.weights.view(torch.int32))  # bits: NaN equals NaN
        assert torch.equal(e.kept, e2.kept) and torch.equal(e.dst_lens, e2.dst_lens)
        assert torch.equal(e.kv.k_pool.view(torch.int16), e2.kv.k_pool.view(torch.int16))
        assert c2.ws.status()[0] == 0 and e2.ws.status()[0] == 0


def test_evict_captured_and_replayed_with_other_budgets():
    c = Evict("g8", [800, 130], [300, 100], seed=12)
    pools = c.kv.k_pool.clone(), c.kv.v_pool.clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        c.launch(torch.cuda.current_stream())
    for budgets, w_seed in (([300, 100], 0), ([799, 5], 1), ([10, 500], 2)):
        c.kv.k_pool.copy_(pools[0])
        c.kv.v_pool.copy_(pools[1])
        c.budgets = budgets
        c.dev_budgets.copy_(H.dev_i32(budgets))
        c.old_w = np.random.default_rng(w_seed).exponential(1.0, c.old_w.shape).astype(np.float32)
        c.weights.copy_(torch.from_numpy(c.old_w))
        c.kept.fill_(-1)
        c.launch = lambda: (g.replay(), torch.cuda.synchronize())
        c.check(budgets)


def test_lengths_out_of_range_count_as_the_nearest_in_range():
    """A length beyond the page table is the table's end, a negative one is zero: the same bits as with those lengths."""
    for wrong, right in (([1000, -3], [128, 0]), ([2**31 - 1, 128], [128, 128])):
        a, b = Weighted("g4", [128, 128], seed=30, decay=0.5), Weighted("g4", [128, 128], seed=30, decay=0.5)
        a.kv.seq_lens.copy_(torch.tensor(wrong, dtype=torch.int32))
        b.kv.seq_lens.copy_(H.dev_i32(right))
        a.launch()
        b.launch()
        assert torch.equal(a.out.view(torch.int16), b.out.view(torch.int16))
        assert torch.equal(a.weights.view(torch.int32), b.weights.view(torch.int32))
        c, d = Evict("g4", [128, 128], [60, 50], seed=31), Evict("g4", [128, 128], [60, 50], seed=31)
        c.kv.seq_lens.copy_(torch.tensor(wrong, dtype=torch.int32))
        d.kv.seq_lens.copy_(H.dev_i32(right))
        c.launch()
        d.launch()
        assert torch.equal(c.dst_lens, d.dst_lens) and torch.equal(c.kept, d.kept) and torch.equal(c.dst_w, d.dst_w)
        assert torch.equal(c.kv.k_pool.view(torch.int16), d.kv.k_pool.view(torch.int16))
        assert c.ws.status()[0] == 0 and a.ws.status()[0] == 0


def test_a_serving_loop_with_a_tree_and_a_budget():
    """A drafted tree is attended, accepted and committed; the weights of the next steps are kept; the cache is cut to a budget in
    place; the decode layer goes on with it.  Every stage against the oracle on what the stage really saw."""
    cfg = dict(synth.WORKLOADS["tiny"], rope_theta=10000.0)
    shape, oshape = H.make_shapes(cfg, n_sink=2, n_window=4)
    B, N, mp = 3, 12, 6
    context, counts = [150, 64, 201], [12, 7, 12]
    rng = np.random.default_rng(1)
    lens = np.array([c + n for c, n in zip(context, counts)], np.int32)
    pages = B * mp
    table = rng.permutation(pages).astype(np.int32).reshape(B, mp)
    k, v = synth.make_kv_pool(cfg, pages, 3)
    kv = H.device_kv(k, v, table, lens)
    weights = torch.zeros((B, 2, mp * 64), device=H.DEV)
    ws = H.Workspace(shape, B, mp)
    tws = CC.TreeWorkspace(shape, B, mp, N)

    parents = CC.random_trees(rng, counts, N, 3)
    n_nodes, dparents = H.dev_i32(counts), H.dev_i32(parents)
    mask = torch.zeros((B, N), dtype=torch.int64, device=H.DEV)
    sol.tree_build(B, N, n_nodes, dparents, mask)
    tree = sol.make_tree(N, n_nodes, mask)
    q = synth.normal_bf16(rng, (B, N, 4, 64), 0.0, 1.0)
    out = torch.zeros((B, N, 4, 64), dtype=torch.bfloat16, device=H.DEV)
    sol.tree_attn(shape, H.dev_bf16(q), kv.struct(), tree, B, out, tws.buf, tws.bytes)
    masks = [OC.ancestor_masks(p[:n])[0] for p, n in zip(parents, counts)]
    want, mass, err = OC.tree_attn(oshape, q, kv.to_oracle(), counts, masks)
    for b, n in enumerate(counts):
        CC.assert_attention(H.host_u16(out)[b, :n], want[b, :n], mass[b, :n], err[b, :n], b)

    draft, target = rng.integers(0, 2, (B, N)).astype(np.int32), rng.integers(0, 2, (B, N)).astype(np.int32)
    path, count, token = (torch.zeros(s, dtype=torch.int32, device=H.DEV) for s in ((B, N), (B,), (B,)))
    new_lens = H.dev_i32([0] * B)
    okv = kv.to_oracle()
    sol.tree_accept(B, N, n_nodes, dparents, H.dev_i32(draft), H.dev_i32(target), path, count, token)
    sol.tree_commit(shape, [kv.struct()], tree, B, path, count, new_lens, ws.buf)
    paths = [OC.tree_accept(p[:n], d, t)[0] for p, n, d, t in zip(parents, counts, draft, target)]
    assert list(new_lens.cpu().numpy()) == OC.tree_commit(okv, counts, paths)
    assert np.array_equal(H.host_u16(kv.k_pool), okv.k_pool) and np.array_equal(H.host_u16(kv.v_pool), okv.v_pool)

    kv.seq_lens = new_lens
    old = np.zeros((B, 2, mp * 64))
    for step in range(3):
        q1 = synth.normal_bf16(rng, (B, 4, 64), 0.0, 1.0)
        out1 = torch.zeros((B, 4, 64), dtype=torch.bfloat16, device=H.DEV)
        sol.weighted_decode_attn(shape, H.dev_bf16(q1), kv.struct(), B, 0.9, weights, out1, ws.buf, ws.bytes)
        want, mass, err, old, _ = OC.weighted_decode_attn(oshape, q1, kv.to_oracle(), 0.9, old)
        CC.assert_attention(H.host_u16(out1), want, mass, err, step, 2.0 ** -16)
    assert np.allclose(weights.cpu().numpy(), old, rtol=1e-4, atol=1e-6)

    w = weights.cpu().numpy()
    before = kv.to_oracle()
    short = H.dev_i32([0] * B)
    sol.kv_evict(shape, kv.struct(), B, H.dev_i32([70, 40, 100]), weights, kv.page_table, weights, short, None, ws.buf, ws.bytes)
    kept, keys, values = OC.kv_evict(oshape, before, [70, 40, 100], w, 2, 4)
    assert list(short.cpu().numpy()) == [len(x[0]) for x in kept] == [70, 40, 100]
    got = kv.to_oracle()
    for b in range(B):
        for h in range(2):
            j = np.arange(len(kept[b][h]))
            assert np.array_equal(O.bf16_to_f64(got.v_pool[table[b][j // 64], h, j % 64]), values[b][h])
            assert np.abs(O.bf16_to_f64(got.k_pool[table[b][j // 64], h, j % 64]) - keys[b][h]).max() < 0.02

    kv.seq_lens = short + 1  # the next token's slot
    lw = synth.make_layer_weights(cfg, 0)
    h_in = synth.normal_bf16(rng, (B, cfg["d_model"]), 0.0, 1.0)
    r, p, bits = [1000, 500, 1000], [0, 0, 0], [16, 16, 16]
    okv = kv.to_oracle()
    got_out, _, st = H.gpu_layer(shape, H.device_weights(lw, shape), kv, h_in, r, p, bits)
    want_out, _ = O.decode_layer(oshape, H.oracle_weights(lw), okv, O.bf16_to_f64(h_in), r, p, bits)
    m, rel = checker.output_errors(want_out, got_out)
    assert st[0] == 0 and m <= checker.OUT_MAX_ABS and rel <= checker.OUT_REL_L2, (m, rel)
    assert ws.status()[0] == 0 and tws.status()[0] == 0
