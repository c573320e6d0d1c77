"""Evictions one after the other, as a server that stays inside a budget makes them."""
import numpy as np
import pytest
import torch

from oracle import sol_oracle as O
from paper_2605_10875_b200 import binding as sol
from paper_2605_10875_b200 import synth
from tests import cache_cases as CC
from tests import harness as H

pytestmark = pytest.mark.gpu


class Run:
    """Caches at their budgets to which every round adds tokens and out of which it takes as many.  On the host: per slot the key as
    it was when it was added (bf16 bits), the value, and the position it was added at."""

    def __init__(self, heads, lens, theta, in_place, tracked, seed=0, sink=2, window=3):
        self.cfg = CC.config(heads, theta)
        self.shape, self.oshape = H.make_shapes(self.cfg, n_sink=sink, n_window=window)
        self.theta, self.tracked, self.B, self.Hkv, self.hd = theta, tracked, len(lens), self.cfg["n_kv_heads"], self.cfg["head_dim"]
        self.rng = np.random.default_rng(seed)
        self.lens = np.array(lens)
        self.mp = int(-(-(self.lens.max() + 40) // 64))
        pages = self.B * self.mp
        k, v = synth.make_kv_pool(self.cfg, 2 * pages, seed)
        order = self.rng.permutation(2 * pages).astype(np.int32).reshape(2, self.B, self.mp)
        self.tables = [order[0], order[0] if in_place else order[1]]
        self.kv = H.device_kv(k, v, self.tables[0], self.lens.astype(np.int32))
        bits = lambda pool: [[[pool[order[0][b][t // 64], h, t % 64].copy() for t in range(n)] for h in range(self.Hkv)]  # noqa: E731
                             for b, n in enumerate(lens)]
        self.keys, self.values = bits(k), bits(v)
        self.born = [[list(range(n)) for _ in range(self.Hkv)] for n in lens]
        stride = (self.B, self.Hkv, self.mp * 64)
        self.weights = torch.from_numpy(self.rng.exponential(1.0, stride).astype(np.float32)).to(H.DEV)
        self.moved = [torch.zeros(stride, dtype=torch.int32, device=H.DEV) for _ in range(1 if in_place else 2)]
        if not in_place:
            self.moved[1].fill_(-77)  # whatever a fresh array holds
        self.first_keys = torch.full_like(self.kv.k_pool, float("nan")) if tracked else None
        self.ws = H.Workspace(self.shape, self.B, self.mp)
        self.kept = torch.zeros(stride, dtype=torch.int32, device=H.DEV)
        self.now = 0

    def add(self, count):
        """`count` more tokens a sequence, their keys rotated for their slots."""
        table = self.tables[self.now]
        at, k, v = [], [], []
        for b in range(self.B):
            for _ in range(count):
                t = int(self.lens[b])
                new = synth.normal_bf16(self.rng, (2, self.Hkv, self.hd), 0.0, 1.0)
                at.append((int(table[b][t // 64]), t % 64))
                k.append(new[0])
                v.append(new[1])
                for h in range(self.Hkv):
                    self.keys[b][h].append(new[0][h])
                    self.values[b][h].append(new[1][h])
                    self.born[b][h].append(t)
                self.lens[b] += 1
        page, slot = (torch.tensor(x, device=H.DEV) for x in zip(*at))
        self.kv.k_pool[page, :, slot] = H.dev_bf16(np.array(k))
        self.kv.v_pool[page, :, slot] = H.dev_bf16(np.array(v))
        self.kv.seq_lens.copy_(H.dev_i32(self.lens))

    def evict(self, budgets):
        """The weights are drawn anew; the host follows the list of what stays (which other tests check)."""
        self.weights.copy_(torch.from_numpy(self.rng.exponential(1.0, self.weights.shape).astype(np.float32)))
        src, self.now = self.now, self.now ^ 1
        origin = None
        if self.tracked:
            moved = (self.moved[0], self.moved[0]) if len(self.moved) == 1 else (self.moved[src], self.moved[src ^ 1])
            origin = sol.make_key_origin(self.first_keys, *moved)
        lens, table = H.dev_i32([0] * self.B), H.dev_i32(self.tables[self.now])
        more = dict(origin=origin) if self.tracked else {}
        sol.kv_evict(self.shape, self.kv.struct(), self.B, H.dev_i32(budgets), self.weights, table, self.weights, lens, self.kept,
                     self.ws.buf, self.ws.bytes, **more)
        assert self.ws.status()[0] == 0
        kept = self.kept.cpu().numpy()
        self.lens = np.minimum(self.lens, budgets)
        assert np.array_equal(lens.cpu().numpy(), self.lens)
        for b, n in enumerate(self.lens):
            for h in range(self.Hkv):
                for x in (self.keys, self.values, self.born):
                    x[b][h] = [x[b][h][i] for i in kept[b, h, :n]]
        self.kv.page_table, self.kv.seq_lens = table, lens

    def check(self, what):
        """Every slot holds the key as it was added, rotated once by the whole distance and rounded once."""
        got_k, got_v = O.bf16_to_f64(H.host_u16(self.kv.k_pool)), H.host_u16(self.kv.v_pool)
        table = self.tables[self.now]
        for b, n in enumerate(self.lens):
            for h in range(self.Hkv if n else 0):
                j = np.arange(n)
                page, slot = table[b][j // 64], j % 64
                assert np.array_equal(got_v[page, h, slot], np.array(self.values[b][h])), what
                first = O.bf16_to_f64(np.array(self.keys[b][h]))
                x = np.array([O.rope_rotate(k, int(t) - int(p), self.theta) for k, t, p in zip(first, j, self.born[b][h])])
                pair = np.hypot(x, np.roll(x, self.hd // 2, 1))
                # one rounding to bf16, 2^-8 of the value; sine, cosine and products in float32, of the pair's length
                bad = ~(np.abs(got_k[page, h, slot] - x) <= np.abs(x) * 2.0 ** -8 + pair * 2.0 ** -20)
                rel = np.linalg.norm(got_k[page, h, slot] - x) / np.linalg.norm(x)
                assert not bad.any(), (what, b, h, int(bad.sum()), rel)
        if self.tracked:
            moved = self.moved[self.now if len(self.moved) == 2 else 0].cpu().numpy()
            for b, n in enumerate(self.lens):
                assert np.all(moved[b, :, n:] == 0), what  # what comes next into these slots has never been moved
                for h in range(self.Hkv):
                    assert np.array_equal(moved[b, h, :n], np.array(self.born[b][h]) - np.arange(n)), what


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("heads,theta", [("g2", 10000.0), ("g4", 500000.0), ("g1", 500000.0)])
def test_a_token_out_for_a_token_in(heads, theta, in_place):
    """The textbook use of a budget: the keys are as good after 200 evictions as after one."""
    run = Run(heads, [150, 70, 33], theta, in_place, True, seed=1)
    for i in range(200):
        run.add(1)
        run.evict([150, 70, 33])
        if i in (0, 1, 50):
            run.check(i)
    run.check("end")


@pytest.mark.parametrize("in_place", [True, False])
def test_evictions_of_every_size(in_place):
    """Rounds that take out nothing, a few tokens, most of them or all; budgets that grow and shrink; long rows and short ones."""
    run = Run("g8", [3000, 1, 500, 64], 500000.0, in_place, True, seed=2, sink=0, window=0)
    for i, (more, budgets) in enumerate([(0, [3000, 5, 500, 64]), (3, [2990, 2, 100, 60]), (30, [2000, 32, 130, 10]), (1, [2001, 0, 3, 11]),
                                         (20, [64, 20, 23, 0]), (33, [97, 40, 56, 33])]):
        if more:
            run.add(more)
        run.evict(budgets)
        run.check(i)


@pytest.mark.parametrize("heads", ["g2", "g8"])
def test_batches_whose_ctas_share_an_sm(heads):
    lens = [5 + (37 * b * b + 5 * b) % 300 for b in range(70)]
    run = Run(heads, lens, 500000.0, True, True, seed=3, sink=1, window=2)
    for i in range(6):
        run.add(1 + i % 3)
        run.evict([max(5, n - i % 2) for n in lens])
    run.check(heads)


def test_a_captured_run():
    """One eviction as a graph, replayed step by step, against the same steps called one by one."""
    a, b = (Run("g4", [120, 64, 300], 500000.0, True, True, seed=4) for _ in range(2))
    budgets, graph, lens = H.dev_i32([118, 60, 300]), torch.cuda.CUDAGraph(), H.dev_i32([0] * 3)
    origin = sol.make_key_origin(b.first_keys, b.moved[0])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=s):
        sol.kv_evict(b.shape, b.kv.struct(), 3, budgets, b.weights, b.kv.page_table, b.weights, lens, b.kept, b.ws.buf, b.ws.bytes,
                     torch.cuda.current_stream(), origin=origin)
    seq_lens = b.kv.seq_lens  # the words that the graph reads
    for i in range(5):
        for r in (a, b):
            r.add(2)
        a.evict([118, 60, 300])
        b.weights.copy_(torch.from_numpy(b.rng.exponential(1.0, b.weights.shape).astype(np.float32)))
        graph.replay()
        torch.cuda.synchronize()
        seq_lens.copy_(lens)
        b.lens = np.minimum(b.lens, [118, 60, 300])
        assert torch.equal(a.kv.seq_lens, lens) and torch.equal(a.moved[0], b.moved[0])
        assert torch.equal(a.kv.k_pool.view(torch.int16), b.kv.k_pool.view(torch.int16))
        assert torch.equal(a.kv.v_pool.view(torch.int16), b.kv.v_pool.view(torch.int16))
    a.check("run")
