"""The decode step, the attention that keeps its weights and the eviction in one workspace, one after the other: each leaves there what the
next does not mind."""
import numpy as np
import pytest
import torch

from oracle import checker
from oracle import sol_oracle as O
from paper_2605_10875_b200 import binding as sol
from paper_2605_10875_b200 import synth
from tests import harness as H

pytestmark = pytest.mark.gpu

CFG = dict(synth.WORKLOADS["tiny"], rope_theta=10000.0)


class Server:
    """A layer over a cache with a budget; `shared` or not: with a workspace of its own for every call."""

    def __init__(self, lens, shared, select, seed=1):
        quest = dict(token_select=sol.SELECT_QUEST_PAGES, quest_page_size=8) if select else {}
        self.shape, self.oshape = H.make_shapes(CFG, n_sink=2, n_window=4, **quest)
        self.B, self.mp, self.select = len(lens), -(-(max(lens) + 20) // 64), select
        pages = self.B * self.mp
        rng = np.random.default_rng(seed)
        table = rng.permutation(pages).astype(np.int32).reshape(self.B, self.mp)
        self.kv = H.device_kv(*synth.make_kv_pool(CFG, pages, seed), table, np.asarray(lens, np.int32))
        if select:
            self.kv.build_quest_meta(self.shape, self.B)
        self.layer = synth.make_layer_weights(CFG, 0)
        self.w = H.device_weights(self.layer, self.shape)
        self.weights = torch.from_numpy(rng.exponential(1.0, (self.B, 2, self.mp * 64)).astype(np.float32)).to(H.DEV)
        self.one = H.Workspace(self.shape, self.B, self.mp) if shared else None
        self.rng = rng

    def ws(self):
        return self.one or H.Workspace(self.shape, self.B, self.mp)

    def decode(self):
        self.kv.seq_lens += 1
        h = synth.normal_bf16(self.rng, (self.B, CFG["d_model"]), 0.0, 1.0)
        okv = self.kv.to_oracle()
        act = [300] * self.B, [0] * self.B, [16] * self.B
        got, _, st = H.gpu_layer(self.shape, self.w, self.kv, h, *act, ws=self.ws(), trace=False)
        quest = dict(token_select=O.SELECT_QUEST_PAGES, quest_page_size=8) if self.select else {}
        want, _ = O.decode_layer(self.oshape, H.oracle_weights(self.layer), okv, O.bf16_to_f64(h), *act, **quest)
        m, rel = checker.output_errors(want, got)
        assert st[0] == 0 and rel <= checker.OUT_REL_L2, (m, rel)
        return got

    def weigh(self):
        q, ws = H.dev_bf16(synth.normal_bf16(self.rng, (self.B, 4, 64), 0.0, 1.0)), self.ws()
        out = torch.zeros((self.B, 4, 64), dtype=torch.bfloat16, device=H.DEV)
        sol.weighted_decode_attn(self.shape, q, self.kv.struct(), self.B, 0.9, self.weights, out, ws.buf, ws.bytes)
        assert ws.status()[0] == 0
        return H.host_u16(out)

    def evict(self, budgets):
        lens, ws = H.dev_i32([0] * self.B), self.ws()
        sol.kv_evict(self.shape, self.kv.struct(), self.B, H.dev_i32(budgets), self.weights, self.kv.page_table, self.weights, lens,
                     None, ws.buf, ws.bytes)
        assert ws.status()[0] == 0
        self.kv.seq_lens = lens
        if self.select:
            sol.quest_build_meta(self.shape, self.kv.struct(), self.B)


@pytest.mark.parametrize("select", [False, True])
@pytest.mark.parametrize("lens", [[150, 64, 201], [9000, 3, 500, 40]])
def test_every_order_in_one_workspace(lens, select):
    """Against the oracle for the layer, and bit for bit against the same calls with a workspace of their own each."""
    a, b = (Server(lens, shared, select) for shared in (True, False))
    for s in "dwdewdwwedd":
        results = []
        for x in (a, b):
            results.append(x.decode() if s == "d" else x.weigh() if s == "w" else x.evict([max(10, int(n) * 3 // 4) for n in x.kv.seq_lens]))
        if s != "e":
            assert np.array_equal(*results), s
        for y in ("k_pool", "v_pool"):
            assert torch.equal(getattr(a.kv, y).view(torch.int16), getattr(b.kv, y).view(torch.int16)), s
        assert torch.equal(a.weights, b.weights) and torch.equal(a.kv.seq_lens, b.kv.seq_lens)
