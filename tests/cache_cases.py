"""Inputs and comparisons shared by the tests of the tree and cache-budget calls."""
from __future__ import annotations

import numpy as np
import torch

from oracle import sol_oracle as O
from paper_2605_10875_b200 import binding as sol
from paper_2605_10875_b200 import synth
from tests import harness as H

# (query heads, kv-heads, head_dim): groups of 1, 2, 3, 4, 6 and 8
HEADS = {"g2": (4, 2, 64), "g1": (4, 4, 64), "g3": (12, 4, 64), "g4": (8, 2, 128), "g6": (12, 2, 64), "g8": (16, 2, 128)}


def config(heads, theta=0.0):
    hq, hkv, hd = HEADS[heads]
    return dict(d_model=256, n_q_heads=hq, n_kv_heads=hkv, head_dim=hd, d_ff=1024, rope_theta=theta, shuffle_pages=True)


def make_cache(cfg, lens, seed=0, spare_pages=0):
    """A cache of the given lengths whose slots behind the sequences hold NaN; spare pages at the end of the pool."""
    lens = np.asarray(lens, np.int32)
    table, n = synth.make_page_table(np.maximum(lens, 1), True, seed)
    k, v = synth.make_kv_pool(cfg, n + spare_pages, seed)
    for b, T in enumerate(lens):
        for t in range(int(T), -(-max(int(T), 1) // 64) * 64):
            k[table[b, t // 64], :, t % 64] = v[table[b, t // 64], :, t % 64] = 0x7FC0
    return H.device_kv(k, v, table, lens), n


def poke(pool, table, b, slot, bits):
    """Sets every head's row of a cached token to a bf16 bit pattern."""
    page = int(table[b, slot // 64])
    pool[page, :, slot % 64] = torch.tensor(bits, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).to(pool.device)


def random_trees(rng, counts, N, near=8):
    parents = np.full((len(counts), N), -1, np.int32)
    for b, n in enumerate(counts):
        for i in range(1, n):
            parents[b, i] = rng.integers(max(0, i - near), i)
    return parents


def dev_masks(masks, N):
    out = np.zeros((len(masks), N), np.uint64)
    for b, row in enumerate(masks):
        for i, m in enumerate(row):
            out[b, i] = np.uint64(m)
    return torch.from_numpy(out.view(np.int64)).to(H.DEV)


class TreeWorkspace:
    def __init__(self, shape, B, max_pages, N):
        self.bytes = sol.tree_workspace_bytes(shape, B, max_pages, N)
        assert self.bytes > 0
        self.buf = torch.empty(self.bytes, dtype=torch.uint8, device=H.DEV)
        sol.workspace_init(self.buf, self.bytes)

    def status(self):
        return sol.read_device_status(self.buf)


def assert_attention(got_u16, out, mass, dscore, what, p_rounding=2.0 ** -8):
    """The output is rounded to bf16 (2^-8 of the value); the weights of the products with V may be (p_rounding of each); a score that is off by d
    changes a weight by a factor e^d and the sum by no more; float32 sums of up to a few thousand terms add 2^-18 of the mass."""
    got = O.bf16_to_f64(got_u16)
    nan = np.isnan(out)
    assert np.array_equal(np.isnan(got), nan), what
    tol = np.abs(out) * 2.0 ** -8 + mass * (p_rounding + 2.0 ** -18 + 2.1 * dscore[..., None]) * (1 + 2.0 ** -7) + 1e-38
    bad = ~nan & ~(np.abs(got - out) <= tol)
    assert not bad.any(), (what, int(bad.sum()), float(np.nanmax(np.abs(got - out) / tol)))
