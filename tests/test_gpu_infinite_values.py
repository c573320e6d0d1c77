"""Infinities in the values of cached tokens: an element of the output is infinite where a token that its row sees is, NaN where NaN or
both infinities meet, and a number elsewhere, whatever form of the dense attention a call takes."""
import numpy as np
import pytest
import torch

from oracle import cache_ops as OC
from oracle import sol_oracle as O
from paper_2605_10875_b200 import binding as sol
from tests import cache_cases as CC
from tests import harness as H
from tests.test_gpu_cache_budget import Weighted
from tests.test_gpu_tree import Case

pytestmark = pytest.mark.gpu

PLUS, MINUS, NAN = 0x7F80, 0xFF80, 0x7FC0


def put(kv, b, slot, col, bits):
    """In one column of every head's value."""
    page = int(kv.page_table[b, slot // 64])
    kv.v_pool.view(torch.int16)[page, :, slot % 64, col] = int(np.array(bits, np.uint16).view(np.int16))


def put_some(kv, b, C, n):
    """Columns with one infinity in the context, with both, with infinities of one sign far apart, with NaN beside one; in node 0."""
    for slot, col, bits in ((0, 1, PLUS), (C - 1, 2, MINUS), (C // 2, 5, PLUS), (C // 3, 5, MINUS), (0, 9, MINUS), (C - 1, 9, MINUS),
                            (C // 2, 30, NAN), (3, 30, PLUS), (C // 2, 63, PLUS), (C // 3, 40, NAN)):
        put(kv, b, slot, col, bits)
    if n:  # a node that only some rows see: alone in its column, beside its like, and against the context
        put(kv, b, C, 11, MINUS)
        put(kv, b, C, 1, PLUS)
        put(kv, b, C, 2, PLUS)


def check(got, out, mass, err, what, p_rounding):
    bad = ~np.isfinite(out)
    got = O.bf16_to_f64(got)
    assert np.array_equal(got[bad], out[bad], equal_nan=True), what
    assert np.isfinite(got[~bad]).all(), what
    tol = np.where(bad, 0, np.abs(np.where(bad, 0, out)) * 2.0 ** -8 +
                   np.where(bad, 0, mass) * (p_rounding + 2.0 ** -18 + 2.1 * err[..., None]) * (1 + 2.0 ** -7) + 1e-38)
    assert np.all(np.abs(np.where(bad, 0, got) - np.where(bad, 0, out)) <= tol), what


@pytest.mark.parametrize("heads,n", [("g4", 1), ("g4", 2), ("g4", 4), ("g1", 9), ("g4", 8), ("g4", 16), ("g2", 17), ("g4", 32), ("g4", 64),
                                     ("g8", 64)])
def test_trees(heads, n):
    """On both sides of every change of form: 4, 8, 16, 32, 64, 128, 256 query rows, two blocks."""
    contexts = [70, 5, 300, 4000, 200]
    masks = [[(1 << i) | (1 if i % 2 else 0) for i in range(n)]] * 5
    c = Case(heads, contexts, [n] * 5, n, seed=n, masks=masks)
    for b, C in enumerate(contexts[:4]):
        put_some(c.kv, b, C, n)
    c.launch()
    assert c.ws.status()[0] == 0
    with np.errstate(all="ignore"):
        out, mass, err = OC.tree_attn(c.oshape, c.q, c.kv.to_oracle(), c.counts, c.masks)
    assert np.isfinite(out[4]).all() and np.isposinf(out).any() and np.isneginf(out).any() and np.isnan(out).any()
    check(H.host_u16(c.out), out, mass, err, (heads, n), 2.0 ** -8)


@pytest.mark.parametrize("n", [3, 30])
def test_a_long_cut_chain(n):
    c = Case("g4", [20000], [n], n, seed=2)
    put_some(c.kv, 0, 20000, 0)
    c.launch()
    with np.errstate(all="ignore"):
        out, mass, err = OC.tree_attn(c.oshape, c.q, c.kv.to_oracle(), c.counts, c.masks)
    check(H.host_u16(c.out), out, mass, err, n, 2.0 ** -8)


@pytest.mark.parametrize("heads", sorted(CC.HEADS))
def test_decode_steps_with_weights(heads):
    lens = [1, 40, 64, 200, 3000]
    c = Weighted(heads, lens, seed=3)
    for b, T in enumerate(lens[1:], 1):
        put_some(c.kv, b, T - 1, 0)
        put(c.kv, b, T - 1, 20, MINUS)  # the newest token
    c.launch()
    assert c.ws.status()[0] == 0
    with np.errstate(all="ignore"):
        out, mass, err, new, _ = OC.weighted_decode_attn(c.oshape, c.q, c.kv.to_oracle(), c.decay, c.old)
    check(H.host_u16(c.out), out, mass, err, heads, 2.0 ** -16)
    w = c.weights.cpu().numpy()
    for b, T in enumerate(lens):
        assert np.allclose(w[b, :, :T], new[b, :, :T], rtol=1e-4, atol=1e-6)  # weights know nothing of values


@pytest.mark.parametrize("n", [2, 7, 20, 50])
def test_scores_that_are_no_numbers_stay_nan(n):
    """A context key of NaN: every weight of its head's rows is NaN, whatever the values are."""
    c = Case("g4", [150, 100], [n, n], n, seed=4)
    CC.poke(c.kv.k_pool, c.kv.page_table.cpu().numpy(), 0, 33, NAN)
    put_some(c.kv, 0, 150, 0)
    c.launch()
    got = O.bf16_to_f64(H.host_u16(c.out))
    assert np.isnan(got[0]).all() and np.isfinite(got[1]).all()


@pytest.mark.parametrize("nodes", [0, 1, 24])
def test_the_longest_pieces(nodes):
    """The longest contexts, so many of them that a CTA has whole ones: all the values of a piece are looked through, and nobody who waits
    meanwhile gives up.  (The sequences share their pages, which are only read.)"""
    cfg = CC.config("g2")
    shape, _ = H.make_shapes(cfg)
    B, pages = 128, 768
    T = pages * 64
    gen = torch.Generator(device=H.DEV).manual_seed(1)
    k, v = (torch.empty((pages, 2, 64, 64), dtype=torch.bfloat16, device=H.DEV).normal_(generator=gen) for _ in range(2))
    v[5, :, 7, 3] = float("inf")
    v[700, :, 1, 8] = -float("inf")
    v[701, 0, 1, 8] = float("nan")
    table = torch.arange(pages, dtype=torch.int32, device=H.DEV).repeat(B, 1)
    kv = H.DeviceKV(k, v, table, H.dev_i32([T] * B), pages, pages)
    q = torch.empty((B, max(1, nodes), 4, 64), dtype=torch.bfloat16, device=H.DEV).normal_(generator=gen)
    out = torch.zeros_like(q)
    if nodes:
        mask = torch.full((B, nodes), -1, dtype=torch.int64, device=H.DEV)
        ws = CC.TreeWorkspace(shape, B, pages, nodes)
        sol.tree_attn(shape, q, kv.struct(), sol.make_tree(nodes, H.dev_i32([nodes] * B), mask), B, out, ws.buf, ws.bytes)
    else:
        ws = H.Workspace(shape, B, pages)
        weights = torch.zeros((B, 2, T), device=H.DEV)
        sol.weighted_decode_attn(shape, q, kv.struct(), B, 1.0, weights, out, ws.buf, ws.bytes)
    assert ws.status()[0] == 0
    got = out.float()
    assert torch.isposinf(got[..., 3]).all() and torch.isnan(got[:, :, :2, 8]).all() and torch.isneginf(got[:, :, 2:, 8]).all()
    rest = [c for c in range(64) if c not in (3, 8)]
    assert torch.isfinite(got[..., rest]).all()
