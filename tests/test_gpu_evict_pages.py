"""Evictions whose page tables name pages that are not there: those rows stay where they are, and all others move."""
import numpy as np
import pytest

from oracle import cache_ops as OC
from oracle import sol_oracle as O
from tests import harness as H
from tests.test_gpu_cache_budget import Evict

pytestmark = pytest.mark.gpu

BAD_PAGE = 2


def check(c, bad_from, bad_to, what):
    """bad_from, bad_to: (sequence, logical page) that the old and the new table do not have."""
    kept, keys, values = OC.kv_evict(c.oshape, c.old, c.budgets, c.old_w, c.sink, c.window)
    got_k, got_v = O.bf16_to_f64(H.host_u16(c.kv.k_pool)), H.host_u16(c.kv.v_pool)
    table = c.good_table
    written = np.zeros(got_k.shape[:3], bool)
    for b in range(c.B):
        assert int(c.dst_lens[b]) == len(kept[b][0])
        for h, idx in enumerate(kept[b]):
            j = np.arange(len(idx))
            moves = np.array([(b, int(i) // 64) not in bad_from and (b, int(t) // 64) not in bad_to for t, i in zip(j, idx)], bool)
            page, slot = table[b][j // 64][moves], (j % 64)[moves]
            written[page, h, slot] = True
            src = c.old.v_pool[c.old.page_table[b][idx // 64], h, idx % 64]
            assert np.array_equal(got_v[page, h, slot], src[moves]), (what, b, h)
            x = keys[b][h]
            pair = np.hypot(x, np.roll(x, x.shape[1] // 2, 1))
            assert np.all(np.abs(got_k[page, h, slot] - x[moves]) <= (np.abs(x) * 2.0 ** -8 + pair * 2.0 ** -20)[moves]), (what, b, h)
            assert moves.any() and not moves.all() or not any(y[0] == b for y in (*bad_from, *bad_to)), (what, b, h)
    for got, old in ((H.host_u16(c.kv.k_pool), c.old.k_pool), (got_v, c.old.v_pool)):
        assert np.array_equal(got[~written], old[~written]), what  # what has no page is where it was, and nothing else was written
    w = c.dst_w.cpu().numpy()
    for b in range(c.B):  # the weights and the list are as if all pages were there
        for h, idx in enumerate(kept[b]):
            assert np.array_equal(w[b, h, : len(idx)], c.old_w[b, h, idx])
            assert np.array_equal(c.kept.cpu().numpy()[b, h, : len(idx)], idx)


@pytest.mark.parametrize("theta", [0.0, 500000.0])
@pytest.mark.parametrize("heads,lens,budgets", [("g2", [200, 130], [150, 100]), ("g4", [6000, 300], [4000, 250]), ("g8", [3000, 64, 700], [1500, 60, 690])])
@pytest.mark.parametrize("side,in_place", [("old", False), ("new", False), ("old", True)])
def test_rows_without_a_page_stay(heads, lens, budgets, theta, side, in_place):
    """The bad page early and in the middle of a row longer than the ring; numbers below zero, just behind the pool and far behind it."""
    c = Evict(heads, lens, budgets, theta=theta, in_place=in_place, seed=5)
    at = [(0, 1), (0, (budgets[0] // 64) // 2)] + ([(1, 0)] if lens[1] > 64 else [])
    if in_place:
        c.dst_table = c.kv.page_table  # one table: a page that is missing is missing on both sides
    c.good_table = c.dst_table.cpu().numpy().copy()
    for n, (b, p) in enumerate(at):
        (c.kv.page_table if side == "old" else c.dst_table)[b, p] = (-1, c.kv.num_pages, 2**31 - 1)[n]
    c.launch()
    assert c.ws.status()[0] == BAD_PAGE
    check(c, at if side == "old" else [], at if side == "new" or in_place else [], (heads, theta, in_place, side))
