"""The attention of drafted trees with its weights in two bf16 parts: for few query rows always, for many as the caller chooses."""
import numpy as np
import numpy as np
import pytest

from oracle import cache_ops as OC
from paper_2605_10875_b200 import binding as sol
from oracle import sol_oracle as O
from tests import cache_cases as CC
from tests import harness as H
from tests.test_gpu_tree import Case

pytestmark = pytest.mark.gpu

TWO_PARTS = 2.0 ** -16  # of a weight in the products with V: the high part is off by 2^-8 of it, the low part by 2^-8 of that


def check(c, what, parts=2):
    sol.tree_attn(c.shape, c.dq, c.kv.struct(), sol.make_tree(c.N, c.n_nodes, c.dmask, parts), c.B, c.out, c.ws.buf, c.ws.bytes)
    got = H.host_u16(c.out)
    assert c.ws.status()[0] == 0
    out, mass, err = OC.tree_attn(c.oshape, c.q, c.kv.to_oracle(), c.counts, c.masks)
    for b, n in enumerate(c.counts):
        CC.assert_attention(got[b, :n], out[b, :n], mass[b, :n], err[b, :n], (what, b), TWO_PARTS)


@pytest.mark.parametrize("heads,n", [("g4", 1), ("g4", 2), ("g2", 7), ("g1", 9), ("g4", 4), ("g8", 2),  # up to 16 query rows
                                     ("g4", 5), ("g4", 8), ("g1", 32),       # ... 32
                                     ("g4", 9), ("g2", 32), ("g1", 33),      # ... 64
                                     ("g4", 17), ("g8", 9), ("g6", 21),      # ... 128
                                     ("g4", 33), ("g8", 32), ("g4", 64),     # ... 256
                                     ("g8", 33), ("g8", 64)])                # two blocks
def test_weights_keep_two_parts(heads, n):
    """Sizes on both sides of every change of form, short contexts (few weights: no rounding averages out) and cut chains."""
    check(Case(heads, [0, 1, 63, 130, 700], [n] * 5, n, seed=n), (heads, n))


@pytest.mark.parametrize("heads,n", [("g4", 4), ("g4", 7), ("g2", 25), ("g4", 30), ("g4", 64)])
def test_weights_keep_two_parts_in_cut_chains(heads, n):
    check(Case(heads, [6000], [n], n, seed=n + 1), (heads, n))


@pytest.mark.parametrize("heads,n", [("g4", 1), ("g2", 4), ("g4", 2), ("g2", 7), ("g1", 9), ("g4", 4), ("g8", 2), ("g6", 2)])
def test_few_query_rows_have_both_parts_in_any_case(heads, n):
    check(Case(heads, [0, 1, 63, 130, 700, 6000], [n] * 6, n, seed=n), (heads, n), 1)


@pytest.mark.parametrize("n", [7, 14, 25, 40])
def test_masks_infinities_and_empty_rows_with_two_parts(n):
    """What the mask hides may hold anything, with two parts too; rows that see nothing are zero."""
    masks = [[(1 << i) | (4 if i in (2, 5) else 0) for i in range(n)], [0, 1] + [0] * (n - 2)]
    c = Case("g4", [100, 0], [n, n], n, seed=3, masks=masks)
    CC.poke(c.kv.v_pool, c.kv.page_table.cpu().numpy(), 0, 102, 0x7F80)
    sol.tree_attn(c.shape, c.dq, c.kv.struct(), sol.make_tree(n, c.n_nodes, c.dmask, 2), 2, c.out, c.ws.buf, c.ws.bytes)
    got = H.host_u16(c.out)
    with np.errstate(all="ignore"):
        out, mass, err = OC.tree_attn(c.oshape, c.q, c.kv.to_oracle(), c.counts, c.masks)
    for i in range(n):
        if i in (2, 5):
            assert np.all(got[0, i] == 0x7F80)
        else:
            CC.assert_attention(got[0, i], out[0, i], mass[0, i], err[0, i], i, TWO_PARTS)
    CC.assert_attention(got[1], out[1], mass[1], err[1], n, TWO_PARTS)
    assert not got[1, 0].any() and not got[1, 2:].any()


def test_outputs_that_cancel():
    """Two tokens with opposite values and nearly equal weights: what is left is what one part of the weights would lose."""
    for n in (3, 5, 12, 20, 40):
        c = Case("g4", [2], [n], n, seed=n, masks=[[0] * n])
        k, v = c.kv.k_pool, c.kv.v_pool
        page = int(c.kv.page_table[0, 0])
        k[page, :, 1] = k[page, :, 0]
        k[page, :, 1, 0] += 0.5
        v[page, :, 1] = -v[page, :, 0]
        check(c, n)
