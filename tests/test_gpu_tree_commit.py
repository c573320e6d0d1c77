"""sol_tree_commit beyond the ordinary path: counts and lengths out of range."""
import numpy as np
import pytest
import torch

from oracle import cache_ops as OC
from oracle import sol_oracle as O
from paper_2605_10875_b200 import binding as sol
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
