"""Where a sequence goes on after a commit in which one of its heads could not take part."""
import numpy as np
import pytest
import torch

from paper_2502_13176_b200 import binding as bk
from tests.test_gpu_tree_commit import commit, lse_of, nodes_of, paths_of
from tests.tree_cases import Held

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kv,flags", [("bf16", 0), ("bf16", bk.FLAG_NO_SCORE), ("fp8", 0), ("int4", 0), ("bf16", bk.FLAG_NO_EVICT)])
@pytest.mark.parametrize("layer,head", [(0, 0), (0, 1), (1, 0), (1, 1)])
@pytest.mark.parametrize("where,value", [("len", 999), ("free_slot", -1)])
def test_the_other_heads_have_taken_the_path(kv, flags, layer, head, where, value):
    rng = np.random.default_rng(layer * 2 + head)
    sh = bk.make_shape(2, 4, 2, 128)
    B, T = 3, 5
    c = Held(sh, [[64, 48], [80, 96]], B, kv, np.full((B, 2, 2), 20), np.full((B, 2, 2), 20), seed=3)
    q, k, v = nodes_of(rng, sh, B, T)
    path, n = paths_of(rng, B, T, 3, "chain")
    n[2] = 4                                                  # longer than max_path: this sequence is skipped
    lse = lse_of(c, q, k, path, np.minimum(n, 3))
    getattr(c.cache, where)[1, layer, head] = value
    first = [9000, 8000, 7000]
    nxt = commit(c, q, k, v, lse, path, n, 3, first, flags)
    assert int(c.cache.status.item()) == bk.STATUS_BAD_STATE
    assert nxt.tolist() == [9000 + n[0], 8000 + n[1], 7000]
    pos, length = c.cache.pos.cpu().numpy(), c.cache.len.cpu().numpy()
    for b in range(B):
        for l in range(2):
            for h in range(2):
                rows = slice(b * c.stride + int(c.off[l, h]), b * c.stride + int(c.off[l, h]) + int(c.cap[l, h]))
                joined = pos[rows][pos[rows] >= 7000].tolist()
                if b == 2 or (b, l, h) == (1, layer, head):
                    assert joined == [] and (b == 1 and where == "len" or length[b, l, h] == 20)
                else:
                    assert joined == list(range(first[b], first[b] + n[b])) and length[b, l, h] == 20 + n[b]
