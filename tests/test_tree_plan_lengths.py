"""Chunks of attention over drafted tokens: how long one may be at most."""
import numpy as np
import pytest

from paper_2502_13176_b200 import binding as bk
from paper_2502_13176_b200 import build as bkbuild

LONGEST = 1 << 19


@pytest.fixture(scope="module", autouse=True)
def _built():
    bkbuild.build()


@pytest.mark.parametrize("B", [65536, 1 << 20, 2147483647])
def test_more_sequences_than_a_call_takes(B):
    """Refused as the call refuses them, before a list of billions of chunks is gone through."""
    with pytest.raises(bk.BaklavaError) as e:
        bk.baklava_tree_plan(bk.make_shape(1, 4, 1, 128), [[16]], B, 0, 8)
    assert e.value.code == -7


def test_as_many_as_it_takes():
    assert len(bk.baklava_tree_plan(bk.make_shape(1, 4, 1, 128), [[16]], 65535, 0, 8).items) == 65535


@pytest.mark.parametrize("kv", [bk.KV_BF16, bk.KV_INT4])
@pytest.mark.parametrize("B,caps,chunk", [(148, [[1 << 22]], 0), (1, [[1 << 24, 4096]], 1 << 30), (1, [[1 << 24, 4096]], 0), (300, [[600000, 16]], 0),
                                          (2, [[LONGEST, LONGEST + 16]], 1 << 30), (1, [[2147483376, 16]], 2147483647), (1, [[2147483376, 16]], 0)])
def test_no_chunk_outlasts_a_wait(B, caps, chunk, kv):
    """Some of a block's warps wait from a chunk's beginning to its end; a wait is given up after 10^8 cycles, and a row takes up to 60."""
    caps = np.array(caps)
    H = caps.shape[1]
    plan = bk.baklava_tree_plan(bk.make_shape(1, 4 * H, H, 128), caps, B, 0, 64, chunk_tokens=chunk, kv_dtype=kv)
    items = plan.items
    assert items[:, 2].max() <= LONGEST and 0 < plan.info.chunk_tokens <= LONGEST
    first = items[(items[:, 3] & 0xffff) == 0]
    assert sorted(first[:, 0].tolist()) == list(range(B * H))
    for i in range(H):                                        # and they are all there
        mine = items[items[:, 0] == i]
        assert mine[-1, 1] < caps[0, i] <= int(mine[-1, 1]) + int(mine[-1, 2]) and len(mine) == mine[0, 3] >> 16
