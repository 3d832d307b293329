"""What follows a call in which no tree has a row to be written begins behind it: it may take the same workspace."""
import numpy as np
import pytest
import torch

from paper_2502_13176_b200 import binding as bk
from tests.tree_cases import bf16_normal

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("why", ["a tree that cannot be", "no nodes", "a tree that cannot be among empty sequences"])
def test_the_next_call_on_the_same_workspace(why):
    rng = np.random.default_rng(3)
    B, T = (3 if "among" in why else 1), 16
    sh = bk.make_shape(1, 32, 8, 128)
    caps = np.full((1, 8), 100000, dtype=np.int32)            # long enough for the first kernel to take a hundred microseconds
    off = np.arange(8, dtype=np.int64).reshape(1, 8) * 100000
    c = bk.Cache(sh, caps, off, 800000, B)
    gen = torch.Generator(device="cuda").manual_seed(4)
    for slab in (c.k_slab, c.v_slab):
        slab.normal_(generator=gen)
    c.len.fill_(99999)
    c.free_slot.fill_(99999)
    q, other = (bf16_normal(rng, (B, 32, T, 128)).cuda() for _ in range(2))
    k, v = (bf16_normal(rng, (B, 8, T, 128)).cuda() for _ in range(2))
    good = torch.arange(-1, T - 1, dtype=torch.int32, device="cuda").repeat(B, 1)
    bad, nodes = good.clone(), None
    if "cannot" in why:
        bad[-1, 3] = 7
    if "no nodes" in why:
        nodes = torch.zeros((B,), dtype=torch.int32, device="cuda")
    elif "among" in why:
        nodes = torch.tensor([0, 0, T], dtype=torch.int32, device="cuda")
    plan = bk.baklava_tree_plan(sh, caps, B, 0, T).to("cuda")
    ws, fresh = (bk.decode_workspace(plan) for _ in range(2))
    want, out = torch.zeros_like(q), torch.zeros_like(q)
    wz, z = (torch.zeros((B, 32, T), device="cuda") for _ in range(2))
    bk.baklava_tree_attn(sh, c, q, k, v, good, None, want, wz, plan, fresh)
    for _ in range(10):
        bk.baklava_tree_attn(sh, c, other, k, v, bad, nodes, out, z, plan, ws)
        bk.baklava_tree_attn(sh, c, q, k, v, good, None, out, z, plan, ws)
        assert torch.equal(out, want) and torch.equal(z, wz)
    assert int(c.status.item()) == (bk.STATUS_BAD_STATE if "cannot" in why else 0)
