"""Values that only their scales make large, under probabilities far above one: the first rows' logits, which a chunk's probabilities
are taken relative to, lie 2^114 below the others'.  The average of equal values is that value."""
import numpy as np
import pytest
import torch

from oracle import int4 as o4
from paper_2502_13176_b200 import binding as bk
from tests.test_gpu_tree_attn import run
from tests.tree_cases import Held

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kv,T", [("fp8", 2), ("fp8", 40), ("int4", 2)])
def test_scaled_values_beside_a_low_reference(kv, T):
    g, n, high = 4, 200, 4
    sh = bk.make_shape(1, g, 1, 128)
    c = Held(sh, [[208]], 1, kv, [[[n]]], [[[n]]], seed=1, poison=False)
    k_rows, v_scale = torch.zeros((208, 128)), 64.0
    k_rows[100:100 + high, 0] = 7.0                           # the only channel with anything in it
    if kv == "fp8":
        data = torch.stack([k_rows.to(torch.float8_e4m3fn), torch.full((208, 128), 448.0).to(torch.float8_e4m3fn)]).view(torch.uint8)
        scale, value = [[[1.0, 1.0, v_scale, 1 / v_scale]]], 448 * v_scale
        c.cache.kv_scale.copy_(torch.tensor(scale))
    else:
        codes = (k_rows + 8).to(torch.uint8).numpy()
        data = torch.from_numpy(np.stack([o4.pack(codes), o4.pack(np.full((208, 128), 15, np.uint8))]))
        four = torch.ones((1, 1, 4, 128))
        four[:, :, 2], four[:, :, 3] = v_scale, 1 / v_scale
        c.cache.kv_scale.copy_(four)
        c.cache.row_scale.copy_(torch.tensor([1.0, 64.0]).repeat(208, 1))
        value = 7 * 64 * v_scale
    c.cache.k_slab.copy_(data[0])
    c.cache.v_slab.copy_(data[1])
    # logits in powers of two: 7 q log2(e) / sqrt(128).  `high` probabilities of 2^logit add up to 2^117; times the value without its
    # channel's (FP8: the head's) scale 2^126, which fp32 holds, with it 2^132, which it does not
    q0 = torch.tensor(115.0 / (7 * np.log2(np.e) / np.sqrt(128))).bfloat16()
    logit = float(q0) * 7 * np.log2(np.e) / np.sqrt(128)
    assert 2.0 ** 125 < high * 2.0 ** logit * value / v_scale < 2.0 ** 127.9 and high * 2.0 ** logit < 2.0 ** 119
    q = torch.zeros((1, g, T, 128), dtype=torch.bfloat16, device="cuda")
    q[..., 0] = q0
    k = torch.zeros((1, 1, T, 128), dtype=torch.bfloat16, device="cuda")
    v = torch.full((1, 1, T, 128), value, dtype=torch.bfloat16, device="cuda")
    parent = torch.arange(-1, T - 1, dtype=torch.int32, device="cuda").reshape(1, T)
    out, z = run(c, q, k, v, parent, None)
    # all values are alike (and bf16 holds them): what is off is the probabilities' rounding against their sum's terms, 2^-8 of
    # it at most, and the result's own, 2^-8
    assert torch.isfinite(out).all() and (out.double() / value - 1).abs().max() <= 2.0 ** -8 + 2.0 ** -8 + 2.0 ** -15
    want = (logit + np.log2(high)) / np.log2(np.e)            # (the others add 2^-100 of it)
    assert (z.double() - want).abs().max() <= 128 * 2.0 ** -24 * want + 2.0 ** -18 + 2.0 ** -22 * want
