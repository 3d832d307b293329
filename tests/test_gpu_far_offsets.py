"""Elements past the 2^31st and rows of 4-bit slabs past the 2^31st byte: the same bits as from tensors that lie close."""
import numpy as np
import pytest
import torch

from paper_2502_13176_b200 import binding as bk

pytestmark = pytest.mark.gpu


def far(x, stride, axis):
    """A copy of x [B, H, T, D] whose `axis` (0 .. 2) steps by `stride` elements."""
    order = [a for a in range(3) if a != axis]
    st = [0, 0, 0, 1]
    st[order[1]] = x.shape[3]
    st[order[0]] = x.shape[3] * x.shape[order[1]]
    st[axis] = stride
    room = torch.empty((x.shape[axis] - 1) * stride + x[0, 0].numel() * x.shape[0] * x.shape[1], dtype=x.dtype, device=x.device)
    view = room.as_strided(x.shape, st)
    view.copy_(x)
    return view


# (extent, stride) of the axis that reaches past 2^31 elements
@pytest.mark.parametrize("axis,shape,stride", [(2, (1, 4, 300, 128), 8_000_000), (1, (1, 16, 200, 64), 160_000_000), (0, (9, 2, 70, 128), 280_000_000)])
def test_prompt_attention_and_norm_rope(axis, shape, stride):
    B, Hq, T, D = shape
    Hkv = Hq // 2
    g = torch.Generator(device="cuda").manual_seed(axis)
    q, k, v = (torch.randn((B, h, T, D), generator=g, device="cuda").bfloat16() for h in (Hq, Hkv, Hkv))
    sh, status = bk.make_shape(1, Hq, Hkv, D), torch.zeros(1, dtype=torch.int32, device="cuda")
    pos = torch.arange(T, dtype=torch.int32, device="cuda").repeat(B, 1)
    freq = (10000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)).float().cuda()
    near = [torch.zeros_like(x) for x in (q, q, k)]
    bk.baklava_prefill_attn(sh, q, k, v, None, near[0], None, status)
    bk.baklava_qk_norm_rope(sh, q, k, pos, freq, None, None, 0.0, near[1], near[2])
    # the keys have fewer heads: their head axis takes twice the stride
    qs, ks = stride, stride * (Hq // Hkv) if axis == 1 else stride
    fq, fk = far(q, qs, axis), far(k, ks, axis)
    out = far(torch.zeros_like(q), qs, axis)
    bk.baklava_prefill_attn(sh, fq, fk, v, None, out, None, status)
    assert torch.equal(out, near[0])
    fv = far(v, ks, axis)
    out.zero_()
    bk.baklava_prefill_attn(sh, q, k, fv, None, out, None, status)
    assert torch.equal(out, near[0])
    del fv
    ko = far(torch.zeros_like(k), ks, axis)
    bk.baklava_qk_norm_rope(sh, fq, fk, pos, freq, None, None, 0.0, out, ko)
    assert torch.equal(out, near[1]) and torch.equal(ko, near[2])
    if axis == 2:                                            # the same as packed prompts
        cu = torch.tensor([0, 130, T], dtype=torch.int32, device="cuda")
        a, z = near[0][0], out[0]
        bk.baklava_prefill_attn_packed(sh, q[0], k[0], v[0], cu, T, a, None, status)
        bk.baklava_prefill_attn_packed(sh, fq[0], fk[0], v[0], cu, T, z, None, status)
        assert torch.equal(a, z)
    assert int(status.item()) == 0


@pytest.mark.parametrize("g", [2, 7])
def test_4bit_slabs(g):
    # the second sequence's rows begin at row 40 000 000: byte 2.56e9 of a slab, element 5.1e9 of what it stands for
    L, Hkv, B, D, T, steps = 1, 2, 2, 128, 300, 40
    sh, caps = bk.make_shape(L, g * Hkv, Hkv, D), np.array([[320, 208]], dtype=np.int32)
    off = np.array([[0, 320]], dtype=np.int64)
    gen = torch.Generator(device="cuda").manual_seed(g)
    four = np.ones((L, Hkv, 4, D), np.float32)
    k, v = (torch.randn((B, Hkv, T, D), generator=gen, device="cuda").bfloat16() for _ in range(2))
    score = torch.rand((B, Hkv, T), generator=gen, device="cuda")
    feeds = [[torch.randn((L, B, h, D), generator=gen, device="cuda").bfloat16() for h in (g * Hkv, Hkv, Hkv)] for _ in range(steps)]
    states = []
    for stride in (528, 40_000_000):
        cache = bk.Cache(sh, caps, off, stride, B, kv_dtype=bk.KV_INT4, kv_scale=four)
        ews = torch.empty((bk.baklava_evict_workspace_size(sh, B, 1, T),), dtype=torch.uint8, device="cuda")
        bk.baklava_evict(sh, cache, 0, 1, k, v, score, T, 0, Hkv * T, T, 1, ews)
        plan = bk.baklava_decode_plan(sh, caps, B, 0, 1, stride, chunk_tokens=64, kv_dtype=bk.KV_INT4).to("cuda")
        ws = bk.decode_workspace(plan)
        outs = []
        for i, (q, kn, vn) in enumerate(feeds):
            out = torch.zeros((L, B, g * Hkv, D), dtype=torch.bfloat16, device="cuda")
            bk.baklava_decode_attn(sh, cache, q, kn, vn, T + i, out, None, 0, plan, ws)
            outs.append(out)
        # in place, the moves inside a slab too
        bk.baklava_evict(sh, cache, 0, 1, None, None, None, 320, 0, 0, 0, 40, ews.new_empty(bk.baklava_evict_workspace_size(sh, B, 1, 320)))
        assert int(cache.status.item()) == 0
        rows = torch.cat([torch.arange(b * stride, b * stride + 528, device="cuda") for b in range(B)])
        n = torch.cat([torch.arange(c, device="cuda") < int(cache.len[b, 0, h]) for b in range(B) for h, c in enumerate(caps[0])])
        rows = rows[n]
        states.append((torch.stack(outs), cache.len, cache.free_slot,
                       *(x[rows] for x in (cache.k_slab, cache.v_slab, cache.row_scale, cache.pos, cache.score))))
        del cache, ws
    assert int(states[0][1].sum()) == 2 * (280 + 168)
    for a, z in zip(*states):
        assert torch.equal(a, z)
