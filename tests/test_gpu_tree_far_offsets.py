"""Drafted tokens over slabs, tensors and probabilities whose elements lie past the 2^31st: the same bits as where they lie close.  And a
head of more rows than a chunk may have."""
import numpy as np
import pytest
import torch

from paper_2502_13176_b200 import binding as bk
from tests.test_gpu_far_offsets import far

pytestmark = pytest.mark.gpu


# rows between the sequences: the second one's begin at element 2.3e9 (FP8: byte; 4 bits: byte 2.4e9, element 4.9e9) of a slab
@pytest.mark.parametrize("kv,D,stride", [(bk.KV_BF16, 128, 18_000_000), (bk.KV_BF16, 64, 36_000_000), (bk.KV_FP8_E4M3, 128, 18_000_000),
                                         (bk.KV_INT4, 128, 38_000_000)])
def test_slabs(kv, D, stride):
    Hkv, g, B, T, caps = 2, 4, 2, 12, np.array([[1504, 304]], dtype=np.int32)
    sh, off = bk.make_shape(1, g * Hkv, Hkv, D), np.array([[0, 1504]], dtype=np.int64)
    rng = np.random.default_rng(D)
    scale = {bk.KV_FP8_E4M3: np.array([[[0.25, 4.0, 0.25, 4.0]] * Hkv]), bk.KV_INT4: np.ones((1, Hkv, 4, D))}.get(kv)
    width = D // 2 if kv == bk.KV_INT4 else D
    if kv == bk.KV_BF16:
        data = torch.from_numpy(rng.normal(0, 1, (2, B, 1808, D)).astype(np.float32)).bfloat16().cuda()
    else:
        data = torch.from_numpy(rng.integers(0x11 if kv == bk.KV_INT4 else 0, 0x60, (2, B, 1808, width)).astype(np.uint8)).cuda()
    score = torch.from_numpy(rng.random((B, 1808)).astype(np.float32)).cuda()
    rs = torch.from_numpy(rng.uniform(0.1, 0.3, (B, 1808, 2)).astype(np.float32)).cuda()
    q, k, v = (torch.from_numpy(rng.normal(0, 1, (1, B, h, T, D)).astype(np.float32)).bfloat16().cuda() for h in (g * Hkv, Hkv, Hkv))
    i32 = lambda x: torch.as_tensor(np.asarray(x), dtype=torch.int32).cuda()                  # noqa: E731
    parent, path, n = i32([np.arange(T) - 1] * B), i32([list(range(5)) + [-1] * (T - 5)] * B), i32([5, 4])
    states = []
    for st in (1808, stride):
        c = bk.Cache(sh, caps, off, st, B, kv_dtype=kv, kv_scale=scale)
        at = torch.cat([torch.arange(b * st, b * st + 1808, device="cuda") for b in range(B)])
        for b in range(B):
            here = slice(b * st, b * st + 1808)
            c.k_slab[here], c.v_slab[here], c.score[here] = data[0, b], data[1, b], score[b]
            c.pos[here] = torch.arange(1808, dtype=torch.int32, device="cuda")
            if kv == bk.KV_INT4:
                c.row_scale[here] = rs[b]
        c.len[:] = i32([[1503, 303]])
        c.free_slot[:] = i32([[700, 303]])
        plan = bk.baklava_tree_plan(sh, caps, B, 0, T, kv_dtype=kv).to("cuda")
        out, lse = torch.zeros_like(q[0]), torch.zeros((1, B, g * Hkv, T), device="cuda")
        bk.baklava_tree_attn(sh, c, q[0], k[0], v[0], parent, None, out, lse[0], plan, bk.decode_workspace(plan))
        plan = bk.baklava_decode_plan(sh, caps, B, 0, 1, st, kv_dtype=kv).to("cuda")
        nxt, t_pos = i32([0, 0]), i32([5000, 6000])
        bk.baklava_tree_commit(sh, c, q, k, v, lse, path, n, 5, t_pos, nxt, 0, plan, bk.tree_commit_workspace(sh, plan, 5))
        assert int(c.status.item()) == 0 and nxt.tolist() == [5005, 6004]
        assert c.len.flatten().tolist() == [1503, 303] * 2
        live = torch.ones((B, 1808), dtype=torch.bool, device="cuda")
        for b in range(B):
            live[b, int(c.free_slot[b, 0, 0])] = live[b, 1504 + int(c.free_slot[b, 0, 1])] = False
        rows = at[live.flatten()]
        states.append([out, lse, c.free_slot.clone()] + [x[rows].clone() for x in (c.k_slab, c.v_slab, c.pos, c.score) + (() if c.row_scale is None else (c.row_scale,))])
        del c
    assert all(torch.equal(a, z) for a, z in zip(*states))


@pytest.mark.parametrize("axis,stride", [(0, 2_400_000_000), (1, 320_000_000), (2, 240_000_000)])
def test_tensors(axis, stride):
    """Queries, keys and values of the nodes, and the rows out, at such distances along each axis."""
    sh, caps = bk.make_shape(1, 8, 8, 64), np.full((1, 8), 64, dtype=np.int32)
    B, T = 2, 11
    rng = np.random.default_rng(axis)
    q, k, v = (torch.from_numpy(rng.normal(0, 1, (B, 8, T, 64)).astype(np.float32)).bfloat16().cuda() for _ in range(3))
    c = bk.Cache(sh, caps, np.arange(8, dtype=np.int64).reshape(1, 8) * 64, 512, B)
    for slab in (c.k_slab, c.v_slab):
        slab.copy_(torch.from_numpy(rng.normal(0, 1, (1024, 64)).astype(np.float32)))
    c.len.fill_(50)
    c.free_slot.fill_(50)
    parent = torch.arange(-1, T - 1, dtype=torch.int32, device="cuda").repeat(B, 1)
    plan = bk.baklava_tree_plan(sh, caps, B, 0, T).to("cuda")
    ws, near, z = bk.decode_workspace(plan), torch.zeros_like(q), torch.zeros((B, 8, T), device="cuda")
    bk.baklava_tree_attn(sh, c, q, k, v, parent, None, near, z, plan, ws)
    for which in range(4):
        a = [q, k, v, torch.zeros_like(q)]
        a[which] = far(a[which], stride, axis)
        bk.baklava_tree_attn(sh, c, *a[:3], parent, None, a[3], z, plan, ws)
        assert torch.equal(a[3], near), which
        del a
    assert int(c.status.item()) == 0


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
def test_probabilities(kind):
    """33 rows of 151 669 tokens, 70 million elements apart."""
    B, T, V, stride = 3, 11, 151669, 70_000_000
    gen = torch.Generator(device="cuda").manual_seed(3)
    near = [torch.softmax(2 * torch.randn((B, T, V), generator=gen, device="cuda"), -1).to(kind) for _ in range(2)]
    room = torch.empty(B * T * stride, dtype=kind, device="cuda")
    away = []
    for i, x in enumerate(near):                              # both in the same room, in turn
        y = room[i * 1_000_000:].as_strided((B, T, V), (T * stride, stride, 1))
        y.copy_(x)
        away.append(y)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")                         # noqa: E731
    parent = torch.tensor([-1, 0, 0, 0, 1, 1, 2, 2, 3, 3, 4], dtype=torch.int32, device="cuda").repeat(B, 1)
    tokens = torch.randint(0, V, (B, T), generator=gen, device="cuda", dtype=torch.int32)
    ua, us = torch.rand((B, T), generator=gen, device="cuda"), torch.rand((B,), generator=gen, device="cuda")
    got = []
    for target, draft in (near, away, (near[0], None), (away[0], None)):
        got.append([i32(B, T), i32(B), i32(B), i32(1)])
        bk.baklava_tree_verify(target, draft, tokens, parent, None, ua, us, *got[-1])
    for a, z in ((0, 1), (2, 3)):
        assert all(torch.equal(x, y) for x, y in zip(got[a], got[z])) and int(got[a][3].item()) == 0


@pytest.mark.parametrize("kv,D,g,T", [(bk.KV_BF16, 64, 1, 3), (bk.KV_INT4, 128, 4, 2)])
def test_a_head_longer_than_a_chunk_may_be(kv, D, g, T):
    """Chunks as long as allowed against short ones, over 6.3 million rows."""
    cap = 6_300_000 // 16 * 16
    sh = bk.make_shape(1, g, 1, D)
    c = bk.Cache(sh, [[cap]], [[0]], cap, 1, kv_dtype=kv, kv_scale=np.ones((1, 1, 4, D)) if kv == bk.KV_INT4 else None)
    gen = torch.Generator(device="cuda").manual_seed(D)
    grow = torch.linspace(0.01, 2.0, cap, device="cuda")[:, None]     # values that rise with the rows: a lost chunk moves the average
    if kv == bk.KV_BF16:
        c.k_slab.normal_(generator=gen)
        c.v_slab.copy_(grow)
    else:
        c.k_slab.random_(0x11, 0x100, generator=gen)
        c.v_slab.fill_(0xCC)
        c.row_scale[:, 0].uniform_(0.1, 0.3, generator=gen)
        c.row_scale[:, 1:].copy_(grow / 4)
    c.len.fill_(cap - 5)
    c.free_slot.fill_(cap - 5)
    q, k, v = (torch.randn((1, h, T, D), generator=gen, device="cuda").bfloat16() for h in (g, 1, 1))
    parent = torch.arange(-1, T - 1, dtype=torch.int32, device="cuda").reshape(1, T)
    got = []
    for chunk in (1 << 30, 0):
        plan = bk.baklava_tree_plan(sh, [[cap]], 1, 0, T, chunk_tokens=chunk, kv_dtype=kv).to("cuda")
        out, z = torch.zeros_like(q), torch.zeros((1, g, T), device="cuda")
        bk.baklava_tree_attn(sh, c, q, k, v, parent, None, out, z, plan, bk.decode_workspace(plan))
        assert int(c.status.item()) == 0
        got.append((out, z))
    # A thread adds up to 2^17 probabilities of a chunk in fp32: 2^17 2^-24 of the sum at most, either side, and logits to 2^-11.  A row
    # besides: probabilities and the result to 2^-8, 2^15 additions of the product.  A chunk of the longest is a thirteenth of all.
    assert (got[0][1] - got[1][1]).abs().max() <= 2 * 2.0 ** -7 + 2.0 ** -10
    assert (got[0][0].float() / got[1][0].float() - 1).abs().max() <= 2 * (2.0 ** -7 + 2.0 ** -8 + 2.0 ** -8 + 2.0 ** -9) + 2.0 ** -9
    assert (got[1][0].float() - 1).abs().max() < 0.1 and (got[1][1] > np.log(cap) - 1).all()
