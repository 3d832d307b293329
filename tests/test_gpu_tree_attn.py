"""Attention of drafted trees over budgeted slabs against the fp64 definition."""
import numpy as np
import pytest
import torch

from oracle import tree as ot
from paper_2502_13176_b200 import binding as bk
from tests.tree_cases import FORMATS, Held, bf16_normal, random_tree

pytestmark = pytest.mark.gpu


def bounds(q, keys, vals, out, lse):
    """What the roundings allow of a row: (output, log-sum-exp).

    Probabilities are rounded to 16 bits for the product with V (bf16 at worst: 2^-8 relative each, so 2^-8 sum p |v|) and
    the result once to bf16 (2^-8 |o|).  A logit is an fp32 sum of D products: at most D roundings of 2^-24 relative to the sum of
    magnitudes (4-bit rows: queries held to 2^-21 besides); an error e of logits moves lse by e and a row by 2 e sum p |v|.
    exp2 and the sums behind it: 2^-20 relative."""
    D = q.shape[-1]
    s = q @ keys.T / np.sqrt(D)
    p = np.exp(s - lse[:, None])
    e = (np.abs(q) @ np.abs(keys).T).max(axis=1) / np.sqrt(D) * (D * 2.0 ** -24 + 2.0 ** -20)
    spread = p @ np.abs(vals)
    return 2.0 ** -8 * np.abs(out) + (2.0 ** -8 + 2 * e[:, None] + 2.0 ** -18) * spread + 1e-30, e + 2.0 ** -18 + 2.0 ** -22 * np.abs(lse)


def run(held, q, k, v, parent, n_nodes, layer=0, chunk=0, lse=True):
    sh, B, T = held.shape, held.B, q.shape[2]
    plan = bk.baklava_tree_plan(sh, held.cap, B, layer, T, chunk_tokens=chunk, kv_dtype=FORMATS[held.kv]).to("cuda")
    ws = torch.full((int(plan.info.ws_bytes),), 0xFF, dtype=torch.uint8, device="cuda")       # NaN: nothing is read before it is written
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    z = torch.full(q.shape[:3], 7.0, dtype=torch.float32, device="cuda") if lse else None
    bk.baklava_tree_attn(sh, held.cache, q, k, v, parent, n_nodes, out, z, plan, ws)
    torch.cuda.synchronize()
    return out, z


def check(held, q, k, v, parent, n_nodes, out, z, layer=0, what=""):
    sh, g = held.shape, held.shape.g
    q64, k64, v64 = (x.double().cpu().numpy() for x in (q, k, v))
    parent = parent.cpu().numpy()
    o64, z64 = out.double().cpu().numpy(), z.double().cpu().numpy()
    for b in range(held.B):
        n = q.shape[2] if n_nodes is None else int(np.clip(int(n_nodes[b]), 0, q.shape[2]))
        assert (o64[b, :, n:] == 7.0).all() and (z64[b, :, n:] == 7.0).all(), "%s: nodes behind the last" % what
        for h in range(sh.Hkv):
            rows = held.rows(b, layer, h)
            K, V = held.values(0, rows, layer, h), held.values(1, rows, layer, h)
            y = slice(h * g, h * g + g)
            ref, rz = ot.tree_attention(q64[b, y, :n], k64[b, h, :n], v64[b, h, :n], parent[b], K, V)
            for i in range(n):
                w = ot.way(parent[b], i)
                keys, vals = np.concatenate([K, k64[b, h, w]]), np.concatenate([V, v64[b, h, w]])
                bo, bz = bounds(q64[b, y, i], keys, vals, ref[:, i], rz[:, i])
                eo, ez = np.abs(o64[b, y, i] - ref[:, i]), np.abs(z64[b, y, i] - rz[:, i])
                assert (ez <= bz).all(), "%s: lse of b%d h%d node %d off by %s of %s" % (what, b, h, i, ez, bz)
                assert (eo <= bo).all(), "%s: row of b%d h%d node %d off by %.3g times its bound" % (what, b, h, i, np.nanmax(eo / bo))
    assert int(held.cache.status.item()) == 0


def inputs(rng, sh, B, T, kind="any", spread=1.0):
    q = bf16_normal(rng, (B, sh.Hq, T, sh.D), spread).cuda()
    k, v = (bf16_normal(rng, (B, sh.Hkv, T, sh.D)).cuda() for _ in range(2))
    parent = torch.from_numpy(np.stack([random_tree(rng, T, kind) for _ in range(B)]).astype(np.int32)).cuda()
    return q, k, v, parent


@pytest.mark.parametrize("kv,D,g,T", [("bf16", 128, 4, 16), ("bf16", 64, 2, 5), ("bf16", 128, 7, 27), ("bf16", 64, 8, 64), ("bf16", 128, 1, 1),
                                      ("bf16", 128, 8, 33), ("bf16", 64, 3, 8), ("bf16", 128, 5, 64), ("fp8", 128, 4, 16), ("fp8", 128, 7, 40),
                                      ("fp8", 128, 1, 3), ("fp8", 128, 4, 64), ("int4", 128, 4, 16), ("int4", 128, 7, 25), ("int4", 128, 8, 64),
                                      ("int4", 128, 2, 1)])
def test_matches_the_definition(kv, D, g, T):
    rng = np.random.default_rng(D + 10 * g + T)
    Hkv, B = 2, 3
    sh = bk.make_shape(2, Hkv * g, Hkv, D)
    caps = [[48, 16], [1200, 304]]
    held = np.array([[[47, 15], [1199, 303]], [[0, 1], [700, 128]], [[20, 16], [0, 129]]])
    holes = np.array([[[0, 15], [640, 128]], [[0, 1], [700, 128]], [[20, 16], [0, 5]]])
    c = Held(sh, caps, B, kv, held, holes, seed=T, seq_gap=32)
    q, k, v, parent = inputs(rng, sh, B, T)
    nodes = torch.tensor([T, max(0, T - 1), (T + 1) // 2], dtype=torch.int32, device="cuda")
    for chunk in (0, 128):
        for layer in (0, 1):
            out, z = run(c, q, k, v, parent, nodes, layer, chunk)
            check(c, q, k, v, parent, nodes, out, z, layer, "chunk %d layer %d" % (chunk, layer))


@pytest.mark.parametrize("kind", ["chain", "star"])
def test_chains_and_stars_without_counts(kind):
    rng = np.random.default_rng(5)
    sh = bk.make_shape(1, 8, 2, 128)
    c = Held(sh, [[512, 400]], 2, "bf16", [[[511, 399]], [[300, 260]]], [[[511, 0]], [[300, 259]]], seed=6)
    q, k, v, parent = inputs(rng, sh, 2, 12, kind)
    out, z = run(c, q, k, v, parent, None, chunk=128)
    check(c, q, k, v, parent, None, out, z, what=kind)


@pytest.mark.parametrize("kv", ["bf16", "fp8", "int4"])
def test_an_empty_cache_leaves_the_tree_alone(kv):
    rng = np.random.default_rng(8)
    sh = bk.make_shape(1, 4, 2, 128)
    c = Held(sh, [[64, 32]], 2, kv, np.zeros((2, 1, 2)), np.zeros((2, 1, 2)), seed=1)
    q, k, v, parent = inputs(rng, sh, 2, 9)
    out, z = run(c, q, k, v, parent, None)
    check(c, q, k, v, parent, None, out, z)


def test_nothing_of_other_branches_gets_in():
    """NaN and infinities in nodes that are neither a node nor above it, and in nodes behind the last."""
    rng = np.random.default_rng(9)
    sh = bk.make_shape(1, 4, 2, 128)
    c = Held(sh, [[64, 160]], 1, "bf16", [[[63, 159]]], [[[5, 100]]], seed=2)
    q, k, v, _ = inputs(rng, sh, 1, 6)
    parent = torch.tensor([[-1, 0, 0, 1, 2, 4]], dtype=torch.int32, device="cuda")
    clean = [x.clone() for x in (q, k, v)]
    for x in (q, k, v):
        x[:, :, 1], x[:, :, 3], x[:, :, 5] = float("nan"), float("inf"), float("nan")
    nodes = torch.tensor([5], dtype=torch.int32, device="cuda")
    out, z = run(c, q, k, v, parent, nodes)
    good, gz = run(c, *clean, parent, nodes)
    for i in (0, 2, 4):
        assert torch.equal(out[:, :, i], good[:, :, i]) and torch.equal(z[:, :, i], gz[:, :, i])
    assert torch.isnan(out[:, :, 1].float()).all() and (out[:, :, 5] == 7.0).all()


@pytest.mark.parametrize("kv", ["bf16", "fp8", "int4"])
def test_logits_far_apart(kv):
    """Later rows tower over the ones before (and the other way round), chunk by chunk and inside a tile."""
    rng = np.random.default_rng(10)
    sh = bk.make_shape(1, 4, 1, 128)
    n = 700
    c = Held(sh, [[704]], 1, kv, [[[n]]], [[[n]]], seed=3)
    if kv == "bf16":                                          # one direction, growing along the slots
        grow = torch.linspace(-60, 60, 704)[:, None] * torch.sign(torch.randn(128, generator=torch.Generator().manual_seed(1)))[None, :]
        grow[300] *= 8
        c.data[0] = torch.where(torch.from_numpy(c.live)[:, None], grow.bfloat16(), c.data[0])
        c.cache.k_slab.copy_(c.data[0])
    q, k, v, parent = inputs(rng, sh, 1, 8, spread=20.0 if kv != "bf16" else 3.0)
    for chunk in (0, 128):
        out, z = run(c, q, k, v, parent, None, chunk=chunk)
        check(c, q, k, v, parent, None, out, z, what="chunk %d" % chunk)


def test_values_near_the_end_of_the_range():
    rng = np.random.default_rng(11)
    sh = bk.make_shape(1, 4, 1, 128)
    c = Held(sh, [[512]], 1, "bf16", [[[500]]], [[[500]]], seed=3)
    c.data[1] = torch.where(torch.from_numpy(c.live)[:, None], torch.full((512, 128), 3e38).bfloat16(), c.data[1])
    c.cache.v_slab.copy_(c.data[1])
    q, k, v, parent = inputs(rng, sh, 1, 4)
    v.fill_(3e38)
    out, z = run(c, q, k, v, parent, None, chunk=128)
    assert torch.isfinite(out.float()).all()
    check(c, q, k, v, parent, None, out, z)


def test_any_layout_of_the_tensors():
    """Views of the projection's rows, token-major outputs, gaps: bit for bit what dense tensors give."""
    rng = np.random.default_rng(12)
    sh = bk.make_shape(1, 6, 2, 64)
    B, T = 2, 11
    c = Held(sh, [[256, 176]], B, "bf16", [[[255, 175]], [[100, 90]]], [[[0, 60]], [[100, 90]]], seed=4)
    q, k, v, parent = inputs(rng, sh, B, T)
    ref, rz = run(c, q, k, v, parent, None)
    rows = torch.full((B, T, 12, 64), float("nan"), dtype=torch.bfloat16, device="cuda")
    rows[:, :, :6], rows[:, :, 6:8], rows[:, :, 9:11] = q.transpose(1, 2), k.transpose(1, 2), v.transpose(1, 2)
    heads = rows.transpose(1, 2)
    plan = bk.baklava_tree_plan(sh, c.cap, B, 0, T).to("cuda")
    ws = bk.decode_workspace(plan)
    out = torch.zeros((B, T, 6, 64), dtype=torch.bfloat16, device="cuda")
    bk.baklava_tree_attn(sh, c.cache, heads[:, :6], heads[:, 6:8], heads[:, 9:11], parent, None, out.transpose(1, 2), None, plan, ws)
    assert torch.equal(out.transpose(1, 2), ref)


@pytest.mark.parametrize("parent", [[-1, 0, 2], [-1, 1, 0], [-1, -2, 0], [0, 0, 0], [-1, 0, 1 << 30]])
def test_trees_that_cannot_be_are_skipped(parent):
    rng = np.random.default_rng(13)
    sh = bk.make_shape(1, 4, 2, 64)
    c = Held(sh, [[64, 64]], 2, "bf16", [[[30, 30]]], [[[30, 30]]], seed=5)
    q, k, v, good = inputs(rng, sh, 2, 3)
    good[1] = torch.tensor(parent, dtype=torch.int32)
    out, z = run(c, q, k, v, good, None)
    assert int(c.cache.status.item()) == bk.STATUS_BAD_STATE
    assert (out[1] == 7.0).all() and (z[1] == 7.0).all()
    c.cache.status.zero_()
    ok = run(c, q, k, v, good, torch.tensor([3, 0], dtype=torch.int32, device="cuda"))        # (nobody looks behind the last node)
    assert int(c.cache.status.item()) == 0
    assert torch.equal(ok[0][0], out[0]) and (ok[0][1] == 7.0).all()


def test_heads_in_a_bad_state_are_skipped():
    rng = np.random.default_rng(14)
    sh = bk.make_shape(1, 4, 2, 64)
    c = Held(sh, [[64, 64]], 2, "bf16", [[[30, 30]]], [[[30, 30]]], seed=5)
    q, k, v, parent = inputs(rng, sh, 2, 3)
    ref, rz = run(c, q, k, v, parent, None)
    for where, value in (("len", 65), ("len", -1), ("free_slot", 65), ("free_slot", -3)):
        t = getattr(c.cache, where)
        keep = t.clone()
        t[1, 0, 0] = value
        out, z = run(c, q, k, v, parent, None)
        assert int(c.cache.status.item()) == bk.STATUS_BAD_STATE
        assert (out[1, :2] == 7.0).all() and torch.equal(out[0], ref[0]) and torch.equal(out[1, 2:], ref[1, 2:])
        t.copy_(keep)
        c.cache.status.zero_()


def test_repeated_replayed_and_side_by_side():
    """The same bits from every call: again, on another stream, from a graph, and two at once with their own workspaces."""
    rng = np.random.default_rng(15)
    sh = bk.make_shape(1, 32, 8, 128)
    n = rng.integers(1, 1000, (2, 1, 8))
    c = Held(sh, [[1008] * 8], 2, "bf16", n, n, seed=6)
    q, k, v, parent = inputs(rng, sh, 2, 16)
    ref, rz = run(c, q, k, v, parent, None)
    plan = bk.baklava_tree_plan(sh, c.cap, 2, 0, 16).to("cuda")
    spaces = [bk.decode_workspace(plan) for _ in range(3)]
    outs = [torch.zeros_like(ref) for _ in range(3)]
    lses = [torch.zeros_like(rz) for _ in range(3)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        for i, s in enumerate(streams):
            bk.baklava_tree_attn(sh, c.cache, q, k, v, parent, None, outs[i], lses[i], plan, spaces[i], stream=s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        bk.baklava_tree_attn(sh, c.cache, q, k, v, parent, None, outs[2], lses[2], plan, spaces[2])
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for o, z in zip(outs, lses):
        assert torch.equal(o, ref) and torch.equal(z, rz)
    q2 = bf16_normal(rng, q.shape).cuda()
    q.copy_(q2)
    graph.replay()
    torch.cuda.synchronize()
    again, _ = run(c, q2, k, v, parent, None)
    assert torch.equal(outs[2], again)


@pytest.mark.parametrize("kv,T,D,chunk", [("bf16", 8, 128, 0), ("bf16", 64, 128, 0), ("bf16", 64, 128, 1024), ("bf16", 16, 64, 0), ("bf16", 64, 64, 1536),
                                          ("fp8", 8, 128, 0), ("fp8", 64, 128, 0), ("int4", 8, 128, 0), ("int4", 40, 128, 0), ("int4", 40, 128, 640)])
def test_long_heads_side_by_side(kv, T, D, chunk):
    """A device full of long items, where loads are late: the same bits every time and for other inputs in between, right where
    looked at."""
    rng = np.random.default_rng(16)
    sh = bk.make_shape(1, 32, 8, D)
    B = 6
    caps = [[9008, 2000, 5008, 7008, 12000, 10000, 16000, 3008]]
    held = np.array(caps)[None] - 1 - rng.integers(0, 900, (B, 1, 8))
    c = Held(sh, caps, B, kv, held, np.minimum(held, rng.integers(0, 16000, held.shape)), seed=7, poison=kv != "bf16")
    q, k, v, parent = inputs(rng, sh, B, T)
    ref, rz = run(c, q, k, v, parent, None, chunk=chunk)
    for i in range(6):
        out, z = run(c, q, k, v, parent, None, chunk=chunk)
        assert torch.equal(out, ref) and torch.equal(z, rz), i
    for b, h in ((0, 0), (5, 6), (3, 1)):
        rows = c.rows(b, 0, h)
        K, V = c.values(0, rows, 0, h), c.values(1, rows, 0, h)
        y = slice(4 * h, 4 * h + 4)
        q64, k64, v64, par = (x[b].double().cpu().numpy() for x in (q, k, v, parent))
        want, wz = ot.tree_attention(q64[y], k64[h], v64[h], par.astype(int), K, V)
        for i in (0, T // 2, T - 1):
            w = ot.way(par.astype(int), i)
            keys, vals = np.concatenate([K, k64[h, w]]), np.concatenate([V, v64[h, w]])
            bo, bz = bounds(q64[y, i], keys, vals, want[:, i], wz[:, i])
            assert (np.abs(rz[b, y, i].double().cpu().numpy() - wz[:, i]) <= bz).all()
            assert (np.abs(ref[b, y, i].double().cpu().numpy() - want[:, i]) <= bo).all()


@pytest.mark.parametrize("kv,T,D", [("bf16", 8, 128), ("bf16", 64, 128), ("bf16", 16, 64), ("bf16", 47, 64), ("fp8", 16, 128), ("fp8", 64, 128),
                                    ("int4", 16, 128), ("int4", 48, 128)])
def test_many_short_heads(kv, T, D):
    """Several items to a block, most of them of one tile, some of more, some of none: the same bits every time, and right
    where looked at."""
    rng = np.random.default_rng(17)
    sh = bk.make_shape(1, 32, 8, D)
    B = 64
    caps = [[16, 112, 128, 304, 64, 16, 1008, 144]]
    held = np.array(caps)[None] - 1 - rng.integers(0, 15, (B, 1, 8))
    held[rng.random(held.shape) < 0.1] = 0
    c = Held(sh, caps, B, kv, held, np.minimum(held, rng.integers(0, 100, held.shape)), seed=8, poison=kv != "bf16")
    q, k, v, parent = inputs(rng, sh, B, T)
    ref, rz = run(c, q, k, v, parent, None)
    for i in range(6):
        out, z = run(c, q, k, v, parent, None)
        assert torch.equal(out, ref) and torch.equal(z, rz), i
    for b in (0, 31, 63):
        for h in range(8):
            rows = c.rows(b, 0, h)
            K, V = c.values(0, rows, 0, h), c.values(1, rows, 0, h)
            y = slice(4 * h, 4 * h + 4)
            q64, k64, v64, par = (x[b].double().cpu().numpy() for x in (q, k, v, parent))
            want, wz = ot.tree_attention(q64[y], k64[h], v64[h], par.astype(int), K, V)
            for i in (0, T - 1):
                w = ot.way(par.astype(int), i)
                bo, bz = bounds(q64[y, i], np.concatenate([K, k64[h, w]]), np.concatenate([V, v64[h, w]]), want[:, i], wz[:, i])
                assert (np.abs(rz[b, y, i].double().cpu().numpy() - wz[:, i]) <= bz).all()
                assert (np.abs(ref[b, y, i].double().cpu().numpy() - want[:, i]) <= bo).all()
