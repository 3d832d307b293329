"""The accepted path into the slabs against the oracle: places and positions exact, rows bit for bit, scores to rounding."""
import numpy as np
import pytest
import torch

from oracle import int4 as o4
from oracle import tree as ot
from paper_2502_13176_b200 import binding as bk
from tests.tree_cases import FORMATS, Held, bf16_normal, random_tree

pytestmark = pytest.mark.gpu


def nodes_of(rng, sh, B, T, spread=1.0):
    q = bf16_normal(rng, (sh.L, B, sh.Hq, T, sh.D), spread)
    k, v = (bf16_normal(rng, (sh.L, B, sh.Hkv, T, sh.D)) for _ in range(2))
    return q, k, v


def paths_of(rng, B, T, longest, kind="any"):
    """Accepted paths: random nodes' ways from their roots, cut."""
    path = np.full((B, T), -1, dtype=np.int32)
    n = np.zeros(B, dtype=np.int32)
    for b in range(B):
        w = ot.way(random_tree(rng, T, kind), T - 1)[:longest]
        path[b, :len(w)], n[b] = w, len(w)
    return path, n


def lse_of(held, q, k, path, n):
    """What attention left for the path's nodes (fp64, rounded once), anything for the others."""
    sh, g = held.shape, held.shape.g
    lse = np.full((sh.L, held.B, sh.Hq, q.shape[3]), 1e9, dtype=np.float32)
    q64, k64 = q.double().numpy(), k.double().numpy()
    for b in range(held.B):
        for l in range(sh.L):
            for h in range(sh.Hkv):
                K = held.values(0, held.rows(b, l, h), l, h)
                for i in range(n[b]):
                    w = path[b, :i + 1]
                    s = q64[l, b, h * g:h * g + g, w[-1]] @ np.concatenate([K, k64[l, b, h, w]]).T / np.sqrt(sh.D)
                    lse[l, b, h * g:h * g + g, w[-1]] = np.log(np.exp(s - s.max(1)[:, None]).sum(1)) + s.max(1)
    return torch.from_numpy(lse)


def commit(held, q, k, v, lse, path, n, max_path, t_pos, flags=0, chunk=0, layers=None):
    sh = held.shape
    lb, le = layers or (0, sh.L)
    plan = bk.baklava_decode_plan(sh, held.cap, held.B, lb, le, held.stride, chunk_tokens=chunk, kv_dtype=FORMATS[held.kv]).to("cuda")
    ws = bk.tree_commit_workspace(sh, plan, max_path).fill_(0xFF)
    i32 = lambda x: torch.as_tensor(np.asarray(x), dtype=torch.int32).cuda()                  # noqa: E731
    nxt = torch.full((held.B,), 12345, dtype=torch.int32, device="cuda")
    dev = [None if x is None else x[lb:le].contiguous().cuda() for x in (q, k, v, lse)]
    bk.baklava_tree_commit(sh, held.cache, *dev, i32(path), i32(n), max_path, i32(t_pos), nxt, flags, plan, ws)
    torch.cuda.synchronize()
    return nxt.cpu().numpy()


def check(held, q, k, v, lse, path, n, t_pos, scored=True, evict=True, layers=None, before=None):
    """The device against oracle twins made from the state before the call."""
    sh, g, c = held.shape, held.shape.g, held.cache
    pos, score, length, free = (x.cpu().numpy() for x in (c.pos, c.score, c.len, c.free_slot))
    slabs = [c.k_slab.cpu(), c.v_slab.cpu()]
    row_scale = None if c.row_scale is None else c.row_scale.cpu().numpy()
    touched = np.zeros(held.live.shape, dtype=bool)
    for b in range(held.B):
        for l in range(*(layers or (0, sh.L))):
            for h in range(sh.Hkv):
                what = "b%d l%d h%d" % (b, l, h)
                hc, lo = held.twin(b, l, h), b * held.stride + int(held.off[l, h])
                old_slots = set(hc.valid_slots().tolist())
                a = int(n[b]) if t_pos[b] >= 0 else 0
                y = slice(h * g, h * g + g)
                w = path[b, :a].tolist()
                joined = True
                base = hc.score.copy()
                if a:
                    joined = ot.commit(hc, q[l, b, y].double().numpy(), k[l, b, h].double().numpy(), v[l, b, h].double().numpy(),
                                       lse[l, b, y].double().numpy(), w, int(t_pos[b]), scored, evict)
                assert (length[b, l, h], free[b, l, h]) == (hc.length, hc.free_slot), what
                here = slice(lo, lo + hc.C)
                touched[here] = True
                valid = hc.valid_slots()
                np.testing.assert_array_equal(pos[here][valid], hc.pos[valid], err_msg=what)
                # a share is exp(s - lse): an fp32 sum of D products (at most D 2^-24 of the sum of magnitudes, which is below 64
                # here), exp2's and the sums' own roundings 2^-18; adding to a score rounds it once more
                both = sorted(old_slots | set(valid.tolist()))
                gain = np.abs(hc.score[both] - np.where([s in old_slots and hc.pos[s] < t_pos[b] for s in both], base[both], 0))
                tol = gain * (64 * 128 * 2.0 ** -24 + 2.0 ** -18) + 2.0 ** -23 * hc.score[both] + 1e-30
                err = np.abs(score[here][both].astype(np.float64) - hc.score[both])
                assert (err <= tol).all(), (what, (err / tol).max())
                fresh = [s for s in valid if joined and a and hc.pos[s] >= t_pos[b]]
                for which, x in enumerate((k, v)):
                    want = held.data[which][here].clone()
                    rows = x[l, b, h][[w[int(hc.pos[s]) - int(t_pos[b])] for s in fresh]]
                    if held.kv == "bf16":
                        want[fresh] = rows
                    elif held.kv == "fp8":
                        inv = c.kv_scale_host[l, h, 2 * which + 1]
                        want[fresh] = (rows.float() * float(inv)).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
                    else:
                        # (the scale is max |y| times the reciprocal of 7; oracle/int4.py has the quotient)
                        y = rows.float().numpy() * c.kv_scale_host[l, h, 2 * which + 1]
                        s = np.abs(y).max(axis=-1) * (np.float32(1) / np.float32(7))
                        codes = (np.clip(np.rint(y / s[:, None]), -7, 7) + 8).astype(np.uint8)
                        want[fresh] = torch.from_numpy(o4.pack(codes))
                        ref = held.row_scale[here, which].copy()
                        ref[fresh] = s
                        np.testing.assert_array_equal(row_scale[here, which].view(np.int32), ref.view(np.int32), err_msg=what)
                    assert torch.equal(slabs[which][here].view(torch.uint8), want.view(torch.uint8)), what
    outside = ~touched                                        # what belongs to no head of the call
    np.testing.assert_array_equal(pos[outside], held.pos[outside])
    np.testing.assert_array_equal(score[outside], held.score[outside])


@pytest.mark.parametrize("kv,D,g,T,longest", [("bf16", 128, 4, 16, 6), ("bf16", 64, 7, 9, 9), ("bf16", 128, 8, 64, 64), ("bf16", 64, 1, 1, 1),
                                              ("bf16", 128, 5, 33, 12), ("fp8", 128, 4, 16, 6), ("fp8", 128, 3, 20, 20), ("int4", 128, 4, 16, 6),
                                              ("int4", 128, 8, 64, 64), ("int4", 128, 7, 5, 5)])
@pytest.mark.parametrize("policy", ["heavy", "window", "no score", "no evict"])
def test_matches_the_definition(kv, D, g, T, longest, policy):
    rng = np.random.default_rng(D + g + T)
    B, Hkv = 3, 2
    sh = bk.make_shape(2, Hkv * g, Hkv, D, n_sink=3, recent_num=1, recent_den=1 if policy == "window" else 3)
    caps = [[160, 96], [1296, 2160]]
    held = np.array([[[159, 95], [1295, 2159]], [[0, 1], [700, 128]], [[150, 96], [1296, 2100]]])
    holes = np.array([[[0, 95], [640, 128]], [[0, 1], [700, 128]], [[150, 96], [1296, 2100]]])
    c = Held(sh, caps, B, kv, held, holes, seed=T)
    q, k, v = nodes_of(rng, sh, B, T)
    path, n = paths_of(rng, B, T, longest, "chain" if longest == T else "any")
    scored, evict = policy in ("heavy", "no evict"), policy in ("heavy", "window")
    lse = lse_of(c, q, k, path, n)
    t_pos = [20000, 20000, 30000]
    flags = (0 if scored else bk.FLAG_NO_SCORE) | (bk.FLAG_NO_EVICT if policy == "no evict" else 0)
    full = not evict
    nxt = commit(c, q, k, v, lse, path, n, longest, t_pos, flags)
    check(c, q, k, v, lse, path, n, t_pos, scored, evict)
    np.testing.assert_array_equal(nxt, np.array(t_pos) + n)
    assert int(c.cache.status.item()) == (bk.STATUS_OVERFLOW if full else 0)


@pytest.mark.parametrize("chunk", [64, 128, 1024, 1088, 8192])
def test_any_chunks_and_a_layer_range(chunk):
    rng = np.random.default_rng(chunk)
    sh = bk.make_shape(3, 4, 2, 128, n_sink=4, recent_num=1, recent_den=2)
    caps = [[16, 32], [5200, 3008], [48, 1024]]
    held = np.array(caps)[None] - 1
    c = Held(sh, caps, 1, "bf16", held, held // 2, seed=chunk)
    q, k, v = nodes_of(rng, sh, 1, 12)
    path, n = paths_of(rng, 1, 12, 9, "chain")
    lse = lse_of(c, q, k, path, n)
    commit(c, q, k, v, lse, path, n, 9, [50000], chunk=chunk, layers=(1, 3))
    check(c, q, k, v, lse, path, n, [50000], layers=(1, 3))
    assert int(c.cache.status.item()) == 0


def test_paths_longer_than_the_window_and_than_the_cache():
    """Joining rows that are not protected compete with the others, and with one another."""
    rng = np.random.default_rng(3)
    for recent in (0, 1):
        sh = bk.make_shape(1, 2, 2, 64, n_sink=4, recent_num=recent, recent_den=8)
        c = Held(sh, [[16, 32]], 2, "bf16", [[[15, 31]], [[16, 10]]], [[[4, 31]], [[16, 10]]], seed=4)
        q, k, v = nodes_of(rng, sh, 2, 40)
        path, n = paths_of(rng, 2, 40, 40, "chain")
        lse = lse_of(c, q, k, path, n)
        commit(c, q, k, v, lse, path, n, 40, [5000, 5000])
        check(c, q, k, v, lse, path, n, [5000, 5000])
        assert int(c.cache.status.item()) == 0


def test_equal_scores_the_latest_goes():
    sh = bk.make_shape(1, 1, 1, 64, n_sink=2, recent_num=1, recent_den=4)
    c = Held(sh, [[128]], 1, "bf16", [[[127]]], [[[127]]], seed=1)
    c.score[:] = 1.0
    c.cache.score.fill_(1.0)
    q = torch.zeros((1, 1, 1, 3, 64), dtype=torch.bfloat16)
    k = v = torch.ones((1, 1, 1, 3, 64), dtype=torch.bfloat16)
    path, n = np.array([[0, 1, 2]], dtype=np.int32), np.array([3], dtype=np.int32)
    lse = torch.full((1, 1, 1, 3), 200.0)                     # exp(-200): adds nothing that fp32 holds beside 1
    commit(c, q, k, v, lse, path, n, 3, [5000])
    check(c, q, k, v, lse, path, n, [5000])


def test_many_short_lists():
    """More blocks to a head than threads that join their lists."""
    rng = np.random.default_rng(6)
    sh = bk.make_shape(1, 1, 1, 64, n_sink=4)
    cap = 64 * 2600
    c = Held(sh, [[cap]], 1, "bf16", [[[cap - 1]]], [[[77]]], seed=2, poison=False)
    q, k, v = nodes_of(rng, sh, 1, 8)
    path, n = paths_of(rng, 1, 8, 8, "chain")
    lse = lse_of(c, q, k, path, n)
    commit(c, q, k, v, lse, path, n, 8, [1 << 20], chunk=64)
    check(c, q, k, v, lse, path, n, [1 << 20])


def test_who_sits_out_and_who_cannot_be():
    rng = np.random.default_rng(7)
    sh = bk.make_shape(1, 2, 1, 64)
    B, T = 7, 4
    c = Held(sh, [[64]], B, "bf16", np.full((B, 1, 1), 40), np.full((B, 1, 1), 40), seed=3)
    q, k, v = nodes_of(rng, sh, B, T)
    path = np.tile(np.arange(T, dtype=np.int32), (B, 1))
    n = np.array([2, 0, 2, 5, 2, 2, -1], dtype=np.int32)       # 3: longer than max_path
    t_pos = [9000, 9000, -1, 9000, 9000, 9000, 9000]
    path[4, 1], path[5, 0] = T, -1                            # nodes that are none
    lse = torch.zeros((1, B, 2, T))
    keep = [x.clone() for x in (c.cache.k_slab, c.cache.v_slab, c.cache.pos, c.cache.score, c.cache.len, c.cache.free_slot)]
    nxt = commit(c, q, k, v, lse, path, n, 3, t_pos)
    assert int(c.cache.status.item()) == bk.STATUS_BAD_STATE
    assert nxt.tolist() == [9002] + t_pos[1:]
    assert c.cache.len[:, 0, 0].tolist() == [42] + [40] * 6
    for x, was in zip((c.cache.k_slab, c.cache.v_slab, c.cache.pos, c.cache.score), keep):
        assert torch.equal(x[64:].view(torch.uint8), was[64:].view(torch.uint8))
    c.cache.status.zero_()
    c.cache.len[0, 0, 0] = 99
    commit(c, q, k, v, lse, path, np.array([2] + [0] * 6, dtype=np.int32), 3, t_pos)
    assert int(c.cache.status.item()) == bk.STATUS_BAD_STATE and int(c.cache.len[0, 0, 0]) == 99


def test_a_capacity_without_room_for_the_sinks():
    rng = np.random.default_rng(8)
    sh = bk.make_shape(1, 2, 1, 64, n_sink=40)
    c = Held(sh, [[16]], 1, "bf16", [[[15]]], [[[15]]], seed=3)
    c.cache.pos.copy_(torch.arange(16, dtype=torch.int32))
    q, k, v = nodes_of(rng, sh, 1, 2)
    commit(c, q, k, v, torch.zeros((1, 1, 2, 2)), np.array([[0, 1]], dtype=np.int32), np.array([2], dtype=np.int32), 2, [20])
    assert int(c.cache.status.item()) == bk.STATUS_BAD_STATE and int(c.cache.len[0, 0, 0]) == 15


@pytest.mark.parametrize("kv", ["fp8", "int4"])
@pytest.mark.parametrize("chunk", [64, 128, 320, 1024])
def test_rows_of_codes_in_any_chunks(kv, chunk):
    """Heads and chunks that end inside a group of 128 rows, on it, one before and one behind; holes at both ends; one to many columns."""
    rng = np.random.default_rng(chunk)
    sh = bk.make_shape(1, 14, 2, 128, n_sink=2, recent_num=1, recent_den=4)
    B, T = 9, 40
    c = Held(sh, [[1104, 400]], B, kv, [[[n, m]] for n, m in ((1, 2), (127, 15), (128, 16), (129, 17), (255, 127), (256, 128), (1023, 257), (1025, 385),
                                                             (1103, 399))],
             [[[n, m]] for n, m in ((0, 0), (0, 15), (127, 3), (128, 17), (255, 0), (1, 127), (1023, 256), (77, 384), (1102, 399))], seed=chunk)
    q, k, v = nodes_of(rng, sh, B, T)
    path, n = paths_of(rng, B, T, T, "chain")
    n[:] = [1, 2, 3, 5, 9, 10, 0, 37, 40]                     # 7 to 280 columns
    lse = lse_of(c, q, k, path, n)
    commit(c, q, k, v, lse, path, n, T, [40000] * B, chunk=chunk)
    check(c, q, k, v, lse, path, n, [40000] * B)
    assert int(c.cache.status.item()) == 0


@pytest.mark.parametrize("kv", ["bf16", "fp8", "int4"])
def test_beside_other_calls_and_replayed(kv):
    """Bit for bit what the calls leave alone: while attention of a tree and another commit run on other streams, and from a graph."""
    rng = np.random.default_rng(12)
    sh = bk.make_shape(2, 8, 2, 128, n_sink=3)
    B, T = 6, 12
    caps = [[3008, 400], [800, 5008]]
    held = np.array(caps)[None] - 1 - rng.integers(0, 300, (B, 2, 2))
    holes = np.minimum(held, rng.integers(0, 400, held.shape))
    q, k, v = nodes_of(rng, sh, B, T)
    path, n = paths_of(rng, B, T, 7, "chain")
    i32 = lambda x: torch.as_tensor(np.asarray(x), dtype=torch.int32).cuda()                  # noqa: E731

    class Call:
        def __init__(self):
            self.c = Held(sh, caps, B, kv, held, holes, seed=5)
            self.plan = bk.baklava_decode_plan(sh, self.c.cap, B, 0, 2, self.c.stride, kv_dtype=FORMATS[kv]).to("cuda")
            self.ws = bk.tree_commit_workspace(sh, self.plan, 7)
            self.at = [i32([30000] * B), i32([0] * B)]
            self.dev = [x.cuda() for x in (q, k, v, torch.full((2, B, 8, T), 9.0))] + [i32(path), i32(n)]
            torch.cuda.synchronize()

        def __call__(self):
            bk.baklava_tree_commit(sh, self.c.cache, *self.dev, 7, *self.at, 0, self.plan, self.ws)
            self.at.reverse()

        def state(self):
            torch.cuda.synchronize()
            c = self.c.cache
            return [x.clone().view(torch.uint8) for x in (c.k_slab, c.v_slab, c.pos, c.score, c.len, c.free_slot)]

    alone, two, three = Call(), Call(), Call()
    for _ in range(4):
        alone()
    want = alone.state()
    other = Held(sh, caps, B, kv, held, holes, seed=6)
    tree_plan = bk.baklava_tree_plan(sh, other.cap, B, 1, T, kv_dtype=FORMATS[kv]).to("cuda")
    tree_ws = bk.decode_workspace(tree_plan)
    parent = i32(np.tile(np.arange(-1, T - 1), (B, 1)))
    out, lse = torch.empty((B, 8, T, 128), dtype=torch.bfloat16, device="cuda"), torch.empty((B, 8, T), device="cuda")
    layer = [x[1].contiguous().cuda() for x in (q, k, v)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        three()
        three()
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    for i in range(4):
        with torch.cuda.stream(streams[0]):
            two()
        with torch.cuda.stream(streams[1]):
            bk.baklava_tree_attn(sh, other.cache, *layer, parent, None, out, lse, tree_plan, tree_ws)
        if i % 2 == 0:
            with torch.cuda.stream(streams[2]):
                graph.replay()
    for call in (two, three):
        for x, y in zip(call.state(), want):
            assert torch.equal(x, y)
        assert int(call.c.cache.status.item()) == 0
