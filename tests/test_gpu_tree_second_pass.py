"""Attention of drafted trees where a chunk's first rows tell nothing of its largest logits: the chunk is done again with the rows' true
maxima, in every format and number of accumulators, for the rows that need it and no others."""
import numpy as np
import pytest
import torch

from oracle import int4 as o4
from oracle import tree as ot
from paper_2502_13176_b200 import binding as bk
from tests.test_gpu_tree_attn import run
from tests.tree_cases import Held, bf16_normal, random_tree

pytestmark = pytest.mark.gpu

CHUNK = 256


def towering(kv, D, B, caps, held, holes, seed):
    """A cache whose chunks begin with small rows; in two of three, rows of one direction follow that tower over them."""
    H = len(caps)
    sh = bk.make_shape(1, H, H, D)
    c = Held(sh, [caps], B, kv, held, holes, seed=seed, poison=False)
    rng = np.random.default_rng(seed)
    way = np.sign(rng.normal(size=D))
    for b in range(B):
        for h in range(H):
            lo = b * c.stride + int(c.off[0, h])
            slot = np.arange(caps[h])
            high = (slot % CHUNK >= 8) & (slot // CHUNK % 3 != b % 3) & (rng.random(caps[h]) < 0.3)
            size = np.where(high, rng.uniform(0.7, 1.0, caps[h]), rng.uniform(0.0, 0.02, caps[h]))
            if kv == "bf16":
                c.data[0][lo:lo + caps[h]] = torch.from_numpy(60 * size[:, None] * way[None]).bfloat16()
            elif kv == "fp8":
                codes = torch.from_numpy(60 * size[:, None] * way[None] / float(c.cache.kv_scale_host[0, h, 0])).clamp(-448, 448)
                c.data[0][lo:lo + caps[h]] = codes.to(torch.float8_e4m3fn).view(torch.uint8)
            else:
                c.data[0][lo:lo + caps[h]] = torch.from_numpy(o4.pack(np.broadcast_to(8 + 7 * way, (caps[h], D)).astype(np.uint8)))
                c.row_scale[lo:lo + caps[h], 0] = (60 / 7 * size).astype(np.float32)
    dead = torch.from_numpy(~c.live)
    if kv == "bf16":
        c.data[:, dead] = float("nan")
    elif kv == "fp8":
        c.data[:, dead] = 0x7F
    else:
        c.row_scale[~c.live] = np.nan
        c.cache.row_scale.copy_(torch.from_numpy(c.row_scale))
    c.cache.k_slab.copy_(c.data[0])
    c.cache.v_slab.copy_(c.data[1])
    return c


# (the accumulators: rows of a block's queries, 128 to each; bf16 has two where a launch has more chunks than SMs besides)
@pytest.mark.parametrize("kv,D,g,T,accs", [("bf16", 128, 4, 16, 1), ("bf16", 128, 4, 61, 2), ("bf16", 64, 2, 40, 1), ("bf16", 64, 7, 33, 2),
                                           ("fp8", 128, 4, 25, 1), ("fp8", 128, 4, 64, 2), ("fp8", 128, 7, 35, 2), ("int4", 128, 4, 31, 1),
                                           ("int4", 128, 3, 64, 1)])
def test_rows_that_have_to_be_done_again(kv, D, g, T, accs):
    B, caps = 3, [16000, 12816, 400, 9872]
    H = len(caps)
    held = np.array([[[15990, 12800, 390, 9870]], [[15999, 12001, 130, 9728]], [[8000, 12815, 0, 9857]]])
    holes = np.array([[[100, 12800, 389, 4000]], [[255, 8, 130, 9728]], [[8000, 300, 0, 9601]]])
    c = towering(kv, D, B, caps, held, holes, seed=T)
    c.shape = sh = bk.make_shape(1, H * g, H, D)
    rng = np.random.default_rng(g)
    q = bf16_normal(rng, (B, H * g, T, D), 2.0)
    k, v = (bf16_normal(rng, (B, H, T, D)) for _ in range(2))
    q[:, :, 1::5] *= 2.0 ** -9                                # rows that need nothing, beside those that do
    parent = np.stack([random_tree(rng, T, "any") for _ in range(B)]).astype(np.int32)
    nodes = np.array([T, max(1, T - 3), T // 2], dtype=np.int32)
    dev = [x.cuda() for x in (q, k, v)] + [torch.from_numpy(parent).cuda(), torch.from_numpy(nodes).cuda()]
    out, z = run(c, *dev, chunk=CHUNK)
    first = [out.clone(), z.clone()]
    for _ in range(3):                                        # the same bits every time
        again = run(c, *dev, chunk=CHUNK)
        assert all(torch.equal(x, y) for x, y in zip(again, first))
    assert int(c.cache.status.item()) == 0
    rows_per_head = (T + 7) // 8 * 8
    parts = -(-g // (accs * 128 // rows_per_head))
    heads = -(-g // parts)                                    # query heads to a block
    assert accs == 1 or heads * rows_per_head > 128 and len(bk.baklava_tree_plan(sh, c.cap, B, 0, T, chunk_tokens=CHUNK).items) > 148
    again_rows, other_rows = np.zeros(2, dtype=int), np.zeros(2, dtype=int)
    for b in range(B):
        n = int(nodes[b])
        assert (out[b, :, n:] == 7.0).all() and (z[b, :, n:] == 7.0).all()
        below = torch.full((n, T), float("-inf"), dtype=torch.float64)
        for i in range(n):
            below[i, ot.way(parent[b], i)] = 0.0
        below = below.cuda()
        for h in range(H):
            rows = c.rows(b, 0, h)
            chunk_of = (rows - b * c.stride - int(c.off[0, h])) // CHUNK
            K, V = (torch.from_numpy(np.ascontiguousarray(c.values(w, rows, 0, h))).cuda() for w in range(2))
            keys, vals = torch.cat([K, k[b, h].double().cuda()]), torch.cat([V, v[b, h].double().cuda()])
            for a in range(g):
                x = q[b, h * g + a, :n].double().cuda()
                s = x @ keys.t() / D ** 0.5
                # which rows leave 2^120 in some chunk, counted by accumulator
                if len(rows):
                    s2 = s[:, :len(rows)].cpu().numpy() / np.log(2)
                    marked = np.zeros(n, dtype=bool)
                    for ch in np.unique(chunk_of):
                        at = np.nonzero(chunk_of == ch)[0]
                        slot = rows[at] - b * c.stride - int(c.off[0, h]) - ch * CHUNK
                        ref = s2[:, at[slot < 8]].max(axis=1)
                        marked |= s2[:, at].max(axis=1) - ref > 121
                    which = ((a % heads) * rows_per_head + np.arange(n)) // 128
                    for w in range(2):
                        again_rows[w] += int((marked & (which == w)).sum())
                        other_rows[w] += int((~marked & (which == w)).sum())
                s[:, len(rows):] += below
                want_z = torch.logsumexp(s, dim=1)
                p = torch.exp(s - want_z[:, None])
                want = p @ vals
                # the bounds of test_gpu_tree_attn.bounds, for all nodes at once: probabilities to 2^-8 (bf16) and the result once,
                # logits to D roundings of 2^-24 of their terms' magnitudes (and 2^-20 for 4-bit rows' queries)
                e = ((x.abs() @ keys.abs().t()) * (s > float("-inf"))).amax(dim=1) / D ** 0.5 * (D * 2.0 ** -24 + 2.0 ** -20)
                bound = 2.0 ** -8 * want.abs() + (2.0 ** -8 + 2 * e[:, None] + 2.0 ** -18) * (p @ vals.abs()) + 1e-30
                far, far_z = (out[b, h * g + a, :n].double() - want).abs(), (z[b, h * g + a, :n].double() - want_z).abs()
                assert (far_z <= e + 2.0 ** -18 + 2.0 ** -22 * want_z.abs()).all(), (b, h, a, (far_z / e).max())
                assert (far <= bound).all(), (b, h, a, (far / bound).max())
    assert (again_rows[:accs] > 20).all() and (other_rows[:accs] > 20).all(), (again_rows, other_rows)
