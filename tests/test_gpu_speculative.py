"""Steps with drafted tokens as a model would take them: the nodes normed and rotated to their places, attention of the tree layer by
layer, verification, commit, the next step, an ordinary decode step in between.  Each stage is judged on what the stage before it left
on the device."""
import numpy as np
import pytest
import torch

from oracle import rope as orope
from oracle import tree as ot
from oracle.cache import HeadCache
from paper_2502_13176_b200 import binding as bk
from paper_2502_13176_b200 import engine
from paper_2502_13176_b200 import workloads as wl
from tests.harness import assert_close, f64
from tests.test_gpu_serving import rows_held
from tests.tree_cases import random_tree

pytestmark = pytest.mark.gpu

LENS = [200, 131, 60]


def session(kv, **kw):
    w = wl.scaled(wl.TINY, name="speculative", L=2, Hq=6, Hkv=2, D=128, B=3, T=200, budget=0.4, **kw)
    sess = engine.DecodeSession(w, chunk_tokens=64, kv_dtype=kv)
    gen = torch.Generator(device="cuda").manual_seed(5)
    lens = torch.tensor(LENS, dtype=torch.int32, device="cuda")
    for l in range(w.L):
        q, k, v = (torch.randn((w.B, h, w.T, w.D), generator=gen, device="cuda").bfloat16() for h in (w.Hq, w.Hkv, w.Hkv))
        sess.prefill_layer(l, q, k, v, lens)
    sess.check_status()
    return sess, gen


def twin(sess, b, l, h, held):
    """The device head as an oracle cache; `held`: rows_held of it (FP8 heads are decoded here)."""
    w, c = sess.w, sess.cache
    lo, hi = c.rows(b, l, h)
    hc = HeadCache(hi - lo, w.D, w.n_sink, w.recent_num, w.recent_den)
    hc.length, hc.free_slot = int(c.len[b, l, h]), int(c.free_slot[b, l, h])
    slots = hc.valid_slots()
    hc.K[slots], hc.V[slots] = held[0][slots], held[1][slots]
    hc.pos[slots] = c.pos[lo:hi].cpu().numpy()[slots]
    hc.score[slots] = f64(c.score[lo:hi])[slots]
    return hc


def held_rows(sess, b, l, h):
    if sess.kv_dtype != bk.KV_FP8_E4M3:
        return rows_held(sess, b, l, h)
    from oracle import fp8 as ofp8
    lo, hi = sess.cache.rows(b, l, h)
    return [ofp8.decode(s[lo:hi].cpu().numpy()) * float(sess.cache.kv_scale_host[l, h, 2 * i]) for i, s in enumerate((sess.cache.k_slab, sess.cache.v_slab))]


@pytest.mark.parametrize("kv", [bk.KV_BF16, bk.KV_FP8_E4M3, bk.KV_INT4], ids=["bf16", "fp8", "int4"])
def test_drafts_to_tokens(kv):
    sess, gen = session(kv)
    w, g, T, V = sess.w, sess.w.g, 11, 97
    sess.drafts(T, max_path=6)
    rng = np.random.default_rng(9)
    inv_freq = (10000.0 ** (-torch.arange(0, w.D, 2, dtype=torch.float64) / w.D)).float().cuda()
    t_pos = torch.tensor(LENS, dtype=torch.int32, device="cuda")
    accepted = []
    for step in range(6):
        parents = np.stack([np.maximum(random_tree(rng, T, "any"), np.where(np.arange(T) > 0, 0, -1)) for _ in range(w.B)])
        if step % 2:
            parents[:] = np.arange(T) - 1
        nodes = np.array([T, 7, 0 if step == 3 else 3])
        depth = np.array([[len(ot.way(parents[b], i)) - 1 for i in range(T)] for b in range(w.B)])
        parent, n_nodes = torch.from_numpy(parents.astype(np.int32)).cuda(), torch.from_numpy(nodes.astype(np.int32)).cuda()
        positions = t_pos[:, None] + torch.from_numpy(depth.astype(np.int32)).cuda()
        before = {}
        for l in range(w.L):
            raw_q, raw_k, raw_v = (torch.randn((w.B, h, T, w.D), generator=gen, device="cuda").bfloat16() for h in (w.Hq, w.Hkv, w.Hkv))
            bk.baklava_qk_norm_rope(sess.shape, raw_q, raw_k, positions, inv_freq, None, None, 1e-6, sess.tree_q[l], sess.tree_k[l])
            sess.tree_v[l].copy_(raw_v)
            out = sess.tree_layer(l, parent, n_nodes)
            sess.check_status()
            assert_close(f64(sess.tree_q[l][0]), orope.rotate(f64(raw_q[0]), f64(positions[0]), f64(inv_freq)), "queries")
            for b in range(w.B):
                for h in range(w.Hkv):
                    hc = before[b, l, h] = twin(sess, b, l, h, held_rows(sess, b, l, h))
                    s, y, n = hc.valid_slots(), slice(h * g, h * g + g), nodes[b]
                    ref, lse = ot.tree_attention(f64(sess.tree_q[l, b, y, :n]), f64(sess.tree_k[l, b, h, :n]), f64(sess.tree_v[l, b, h, :n]),
                                                 parents[b], hc.K[s], hc.V[s])
                    assert_close(f64(out[b, y, :n]), ref, "step %d tree b%d l%d h%d" % (step, b, l, h))
                    assert_close(f64(sess.tree_lse[l, b, y, :n]), lse, "log-sum-exp")
        # the target's probabilities are made of the last layer's output, the draft's are a blurred copy
        logits = torch.tanh(out.float().mean(dim=1))[:, :, :1] * torch.linspace(-3, 3, V, device="cuda") + torch.randn((w.B, T, V), generator=gen, device="cuda")
        target, draft = torch.softmax(logits, -1), torch.softmax(logits + 0.3 * torch.randn((w.B, T, V), generator=gen, device="cuda"), -1)
        tokens = torch.zeros((w.B, T), dtype=torch.int32, device="cuda")
        for b in range(w.B):
            for i in range(1, T):
                tokens[b, i] = torch.multinomial(draft[b, parents[b, i]], 1, generator=gen)[0]
        ua, us = torch.rand((w.B, T), generator=gen, device="cuda"), torch.rand((w.B,), generator=gen, device="cuda")
        path, n_path, token, status = engine.verify(target, draft, tokens, parent, ua, us, n_nodes)
        assert int(status.item()) == 0
        for b in range(w.B):
            want, nxt = ot.verify(target[b].double().cpu().numpy(), draft[b].double().cpu().numpy(), tokens[b].cpu().numpy(), parents[b], int(nodes[b]),
                                  ua[b].cpu().numpy(), float(us[b]))
            assert path[b].tolist() == want + [-1] * (T - len(want)) and int(token[b]) == nxt
            accepted.append(len(want))
        n_path = torch.clamp(n_path, max=sess.max_path)       # (a longer path goes on in the next step)
        was = t_pos
        t_pos = sess.commit(path, n_path, t_pos)
        sess.check_status()
        assert torch.equal(t_pos, was + n_path)
        for (b, l, h), hc in before.items():
            a, y = int(n_path[b]), slice(h * g, h * g + g)
            w_ = path[b, :a].tolist()
            if a:
                assert ot.commit(hc, f64(sess.tree_q[l, b, y]), f64(sess.tree_k[l, b, h]), f64(sess.tree_v[l, b, h]), f64(sess.tree_lse[l, b, y]), w_, int(was[b]))
            lo, hi = sess.cache.rows(b, l, h)
            s = hc.valid_slots()
            assert (int(sess.cache.len[b, l, h]), int(sess.cache.free_slot[b, l, h])) == (hc.length, hc.free_slot)
            np.testing.assert_array_equal(sess.cache.pos[lo:hi].cpu().numpy()[s], hc.pos[s])
            assert_close(f64(sess.cache.score[lo:hi])[s], hc.score[s], "scores")
            if kv == bk.KV_BF16:
                np.testing.assert_array_equal(f64(sess.cache.k_slab[lo:hi])[s], hc.K[s])
                np.testing.assert_array_equal(f64(sess.cache.v_slab[lo:hi])[s], hc.V[s])
        if step == 2:                                         # an ordinary step over the same slabs
            q, k, v = (torch.randn((w.L, w.B, h, w.D), generator=gen, device="cuda").bfloat16() for h in (w.Hq, w.Hkv, w.Hkv))
            sess.step_varlen(q, k, v, t_pos)
            sess.check_status()
            t_pos = t_pos + 1
    assert max(accepted) > 2 and min(accepted) == 0


def test_one_node_is_a_decode_step():
    """A tree of one node, committed, leaves what the decode step leaves: rows, places and positions alike, outputs and scores to
    rounding."""
    a, gen = session(bk.KV_BF16)
    b, _ = session(bk.KV_BF16)
    w = a.w
    a.drafts(1)
    t_pos = torch.tensor(LENS, dtype=torch.int32, device="cuda")
    parent, path, one = torch.full((w.B, 1), -1, dtype=torch.int32, device="cuda"), torch.zeros((w.B, 1), dtype=torch.int32, device="cuda"), torch.ones((w.B,), dtype=torch.int32, device="cuda")
    for _ in range(30):
        q, k, v = (torch.randn((w.L, w.B, h, w.D), generator=gen, device="cuda").bfloat16() for h in (w.Hq, w.Hkv, w.Hkv))
        a.tree_q.copy_(q[:, :, :, None])
        a.tree_k.copy_(k[:, :, :, None])
        a.tree_v.copy_(v[:, :, :, None])
        for l in range(w.L):
            a.tree_layer(l, parent)
        out = b.step_varlen(q, k, v, t_pos)
        assert_close(f64(a.tree_out[:, :, :, 0]), f64(out), "output")
        t_pos = a.commit(path, one, t_pos)
    for s in (a, b):
        s.check_status()
    assert torch.equal(a.cache.len, b.cache.len)
    for bb in range(w.B):
        for l in range(w.L):
            for h in range(w.Hkv):
                x, y = (twin(s, bb, l, h, held_rows(s, bb, l, h)).retained() for s in (a, b))
                np.testing.assert_array_equal(x[0], y[0])
                assert_close(x[1], y[1], "scores")
                np.testing.assert_array_equal(x[2], y[2])


def test_a_step_from_a_graph():
    """Attention of two layers, verification and commit captured together and replayed: the same state as calls one by one."""
    runs = []
    for captured in (False, True):
        sess, _ = session(bk.KV_BF16)
        w, T, V = sess.w, 8, 50
        sess.drafts(T)
        gen = torch.Generator(device="cuda").manual_seed(21)
        parent = torch.from_numpy(np.stack([np.maximum(random_tree(np.random.default_rng(3), T, "any"), np.where(np.arange(T) > 0, 0, -1))] * w.B).astype(np.int32)).cuda()
        t_pos = torch.tensor(LENS, dtype=torch.int32, device="cuda")
        target, draft = (torch.empty((w.B, T, V), device="cuda") for _ in range(2))
        tokens = torch.empty((w.B, T), dtype=torch.int32, device="cuda")
        ua, us = torch.empty((w.B, T), device="cuda"), torch.empty((w.B,), device="cuda")
        got = torch.zeros((w.B,), dtype=torch.int32, device="cuda")

        def inputs():
            for x in (sess.tree_q, sess.tree_k, sess.tree_v):
                x.copy_(torch.randn(x.shape, generator=gen, device="cuda"))
            target.copy_(torch.softmax(torch.randn(target.shape, generator=gen, device="cuda"), -1))
            draft.copy_(target)
            tokens.copy_(torch.randint(0, V, tokens.shape, generator=gen, device="cuda"))
            ua.copy_(torch.rand(ua.shape, generator=gen, device="cuda"))
            us.copy_(torch.rand(us.shape, generator=gen, device="cuda"))

        def step():
            for l in range(w.L):
                sess.tree_layer(l, parent)
            path, n_path, token, _ = engine.verify(target, draft, tokens, parent, ua, us)
            t_pos.copy_(sess.commit(path, n_path, t_pos))
            got.copy_(token)

        inputs()
        step()                                                # (first calls look things up)
        graph = None
        if captured:
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
        tokens_out = []
        for _ in range(12):
            inputs()
            graph.replay() if captured else step()
            tokens_out.append(got.tolist())
        sess.check_status()
        c = sess.cache
        live = torch.cat([torch.arange(*c.rows(b, l, h))[torch.from_numpy(twin(sess, b, l, h, held_rows(sess, b, l, h)).valid_slots())]
                          for b in range(w.B) for l in range(w.L) for h in range(w.Hkv)])
        runs.append((tokens_out, t_pos.tolist(), c.len.tolist(), c.pos.cpu()[live], c.score.cpu()[live], c.k_slab.cpu()[live], c.v_slab.cpu()[live]))
    for x, y in zip(*runs):
        assert torch.equal(x, y) if isinstance(x, torch.Tensor) else x == y
