"""A served request from projections to tokens: queries and keys normed and rotated, prompt attention, scores from its
log-sum-exp, bulk eviction into the slabs, decode steps at every sequence's own position.  Each stage is judged on
what the stage before it left on the device, so that a deviation is found where it arises."""
import numpy as np
import pytest
import torch

from oracle import eviction as oevict
from oracle import int4 as o4
from oracle import prefill as oprefill
from oracle import rope as orope
from oracle.cache import HeadCache
from paper_2502_13176_b200 import binding as bk
from paper_2502_13176_b200 import engine
from paper_2502_13176_b200 import workloads as wl
from tests.harness import assert_close, f64
from tests.test_gpu_prompt_attn import check_head

pytestmark = pytest.mark.gpu

W = wl.scaled(wl.TINY, name="serving", L=2, Hq=6, Hkv=2, D=128, B=3, T=200, budget=0.4)
LENS = [200, 131, 60]


def rows_held(sess, b, l, h):
    """K and V values of a head's slab."""
    c = sess.cache
    lo, hi = c.rows(b, l, h)
    if sess.kv_dtype == bk.KV_INT4:
        rs = c.row_scale[lo:hi].cpu().numpy()
        return [o4.values(o4.unpack(s[lo:hi].cpu().numpy()), rs[:, i], c.kv_scale_host[l, h, 2 * i]) for i, s in enumerate((c.k_slab, c.v_slab))]
    return [f64(s[lo:hi]) for s in (c.k_slab, c.v_slab)]


def as_stored(sess, rows, l, h, which):
    if sess.kv_dtype != bk.KV_INT4:
        return rows
    four = sess.cache.kv_scale_host[l, h]
    codes, s = o4.quantise_rows(rows, four[2 * which + 1])
    return o4.values(codes, s, four[2 * which])


@pytest.mark.parametrize("kv", [bk.KV_BF16, bk.KV_INT4], ids=["bf16", "int4"])
def test_prompt_to_tokens(kv):
    w, g = W, W.g
    gen = torch.Generator(device="cuda").manual_seed(77)
    sess = engine.DecodeSession(w, chunk_tokens=64, kv_dtype=kv)
    lens = torch.tensor(LENS, dtype=torch.int32, device="cuda")
    inv_freq = (10000.0 ** (-torch.arange(0, w.D, 2, dtype=torch.float64) / w.D)).float().cuda()
    weights = [(1 + 0.2 * torch.randn(w.D, generator=gen, device="cuda")).bfloat16() for _ in range(2)]

    def project(T):
        rows = torch.randn((w.B, T, (w.Hq + 2 * w.Hkv) * w.D), generator=gen, device="cuda").bfloat16()
        heads = rows.unflatten(-1, (w.Hq + 2 * w.Hkv, w.D)).transpose(1, 2)
        return heads[:, :w.Hq], heads[:, w.Hq:w.Hq + w.Hkv], heads[:, w.Hq + w.Hkv:].contiguous()

    def rotated(x, pos, wt, b):
        return orope.rotate(orope.norm_heads(f64(x[b]), f64(wt), 1e-6), pos, f64(inv_freq))

    pos = torch.arange(w.T, device="cuda", dtype=torch.int32).repeat(w.B, 1)
    for l in range(w.L):
        q_raw, k_raw, v = project(w.T)
        q, k = engine.norm_rope(sess.shape, q_raw, k_raw, pos, inv_freq, *weights)
        for b in range(w.B):
            for got, raw, wt in ((q, q_raw, weights[0]), (k, k_raw, weights[1])):
                ref = rotated(raw, np.arange(w.T), wt, b)
                assert np.all(np.abs(f64(got[b]) - ref) <= 2.0 ** -8 * np.abs(ref) + 1e-4)
        out = sess.prefill_layer(l, q, k, v, lens)
        torch.cuda.synchronize()
        sess.check_status()
        for b, n in enumerate(LENS):
            for h in range(w.Hq):
                check_head(q[b, h, :n], k[b, h // g, :n], v[b, h // g, :n], out[b, h, :n], None, "layer %d sequence %d head %d" % (l, b, h))
            for h in range(w.Hkv):
                C = int(sess.cap[l, h])
                lo, _ = sess.cache.rows(b, l, h)
                kept = int(sess.cache.len[b, l, h])
                at = sess.cache.pos[lo:lo + kept].cpu().numpy()
                score = sess.cache.score[lo:lo + kept].cpu().numpy()
                assert kept == min(n, C - 1) and (np.diff(at) > 0).all()
                ref = oprefill.prefill_scores(f64(q[b, h * g:h * g + g, :n]), f64(k[b, h, :n]))
                assert_close(score, ref[at], "scores")
                if kept < n:                                 # sinks and window are there; the rest outranks what is not
                    keep = oevict.select_keep(np.arange(n), ref, C - 1, w.n_sink, w.recent_num, w.recent_den)
                    gone, extra = np.setdiff1d(keep, at), np.setdiff1d(at, keep)
                    if len(gone):                            # only near ties may be settled differently
                        assert ref[gone].max() - ref[extra].min() <= 2e-3 * ref[gone].max()
                K, V = rows_held(sess, b, l, h)
                for got, src, i in ((K, k, 0), (V, v, 1)):
                    np.testing.assert_array_equal(got[:kept], as_stored(sess, f64(src[b, h, :n])[at], l, h, i))
    t_pos = lens.clone()
    for step in range(4):
        raws = [project(1) for _ in range(w.L)]
        qk = [engine.norm_rope(sess.shape, r[0], r[1], t_pos[:, None].contiguous(), inv_freq, *weights) for r in raws]
        qd = torch.stack([x[0].squeeze(2) for x in qk])                       # [L, B, Hq, D]
        kd = torch.stack([x[1].squeeze(2) for x in qk])
        vd = torch.stack([r[2].squeeze(2) for r in raws])
        twins = {}
        for l in range(w.L):
            for b in range(w.B):
                for h in range(w.Hkv):
                    lo, hi = sess.cache.rows(b, l, h)
                    tw = HeadCache(int(sess.cap[l, h]), w.D, w.n_sink, w.recent_num, w.recent_den)
                    tw.K, tw.V = rows_held(sess, b, l, h)
                    tw.pos = sess.cache.pos[lo:hi].cpu().numpy().astype(np.int64)
                    tw.score = sess.cache.score[lo:hi].cpu().numpy().astype(np.float64)
                    tw.length, tw.free_slot = int(sess.cache.len[b, l, h]), int(sess.cache.free_slot[b, l, h])
                    twins[(l, b, h)] = tw
        out = sess.step_varlen(qd, kd, vd, t_pos)
        torch.cuda.synchronize()
        sess.check_status()
        for (l, b, h), tw in twins.items():
            ref, lse, _ = tw.step(f64(qd)[l, b, h * g:h * g + g], as_stored(sess, f64(kd)[l, b, h], l, h, 0),
                                  as_stored(sess, f64(vd)[l, b, h], l, h, 1), int(t_pos[b]))
            assert_close(f64(out)[l, b, h * g:h * g + g], ref, "step %d out" % step)
            assert_close(f64(sess.lse)[l, b, h * g:h * g + g], lse, "step %d lse" % step)
            assert int(sess.cache.len[b, l, h]) == tw.length
        t_pos += 1
