"""An ordinary step after drafted tokens: the session's own counter knows nothing of where the sequences are by then."""
import pytest
import torch

from paper_2502_13176_b200 import binding as bk
from tests.test_gpu_speculative import LENS, session

pytestmark = pytest.mark.gpu


def test_the_uniform_step_is_refused_and_the_other_goes_on():
    sess, gen = session(bk.KV_BF16)
    w = sess.w
    sess.drafts(4)
    feed = [torch.randn((w.L, w.B, h, w.D), generator=gen, device="cuda").bfloat16() for h in (w.Hq, w.Hkv, w.Hkv)]
    for x in (sess.tree_q, sess.tree_k, sess.tree_v):
        x.copy_(torch.randn(x.shape, generator=gen, device="cuda"))
    parent = torch.tensor([[-1, 0, 1, 2]] * w.B, dtype=torch.int32, device="cuda")
    path, n = torch.tensor([[0, 1, 2, -1]] * w.B, dtype=torch.int32, device="cuda"), torch.full((w.B,), 3, dtype=torch.int32, device="cuda")
    t_pos = torch.tensor(LENS, dtype=torch.int32, device="cuda")
    for l in range(w.L):
        sess.tree_layer(l, parent)
    t_pos = sess.commit(path, n, t_pos)
    before = [x.clone() for x in (sess.cache.len, sess.cache.pos, sess.cache.free_slot)]
    for flags in (0, bk.FLAG_NO_EVICT):
        with pytest.raises(RuntimeError, match="step_varlen"):
            sess.step(*feed, flags)
    sess.step(*feed, bk.FLAG_NO_APPEND | bk.FLAG_NO_SCORE)    # takes no position: over the rows as they are
    assert all(torch.equal(x, y) for x, y in zip(before, (sess.cache.len, sess.cache.pos, sess.cache.free_slot)))
    sess.step_varlen(*feed, t_pos)
    sess.check_status()
    for b in range(w.B):                                      # every position once
        for l in range(w.L):
            for h in range(w.Hkv):
                lo, hi = sess.cache.rows(b, l, h)
                ln, hole = int(sess.cache.len[b, l, h]), int(sess.cache.free_slot[b, l, h])
                pos = [p for s, p in enumerate(sess.cache.pos[lo:hi].tolist()) if s != hole and s <= ln][:ln]
                assert len(set(pos)) == ln and {LENS[b], LENS[b] + 1, LENS[b] + 2, LENS[b] + 3} <= set(pos)
    # positions that the caller knows to be the same, or a new prompt, and the counter holds again
    sess.t = 300
    sess.step(*feed)
    assert sess.t == 301
    for x in (sess.cache.len, sess.cache.free_slot):
        x.zero_()
    q, k, v = (torch.randn((w.B, h, w.T, w.D), generator=gen, device="cuda").bfloat16() for h in (w.Hq, w.Hkv, w.Hkv))
    for l in range(w.L):
        sess.prefill_layer(l, q, k, v)
    sess.step(*feed)
    sess.check_status()
    assert sess.t == w.T + 1
