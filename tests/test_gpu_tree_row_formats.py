"""One token, one form in the slab: a row that joins as an accepted draft through the session has the bits that the decode step gives it."""
import numpy as np
import pytest
import torch

from oracle import int4 as o4
from paper_2502_13176_b200 import binding as bk
from tests.harness import assert_close, f64
from tests.test_gpu_speculative import LENS, held_rows, session, twin

pytestmark = pytest.mark.gpu


def stored(sess, b, l, h):
    """(positions ascending, bytes of K and V, row scales or nothing) of a head's rows."""
    c = sess.cache
    lo, hi = c.rows(b, l, h)
    slots = torch.from_numpy(twin(sess, b, l, h, held_rows(sess, b, l, h)).valid_slots())
    pos, order = torch.sort(c.pos[lo:hi].cpu()[slots])
    bits = [x[lo:hi].cpu()[slots][order].contiguous().view(torch.uint8) for x in (c.k_slab, c.v_slab) + (() if c.row_scale is None else (c.row_scale,))]
    return [pos] + bits


@pytest.mark.parametrize("kv", [bk.KV_BF16, bk.KV_FP8_E4M3, bk.KV_INT4], ids=["bf16", "fp8", "int4"])
def test_an_accepted_draft_is_stored_as_a_decoded_token(kv):
    a, gen = session(kv)
    b, _ = session(kv)
    w = a.w
    a.drafts(1)
    t_pos = torch.tensor(LENS, dtype=torch.int32, device="cuda")
    parent, path, one = torch.full((w.B, 1), -1, dtype=torch.int32, device="cuda"), torch.zeros((w.B, 1), dtype=torch.int32, device="cuda"), torch.ones((w.B,), dtype=torch.int32, device="cuda")
    made = []
    for _ in range(30):
        q, k, v = (torch.randn((w.L, w.B, h, w.D), generator=gen, device="cuda").bfloat16() for h in (w.Hq, w.Hkv, w.Hkv))
        a.tree_q.copy_(q[:, :, :, None])
        a.tree_k.copy_(k[:, :, :, None])
        a.tree_v.copy_(v[:, :, :, None])
        for l in range(w.L):
            a.tree_layer(l, parent)
        out = b.step_varlen(q, k, v, t_pos)
        if kv == bk.KV_BF16:                                  # (over codes the step attends to its own row as stored, the tree as given)
            assert_close(f64(a.tree_out[:, :, :, 0]), f64(out), "output")
        made.append([x.cpu() for x in (k, v)])
        t_pos = a.commit(path, one, t_pos)
    for s in (a, b):
        s.check_status()
    assert torch.equal(a.cache.len, b.cache.len)
    joined = 0
    for bb in range(w.B):
        for l in range(w.L):
            for h in range(w.Hkv):
                x, y = stored(a, bb, l, h), stored(b, bb, l, h)
                # over codes the scores differ by that own row, so that here and there another row may have left
                both = sorted(set(x[0].tolist()) & set(y[0].tolist()))
                assert len(both) == len(x[0]) if kv == bk.KV_BF16 else len(both) > 0.8 * len(x[0])
                for m, n in zip(x, y):
                    assert torch.equal(m[torch.isin(x[0], torch.tensor(both))], n[torch.isin(y[0], torch.tensor(both))]), (bb, l, h)
                if kv != bk.KV_INT4:
                    continue
                for i, p in enumerate(x[0].tolist()):         # and they are what the format's definition says
                    if p < LENS[bb]:
                        continue
                    joined += 1
                    for which in range(2):
                        codes, s = o4.quantise_rows(made[p - LENS[bb]][which][l, bb, h].float().numpy(), a.cache.kv_scale_host[l, h, 2 * which + 1])
                        assert x[3].view(torch.float32)[i, which].item() == s and x[1 + which][i].numpy().tolist() == o4.pack(codes).tolist()
    assert kv != bk.KV_INT4 or joined > 100
