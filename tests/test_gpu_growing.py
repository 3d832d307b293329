"""Caches that grow row by row over the ends of their chunks, in launches of several waves of blocks.  A step changes a
head's length while blocks of the same head, whose pieces hold no rows yet, may not have started; nothing they read then
may count.  Every step's lengths, slots, outputs, scores and arrival counters are checked, in batches whose sequences
join at different steps, so that some head ends a chunk at nearly every step.

The rows are multiples of 1/4 up to 7/4 with one element of 7/4 each, which every slab format holds exactly, so that one
float64 reference serves all of them."""
import numpy as np
import pytest
import torch

from paper_2502_13176_b200 import binding as bk
from tests.harness import assert_close

pytestmark = pytest.mark.gpu

FORMATS = {"bf16": bk.KV_BF16, "fp8": bk.KV_FP8_E4M3, "int4": bk.KV_INT4}


def exact_rows(shape, gen):
    x = torch.randint(-7, 8, shape, generator=gen, device="cuda").float() / 4
    x[..., 0] = 1.75
    return x.bfloat16()


def counters(plan, ws):
    """The heads' arrival counters: behind the workspace's first 256 bytes."""
    return ws[256:256 + 4 * plan.info.n_units].view(torch.int32)


def grow(kv, g, D, L, Hkv, B, cap, chunk, steps, flags, n_sm=148, recent=(1, 2), per_layer=False):
    gen = torch.Generator(device="cuda").manual_seed(cap + 31 * g + steps)
    sh = bk.make_shape(L, g * Hkv, Hkv, D, recent_num=recent[0], recent_den=recent[1])
    caps = np.full((L, Hkv), cap, dtype=np.int32)
    off = (np.arange(L * Hkv, dtype=np.int64) * cap).reshape(L, Hkv)
    one = {bk.KV_FP8_E4M3: np.ones((L, Hkv, 4), np.float32), bk.KV_INT4: np.ones((L, Hkv, 4, D), np.float32)}.get(kv)
    cache = bk.Cache(sh, caps, off, L * Hkv * cap, B, kv_dtype=kv, kv_scale=one)
    spans = [(l, l + 1) for l in range(L)] if per_layer else [(0, L)]
    plans = [bk.baklava_decode_plan(sh, caps, B, a, z, L * Hkv * cap, chunk_tokens=chunk, n_sm=n_sm, kv_dtype=kv).to("cuda") for a, z in spans]
    wss = [bk.decode_workspace(p) for p in plans]
    hist = torch.zeros((2, L, B, Hkv, steps, D), dtype=torch.float64, device="cuda")
    held = torch.zeros((L, B, Hkv, steps), dtype=torch.float64, device="cuda")          # reference scores
    out = torch.zeros((L, B, g * Hkv, D), dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros((L, B, g * Hkv), device="cuda")
    joins = torch.arange(B, device="cuda", dtype=torch.int32)                           # sequence b joins at step b
    for step in range(steps):
        t = torch.where(step >= joins, step - joins, torch.full_like(joins, -1))
        q = (torch.randn((L, B, g * Hkv, D), generator=gen, device="cuda") * 0.7).bfloat16()
        kn, vn = exact_rows((L, B, Hkv, D), gen), exact_rows((L, B, Hkv, D), gen)
        torch.cuda.synchronize()
        for i, ((a, z), plan, ws) in enumerate(zip(spans, plans, wss)):
            bk.baklava_decode_attn_varlen(sh, cache, q[a:z], kn[a:z], vn[a:z], t, out[a:z], lse[a:z],
                                          flags | (bk.FLAG_OVERLAP_PREV if i else 0), plan, ws)
        torch.cuda.synchronize()
        assert int(cache.status.item()) == 0
        n = t + 1                                                                       # rows now (0: not joined)
        for state in (cache.len, cache.free_slot):
            assert torch.equal(state, n.view(B, 1, 1).expand(B, L, Hkv)), "step %d" % step
        for plan, ws in zip(plans, wss):
            assert not bool(counters(plan, ws).any()), "step %d: arrivals left behind" % step
        on = t >= 0
        at = t.clamp(min=0).long()
        b = torch.arange(B, device="cuda")
        for which, x in enumerate((kn, vn)):
            hist[which, :, b, :, at] = torch.where(on.view(B, 1, 1, 1), x.double().transpose(0, 1), hist[which, :, b, :, at])
        top = int(n.max())
        K, V = hist[0, ..., :top, :], hist[1, ..., :top, :]
        s = torch.einsum("lbhgd,lbhtd->lbhgt", q.double().view(L, B, Hkv, g, D), K) / D ** 0.5
        hidden = torch.arange(top, device="cuda") >= n.view(B, 1)
        s = s.masked_fill(hidden.view(1, B, 1, 1, top), float("-inf"))
        p = torch.softmax(s, dim=-1).nan_to_num(0.0)
        ref, ref_lse = torch.einsum("lbhgt,lbhtd->lbhgd", p, V), torch.logsumexp(s, dim=-1)
        live = on.cpu().numpy()
        assert_close(out.view(L, B, Hkv, g, D)[:, live].double().cpu(), ref[:, live].cpu(), "step %d out" % step)
        assert_close(lse.view(L, B, Hkv, g)[:, live].double().cpu(), ref_lse[:, live].cpu(), "step %d lse" % step)
        held[..., :top] += p.sum(dim=3)
    score = cache.score.view(B, L, Hkv, cap)[..., :steps].transpose(0, 1).double()
    valid = torch.arange(steps, device="cuda") < n.view(1, B, 1, 1)
    want = torch.zeros_like(held) if flags & bk.FLAG_NO_SCORE else held
    assert_close(torch.where(valid, score, 0.0).cpu(), torch.where(valid, want, 0.0).cpu(), "scores")
    rows = torch.arange(cap, device="cuda").view(1, 1, 1, cap).expand(B, L, Hkv, cap)
    there = rows < n.view(B, 1, 1, 1)
    assert torch.equal(cache.pos.view(B, L, Hkv, cap)[there].long(), rows[there])        # no row was written twice


# (heads, pieces of 64 rows): 1 024 heads of 8 pieces are 8 192 blocks, at least six waves of them
@pytest.mark.parametrize("flags", [0, bk.FLAG_NO_SCORE, bk.FLAG_NO_EVICT], ids=["scores", "no scores", "no evict"])
@pytest.mark.parametrize("kv,g,D", [("bf16", 4, 128), ("bf16", 2, 64), ("fp8", 4, 128), ("int4", 4, 128), ("int4", 7, 128)])
def test_lengths_over_the_ends_of_chunks(kv, g, D, flags):
    grow(FORMATS[kv], g, D, L=2, Hkv=8, B=64, cap=512, chunk=64, steps=140, flags=flags)


@pytest.mark.parametrize("kv,g", [("bf16", 4), ("int4", 4), ("int4", 5)])
def test_window_policy(kv, g):
    grow(FORMATS[kv], g, 128, L=2, Hkv=8, B=64, cap=512, chunk=64, steps=140, flags=bk.FLAG_NO_SCORE, recent=(1, 1))


def test_score_pass_of_its_own():
    # told of a very large device, the plan takes the launch for a short one and lists the score pieces: four of 256 rows
    # to a head, 8 192 blocks of the second kernel
    sh, caps = bk.make_shape(1, 64, 32, 128), np.full((1, 32), 1024, dtype=np.int32)
    assert bk.baklava_decode_plan(sh, caps, 64, 0, 1, 32768, chunk_tokens=256, n_sm=1 << 16).info.n_score_items == 8192
    grow(bk.KV_BF16, 2, 128, L=1, Hkv=32, B=64, cap=1024, chunk=256, steps=330, flags=0, n_sm=1 << 16)


def test_score_pass_of_long_4bit_heads():
    grow(bk.KV_INT4, 2, 128, L=1, Hkv=1, B=2, cap=65536, chunk=256, steps=520, flags=0)


@pytest.mark.parametrize("kv", ["bf16", "int4"])
def test_overlapping_calls_layer_by_layer(kv):
    grow(FORMATS[kv], 4, 128, L=4, Hkv=8, B=32, cap=256, chunk=64, steps=100, flags=0, per_layer=True)


@pytest.mark.parametrize("kv", ["bf16", "fp8", "int4"])
@pytest.mark.parametrize("flags,n_sm", [(0, 148), (0, 1), (bk.FLAG_NO_SCORE, 148)], ids=["two kernels", "one kernel", "no scores"])
def test_a_lost_step_of_a_growing_head(kv, flags, n_sm):
    # the first piece gives up its wait, the pieces without rows arrive: nothing of the step counts, the counters are zero
    # again, and the head grows on over the end of the piece
    L, Hkv, g, D, cap = 1, 3, 4, 128, 512
    sh = bk.make_shape(L, g * Hkv, Hkv, D)
    caps = np.full((L, Hkv), cap, dtype=np.int32)
    off = (np.arange(L * Hkv, dtype=np.int64) * cap).reshape(L, Hkv)
    kind = FORMATS[kv]
    one = {bk.KV_FP8_E4M3: np.ones((L, Hkv, 4), np.float32), bk.KV_INT4: np.ones((L, Hkv, 4, D), np.float32)}.get(kind)
    cache = bk.Cache(sh, caps, off, Hkv * cap, 1, kv_dtype=kind, kv_scale=one)
    plan = bk.baklava_decode_plan(sh, caps, 1, 0, 1, Hkv * cap, chunk_tokens=128 if kind != bk.KV_FP8_E4M3 else 256, n_sm=n_sm, kv_dtype=kind).to("cuda")
    ws = bk.decode_workspace(plan)
    gen = torch.Generator(device="cuda").manual_seed(5)
    # (256-row pieces are fed 128 rows, 128-row pieces 64)
    at = 100 if kind != bk.KV_FP8_E4M3 else 200
    steps = at + 70
    hist = torch.zeros((2, Hkv, steps, D), dtype=torch.float64, device="cuda")
    out, lse = torch.zeros((L, 1, g * Hkv, D), dtype=torch.bfloat16, device="cuda"), torch.zeros((L, 1, g * Hkv), device="cuda")
    for t in range(steps):
        q = (torch.randn((L, 1, g * Hkv, D), generator=gen, device="cuda") * 0.7).bfloat16()
        kn, vn = exact_rows((L, 1, Hkv, D), gen), exact_rows((L, 1, Hkv, D), gen)
        if t == at:
            score = cache.score.clone()
            out.fill_(7.0)
            bk.baklava_set_wait_limit(2_000_000)                     # about a millisecond
            try:
                bk.baklava_decode_attn(sh, cache, q, kn, vn, t, out, lse, flags | bk.FLAG_TEST_STALL, plan, ws)
                torch.cuda.synchronize()
            finally:
                bk.baklava_set_wait_limit(100_000_000)
            assert int(cache.status.item()) == bk.STATUS_TIMEOUT
            cache.status.zero_()
            assert bool((cache.len == t).all()) and bool((cache.free_slot == t).all()) and bool((out == 7.0).all())
            held = (torch.arange(cap, device="cuda") < t).repeat(Hkv)
            assert torch.equal(cache.score[held], score[held]) and not bool(counters(plan, ws).any())
        bk.baklava_decode_attn(sh, cache, q, kn, vn, t, out, lse, flags, plan, ws)
        torch.cuda.synchronize()
        hist[0, :, t], hist[1, :, t] = kn[0, 0].double(), vn[0, 0].double()
        s = torch.einsum("hgd,htd->hgt", q.double().view(Hkv, g, D), hist[0, :, :t + 1]) / D ** 0.5
        ref = torch.einsum("hgt,htd->hgd", torch.softmax(s, -1), hist[1, :, :t + 1])
        assert_close(out.view(Hkv, g, D).double().cpu(), ref.cpu(), "step %d out" % t)
        assert int(cache.status.item()) == 0 and bool((cache.len == t + 1).all()) and bool((cache.free_slot == t + 1).all())
        assert not bool(counters(plan, ws).any())
