"""4-bit slabs: the quantising bulk eviction and the decode step against the oracle run on the values the codes stand
for.  Codes, scales, positions, kept sets and slots must agree exactly; outputs within the decode tests' tolerance, and
in `test_attention_is_as_exact_as_its_roundings` within the bound of the roundings that are made."""
from unittest import mock

import numpy as np
import pytest
import torch

from oracle import int4 as o4
from paper_2502_13176_b200 import binding as bk
from paper_2502_13176_b200 import workloads as wl
from tests import harness
from tests.harness import Session, f64

pytestmark = pytest.mark.gpu

W4 = wl.scaled(wl.TINY, name="tiny-d128", D=128)


class Session4(Session):
    """The harness's session over 4-bit slabs."""

    def __init__(self, w, **kw):
        self.four = wl.kv_int4_scales(w, wl.kv_scales(w))            # [L, Hkv, 4, D]
        real = bk.Cache
        with mock.patch.object(harness.bk, "Cache", lambda *a, **k: real(*a, **dict(k, kv_scale=self.four))):
            super().__init__(w, kv_dtype=bk.KV_INT4, **kw)

    def as_stored(self, rows, l, h, which):
        codes, s = o4.quantise_rows(rows, self.four[l, h, 2 * which + 1])
        return o4.values(codes, s, self.four[l, h, 2 * which])

    def _rows_host(self, b, l, h):
        lo, hi = self.cache.rows(b, l, h)
        rs = self.cache.row_scale[lo:hi].cpu().numpy()
        return tuple(o4.values(o4.unpack(slab[lo:hi].cpu().numpy()), rs[:, i], self.four[l, h, 2 * i])
                     for i, slab in enumerate((self.cache.k_slab, self.cache.v_slab)))

    def head_state(self, b, l, h):
        lo, hi = self.cache.rows(b, l, h)
        c = self.cache
        K, V = self._rows_host(b, l, h)
        return dict(K=K, V=V, pos=c.pos[lo:hi].cpu().numpy().astype(np.int64), score=c.score[lo:hi].cpu().numpy(),
                    len=int(c.len[b, l, h]), free=int(c.free_slot[b, l, h]))


def test_bulk_evict_quantises_rows_exactly():
    s = Session4(W4)
    for (b, l, h) in s.heads:
        s.check_state(b, l, h, "after bulk evict")
        lo, _ = s.cache.rows(b, l, h)
        n = int(s.cache.len[b, l, h])
        codes = o4.unpack(s.cache.k_slab[lo:lo + n].cpu().numpy())
        assert codes.min() >= 1 and codes.max() == 15


def test_decode_steps_match_oracle_on_dequantised_values():
    s = Session4(W4)
    for i in range(8):
        s.step(i)


@pytest.mark.parametrize("chunk", [64, 128, 192, 320])
def test_chunkings_and_ragged_tails(chunk):
    w = wl.scaled(W4, T=700, budget=0.9)                  # capacities that are no multiple of the 256-token stage
    s = Session4(w, chunk_tokens=chunk)
    for i in range(4):
        s.step(i)


def test_filling_from_empty_then_evicting():
    w = wl.scaled(W4, budget=0.0625, steps=64)
    s = Session4(w, prefill=False)
    for i in range(int(s.cap.max()) + 4):
        s.step(i)


LONG = wl.scaled(W4, L=1, Hq=16, Hkv=2, T=8192, budget=0.6)


@pytest.mark.parametrize("w,chunk,waves", [(LONG, 0, 1), (LONG, 64, 1), (wl.scaled(W4, L=1, Hq=8, Hkv=1, T=36000, budget=0.9), 64, 2)],
                         ids=["one wave", "short chunks", "two waves"])
def test_long_heads_end_in_a_kernel_of_their_own(w, chunk, waves):
    s = Session4(w, chunk_tokens=chunk)
    assert s.plan.info.n_score_items > 0 and (s.plan.info.n_items > 444) == (waves == 2)
    for i in range(3):
        s.step(i)


def test_a_lost_wait_before_the_kernel_of_its_own():
    s = Session4(LONG, chunk_tokens=512)
    assert s.plan.info.n_score_items > 0
    lost_step(s, LONG, 0)


@pytest.mark.parametrize("Hq,Hkv", [(2, 2), (10, 2), (14, 2), (16, 2)])
def test_groups_and_batch(Hq, Hkv):
    w = wl.scaled(W4, Hq=Hq, Hkv=Hkv, B=3, T=256)
    s = Session4(w)
    for i in range(3):
        s.step(i)


def test_window_only_policy_without_scores():
    w = wl.scaled(W4, recent_num=1, recent_den=1)
    s = Session4(w)
    for i in range(6):
        s.step(i, flags=bk.FLAG_NO_SCORE)


def test_flags_no_append_and_no_evict():
    s = Session4(W4)
    s.step(0)
    s.step(1, flags=bk.FLAG_NO_APPEND)
    s.step(2, flags=bk.FLAG_NO_APPEND | bk.FLAG_NO_SCORE)
    s.step(3)


def test_per_layer_overlapping_calls():
    s = Session4(wl.scaled(W4, L=4), per_layer=True)
    for i in range(4):
        s.step(i)


def test_head_dimension_64_is_refused():
    with pytest.raises(bk.BaklavaError) as e:
        Session4(wl.TINY)
    assert e.value.code == -7


def test_varlen_steps_with_an_idle_sequence():
    w = wl.scaled(W4, B=3, T=200)
    s, ref = Session4(w), Session4(w)
    q, kn, vn = wl.decode_inputs(w, 0, s.scales, "cuda")
    t = torch.tensor([w.T, -1, w.T], dtype=torch.int32, device="cuda")
    before = [s.head_state(1, l, h) for l in range(w.L) for h in range(w.Hkv)]
    s.out.fill_(7.0)
    bk.baklava_decode_attn_varlen(s.shape, s.cache, q, kn, vn, t, s.out, s.lse, 0, s.plan, s.ws)
    ref.step(0)
    assert torch.equal(s.out[:, 0], ref.out[:, 0]) and torch.equal(s.out[:, 2], ref.out[:, 2]) and bool((s.out[:, 1] == 7.0).all())
    after = [s.head_state(1, l, h) for l in range(w.L) for h in range(w.Hkv)]
    for a, z in zip(before, after):
        assert a["len"] == z["len"] and a["free"] == z["free"]
        np.testing.assert_array_equal(a["K"], z["K"])


def test_shrinking_in_place_moves_rows_and_scales():
    s = Session4(W4)
    for i in range(3):
        s.step(i)                                          # (a freed slot lies among the rows)
    before = {key: s.head_state(*key) for key in s.heads}
    ws = torch.empty((bk.baklava_evict_workspace_size(s.shape, 1, W4.L, int(s.cap.max())),), dtype=torch.uint8, device="cuda")
    bk.baklava_evict(s.shape, s.cache, 0, W4.L, None, None, None, int(s.cap.max()), 0, 0, 0, 40, ws)
    torch.cuda.synchronize()
    assert int(s.cache.status.item()) == 0
    for key in s.heads:
        a, z = before[key], s.head_state(*key)
        n = int(s.cap[key[1], key[2]]) - 40
        assert z["len"] == n == z["free"]
        at = {int(p): j for j, p in enumerate(a["pos"]) if j != a["free"] and j <= a["len"]}
        src = [at[int(p)] for p in z["pos"][:n]]
        assert src == sorted(src)
        np.testing.assert_array_equal(z["K"][:n], a["K"][src])
        np.testing.assert_array_equal(z["V"][:n], a["V"][src])


def direct(lens, G, chan, seed, q_scale=1.0, row_scale=None, stale=float("nan")):
    """A cache of one layer whose heads hold `lens` random rows, written as codes; stale rows hold `stale` scales."""
    rng = np.random.default_rng(seed)
    H, D = len(lens), 128
    cap = np.array([[-(-(n + 1) // 16) * 16 for n in lens]], dtype=np.int32)
    off = np.concatenate([[0], np.cumsum(cap[0])[:-1]]).astype(np.int64).reshape(1, H)
    stride = int(cap.sum())
    sh = bk.make_shape(1, H * G, H, D)
    four = np.stack([chan[0], np.float32(1) / chan[0], chan[1], np.float32(1) / chan[1]], axis=1)[None].astype(np.float32)
    cache = bk.Cache(sh, cap, off, stride, 1, kv_dtype=bk.KV_INT4, kv_scale=four)
    codes = rng.integers(1, 16, (2, stride, D)).astype(np.uint8)
    scale = (row_scale(rng, (stride, 2)) if row_scale else 0.2 + 0.3 * rng.random((stride, 2))).astype(np.float32)
    free = []
    for h, n in enumerate(lens):
        free.append(int(rng.integers(0, n + 1)))
        lo = int(off[0, h])
        scale[lo + free[-1]] = stale
        scale[lo + n + 1:lo + int(cap[0, h])] = stale
    cache.k_slab.copy_(torch.from_numpy(o4.pack(codes[0])))
    cache.v_slab.copy_(torch.from_numpy(o4.pack(codes[1])))
    cache.row_scale.copy_(torch.from_numpy(scale))
    cache.len.copy_(torch.tensor(lens).reshape(1, 1, H)); cache.free_slot.copy_(torch.tensor(free).reshape(1, 1, H))
    q = (torch.from_numpy(rng.normal(size=(1, 1, H * G, D))).float() * q_scale).bfloat16().cuda()
    return sh, cache, cap, off, stride, codes, scale, free, q, four


def attend(sh, cache, cap, stride, q, chunk=0):
    plan = bk.baklava_decode_plan(sh, cap, 1, 0, 1, stride, chunk_tokens=chunk, kv_dtype=bk.KV_INT4).to("cuda")
    ws = bk.decode_workspace(plan)
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full(q.shape[:3], 7.0, device="cuda")
    bk.baklava_decode_attn(sh, cache, q, None, None, 1 << 20, out, lse, bk.FLAG_NO_APPEND | bk.FLAG_NO_SCORE, plan, ws)
    torch.cuda.synchronize()
    assert int(cache.status.item()) == 0
    return out, lse


def check_direct(lens, G, setup, out, lse):
    """Bound of an output: the probability times V scale is rounded to fp16 (2^-12 of itself, 2^-11 with the products
    around it; below the normal range 2^-25 of the largest V scale per row).  The scaled query is held to 2^-20 of its
    largest element per channel, which a code of up to 7 multiplies (sums of the terms are exact), and a logit has a
    few fp32 factors: 2^-19 of sum 15 |q c| s / sqrt(D) covers them.  The sums over the rows of 16 p s c go in steps of
    16 rows (2^-23 each); the result is rounded once to bf16 (2^-8)."""
    sh, cache, cap, off, stride, codes, scale, free, q, four = setup
    D = 128
    for h, n in enumerate(lens):
        rows = int(off[0, h]) + np.array([j for j in range(n + 1) if j != free[h]][:n])
        K = o4.values(codes[0][rows], scale[rows, 0], four[0, h, 0])
        V = o4.values(codes[1][rows], scale[rows, 1], four[0, h, 2])
        for a in range(G):
            qv = f64(q)[0, 0, h * G + a]
            s = K @ qv / np.sqrt(D)
            m = s.max()
            p = np.exp(s - m)
            l = p.sum()
            ref, ref_lse = p @ V / l, m + np.log(l)
            qc = np.abs(qv * four[0, h, 0])
            e = (2.0 ** -19 * 15 * qc.sum() + 2.0 ** -20 * D * 7 * qc.max()) * np.abs(scale[rows, 0]).max() / np.sqrt(D) + 2.0 ** -21
            span = np.abs(scale[rows, 1]).astype(np.float64)
            bound = ((2.0 ** -11 + 2 * e) * (p @ np.abs(V)) / l
                     + (n / 16 + 40) * 2.0 ** -23 * 16 * (p @ span) / l * four[0, h, 2]
                     + n * 2.0 ** -25 * 7 * span.max() / l * four[0, h, 2] + 2.0 ** -8 * np.abs(ref) + 1e-37)
            err = np.abs(f64(out)[0, 0, h * G + a] - ref)
            assert (err <= bound).all(), "head %d query %d: out, worst %.3g of its bound" % (h, a, (err / bound).max())
            el = abs(float(lse[0, 0, h * G + a]) - ref_lse)
            assert el <= e + (n / 16 + 40) * 2.0 ** -23 + 2.0 ** -22 * (1 + abs(ref_lse)), "head %d query %d: lse off by %.3g" % (h, a, el)


def plain_chan(H, rng):
    return np.stack([[np.exp(0.5 * rng.normal(size=128)) for _ in range(H)] for _ in range(2)]).astype(np.float32)


@pytest.mark.parametrize("G", [1, 3, 4, 7, 8])
def test_attention_is_as_exact_as_its_roundings(G):
    lens = [1, 2, 15, 16, 17, 63, 64, 65, 255, 256, 257, 1000, 5000]
    setup = direct(lens, G, plain_chan(len(lens), np.random.default_rng(G)), G)
    for chunk in (0, 64):
        out, lse = attend(*setup[:3], setup[4], setup[8], chunk)
        check_direct(lens, G, setup, out, lse)


def test_scales_of_any_magnitude():
    lens = [300, 300, 900]
    rng = np.random.default_rng(7)
    chan = plain_chan(3, rng)
    chan[0, 0] *= 1e-6                                     # tiny and huge channel scales, made up for by the row scales
    chan[1, 0] *= 1e5
    chan[0, 1] *= 1e4
    chan[1, 2] *= 1e-12

    def scales(r, shape):
        s = 0.2 + 0.3 * r.random(shape)
        s[:304, 0] *= 1e6; s[304:608, 0] *= 1e-4
        s[:, 1] *= np.exp(6 * r.normal(size=shape[0]))     # V rows of very different size
        s[5:50, 1] = 0.0                                   # and rows of zeros
        return s

    setup = direct(lens, 4, chan, 8, row_scale=scales)
    out, lse = attend(*setup[:3], setup[4], setup[8])
    check_direct(lens, 4, setup, out, lse)
    setup = direct([200], 2, plain_chan(1, rng), 9, row_scale=lambda r, shape: np.zeros(shape))
    out, lse = attend(*setup[:3], setup[4], setup[8])
    assert bool((out == 0).all()) and np.allclose(lse.cpu().numpy(), np.log(200), atol=1e-5)


@pytest.mark.parametrize("q_scale", [0.0, 1e-20, 300.0])
def test_queries_of_any_size(q_scale):
    lens = [100, 700]
    setup = direct(lens, 4, plain_chan(2, np.random.default_rng(3)), 10, q_scale=q_scale)
    out, lse = attend(*setup[:3], setup[4], setup[8])
    check_direct(lens, 4, setup, out, lse)


def test_scales_at_the_ends_of_the_range():
    lens = [130, 130]
    chan = plain_chan(2, np.random.default_rng(21))
    chan[0, 0] *= 1e30                                     # the scaled query is huge, the rows are tiny

    def scales(r, shape):
        s = 0.2 + 0.3 * r.random(shape)
        s[:144, 0] *= 1e-30
        s[144:, 1] = 1e-42                                 # V rows below the normal range: their sum is 0 to 1e-38
        return s

    setup = direct(lens, 4, chan, 22, row_scale=scales)
    out, lse = attend(*setup[:3], setup[4], setup[8])
    check_direct(lens[:1], 4, (setup[0], setup[1], setup[2], setup[3][:, :1], setup[4], setup[5], setup[6], setup[7][:1],
                               setup[8], setup[9][:, :1]), out, lse)
    assert float(out[:, :, 4:].float().abs().max()) <= 1e-37 and bool(torch.isfinite(lse).all())


@pytest.mark.parametrize("flags", [0, bk.FLAG_OVERLAP_PREV, bk.FLAG_NO_SCORE], ids=["two kernels", "one kernel", "no scores"])
def test_a_wait_that_runs_out_loses_the_step_and_nothing_else(flags):
    w = wl.scaled(wl.LLAMA3_8B_32K, L=2, T=3000, steps=4)
    chunk = 256 if flags != bk.FLAG_NO_SCORE else 8192     # (heads of one chunk write their own output)
    s = Session4(w, chunk_tokens=chunk)
    lost_step(s, w, flags)


def lost_step(s, w, flags):
    s.step(0)
    state = [t.clone() for t in (s.cache.len, s.cache.free_slot, s.cache.score)]
    q, kn, vn = wl.decode_inputs(w, 1, s.scales, "cuda")
    bk.baklava_set_wait_limit(2_000_000)                             # about a millisecond
    try:
        s.out.fill_(7.0)
        bk.baklava_decode_attn(s.shape, s.cache, q, kn, vn, s.t, s.out, s.lse, bk.FLAG_TEST_STALL | flags, s.plan, s.ws)
        torch.cuda.synchronize()
    finally:
        bk.baklava_set_wait_limit(100_000_000)
    assert int(s.cache.status.item()) == bk.STATUS_TIMEOUT
    assert torch.equal(state[0], s.cache.len) and torch.equal(state[1], s.cache.free_slot)
    valid = s.cache.pos.ne(-1) & (s.cache.pos < s.t)
    assert torch.equal(state[2][valid], s.cache.score[valid])
    assert torch.all(s.out == 7.0)
    s.cache.status.zero_()
    for i in range(1, 4):                                            # the same workspace, no re-zeroing
        s.step(i)


def test_empty_cache_and_infinite_stale_rows():
    setup = direct([0, 40], 2, plain_chan(2, np.random.default_rng(4)), 11, stale=float("inf"))
    out, lse = attend(*setup[:3], setup[4], setup[8])
    check_direct([0, 40][1:], 2, (setup[0], setup[1], setup[2], setup[3][:, 1:], setup[4], setup[5], setup[6], setup[7][1:],
                                  setup[8][:, :, 2:], setup[9][:, 1:]), out[:, :, 2:], lse[:, :, 2:])
    assert bool((out[:, :, :2] == 0).all()) and bool((lse[:, :, :2] == float("-inf")).all())


def test_repeated_captured_calls_give_the_same_bits():
    lens = [900, 77, 3000]
    setup = direct(lens, 7, plain_chan(3, np.random.default_rng(5)), 12)
    sh, cache, cap, _, stride, _, _, _, q, _ = setup
    out, lse = attend(sh, cache, cap, stride, q)
    plan = bk.baklava_decode_plan(sh, cap, 1, 0, 1, stride, kv_dtype=bk.KV_INT4).to("cuda")
    ws = bk.decode_workspace(plan)
    o, l = torch.zeros_like(out), torch.zeros_like(lse)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        bk.baklava_decode_attn(sh, cache, q, None, None, 1 << 20, o, l, bk.FLAG_NO_APPEND | bk.FLAG_NO_SCORE, plan, ws)
    for _ in range(3):
        o.zero_(); l.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, out) and torch.equal(l, lse)
