"""baklava_prefill_attn and its packed form against Eq. 1 in float64.

Tolerance of an output element, from the roundings the kernel makes: probabilities are rounded to bf16 for the product
with V (2^-8 of each term, hence of sum_j p_j |v_j|), the result once more (2^-8 of itself); a logit is a sum of D
products in fp32 (D + 8 steps of 2^-23 of sum |q_d k_d| / sqrt(D), the factor 2 over 2^-24 for an adder that cuts
off), scaled and shifted by the reference in fp32 (2^-22 of the largest logit) and exponentiated to 2^-21, which moves
a probability by that much relative to itself; row sum and accumulation of P V add T steps of 2^-23.
"""
import numpy as np
import pytest
import torch

from oracle import prefill as oprefill
from paper_2502_13176_b200 import binding as bk

pytestmark = pytest.mark.gpu
TIMEOUT, BAD_STATE = bk.STATUS_TIMEOUT, bk.STATUS_BAD_STATE


def reference(q, k, v):
    """One head in float64: q, k, v [n, D] -> (out, bound of out, lse, bound of lse)."""
    q, k, v = q.double(), k.double(), v.double()
    n, D = q.shape
    hidden = torch.ones((n, n), dtype=torch.bool, device=q.device).triu(1)
    s = (q @ k.T / D ** 0.5).masked_fill(hidden, float("-inf"))
    lse = torch.logsumexp(s, dim=1)
    p = torch.exp(s - lse[:, None])
    out = p @ v
    size = (q.abs() @ k.abs().T / D ** 0.5).masked_fill(hidden, 0.0).amax(dim=1)
    e = (D + 8) * 2.0 ** -23 * size + 2.0 ** -22 * s.masked_fill(hidden, 0.0).abs().amax(dim=1) + 2.0 ** -21
    bound = (2.0 ** -8 + 2 * e[:, None] + n * 2.0 ** -23) * (p @ v.abs()) + 2.0 ** -8 * out.abs() + 1e-37
    return out, bound, lse, e + n * 2.0 ** -23 + 2.0 ** -22 * (1 + lse.abs())


def make(B, T, Hq, Hkv, D, seed=0, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [(torch.randn((B, h, T, D), generator=g, device="cuda") * scale).bfloat16() for h in (Hq, Hkv, Hkv)]


def run(q, k, v, lens=None, want_lse=True, fill=7.0):
    B, Hq, T, D = q.shape
    out = torch.full((B, Hq, T, D), fill, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((B, Hq, T), fill, dtype=torch.float32, device="cuda") if want_lse else None
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    n = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    bk.baklava_prefill_attn(bk.make_shape(1, Hq, k.shape[1], D), q, k, v, n, out, lse, status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    return out, lse


def check_head(q, k, v, out, lse, what):
    ref, bound, rl, bl = reference(q, k, v)
    err = (out.double() - ref).abs()
    assert bool((err <= bound).all()), "%s: out, worst %.3g of its bound" % (what, float((err / bound).max()))
    if lse is not None:
        el = (lse.double() - rl).abs()
        assert bool((el <= bl).all()), "%s: lse, worst %.3g of its bound" % (what, float((el / bl).max()))


def check_padded(q, k, v, out, lse, lens=None, fill=7.0):
    B, Hq, T, D = q.shape
    g = Hq // k.shape[1]
    for b in range(B):
        n = T if lens is None else min(max(lens[b], 0), T)
        for h in range(Hq):
            if n:
                check_head(q[b, h, :n], k[b, h // g, :n], v[b, h // g, :n], out[b, h, :n], None if lse is None else lse[b, h, :n],
                           "sequence %d head %d" % (b, h))
        assert bool((out[b, :, n:] == fill).all()) and (lse is None or bool((lse[b, :, n:] == fill).all()))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T", [1, 2, 7, 8, 9, 64, 127, 128, 129, 255, 256, 300, 513])
def test_lengths_around_the_tiles(D, T):
    q, k, v = make(1, T, 3, 1, D, seed=T)
    out, lse = run(q, k, v)
    check_padded(q, k, v, out, lse)


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (8, 1), (7, 7), (14, 2), (6, 3)])
def test_grouped_heads_and_batches(Hq, Hkv):
    q, k, v = make(3, 170, Hq, Hkv, 128, seed=Hq)
    out, lse = run(q, k, v)
    check_padded(q, k, v, out, lse)


@pytest.mark.parametrize("D", [64, 128])
def test_ragged_padded_batch_with_garbage_in_the_padding(D):
    lens = [300, 0, 1, 129, 1000, 77]
    q, k, v = make(6, 300, 4, 2, D, seed=5)
    for b, n in enumerate(lens):
        for x in (q, k, v):
            x[b, :, min(n, 300):] = float("nan") if b % 2 else float("inf")
    out, lse = run(q, k, v, lens)
    check_padded(q, k, v, out, lse, lens)


def test_long_prompt_and_no_lse():
    q, k, v = make(1, 4500, 2, 1, 128, seed=9)
    out, lse = run(q, k, v)
    check_padded(q, k, v, out, lse)
    assert torch.equal(run(q, k, v, want_lse=False)[0], out)      # and the same bits every time


@pytest.mark.parametrize("D", [64, 128])
def test_packed_token_major_rows(D):
    lens = [5, 0, 128, 300, 1, 0, 259, 127]
    Hq, Hkv, tail = 6, 2, 40
    total = sum(lens) + tail
    g = torch.Generator(device="cuda").manual_seed(3)
    rows = torch.randn((total, (Hq + 2 * Hkv) * D + 16), generator=g, device="cuda").bfloat16()
    rows[sum(lens):] = float("nan")                               # rows behind the last prompt
    heads = rows[:, :(Hq + 2 * Hkv) * D].unflatten(-1, (Hq + 2 * Hkv, D)).transpose(0, 1)
    q, k, v = heads[:Hq], heads[Hq:Hq + Hkv], heads[Hq + Hkv:]
    out = torch.full((total, Hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((Hq, total), 7.0, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    cu = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")
    bk.baklava_prefill_attn_packed(bk.make_shape(1, Hq, Hkv, D), q, k, v, cu, 300, out.transpose(0, 1), lse, status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    at = 0
    for n in lens:
        for h in range(Hq):
            if n:
                check_head(q[h, at:at + n], k[h // 3, at:at + n], v[h // 3, at:at + n], out[at:at + n, h], lse[h, at:at + n],
                           "rows %d.. head %d" % (at, h))
        at += n
    assert bool((out[at:] == 7.0).all()) and bool((lse[:, at:] == 7.0).all())


def test_packed_prompt_does_not_see_its_neighbours():
    Hq, Hkv, D = 2, 1, 128
    q, k, v = (x[0] for x in make(1, 600, Hq, Hkv, D, seed=11))
    cu = torch.tensor([0, 150, 450, 600], dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def go(q, k, v):
        out, lse = torch.zeros((Hq, 600, D), dtype=torch.bfloat16, device="cuda"), torch.zeros((Hq, 600), device="cuda")
        bk.baklava_prefill_attn_packed(bk.make_shape(1, Hq, Hkv, D), q, k, v, cu, 300, out, lse, status)
        return out, lse

    out, lse = go(q, k, v)
    for x in (q, k, v):
        x[:, :150] = float("nan")
        x[:, 450:] = float("inf")
    out2, lse2 = go(q, k, v)
    assert torch.equal(out[:, 150:450], out2[:, 150:450]) and torch.equal(lse[:, 150:450], lse2[:, 150:450])
    assert int(status.item()) == 0


@pytest.mark.parametrize("bounds,bad", [([0, 100, 90, 200], {1}), ([0, 100, 250], {1}), ([-5, 60, 200], {0}), ([0, 180, 200], {0})])
def test_packed_bounds_that_are_none_are_skipped(bounds, bad):
    Hq, Hkv, D, total, T = 2, 2, 64, 200, 150
    q, k, v = (x[0] for x in make(1, total, Hq, Hkv, D))
    out = torch.full((Hq, total, D), 7.0, dtype=torch.bfloat16, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    bk.baklava_prefill_attn_packed(bk.make_shape(1, Hq, Hkv, D), q, k, v, torch.tensor(bounds, dtype=torch.int32, device="cuda"), T,
                                   out, None, status)
    torch.cuda.synchronize()
    assert int(status.item()) == BAD_STATE
    written = torch.zeros(total, dtype=torch.bool)
    for i in range(len(bounds) - 1):
        if i not in bad:
            written[bounds[i]:bounds[i + 1]] = True
            for h in range(Hq):
                a, z = bounds[i], bounds[i + 1]
                if len(bounds) == 3:                              # (prompts that overlap others are written twice)
                    check_head(q[h, a:z], k[h, a:z], v[h, a:z], out[h, a:z], None, "prompt %d" % i)
    assert bool((out[:, ~written.cuda()] == 7.0).all())


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_a_row_does_not_depend_on_later_tokens(D, bad):
    T, at = 400, 200
    q, k, v = make(1, T, 2, 1, D, seed=21)
    out, lse = run(q, k, v)
    for x in (q, k, v):
        x[:, :, at:] = bad
    out2, lse2 = run(q, k, v)
    # the row block that holds token `at` is done again against its rows' true maxima: same values up to rounding
    assert torch.equal(out[:, :, :128], out2[:, :, :128]) and torch.equal(lse[:, :, :128], lse2[:, :, :128])
    check_padded(q[:, :, :at], k[:, :, :at], v[:, :, :at], out2[:, :, :at], lse2[:, :, :at])
    assert out2[:, :, at:].isnan().all()


def test_value_rows_with_infinities_reach_exactly_the_rows_that_see_them():
    T, D = 300, 128
    q, k, v = make(1, T, 2, 1, D, seed=22)
    clean, _ = run(q, k, v)
    v[0, 0, 140, 5] = float("inf")
    v[0, 0, 150, 5] = float("-inf")
    v[0, 0, 10, 70] = float("nan")
    out, lse = run(q, k, v)
    o = out[0].float()
    assert o[:, 10:, 70].isnan().all() and not o[:, :10].isnan().any()
    assert (o[:, 140:150, 5] == float("inf")).all() and o[:, 150:, 5].isnan().all()
    cols = [c for c in range(D) if c not in (5, 70)]
    check = torch.zeros_like(v); check.copy_(v)
    check[~torch.isfinite(check)] = 0.0
    for h in range(2):
        ref, bound, rl, bl = reference(q[0, h], k[0, 0], check[0, 0])
        assert bool(((out[0, h].double() - ref).abs() <= bound)[:, cols].all())
        assert bool(((out[0, h].double() - ref).abs() <= bound)[:140, 5].all())
        assert bool(((lse[0, h].double() - rl).abs() <= bl).all())


@pytest.mark.parametrize("D", [64, 128])
def test_keys_far_above_the_first_eight_are_redone_exactly(D):
    T = 700
    q, k, v = make(1, T, 2, 1, D, seed=23)
    k[0, 0, 333] = (q[0, 0, 500].float() * 40).bfloat16()        # logits of several hundred for some of the rows
    k[0, 0, 80] = (-q[0, 1, 90].float() * 30).bfloat16()
    q[0, 1, 640:] *= 20
    out, lse = run(q, k, v)
    assert float(lse.max()) > 200
    check_padded(q, k, v, out, lse)


def test_large_and_tiny_magnitudes():
    for scale in (1e-3, 12.0):
        q, k, v = make(1, 260, 2, 2, 128, seed=24, scale=scale)
        out, lse = run(q, k, v)
        check_padded(q, k, v, out, lse)


def test_log_sum_exp_feeds_the_prompt_scores():
    B, T, Hq, Hkv, D = 2, 300, 4, 2, 128
    lens = [300, 211]
    q, k, v = make(B, T, Hq, Hkv, D, seed=25)
    _, lse = run(q, k, v, lens)
    sh = bk.make_shape(1, Hq, Hkv, D)
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    ws = torch.empty((bk.baklava_prefill_workspace_size(sh, B, T),), dtype=torch.uint8, device="cuda")
    score = torch.empty((B, Hkv, T), device="cuda")
    bk.baklava_prefill_scores(sh, q, k, n, B, T, score, ws, lse=lse)
    for b in range(B):
        for h in range(Hkv):
            ref = oprefill.prefill_scores(q[b, 2 * h:2 * h + 2, :lens[b]].double().cpu().numpy(), k[b, h, :lens[b]].double().cpu().numpy())
            got = score[b, h, :lens[b]].cpu().numpy()
            assert np.all(np.abs(got - ref) <= 1e-3 + 1e-3 * np.abs(ref))
    assert bk.workspace_error(ws) == 0


def test_two_streams_and_a_captured_graph():
    q, k, v = make(2, 500, 4, 2, 128, seed=26)
    out, lse = run(q, k, v)
    sh = bk.make_shape(1, 4, 2, 128)
    streams = [torch.cuda.Stream() for _ in range(2)]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    res = [(torch.zeros_like(out), torch.zeros_like(lse)) for _ in range(2)]
    torch.cuda.synchronize()
    for s, (o, l) in zip(streams, res):
        bk.baklava_prefill_attn(sh, q, k, v, None, o, l, status, stream=s)
    torch.cuda.synchronize()
    for o, l in res:
        assert torch.equal(o, out) and torch.equal(l, lse)
    graph = torch.cuda.CUDAGraph()
    o, l = torch.zeros_like(out), torch.zeros_like(lse)
    with torch.cuda.graph(graph):
        bk.baklava_prefill_attn(sh, q, k, v, None, o, l, status)
    for _ in range(2):
        o.zero_(); l.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, out) and torch.equal(l, lse)
    assert int(status.item()) == 0


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(2, 1), (6, 2), (14, 2), (8, 1), (20, 4)])
@pytest.mark.parametrize("T", [1, 2, 8, 9, 16, 17, 32, 33, 63, 64])
def test_short_prompts_share_a_tile_among_the_heads_of_a_group(D, Hq, Hkv, T):
    lens = [T, 0, (T + 1) // 2, T]
    q, k, v = make(4, T, Hq, Hkv, D, seed=T + Hq)
    for b, n in enumerate(lens):
        for x in (q, k, v):
            x[b, :, n:] = float("nan")
    out, lse = run(q, k, v, lens)
    check_padded(q, k, v, out, lse, lens)


@pytest.mark.parametrize("D,T", [(64, 20), (128, 7), (128, 50)])
def test_many_short_packed_prompts(D, T):
    # more row blocks than places for CTAs: they go on from one to another
    rng = np.random.default_rng(T)
    lens = rng.integers(0, T + 1, 200)
    Hq, Hkv, total = 15, 5, int(lens.sum()) + 3
    g = torch.Generator(device="cuda").manual_seed(T)
    heads = torch.randn((total, Hq + 2 * Hkv, D), generator=g, device="cuda").bfloat16().transpose(0, 1)
    q, k, v = heads[:Hq], heads[Hq:Hq + Hkv], heads[Hq + Hkv:]
    out = torch.full((total, Hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((Hq, total), 7.0, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    cu = torch.from_numpy(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)).cuda()
    bk.baklava_prefill_attn_packed(bk.make_shape(1, Hq, Hkv, D), q, k, v, cu, T, out.transpose(0, 1), lse, status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    at = 0
    for n in lens:
        for h in range(Hq if n else 0):
            check_head(q[h, at:at + n], k[h // 3, at:at + n], v[h // 3, at:at + n], out[at:at + n, h], lse[h, at:at + n],
                       "rows %d.. head %d" % (at, h))
        at += int(n)
    assert bool((out[at:] == 7.0).all()) and bool((lse[:, at:] == 7.0).all())


@pytest.mark.parametrize("D", [64, 128])
def test_short_prompts_done_again(D):
    # infinite and NaN tokens, in a head of its own and in the keys of all, and logits of several hundred
    T, at = 48, 30
    q, k, v = make(2, T, 6, 2, D, seed=31)
    k[0, 0, 20] = (q[0, 1, 25].float() * 40).bfloat16()
    out, lse = run(q, k, v)
    assert float(lse.max()) > 200
    check_padded(q, k, v, out, lse)
    bad = [x.clone() for x in (q, k, v)]
    bad[0][0, 2, 5] = float("nan")                                # one row of one head
    bad[1][1, :, at:], bad[2][1, :, at:] = float("inf"), float("nan")
    out2, lse2 = run(*bad)
    assert bool(out2[0, 2, 5].isnan().all())
    out2[0, 2, 5], lse2[0, 2, 5] = out[0, 2, 5], lse[0, 2, 5]
    check_padded(q[:1], k[:1], v[:1], out2[:1], lse2[:1])
    check_padded(q[1:, :, :at], k[1:, :, :at], v[1:, :, :at], out2[1:, :, :at], lse2[1:, :, :at])
    assert bool(out2[1, :, at:].isnan().all())


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T,Hq,Hkv", [(128, 4, 4), (100, 6, 1), (40, 16, 2)])
def test_runs_of_one_tile_blocks(D, T, Hq, Hkv):
    # a block of one tile asks nothing of the lower thread of a row before the upper one writes its sum: thousands of them
    # in a row, which every CTA goes through one after the other, give the same bits every time
    q, k, v = make(500, T, Hq, Hkv, D, seed=T)
    lens = [T - b % 7 if b % 5 else T // 2 for b in range(500)]
    out, lse = run(q, k, v, lens)
    for _ in range(10):
        again = run(q, k, v, lens)
        assert torch.equal(again[0], out) and torch.equal(again[1], lse)
    check_padded(q[::25], k[::25], v[::25], out[::25], lse[::25], lens[::25])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T", [50, 300])
def test_values_up_to_the_end_of_the_range(D, T):
    # averages of values between 1e37 and 3.3e38: the terms' sum is far outside fp32, the average is not
    q, k, v = make(1, T, 4, 2, D, seed=33, scale=0.3)
    g = torch.Generator(device="cuda").manual_seed(T)
    v.copy_((1e37 + 3.2e38 * torch.rand(v.shape, generator=g, device="cuda", dtype=torch.float64)).bfloat16())
    v[:, :, :, ::3] *= -1
    out, lse = run(q, k, v)
    check_padded(q, k, v, out, lse)
    # and beside infinities, which are looked for among them
    at = T // 2
    v2 = v.clone()
    v2[0, 0, at, 1] = float("inf")
    out2, lse2 = run(q, k, v2)
    assert bool((out2[0, :2, at:, 1] == float("inf")).all())
    v2[0, 0, at, 1] = 0.0
    for h in range(2):
        ref, bound, rl, bl = reference(q[0, h], k[0, 0], v2[0, 0])
        cols = [c for c in range(D) if c != 1]
        assert bool(((out2[0, h].double() - ref).abs() <= bound)[:, cols].all())
        assert bool(((out2[0, h].double() - ref).abs() <= bound)[:at, 1].all())
        assert bool(((lse2[0, h].double() - rl).abs() <= bl).all())
