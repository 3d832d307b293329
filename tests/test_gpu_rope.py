"""baklava_qk_norm_rope against the float64 oracle.

Tolerance: everything is fp32 until one rounding to bf16 (half a step, 2^-8 of the value).  Before it an output is
u cos - v sin of normed elements; each of u, v carries the norm's few roundings (square root, division, three
products: below 8 * 2^-24 relative) and the sum of squares (D * 2^-24), cosine and sine 2^-22 absolute including the
rounding of the remainder's angle, the products 2 * 2^-24: below (D + 64) * 2^-24 of |u| + |v| altogether.
"""
import numpy as np
import pytest
import torch

from oracle import rope as oracle
from paper_2502_13176_b200 import binding as bk

pytestmark = pytest.mark.gpu


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def reference(x, pos, freq, w, eps, interleaved):
    """(expected, bound) for x [B, H, T, D]."""
    out, bound = [], []
    for b in range(x.shape[0]):
        y = oracle.norm_heads(x[b], w, eps)
        r = oracle.rotate(y, pos[b], freq, interleaved)
        both = np.abs(y).copy()
        rot = 2 * len(freq)
        ia, ib = ((np.arange(0, rot, 2), np.arange(1, rot, 2)) if interleaved
                  else (np.arange(rot // 2), np.arange(rot // 2, rot)))
        s = both[..., ia] + both[..., ib]
        both[..., ia], both[..., ib] = s, s
        out.append(r)
        bound.append(both)
    r, both = np.stack(out), np.stack(bound)
    D = x.shape[-1]
    return r, 2.0 ** -8 * np.abs(r) + (1 + 2.0 ** -8) * (D + 64) * 2.0 ** -24 * both + 1e-38


def call(case, q, k, pos, freq, qw, kw, qo, ko, stream=None):
    Hq, Hkv, D = q.shape[1], k.shape[1], q.shape[3]
    bk.baklava_qk_norm_rope(bk.make_shape(1, Hq, Hkv, D), q, k, pos, freq, qw, kw, 1e-6, qo, ko,
                            bk.ROPE_INTERLEAVED if case["il"] else 0, stream)


def inputs(B, T, Hq, Hkv, D, rot, norm, far=0, seed=0, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    qkv = (torch.randn((B, T, (Hq + 2 * Hkv) * D), generator=g, device="cuda") * scale).bfloat16()
    q = qkv[..., :Hq * D].unflatten(-1, (Hq, D)).transpose(1, 2)
    k = qkv[..., Hq * D:(Hq + Hkv) * D].unflatten(-1, (Hkv, D)).transpose(1, 2)
    pos = (far + torch.randint(0, 5, (B, 1), generator=g, device="cuda") + torch.arange(T, device="cuda")).to(torch.int32)
    freq = (10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)).float().cuda()
    w = [(1 + 0.3 * torch.randn(D, generator=g, device="cuda")).bfloat16() if norm else None for _ in range(2)]
    return q, k, pos, freq, w[0], w[1]


def check(got, x, pos, freq, w, il, what):
    ref, bound = reference(f64(x), pos.cpu().numpy().astype(np.int64), f64(freq), None if w is None else f64(w), 1e-6, il)
    err = np.abs(f64(got) - ref)
    assert (err <= bound).all(), "%s: worst %.3g of its bound" % (what, float((err / bound).max()))


CASES = [
    dict(B=1, T=1, Hq=1, Hkv=1, D=64, rot=64, norm=True, il=False),
    dict(B=1, T=1, Hq=32, Hkv=8, D=128, rot=128, norm=True, il=False, far=1 << 30),
    dict(B=7, T=1, Hq=28, Hkv=4, D=128, rot=128, norm=True, il=True, far=131072),
    dict(B=2, T=37, Hq=6, Hkv=2, D=64, rot=32, norm=False, il=True),
    dict(B=2, T=37, Hq=6, Hkv=3, D=128, rot=96, norm=True, il=False, far=1000),
    dict(B=1, T=200, Hq=5, Hkv=5, D=64, rot=16, norm=True, il=False, far=2 ** 31 - 1 - 300),
    dict(B=3, T=1701, Hq=3, Hkv=1, D=128, rot=128, norm=False, il=False),     # many tokens per CTA,
    dict(B=3, T=1701, Hq=9, Hkv=3, D=64, rot=48, norm=True, il=True),         #   the last CTA's not all there
]


@pytest.mark.parametrize("c", CASES)
def test_matches_the_oracle_from_projection_slices_to_head_major(c):
    q, k, pos, freq, qw, kw = inputs(c["B"], c["T"], c["Hq"], c["Hkv"], c["D"], c["rot"], c["norm"], c.get("far", 0))
    qo, ko = (torch.zeros(x.shape, dtype=torch.bfloat16, device="cuda") for x in (q, k))
    call(c, q, k, pos, freq, qw, kw, qo, ko)
    check(qo, q, pos, freq, qw, c["il"], "q")
    check(ko, k, pos, freq, kw, c["il"], "k")


@pytest.mark.parametrize("D,Hq,Hkv", [(64, 2, 1), (128, 18, 6)])
@pytest.mark.parametrize("B,T", [(1, 296), (1, 297), (2, 296), (1, 593), (2, 592), (5, 237), (1, 2367), (3, 791)])
def test_every_number_of_tokens_per_cta(B, T, D, Hq, Hkv):
    # the numbers change behind 296, 592, 1 184 and 2 368 tokens (few heads go on to sixteen); ragged ends, sequences that
    # end inside a CTA's tokens
    c = dict(il=T % 2 == 0)
    q, k, pos, freq, qw, kw = inputs(B, T, Hq, Hkv, D, D, True, seed=T)
    qo, ko = (torch.zeros(x.shape, dtype=torch.bfloat16, device="cuda") for x in (q, k))
    call(c, q, k, pos, freq, qw, kw, qo, ko)
    check(qo, q, pos, freq, qw, c["il"], "q")
    check(ko, k, pos, freq, kw, c["il"], "k")


def test_one_weight_only_and_extreme_rows():
    q, k, pos, freq, qw, kw = inputs(1, 9, 4, 2, 128, 128, True)
    q = q.contiguous()
    q[0, 0, 0] = 0.0                                         # a row of zeros stays zero
    q[0, 1, 3] *= 1e-18                                      # squares below the normal range
    q[0, 2, 4] *= 1e15
    c = dict(il=False)
    qo, ko = torch.zeros_like(q), torch.zeros(k.shape, dtype=torch.bfloat16, device="cuda")
    call(c, q, k, pos, freq, qw, None, qo, ko)
    check(qo, q, pos, freq, qw, False, "q")
    check(ko, k, pos, freq, None, False, "k")
    assert (qo[0, 0, 0] == 0).all()


def test_a_row_with_nan_or_infinity_leaves_the_others_alone():
    q, k, pos, freq, qw, kw = inputs(1, 40, 4, 2, 64, 64, True)
    clean_q, clean_k = (torch.zeros(x.shape, dtype=torch.bfloat16, device="cuda") for x in (q, k))
    call(dict(il=False), q, k, pos, freq, qw, kw, clean_q, clean_k)
    bad = q.clone()
    bad[0, 1, 5, 3], bad[0, 2, 6, 7] = float("nan"), float("inf")
    qo, ko = torch.zeros_like(clean_q), torch.zeros_like(clean_k)
    call(dict(il=False), bad, k, pos, freq, qw, kw, qo, ko)
    assert qo[0, 1, 5].isnan().any() and qo[0, 2, 6].isnan().any()
    qo[0, 1, 5], qo[0, 2, 6] = clean_q[0, 1, 5], clean_q[0, 2, 6]
    assert torch.equal(qo, clean_q) and torch.equal(ko, clean_k)


def test_in_place_idle_tokens_and_untouched_neighbours():
    q, k, pos, freq, qw, kw = inputs(2, 21, 4, 2, 128, 64, True)
    out = [torch.zeros(x.shape, dtype=torch.bfloat16, device="cuda") for x in (q, k)]
    call(dict(il=False), q, k, pos, freq, qw, kw, *out)
    whole = q._base if q._base is not None else q
    before = whole.clone()
    pos2 = pos.clone()
    pos2[1, 4] = -1
    keep = q[1, :, 4].clone()
    call(dict(il=False), q, k, pos2, freq, qw, kw, q, k)     # over the projection's rows
    assert torch.equal(q[1, :, 4], keep)                     # the idle token is as it was
    q2 = q.clone(); q2[1, :, 4] = out[0][1, :, 4]
    assert torch.equal(q2, out[0])
    D, Hq, Hkv = 128, 4, 2
    assert torch.equal(whole[..., (Hq + Hkv) * D:], before[..., (Hq + Hkv) * D:])     # the values were not touched


def test_decode_layout_other_stream_and_captured_graph():
    q, k, pos, freq, qw, kw = inputs(5, 1, 28, 4, 128, 128, True)
    out = [torch.zeros(x.shape, dtype=torch.bfloat16, device="cuda") for x in (q, k)]
    call(dict(il=False), q, k, pos, freq, qw, kw, *out)
    qd, kd = torch.zeros((5, 28, 128), dtype=torch.bfloat16, device="cuda"), torch.zeros((5, 4, 128), dtype=torch.bfloat16, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):                            # one token of each sequence along the token axis
        args = (q.permute(2, 1, 0, 3), k.permute(2, 1, 0, 3), pos.T.contiguous())
        call(dict(il=False), *args, freq, qw, kw, qd.transpose(0, 1)[None], kd.transpose(0, 1)[None])
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            call(dict(il=False), *args, freq, qw, kw, qd.transpose(0, 1)[None], kd.transpose(0, 1)[None])
    assert torch.equal(qd, out[0][:, :, 0]) and torch.equal(kd, out[1][:, :, 0])
    qd.zero_(); kd.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(qd, out[0][:, :, 0]) and torch.equal(kd, out[1][:, :, 0])
