"""4-bit attention where rows of very different sizes meet: a key that takes nearly all of the probability, thousands of
rows that share the rest, and a value row whose scale stands far above theirs."""
import numpy as np
import pytest
import torch

from oracle import int4 as o4
from tests.harness import f64
from tests.test_gpu_int4 import attend, direct, plain_chan

pytestmark = pytest.mark.gpu


def check(lens, G, setup, out, lse):
    """Bound of an output.  The product of probability and V scale, relative to the largest scale and times 2^15, is
    rounded to fp16: 2^-11 of itself, with the two factors around it 2^-11 + 2^-22, and below the normal range (2^-14)
    2^-25, hence 2^-40 of the largest V scale per row, times a code of up to 7.  The scaled query is held to 2^-20 of its
    largest element per channel, which a code of up to 7 multiplies (sums of the terms are exact), and a logit has a
    few fp32 factors: 2^-19 of sum 15 |q c| s / sqrt(D) covers them.  The accumulators hold sums of u p s with u up to 15
    and eight of the same p s, in steps of 16 rows (2^-23 each).  The result is rounded once to bf16 (2^-8)."""
    sh, cache, cap, off, stride, codes, scale, free, q, four = setup
    D = 128
    for h, n in enumerate(lens):
        rows = int(off[0, h]) + np.array([j for j in range(n + 1) if j != free[h]][:n])
        K = o4.values(codes[0][rows], scale[rows, 0], four[0, h, 0])
        V = o4.values(codes[1][rows], scale[rows, 1], four[0, h, 2])
        top = np.abs(scale[rows, 0]) * 1.0
        span = np.abs(scale[rows, 1]).astype(np.float64)
        for a in range(G):
            qv = f64(q)[0, 0, h * G + a]
            s = K @ qv / np.sqrt(D)
            m = s.max()
            p = np.exp(s - m)
            l = p.sum()
            ref, ref_lse = p @ V / l, m + np.log(l)
            qc = np.abs(qv * four[0, h, 0])
            # of every row's logit, relative to the largest one: the factors move both
            e = (2.0 ** -19 * 15 * qc.sum() + 2.0 ** -20 * D * 7 * qc.max()) * top / np.sqrt(D)
            e = e + e[s.argmax()] + 2.0 ** -21 + 2.0 ** -22 * np.abs(s)
            share = (p * e).sum() / l                                      # of the normaliser
            bound = ((2.0 ** -11 + 2.0 ** -22) * (p @ np.abs(V)) + (p * e) @ np.abs(V)) / l + share * np.abs(ref) \
                + (n / 16 + 40) * 2.0 ** -23 * 23 * (p @ span) / l * four[0, h, 2] \
                + n * 2.0 ** -40 * 7 * span.max() / l * four[0, h, 2] + 2.0 ** -8 * np.abs(ref)
            err = np.abs(f64(out)[0, 0, h * G + a] - ref)
            assert (err <= bound).all(), "head %d query %d: out, worst %.3g of its bound" % (h, a, (err / bound).max())
            el = abs(float(lse[0, 0, h * G + a]) - ref_lse)
            assert el <= e.max() + (n / 16 + 40) * 2.0 ** -23 + 2.0 ** -22 * (1 + abs(ref_lse)), "head %d query %d: lse off by %.3g" % (h, a, el)


@pytest.mark.parametrize("G", [1, 4, 7])
@pytest.mark.parametrize("outlier", [1.0, 300.0, 1024.0, 4096.0])
def test_many_small_shares_beside_a_dominant_key_and_a_large_value_row(G, outlier):
    lens = [60000, 3000]
    rng = np.random.default_rng(int(outlier) + G)
    chan = plain_chan(2, rng)

    def scales(r, shape):
        s = 0.2 + 0.3 * r.random(shape)
        s[:, 0] *= 0.05                                      # logits of the many lie within a few tenths
        return s

    setup = direct(lens, G, chan, 40 + G, row_scale=scales)
    sh, cache, cap, off, stride, codes, scale, free, q, four = setup
    base = torch.randn((1, 1, 2, 1, 128), generator=torch.Generator().manual_seed(G))
    q.copy_((base + 0.1 * torch.randn((1, 1, 2, G, 128), generator=torch.Generator().manual_seed(G + 1))).flatten(2, 3).bfloat16())
    codes[1][:] = rng.integers(12, 16, codes[1].shape)       # values that add up
    for h, n in enumerate(lens):
        lo = int(off[0, h])
        key, big = (lo + (i if free[h] > i else i + 1) for i in (n // 3, n // 2))
        x = base[0, 0, h, 0].numpy() * four[0, h, 0]
        codes[0][key] = np.clip(np.rint(7 * x / np.abs(x).max()), -7, 7) + 8
        unit = o4.values(codes[0][key], np.float32(1), four[0, h, 0]) @ base[0, 0, h, 0].numpy() / np.sqrt(128)
        scale[key] = 12.0 / unit, 0.01                       # a logit of about 12 and next to no value
        scale[big, 1] *= outlier
    cache.k_slab.copy_(torch.from_numpy(o4.pack(codes[0])))
    cache.v_slab.copy_(torch.from_numpy(o4.pack(codes[1])))
    cache.row_scale.copy_(torch.from_numpy(scale))
    for chunk in (0, 2048):
        out, lse = attend(sh, cache, cap, stride, q, chunk)
        check(lens, G, setup, out, lse)


@pytest.mark.parametrize("G", [4, 7])
@pytest.mark.parametrize("power", [-100, 109])
def test_scaled_queries_at_the_ends_of_their_range(G, power):
    # up to 2^112 and down to where 2^-20 of the largest element is still held; the rows' scales make up for it
    lens = [700, 90]
    rng = np.random.default_rng(G + 200 + power)
    chan = plain_chan(2, rng)
    chan = (chan / np.abs(chan).max() * 1.9).astype(np.float32)
    chan[0] *= np.float32(2.0 ** power)
    setup = direct(lens, G, chan, 60 + G, row_scale=lambda r, shape: (0.2 + 0.3 * r.random(shape)) * np.array([2.0 ** -power, 1.0]))
    q = setup[8]
    q.copy_(q.clamp(-4, 4))
    out, lse = attend(*setup[:3], setup[4], q)
    check(lens, G, setup, out, lse)
