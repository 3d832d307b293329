"""Probabilities that count as nothing (zeros of either sign, negative numbers, NaN) and the smallest that do not, anywhere in the rows."""
import numpy as np
import pytest
import torch

from paper_2502_13176_b200 import binding as bk
from tests.test_gpu_tree_verify import case, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["drawn", "distinct", "points"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("nothing", [-0.0, -0.25, float("nan"), -1e-42])
def test_what_counts_as_nothing(kind, dtype, nothing):
    B, T, V = 24, 10, 2011
    t, d, tok, par, n, ua, us, distinct = case(31, B, T, V, kind, dtype, sharp=1.0)
    rng = np.random.default_rng(5)
    keep = rng.random((B, T, V)) < 0.1
    for b in range(B):                                        # (what was drafted keeps its probability in the draft)
        for c in range(1, T):
            keep[b, par[b, c], tok[b, c]] = True
    mask = torch.from_numpy(~keep).cuda()
    t = torch.where(mask, torch.tensor(nothing, dtype=dtype, device="cuda"), 4 * t)
    d = None if d is None else torch.where(mask, torch.tensor(nothing, dtype=dtype, device="cuda"), 4 * d)
    assert nothing != 0.0 or bool((torch.signbit(t) & (t == 0)).any())
    check(t, d, tok, par, n, ua, us, distinct)


@pytest.mark.parametrize("kind", ["drawn", "distinct", "points"])
def test_rows_of_the_smallest_numbers(kind):
    """All of a row below the smallest normal number."""
    t, d, tok, par, n, ua, us, distinct = case(32, 16, 8, 1500, kind, sharp=0.1)
    tiny = 2.0 ** -130
    t = t * tiny
    d = None if d is None else d * tiny
    assert float(t.max()) < 2.0 ** -126 and float(t.max()) > 0
    check(t, d, tok, par, n, ua, us, distinct)
