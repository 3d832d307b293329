"""4-bit slabs under the policies and calls that meet larger groups, batches at different positions and caches that grow:
the sinks + window policy without scores, baklava_decode_attn_varlen, and the bulk eviction without a workspace."""
import numpy as np
import pytest
import torch

from paper_2502_13176_b200 import binding as bk
from paper_2502_13176_b200 import workloads as wl
from tests.test_gpu_int4 import W4, Session4
from tests.test_gpu_varlen import VarlenSession

pytestmark = pytest.mark.gpu


class Varlen4(VarlenSession, Session4):
    """Sequences at their own positions over 4-bit slabs; the twins hold the values the codes stand for."""

    def __init__(self, w, prompt_len, **kw):
        super().__init__(w, prompt_len, **kw)
        for (b, l, h), tw in self.twins.items():
            tw.K, tw.V = self.as_stored(tw.K, l, h, 0), self.as_stored(tw.V, l, h, 1)
            tw.step = self.storing(tw.step, l, h)

    def storing(self, step, l, h):
        def call(q, k, v, t_pos, **kw):
            kw["update_score"] = not self.no_scores
            return step(q, self.as_stored(k, l, h, 0), self.as_stored(v, l, h, 1), t_pos, **kw)
        return call

    def step_varlen(self, step_index, idle=(), flags=0):
        self.no_scores = bool(flags & bk.FLAG_NO_SCORE)
        super().step_varlen(step_index, idle, flags)


@pytest.mark.parametrize("chunk", [0, 64])
@pytest.mark.parametrize("Hq,Hkv", [(2, 2), (10, 2), (12, 2), (14, 2), (16, 2)])
def test_window_policy_for_every_group(Hq, Hkv, chunk):
    w = wl.scaled(W4, Hq=Hq, Hkv=Hkv, B=2, T=400, recent_num=1, recent_den=1)
    s = Session4(w, chunk_tokens=chunk)
    for i in range(5):
        s.step(i, flags=bk.FLAG_NO_SCORE)
    s.step(5, flags=bk.FLAG_NO_SCORE | bk.FLAG_NO_APPEND)
    s.step(6, flags=bk.FLAG_NO_SCORE)


@pytest.mark.parametrize("g", [2, 7])
def test_window_policy_from_empty(g):
    w = wl.scaled(W4, Hq=2 * g, Hkv=2, budget=0.0625, steps=64, recent_num=1, recent_den=1)
    s = Session4(w, prefill=False)
    for i in range(int(s.cap.max()) + 4):
        s.step(i, flags=bk.FLAG_NO_SCORE)


@pytest.mark.parametrize("g", [2, 5])
@pytest.mark.parametrize("window", [False, True], ids=["heavy", "window"])
def test_sequences_that_grow_and_evict_at_their_own_positions(g, window):
    policy = dict(recent_num=1, recent_den=1) if window else {}
    w = wl.scaled(W4, B=4, Hq=2 * g, Hkv=2, budget=0.0625, steps=64, **policy)
    s = Varlen4(w, [512, 300, 3, 0], chunk_tokens=64)
    flags = bk.FLAG_NO_SCORE if window else 0
    for i in range(int(s.cap.min()) + 6):
        s.step_varlen(i, idle=(3,) if i < 2 else (1,) if i % 5 == 0 else (), flags=flags)
    l, h = np.unravel_index(int(np.argmin(s.cap)), s.cap.shape)
    assert s.head_state(2, int(l), int(h))["len"] == int(s.cap.min()) - 1


def test_overlapping_layers_at_their_own_positions():
    s = Varlen4(wl.scaled(W4, B=4, L=4), [512, 128, 37, 0], per_layer=True)
    for i, idle in enumerate([(3,), (1, 3), (0, 1, 2), (), (0, 1, 2, 3), ()]):
        s.step_varlen(i, idle=idle)


@pytest.mark.parametrize("scored", [False, True])
def test_bulk_eviction_without_a_workspace(scored):
    w = wl.scaled(W4, B=2)
    a, b = Session4(w, prefill=False), Session4(w, prefill=False)
    ws = torch.empty((bk.baklava_evict_workspace_size(a.shape, w.B, 1, w.T),), dtype=torch.uint8, device="cuda")
    for l in range(w.L):
        k, v = wl.dense_kv_layer(w, l, a.scales, "cuda")
        score = wl.prefill_scores(w, l, "cuda") if scored else None
        strides = (0, w.Hkv * w.T, w.T)
        bk.baklava_evict(a.shape, a.cache, l, l + 1, k, v, score, w.T, *strides, 1, ws)
        bk.baklava_evict_static(b.shape, b.cache, l, l + 1, k, v, score, w.T, *strides, 1)
    torch.cuda.synchronize()
    assert int(b.cache.status.item()) == 0
    for key in a.heads:
        x, y = a.head_state(*key), b.head_state(*key)
        n = x["len"]
        assert n == y["len"] == int(a.cap[key[1], key[2]]) - 1 and x["free"] == y["free"]
        for name in ("K", "V", "pos", "score"):
            np.testing.assert_array_equal(x[name][:n], y[name][:n])


@pytest.mark.parametrize("seed", range(16))
def test_random_shapes_and_batches(seed):
    rng = np.random.default_rng(900 + seed)
    B, g, Hkv = int(rng.integers(1, 6)), int(rng.integers(1, 9)), int(rng.integers(1, 4))
    window = rng.random() < 0.3
    w = wl.scaled(W4, B=B, L=int(rng.integers(1, 3)), Hq=g * Hkv, Hkv=Hkv, T=int(rng.choice([64, 200, 512, 900])),
                  budget=float(rng.choice([0.125, 0.25, 0.5, 0.9])), seed=wl.MASTER_SEED + 300 + seed,
                  **(dict(recent_num=1, recent_den=1) if window else {}))
    lens = [int(x) for x in rng.integers(0, w.T + 1, size=B)]
    s = Varlen4(w, lens, chunk_tokens=int(rng.choice([0, 64, 128, 192])), per_layer=bool(rng.random() < 0.3))
    for i in range(8):
        idle = tuple(int(b) for b in range(B) if rng.random() < 0.25)
        s.step_varlen(i, idle=idle, flags=bk.FLAG_NO_SCORE if window else 0)
