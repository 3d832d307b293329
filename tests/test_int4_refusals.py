"""CPU tests: what the calls that take a cache refuse of 4-bit slabs, before anything touches a device."""
import ctypes

import numpy as np
import pytest

from paper_2502_13176_b200 import binding as bk
from paper_2502_13176_b200 import build as bkbuild

INVALID, UNSUPPORTED = -1, -7
P = 1 << 20


@pytest.fixture(scope="module", autouse=True)
def _built():
    bkbuild.build()


def cache(**kw):
    a = dict(k_slab=P, v_slab=P, pos=P, score=P, len=P, free_slot=P, cap=P, slab_off=P, seq_stride_tokens=64, B=1, status=P,
             kv_dtype=bk.KV_INT4, kv_scale=P, row_scale=P)
    a.update(kw)
    return bk.CacheStruct(*a.values())


def decode(c, D=128):
    sh = bk.make_shape(1, 2, 1, D)
    info = bk.PlanInfo(n_items=1, n_score_items=0, n_units=1, chunk_tokens=64, layer_begin=0, layer_end=1, B=1, ws_bytes=0)
    return bk.lib().baklava_decode_attn(ctypes.byref(sh), ctypes.byref(c), P, P, P, 5, P, None, 0, P, ctypes.byref(info), P, 1 << 30, None)


def evict(c, D=128):
    sh = bk.make_shape(1, 2, 1, D)
    return bk.lib().baklava_evict(ctypes.byref(sh), ctypes.byref(c), 0, 1, P, P, None, 64, 64, 64, 64, 1, P, 1 << 30, None)


@pytest.mark.parametrize("call", [decode, evict])
@pytest.mark.parametrize("kw,code", [(dict(row_scale=None), INVALID), (dict(kv_scale=None), INVALID), (dict(row_scale=P + 8), INVALID),
                                     (dict(kv_scale=P + 4), INVALID), (dict(seq_stride_tokens=72), INVALID), (dict(kv_dtype=3), INVALID)])
def test_cache_refused(call, kw, code):
    assert call(cache(**kw)) == code


@pytest.mark.parametrize("call", [decode, evict])
def test_other_head_sizes_refused(call):
    assert call(cache(), 64) == UNSUPPORTED


def test_plan_knows_the_format():
    sh = bk.make_shape(1, 4, 2, 128)
    cap = np.array([[40000, 8000]], dtype=np.int32)
    plan = bk.baklava_decode_plan(sh, cap, 4, 0, 1, int(cap.sum()), kv_dtype=bk.KV_INT4)
    assert plan.info.n_items > 0
    with pytest.raises(bk.BaklavaError):
        bk.baklava_decode_plan(sh, cap, 4, 0, 1, int(cap.sum()), kv_dtype=3)


def test_plan_of_one_very_long_head_stays_mergeable():
    for Hq in (1, 8):
        sh = bk.make_shape(1, Hq, 1, 128)
        cap = np.array([[2 << 20]], dtype=np.int32)
        plan = bk.baklava_decode_plan(sh, cap, 1, 0, 1, 2 << 20, kv_dtype=bk.KV_INT4)
        items = plan.items[:plan.info.n_items]
        assert plan.info.n_items * Hq <= 48 * 128
        assert (np.sort(items[:, 1]) == np.cumsum(np.concatenate([[0], items[np.argsort(items[:, 1]), 2]]))[:-1]).all()
        assert items[:, 2].sum() >= 2 << 20 and (items[:, 2] % 64 == 0).all()
