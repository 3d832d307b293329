"""CPU tests of what the calls for drafted tokens refuse before anything touches a device."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2502_13176_b200 import binding as bk
from paper_2502_13176_b200 import build as bkbuild

INVALID, SHAPE, WORKSPACE, UNSUPPORTED = -1, -2, -4, -7
P = 1 << 20


@pytest.fixture(scope="module", autouse=True)
def _built():
    bkbuild.build()


def cache(**kw):
    a = dict(k_slab=P, v_slab=P, pos=P, score=P, len=P, free_slot=P, cap=P, slab_off=P, seq_stride_tokens=64, B=2, status=P,
             kv_dtype=bk.KV_BF16, kv_scale=None, row_scale=None)
    a.update({k: v for k, v in kw.items() if k in a})
    return bk.CacheStruct(*a.values())


def strides(s, h, t):
    return ctypes.byref(bk.Strides(s, h, t))


def attn(**kw):
    T, Hq, Hkv, D, B = (kw.get(k, d) for k, d in (("T", 8), ("Hq", 4), ("Hkv", 2), ("D", 64), ("B", 2)))
    sh, c = bk.make_shape(1, Hq, Hkv, D), cache(**kw)
    info = bk.PlanInfo(n_items=4, n_score_items=kw.get("score_items", 0), n_units=kw.get("units", B * Hkv), chunk_tokens=128,
                       layer_begin=kw.get("layer", 0), layer_end=kw.get("layer", 0) + 1, B=kw.get("plan_B", B), ws_bytes=0)
    s = strides(Hq * T * D, T * D, D)
    a = dict(shape=ctypes.byref(sh), cache=ctypes.byref(c), q=P, qs=s, k=P, ks=s, v=P, vs=s, parent=P, n_nodes=None, T=T, out=P, os=s,
             lse=None, items=P, info=ctypes.byref(info), ws=P, ws_bytes=1 << 40, stream=None)
    a.update({k: v for k, v in kw.items() if k in a})
    return bk.lib().baklava_tree_attn(*a.values())


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(out=None), INVALID), (dict(parent=None), INVALID),
    (dict(items=None), INVALID), (dict(info=None), INVALID), (dict(ws=None), INVALID), (dict(cache=None), INVALID), (dict(shape=None), INVALID),
    (dict(T=0), INVALID), (dict(T=65), UNSUPPORTED), (dict(q=P + 8), INVALID), (dict(parent=P + 2), INVALID), (dict(lse=P + 1), INVALID),
    (dict(n_nodes=P + 2), INVALID), (dict(k_slab=None), INVALID), (dict(k_slab=P + 4), INVALID), (dict(len=None), INVALID), (dict(B=0), INVALID),
    (dict(seq_stride_tokens=72), INVALID), (dict(seq_stride_tokens=1 << 31), UNSUPPORTED), (dict(kv_dtype=3), INVALID),
    (dict(kv_dtype=bk.KV_FP8_E4M3, D=128), INVALID), (dict(kv_dtype=bk.KV_FP8_E4M3, kv_scale=P), UNSUPPORTED),
    (dict(kv_dtype=bk.KV_INT4, kv_scale=P, D=128), INVALID), (dict(layer=1), INVALID), (dict(layer=-1), INVALID), (dict(score_items=1), INVALID),
    (dict(units=3), INVALID), (dict(plan_B=3), INVALID), (dict(ws_bytes=100), WORKSPACE), (dict(qs=None), INVALID),
    (dict(os=strides(2048, 512, 0)), INVALID), (dict(ks=strides(1024, 512, 68)), INVALID), (dict(os=strides(2048, 256, 64)), INVALID),
    (dict(D=80), SHAPE), (dict(Hq=5), SHAPE)])
def test_attention_refuses(kw, code):
    assert attn(**kw) == code


def verify(**kw):
    a = dict(target=P, ts=100, draft=P, ds=100, dtype=0, tokens=P, parent=P, n_nodes=None, B=2, T=4, V=100, ua=P, us=P, flags=0, path=P,
             n_path=P, nxt=P, status=P, stream=None)
    a.update(kw)
    return bk.lib().baklava_tree_verify(*a.values())


@pytest.mark.parametrize("kw,code", [
    (dict(target=None), INVALID), (dict(tokens=None), INVALID), (dict(parent=None), INVALID), (dict(ua=None), INVALID), (dict(us=None), INVALID),
    (dict(path=None), INVALID), (dict(n_path=None), INVALID), (dict(nxt=None), INVALID), (dict(status=None), INVALID), (dict(B=0), INVALID),
    (dict(T=0), INVALID), (dict(V=0), INVALID), (dict(T=65), UNSUPPORTED), (dict(ts=99), INVALID), (dict(ds=99), INVALID), (dict(dtype=2), INVALID),
    (dict(flags=2), INVALID), (dict(target=P + 2), INVALID), (dict(draft=P + 1, dtype=1), INVALID), (dict(tokens=P + 2), INVALID),
    (dict(ts=1 << 50), INVALID)])
def test_verification_refuses(kw, code):
    assert verify(**kw) == code


def commit(**kw):
    T, Hq, Hkv, D, B = (kw.get(k, d) for k, d in (("T", 8), ("Hq", 4), ("Hkv", 2), ("D", 64), ("B", 2)))
    sh, c = bk.make_shape(1, Hq, Hkv, D), cache(**kw)
    info = bk.PlanInfo(n_items=4, n_score_items=0, n_units=kw.get("units", B * Hkv), chunk_tokens=kw.get("chunk", 128), layer_begin=0,
                       layer_end=kw.get("le", 1), B=kw.get("plan_B", B), ws_bytes=0)
    a = dict(shape=ctypes.byref(sh), cache=ctypes.byref(c), q=P, k=P, v=P, lse=P, T=T, path=P, n_path=P, max_path=4, t_pos=P, t_next=None,
             flags=0, items=P, info=ctypes.byref(info), ws=P, ws_bytes=1 << 40, stream=None)
    a.update({k: v for k, v in kw.items() if k in a})
    return bk.lib().baklava_tree_commit(*a.values())


@pytest.mark.parametrize("kw,code", [
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(q=None), INVALID), (dict(lse=None), INVALID), (dict(path=None), INVALID),
    (dict(n_path=None), INVALID), (dict(t_pos=None), INVALID), (dict(items=None), INVALID), (dict(info=None), INVALID), (dict(ws=None), INVALID),
    (dict(T=0), INVALID), (dict(T=65), UNSUPPORTED), (dict(max_path=0), INVALID), (dict(max_path=9), INVALID), (dict(t_next=P), INVALID),
    (dict(flags=1), INVALID), (dict(flags=8), INVALID), (dict(flags=256), INVALID), (dict(ws_bytes=100), WORKSPACE), (dict(units=3), INVALID),
    (dict(le=2), INVALID), (dict(plan_B=1), INVALID), (dict(chunk=0), INVALID), (dict(k=P + 8), INVALID),
    (dict(path=P + 2), INVALID), (dict(score=None), INVALID), (dict(kv_dtype=bk.KV_INT4, kv_scale=P, row_scale=P), UNSUPPORTED), (dict(D=80), SHAPE)])
def test_commit_refuses(kw, code):
    assert commit(**kw) == code


@pytest.mark.parametrize("call,words,other", [(0, 27, 28), (1, 19, 20), (2, 18, 17), (3, 18, 18), (-1, 27, 27)])
def test_calls_from_an_array(call, words, other):
    """A wrong number of words or call is refused, numbers beyond 32 bits too; with the right ones the call's own refusal comes."""
    f = bk.lib().baklava_tree_call
    pack = lambda *x: np.array(x, dtype=np.int64).tobytes()                                   # noqa: E731
    assert f(call, pack(*[0] * other), other) == INVALID and f(call, None, words) == INVALID
    if call == 1:
        good = [P, 100, P, 100, 0, P, P, 0, 2, 4, 100, P, P, 0, P, P, P, P, 0]
        assert f(1, pack(*good[:9], 65, *good[10:]), 19) == UNSUPPORTED and f(1, pack(*good[:9], 1 << 32, *good[10:]), 19) == INVALID
    if call == 0:
        sh, c = bk.make_shape(1, 4, 2, 80), cache()
        assert f(0, pack(ctypes.addressof(sh), ctypes.addressof(c), *[0] * 25), 27) == SHAPE
    if call == 2:
        sh, c = bk.make_shape(1, 4, 2, 80), cache()
        assert f(2, pack(ctypes.addressof(sh), ctypes.addressof(c), *[0] * 16), 18) == SHAPE


def test_workspace_of_nothing():
    sh, info = bk.make_shape(1, 4, 2, 64), bk.PlanInfo(n_items=4, chunk_tokens=128)
    size = lambda i, m: bk.lib().baklava_tree_commit_workspace_size(ctypes.byref(sh), i, m)   # noqa: E731
    assert size(ctypes.byref(info), 4) > 0 and size(None, 4) == 0 and size(ctypes.byref(info), 0) == 0 and size(ctypes.byref(info), 65) == 0


@pytest.mark.parametrize("kw,code", [(dict(B=0), INVALID), (dict(layer=2), INVALID), (dict(layer=-1), INVALID), (dict(T=0), INVALID),
                                     (dict(T=65), UNSUPPORTED), (dict(n_sm=0), INVALID), (dict(chunk_tokens=-1), INVALID), (dict(kv_dtype=3), INVALID),
                                     (dict(cap=[[64, 65], [16, 16]]), INVALID), (dict(cap=[[0, 64], [16, 16]]), INVALID)])
def test_plan_refuses(kw, code):
    a = dict(shape=bk.make_shape(2, 4, 2, 64), cap=[[64, 64], [16, 16]], B=1, layer=0, T=8)
    a.update(kw)
    with pytest.raises(bk.BaklavaError) as e:
        bk.baklava_tree_plan(**a)
    assert e.value.code == code


@pytest.mark.parametrize("chunk", [0, 1, 128, 500, 1 << 30])
def test_plan_covers_every_row_once(chunk):
    rng = np.random.default_rng(chunk)
    cap = 16 * rng.integers(1, 400, (3, 5)).astype(np.int32)
    sh = bk.make_shape(3, 10, 5, 128)
    for B in (1, 7):
        plan = bk.baklava_tree_plan(sh, cap, B, 1, 20, chunk_tokens=chunk)
        items = plan.items
        assert plan.info.n_items == len(items) and plan.info.n_units == 5 * B and (plan.info.layer_begin, plan.info.layer_end) == (1, 2)
        assert plan.info.ws_bytes >= len(items) * 2 * 20 * (128 * 4 + 8)
        at = 0
        seen = set()
        while at < len(items):                                # a head's pieces follow one another from row 0 on
            unit, pieces = items[at, 0], items[at, 3] >> 16
            assert unit not in seen
            seen.add(unit)
            upto = 0
            for i in range(pieces):
                u, start, length, w = items[at + i]
                assert u == unit and w == i | pieces << 16 and start == upto and length % 128 == 0
                upto += length
            assert upto >= cap[1, unit % 5] > upto - items[at, 2]
            at += pieces
        assert seen == set(range(5 * B))


def test_tensors_of_other_kinds_are_refused():
    sh = bk.make_shape(1, 4, 2, 64)
    z = lambda *s, dtype=torch.bfloat16: torch.zeros(s, dtype=dtype)                          # noqa: E731
    c = type("C", (), dict(B=2, k_slab=z(4, 64), struct=cache()))()
    plan = bk.baklava_tree_plan(sh, [[64, 64]], 2, 0, 8)
    good = dict(q=z(2, 4, 8, 64), k=z(2, 2, 8, 64), v=z(2, 2, 8, 64), parent=z(2, 8, dtype=torch.int32), n_nodes=None, out=z(2, 4, 8, 64), lse=None)
    for name, bad in [("q", z(2, 4, 8, 64, dtype=torch.float16)), ("k", z(2, 2, 7, 64)), ("v", z(2, 2, 64, 8).transpose(2, 3)),
                      ("parent", z(2, 8, dtype=torch.int64)), ("n_nodes", z(3, dtype=torch.int32)), ("out", z(2, 4, 8, 32)),
                      ("lse", z(2, 4, 8)), ("q", z(3, 4, 8, 64))]:
        with pytest.raises(ValueError):
            bk.baklava_tree_attn(sh, c, **dict(good, **{name: bad}), plan=plan, ws=z(1024, dtype=torch.uint8))
    p = torch.zeros((2, 4, 100))
    i = lambda *s: torch.zeros(s, dtype=torch.int32)                                          # noqa: E731
    good = dict(target=p, draft=p, tokens=i(2, 4), parent=i(2, 4), n_nodes=None, u_accept=torch.zeros(2, 4), u_sample=torch.zeros(2), path=i(2, 4),
                n_path=i(2), next_token=i(2), status=i(1))
    for name, bad in [("target", p.half()), ("draft", p.bfloat16()), ("draft", p[:, :, :50]), ("target", torch.zeros((2, 100, 4)).transpose(1, 2)),
                      ("target", torch.zeros((2, 8, 100))[:, ::2][:, :4].as_strided((2, 4, 100), (900, 100, 1))), ("tokens", i(4, 2)), ("u_sample", torch.zeros(3))]:
        with pytest.raises(ValueError):
            bk.baklava_tree_verify(**dict(good, **{name: bad}))
