"""CPU tests of the argument checks of the prompt-side attention calls: refused before anything touches a device (the
pointers are never dereferenced)."""
import ctypes
from types import SimpleNamespace

import pytest
import torch

from paper_2502_13176_b200 import binding as bk
from paper_2502_13176_b200 import build as bkbuild
from paper_2502_13176_b200 import engine

INVALID, SHAPE, UNSUPPORTED = -1, -2, -7


@pytest.fixture(scope="module", autouse=True)
def _built():
    bkbuild.build()


P = ctypes.c_void_p(1 << 20)


def strides(seq, head, token):
    return ctypes.byref(bk.Strides(seq, head, token))


def rope(**kw):
    B, T, Hq, Hkv, D = (kw.get(k, d) for k, d in (("B", 2), ("T", 8), ("Hq", 4), ("Hkv", 2), ("D", 64)))
    sh = bk.make_shape(1, Hq, Hkv, D)
    s = strides(Hq * T * D, T * D, D)
    a = dict(shape=ctypes.byref(sh), q=P, qs=s, k=P, ks=s, pos=P, B=B, T=T, freq=P, rot=D, qw=None, kw=None, eps=1e-6, flags=0,
             qo=P, qos=s, ko=P, kos=s, stream=None)
    a.update({k: v for k, v in kw.items() if k in a})
    return bk.lib().baklava_qk_norm_rope(*a.values())


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), INVALID), (dict(k=None), INVALID), (dict(pos=None), INVALID), (dict(freq=None), INVALID),
    (dict(qo=None), INVALID), (dict(ko=None), INVALID), (dict(shape=None), INVALID),
    (dict(q=ctypes.c_void_p((1 << 20) + 8)), INVALID), (dict(qw=ctypes.c_void_p((1 << 20) + 2)), INVALID),
    (dict(pos=ctypes.c_void_p((1 << 20) + 2)), INVALID),
    (dict(B=0), INVALID), (dict(T=0), INVALID), (dict(flags=2), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID),
    (dict(rot=0), SHAPE), (dict(rot=8), SHAPE), (dict(rot=128), SHAPE), (dict(rot=40), SHAPE), (dict(D=80), SHAPE), (dict(Hq=5), SHAPE),
    (dict(qs=None), INVALID), (dict(qos=strides(1024, 512, 0)), INVALID), (dict(kos=strides(1024, 32, 64)), INVALID),
    (dict(ks=strides(1024, 512, 68)), INVALID), (dict(qs=strides(-2048, 512, 64)), INVALID),
    (dict(B=1 << 17, T=1 << 15), UNSUPPORTED)])
def test_norm_rope_refuses(kw, code):
    assert rope(**kw) == code


def attn(packed=False, **kw):
    B, T, Hq, Hkv, D = (kw.get(k, d) for k, d in (("B", 2), ("T", 8), ("Hq", 4), ("Hkv", 2), ("D", 64)))
    sh = bk.make_shape(1, Hq, Hkv, D)
    s = strides(Hq * T * D, T * D, D)
    a = dict(shape=ctypes.byref(sh), q=P, qs=s, k=P, ks=s, v=P, vs=s, len=P if packed else None, B=B, T=T)
    if packed:
        a["total"] = 16
    a.update(out=P, os=s, lse=None, status=P, stream=None)
    a.update({k: v for k, v in kw.items() if k in a})
    return (bk.lib().baklava_prefill_attn_packed if packed else bk.lib().baklava_prefill_attn)(*a.values())


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("kw,code", [
    (dict(q=None), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(out=None), INVALID), (dict(status=None), INVALID),
    (dict(shape=None), INVALID), (dict(v=ctypes.c_void_p((1 << 20) + 4)), INVALID), (dict(lse=ctypes.c_void_p((1 << 20) + 2)), INVALID),
    (dict(status=ctypes.c_void_p((1 << 20) + 1)), INVALID), (dict(len=ctypes.c_void_p((1 << 20) + 2)), INVALID),
    (dict(B=0), INVALID), (dict(T=0), INVALID), (dict(T=-1), INVALID), (dict(B=65536), UNSUPPORTED), (dict(D=96), SHAPE), (dict(Hq=3), SHAPE),
    (dict(Hq=18), SHAPE), (dict(qs=None), INVALID), (dict(os=strides(2048, 512, 32)), INVALID), (dict(ks=strides(2048, 516, 64)), INVALID),
    (dict(vs=strides(2048, 0, 64)), INVALID)])
def test_prompt_attention_refuses(packed, kw, code):
    assert attn(packed, **kw) == code


def test_packed_wants_bounds_and_rows():
    assert attn(True, len=None) == INVALID
    assert attn(True, total=0) == INVALID
    assert attn(True, total=1 << 31) == UNSUPPORTED


def test_binding_refuses_other_types_shapes_and_devices():
    sh = bk.make_shape(1, 4, 2, 64)
    good = torch.zeros((1, 4, 8, 64), dtype=torch.bfloat16)
    kv = torch.zeros((1, 2, 8, 64), dtype=torch.bfloat16)
    status = torch.zeros(1, dtype=torch.int32)
    for q in (good.float(), good[:, :3], good[..., :32], good.transpose(2, 3)):
        with pytest.raises(ValueError):
            bk.baklava_prefill_attn(sh, q, kv, kv, None, good, None, status)
    if not torch.cuda.is_available():
        with pytest.raises((ValueError, RuntimeError, AssertionError)):      # host tensors
            bk.baklava_prefill_attn(sh, good, kv, kv, None, good, None, status)


def session(monkeypatch, scores=lambda ws: None):
    """A session of two sequences whose calls into the library do nothing but what `scores` does to the workspace."""
    sess = engine.DecodeSession.__new__(engine.DecodeSession)
    sess.w = SimpleNamespace(B=2, L=2, Hq=4, Hkv=2, D=64)
    sess.shape, sess.device, sess.prompt_error = None, "cpu", None
    sess.cache = SimpleNamespace(status=torch.zeros(1, dtype=torch.int32))
    calls = []
    for name in ("baklava_prefill_attn", "baklava_evict_varlen"):
        monkeypatch.setattr(bk, name, lambda *a, **kw: calls.append(a))
    for name in ("baklava_prefill_workspace_size", "baklava_evict_workspace_size"):
        monkeypatch.setattr(bk, name, lambda *a: 256)
    monkeypatch.setattr(bk, "baklava_prefill_scores", lambda *a, **kw: scores(a[7]))
    return sess, calls


def prompt(B=2, T=8):
    return [torch.zeros((B, h, T, 64), dtype=torch.bfloat16) for h in (4, 2, 2)]


def test_session_prompt_refuses_other_batches_and_layouts(monkeypatch):
    # the scores and the eviction read the prompt's tensors densely, for as many sequences as the cache has
    sess, calls = session(monkeypatch)
    q, k, v = prompt()
    sess.prefill_layer(1, q, k, v)
    assert len(calls) == 2
    wide = torch.zeros((2, 8, 8, 64), dtype=torch.bfloat16).transpose(1, 2)
    for bad in ((0, *prompt(B=1)), (0, *prompt(B=3)), (0, q, k, prompt(T=9)[2]), (0, q, k[:, :1], v), (0, wide[:, :4], k, v),
                (0, q, wide[:, :2], v), (0, q, k, wide[:, :2]), (2, q, k, v), (-1, q, k, v)):
        with pytest.raises(ValueError):
            sess.prefill_layer(*bad)
    assert len(calls) == 2


@pytest.mark.parametrize("bad_layer", [0, 1])
def test_session_keeps_the_error_of_every_layer(monkeypatch, bad_layer):
    layer = [0]
    sess, _ = session(monkeypatch, lambda ws: ws[:4].view(torch.int32).fill_(int(layer[0] == bad_layer)))
    for layer[0] in range(2):
        sess.prefill_layer(layer[0], *prompt())
    with pytest.raises(RuntimeError, match="prompt scores"):
        sess.check_status()


@pytest.mark.parametrize("seq,head,token,code", [
    (64, 64, 64, INVALID), (2048, 64, 64, INVALID), (64, 512, 64, INVALID), (512, 512, 64, INVALID),
    (2048, 448, 64, INVALID), (2048, 512, 72, INVALID), (2040, 512, 64, INVALID), (2048, 64, 248, INVALID),
    (1 << 38, 1 << 38, 1 << 38, INVALID)])
def test_outputs_that_overlap_themselves_are_refused(seq, head, token, code):
    # [2, 4, 8, 64] in less room than it takes, or with rows across others
    assert rope(qos=strides(seq, head, token)) == code
    assert attn(os=strides(seq, head, token)) == code


def test_output_layouts_that_are_no_overlap():
    # every order of the axes, dense and as slices of something wider; inputs whose rows lie across each other too.  The
    # rotary dimension, which is looked at later, is out of range, so that nothing is enqueued where the strides pass
    import itertools
    for pad in (0, 64, 192):
        for order in itertools.permutations(range(3)):
            step, st = 64 + pad, [0, 0, 0]
            for axis in order:
                st[axis] = step
                step = step * (2, 4, 8)[axis] + pad
            assert rope(qos=strides(*st), rot=8) == SHAPE
    assert rope(qs=strides(64, 64, 64), ks=strides(64, 128, 64), rot=8) == SHAPE
    assert rope(qos=strides(0, 512, 64), kos=strides(-8, 512, 64), B=1, rot=8) == SHAPE
    assert rope(qos=strides(512, 64, 3), kos=strides(512, 64, 0), T=1, rot=8) == SHAPE


@pytest.mark.parametrize("wrong", [64, 32])
def test_head_dimension_of_the_tensors_and_of_the_shape(wrong):
    # rows of 64 elements are not read as rows of 128, however far apart they lie
    sh, st = bk.make_shape(1, 4, 2, 128), torch.zeros(1, dtype=torch.int32)
    q, k = (torch.zeros((1, h, 8, 256), dtype=torch.bfloat16)[..., :wrong] for h in (4, 2))
    pos = torch.zeros((1, 8), dtype=torch.int32)
    freq = torch.ones(wrong // 2)
    with pytest.raises(ValueError, match=r"\[1, 4, 8, 128\]"):
        bk.baklava_prefill_attn(sh, q, k, k, None, q, None, st)
    with pytest.raises(ValueError, match=r"\[1, 4, 8, 128\]"):
        bk.baklava_qk_norm_rope(sh, q, k, pos, freq, None, None, 1e-6, q, k)
    with pytest.raises(ValueError, match=r"\[1, 4, 8, 128\]"):
        bk.baklava_prefill_attn_packed(sh, q[0], k[0], k[0], pos[0, :2], 8, q[0], None, st)
