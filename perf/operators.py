"""The library's prompt-side attention operators and its 4-bit cache as cases to measure: what a serving step calls
between the QKV projection and the output projection.

  norm_rope  per-head RMS norm of queries and keys with the rotary position embedding in the same pass
  prompt     causal attention of whole prompts (grouped heads, padded or packed), with the rows' log-sum-exp
  decode4    single-token attention over budgeted caches whose slabs hold 4-bit codes

Each has a plain form in elementary torch operations, and the call a user makes of the library (`own`).
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"


# ------------------------------------------------------------------ cases
def listed():
    return [
        # one decode step of one sequence: a single token, where the call's latency is everything
        dict(name="norm-rope-1-token", op="norm_rope", B=1, T=1, Hq=32, Hkv=8, D=128, rot=128, interleaved=False,
             norm=True, decode=True, far=32768),
        # a batched decode step: one token of each of 16 sequences, group of seven
        dict(name="norm-rope-batch-16", op="norm_rope", B=16, T=1, Hq=28, Hkv=4, D=128, rot=128, interleaved=False,
             norm=True, decode=True, far=8192),
        # one layer of a 32K prompt, from the projection's token-major rows to head-major tensors
        dict(name="norm-rope-prompt-32k", op="norm_rope", B=1, T=32768, Hq=32, Hkv=8, D=128, rot=128, interleaved=False,
             norm=True, decode=False, far=0),
        # ragged small-head model: pairs side by side, half of the head rotated, no norm, far positions
        dict(name="norm-rope-ragged-d64", op="norm_rope", B=3, T=1667, Hq=12, Hkv=4, D=64, rot=32, interleaved=True,
             norm=False, decode=False, far=1 << 20),
        # a short chat turn
        dict(name="prompt-200", op="prompt", B=1, T=200, Hq=4, Hkv=2, D=64, packed=False, ragged=False),
        # one layer of a 32K prompt
        dict(name="prompt-32k", op="prompt", B=1, T=32768, Hq=32, Hkv=8, D=128, packed=False, ragged=False),
        # a prefill batch of 16 prompts of different lengths, packed token-major as the projection leaves them
        dict(name="prompt-packed-16x8k", op="prompt", B=16, T=8192, Hq=28, Hkv=4, D=128, packed=True, ragged=True),
        # many short prompts, small heads, packed
        dict(name="prompt-packed-64x500-d64", op="prompt", B=64, T=500, Hq=32, Hkv=8, D=64, packed=True, ragged=True),
        # two small caches: latency
        dict(name="decode4-small", op="decode4", L=1, B=1, Hq=4, Hkv=2, mean=256, sigma=1.0, varlen=False),
        # one layer of one sequence, 32K context at 30 %
        dict(name="decode4-layer", op="decode4", L=1, B=1, Hq=32, Hkv=8, mean=9824, sigma=1.0, varlen=False),
        # a whole step of one sequence: 32 layers, 32K context at 30 %
        dict(name="decode4-step", op="decode4", L=32, B=1, Hq=32, Hkv=8, mean=9824, sigma=1.0, varlen=False),
        # a whole step of 16 sequences at different positions, 8K context at 30 %, group of seven
        dict(name="decode4-batch", op="decode4", L=28, B=16, Hq=28, Hkv=4, mean=2448, sigma=1.5, varlen=True),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm_rope", "prompt", "decode4"])
    hkv, g = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 3, 4, 5, 6, 7, 8])
    if op == "norm_rope":
        D = rng.choice([64, 128])
        decode = rng.random() < 0.4
        B = _log_int(rng, 1, 256) if decode else rng.randint(1, 4)
        T = 1 if decode else _log_int(rng, 2, 8192)
        hkv, g = min(hkv, 8), min(g, 32 // max(hkv, 4))
        return dict(op=op, B=B, T=T, Hq=hkv * g, Hkv=hkv, D=D, rot=rng.choice([r for r in (16, 32, 64, 96, 128) if r <= D]),
                    interleaved=rng.random() < 0.5, norm=rng.random() < 0.7, decode=decode,
                    far=rng.choice([0, 4096, 32768, 1 << 20, 1 << 30]))
    if op == "prompt":
        D = rng.choice([64, 128])
        T = _log_int(rng, 1, 16384)
        B = max(1, min(64, _log_int(rng, 1, 64), int(65536 / T), int(2 ** 42 / (T * T * hkv * g * D))))
        return dict(op=op, B=B, T=T, Hq=hkv * g, Hkv=hkv, D=D, packed=rng.random() < 0.6, ragged=rng.random() < 0.7)
    L, B = _log_int(rng, 1, 32), _log_int(rng, 1, 16)
    mean = max(16, min(_log_int(rng, 64, 32768), int(2400000 / (L * B * hkv))))
    return dict(op=op, L=L, B=B, Hq=hkv * g, Hkv=hkv, mean=mean, sigma=rng.choice([0.0, 0.5, 1.0, 1.5]),
                varlen=rng.random() < 0.5)


# ------------------------------------------------------------------ what a user's program has in hand
def _capacities(case):
    """int32 [L, Hkv] tokens, multiples of 16, unequal the way an importance profile leaves them (a model's profile
    and a batch's lengths belong to the case, like its sizes: they do not change with the inputs)."""
    rs = np.random.RandomState(case["L"] * 7919 + case["mean"])
    w = np.exp(rs.standard_normal((case["L"], case["Hkv"])) * case["sigma"])
    w = np.minimum(w / w.mean(), 3.0)
    return (16 * np.maximum(2, np.round(case["mean"] * w / w.mean() / 16))).astype(np.int32)


def _lengths(case):
    rs = np.random.RandomState(case["B"] * 7919 + case["T"])
    n = rs.randint(1, case["T"] + 1, case["B"]) if case["ragged"] else np.full(case["B"], case["T"])
    if case["ragged"]:
        n[rs.randint(0, case["B"])] = case["T"]
    return n.astype(np.int32)


def _held(case, cap):
    """Rows each cache holds, [B, L, Hkv]."""
    full = np.broadcast_to(cap[None].astype(np.int64) - 1, (case["B"],) + cap.shape)
    if not case["varlen"]:
        return full.copy()
    share = np.random.RandomState(case["B"]).uniform(0.125, 1.0, (case["B"], 1, 1))
    return np.maximum(1, (full * share).astype(np.int64))


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    return {"norm_rope": _prepare_norm_rope, "prompt": _prepare_prompt, "decode4": _prepare_decode4}[case["op"]](case, gen)


def _randn(shape, gen, dtype=torch.bfloat16):
    return torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32).to(dtype)


def _prepare_norm_rope(case, gen):
    B, T, Hq, Hkv, D = (case[k] for k in ("B", "T", "Hq", "Hkv", "D"))
    qkv = _randn((B, T, (Hq + 2 * Hkv) * D), gen)            # the projection's rows; queries, keys, values side by side
    st = dict(case, qkv=qkv)
    st["q_in"] = qkv[..., :Hq * D].unflatten(-1, (Hq, D)).transpose(1, 2)                       # [B, Hq, T, D] views
    st["k_in"] = qkv[..., Hq * D:(Hq + Hkv) * D].unflatten(-1, (Hkv, D)).transpose(1, 2)
    start = torch.randint(0, case["far"] + 1, (B, 1), generator=gen, device=DEV)
    st["pos"] = (start + torch.arange(T, device=DEV)).to(torch.int32)
    st["inv_freq"] = (500000.0 ** (-torch.arange(0, case["rot"], 2, dtype=torch.float64) / case["rot"])).float().to(DEV)
    st["qw"] = (1.0 + 0.2 * torch.randn(D, generator=gen, device=DEV)).bfloat16() if case["norm"] else None
    st["kw"] = (1.0 + 0.2 * torch.randn(D, generator=gen, device=DEV)).bfloat16() if case["norm"] else None
    if case["decode"]:                                       # [B, H, D], what the decode step takes
        st["q_out"] = torch.zeros((B, Hq, D), dtype=torch.bfloat16, device=DEV)
        st["k_out"] = torch.zeros((B, Hkv, D), dtype=torch.bfloat16, device=DEV)
    else:                                                    # [B, H, T, D], what the prompt-side calls take
        st["q_out"] = torch.zeros((B, Hq, T, D), dtype=torch.bfloat16, device=DEV)
        st["k_out"] = torch.zeros((B, Hkv, T, D), dtype=torch.bfloat16, device=DEV)
    if own:
        from paper_2502_13176_b200 import binding as bk
        st["shape"] = bk.make_shape(1, Hq, Hkv, D)
    return st


def _prepare_prompt(case, gen):
    B, T, Hq, Hkv, D = (case[k] for k in ("B", "T", "Hq", "Hkv", "D"))
    n = _lengths(case)
    st = dict(case, n=n, total=int(n.sum()))
    if case["packed"]:                                       # token-major rows of all prompts, one after the other
        rows = _randn((st["total"], (Hq + 2 * Hkv) * D), gen)
        heads = rows.unflatten(-1, (Hq + 2 * Hkv, D)).transpose(0, 1)                           # [H, total, D] views
        st["q"], st["k"], st["v"] = heads[:Hq], heads[Hq:Hq + Hkv], heads[Hq + Hkv:]
        st["out"] = torch.zeros((st["total"], Hq, D), dtype=torch.bfloat16, device=DEV)
        st["lse"] = torch.zeros((Hq, st["total"]), dtype=torch.float32, device=DEV)
        st["cu"] = torch.from_numpy(np.concatenate([[0], np.cumsum(n)]).astype(np.int32)).to(DEV)
    else:
        st["q"], st["k"], st["v"] = (_randn((B, h, T, D), gen) for h in (Hq, Hkv, Hkv))
        st["out"] = torch.zeros((B, Hq, T, D), dtype=torch.bfloat16, device=DEV)
        st["lse"] = torch.zeros((B, Hq, T), dtype=torch.float32, device=DEV)
        st["len"] = torch.from_numpy(n).to(DEV) if case["ragged"] else None
    if own:
        from paper_2502_13176_b200 import binding as bk
        st["shape"] = bk.make_shape(1, Hq, Hkv, D)
        st["status"] = torch.zeros((1,), dtype=torch.int32, device=DEV)
    return st


def _quantise4(x, inv_chan):
    """Rows [n, D] -> (codes uint8 [n, D / 2], scale fp32 [n]): y = x / channel scale, scale = max |y| / 7,
    code = round(y / scale) + 8, the even channel in the low half of a byte."""
    y = x * inv_chan
    scale = y.abs().amax(dim=1) / 7.0
    u = (torch.round(y / scale[:, None]).clamp(-7, 7) + 8).to(torch.uint8)
    return u[:, 0::2] | (u[:, 1::2] << 4), scale


def _prepare_decode4(case, gen):
    L, B, Hq, Hkv, D = case["L"], case["B"], case["Hq"], case["Hkv"], 128
    cap = _capacities(case)
    flat = cap.reshape(-1).astype(np.int64)
    off = np.concatenate([[0], np.cumsum(flat)[:-1]]).reshape(L, Hkv)
    stride = int(flat.sum())
    rows = B * stride
    st = dict(case, D=D, cap=cap, off=off, stride=stride)
    # one channel of each head sticks out by 8, as keys and values of real models do; the channel scales know it
    chan = 0.5 + torch.rand((2, L, Hkv, D), generator=gen, device=DEV)
    chan.scatter_(3, torch.randint(0, D, (2, L, Hkv, 1), generator=gen, device=DEV), 8.0)
    head_of = torch.repeat_interleave(torch.arange(L * Hkv, device=DEV), torch.from_numpy(flat).to(DEV), output_size=stride)
    codes, scales = [], []
    for i in range(2):
        c = chan[i].reshape(L * Hkv, D)
        parts = [_quantise4(_randn((stride, D), gen).float() * c[head_of], 1.0 / c[head_of]) for _ in range(B)]
        codes.append(torch.cat([p[0] for p in parts]))
        scales.append(torch.cat([p[1] for p in parts]))
    st["k_codes"], st["v_codes"] = codes
    st["row_scale"] = torch.stack(scales, dim=1).contiguous()                                   # [rows, 2] K, V
    st["chan"] = torch.stack([chan[0], 1.0 / chan[0], chan[1], 1.0 / chan[1]], dim=2).contiguous()   # [L, Hkv, 4, D]
    # a full cache has one freed slot among its rows; a joining sequence is not full yet
    n = _held(case, cap)
    if case["varlen"]:
        free = n.copy()
    else:
        free = np.minimum(n, (torch.rand((B, L, Hkv), generator=gen, device=DEV).cpu().numpy() * (n + 1)).astype(np.int64))
    st["len"] = torch.from_numpy(n.astype(np.int32)).to(DEV)
    st["free"] = torch.from_numpy(free.astype(np.int32)).to(DEV)
    st["q"] = _randn((L, B, Hq, D), gen)
    st["out"] = torch.zeros((L, B, Hq, D), dtype=torch.bfloat16, device=DEV)
    st["lse"] = torch.zeros((L, B, Hq), dtype=torch.float32, device=DEV)
    st["t_pos"] = torch.full((B,), 1 << 20, dtype=torch.int32, device=DEV)
    if own:
        from paper_2502_13176_b200 import binding as bk
        st["shape"] = bk.make_shape(L, Hq, Hkv, D)
        cache = bk.Cache(st["shape"], cap, off, stride, B, kv_dtype=bk.KV_INT4, kv_scale=st["chan"].cpu().numpy())
        cache.k_slab.copy_(st["k_codes"])
        cache.v_slab.copy_(st["v_codes"])
        cache.row_scale.copy_(st["row_scale"])
        cache.len.copy_(st["len"])
        cache.free_slot.copy_(st["free"])
        st["cache"] = cache
        st["plan"] = bk.baklava_decode_plan(st["shape"], cap, B, 0, L, stride, kv_dtype=bk.KV_INT4).to(DEV)
        st["ws"] = bk.decode_workspace(st["plan"])
    return st


# ------------------------------------------------------------------ one pass
def run(st):
    if own:
        return _call(st)
    return {"norm_rope": _plain_norm_rope, "prompt": _plain_prompt, "decode4": _plain_decode4}[st["op"]](st)


def _call(st):
    from paper_2502_13176_b200 import binding as bk
    if st["op"] == "norm_rope":
        flags = bk.ROPE_INTERLEAVED if st["interleaved"] else 0
        qo, ko = (t.unsqueeze(2) if st["decode"] else t for t in (st["q_out"], st["k_out"]))
        bk.baklava_qk_norm_rope(st["shape"], st["q_in"], st["k_in"], st["pos"], st["inv_freq"], st["qw"], st["kw"], 1e-6,
                                qo, ko, flags)
        return {"q": st["q_out"], "k": st["k_out"]}
    if st["op"] == "prompt":
        if st["packed"]:
            bk.baklava_prefill_attn_packed(st["shape"], st["q"], st["k"], st["v"], st["cu"], st["T"],
                                           st["out"].transpose(0, 1), st["lse"], st["status"])
        else:
            bk.baklava_prefill_attn(st["shape"], st["q"], st["k"], st["v"], st["len"], st["out"], st["lse"], st["status"])
        return {"out": st["out"], "lse": st["lse"]}
    flags = bk.FLAG_NO_APPEND | bk.FLAG_NO_SCORE
    if st["varlen"]:
        bk.baklava_decode_attn_varlen(st["shape"], st["cache"], st["q"], None, None, st["t_pos"], st["out"], st["lse"], flags,
                                      st["plan"], st["ws"])
    else:
        bk.baklava_decode_attn(st["shape"], st["cache"], st["q"], None, None, 1 << 20, st["out"], st["lse"], flags,
                               st["plan"], st["ws"])
    return {"out": st["out"], "lse": st["lse"]}


def _plain_norm_rope(st):
    rot, half = st["rot"], st["rot"] // 2
    turns = st["pos"].double()[:, None, :, None] * st["inv_freq"].double()      # angles of far positions: 64 bits
    cos, sin = turns.cos().float(), turns.sin().float()

    def one(x, w):
        x = x.float()
        if w is not None:
            x = x * torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + 1e-6) * w.float()
        head, rest = x[..., :rot], x[..., rot:]
        if st["interleaved"]:
            a, b = head[..., 0::2], head[..., 1::2]
            head = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
        else:
            a, b = head[..., :half], head[..., half:]
            head = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
        return torch.cat([head, rest], dim=-1).bfloat16()

    q, k = one(st["q_in"], st["qw"]), one(st["k_in"], st["kw"])
    return {"q": q[:, :, 0] if st["decode"] else q.contiguous(), "k": k[:, :, 0] if st["decode"] else k.contiguous()}


def _plain_causal(q, k, v):
    """q [g, n, D], k, v [n, D] in fp32, a block of query rows at a time (the whole matrix would not fit)."""
    n, D = k.shape
    step = max(128, min(n, (1 << 27) // max(1, n)))
    outs, lses = [], []
    for r0 in range(0, n, step):
        r1 = min(n, r0 + step)
        s = (q[:, r0:r1] @ k[:r1].T) * (1.0 / math.sqrt(D))
        hidden = torch.arange(r1, device=DEV)[None, :] > torch.arange(r0, r1, device=DEV)[:, None]
        s.masked_fill_(hidden, float("-inf"))
        m = s.amax(dim=-1, keepdim=True)
        p = torch.exp(s - m)
        total = p.sum(dim=-1, keepdim=True)
        outs.append((p @ v[:r1]) / total)
        lses.append((m + torch.log(total)).squeeze(-1))
    return torch.cat(outs, dim=1), torch.cat(lses, dim=1)


def _plain_prompt(st):
    Hq, Hkv, D = st["Hq"], st["Hkv"], st["D"]
    g = Hq // Hkv
    out, lse = torch.zeros_like(st["out"]), torch.zeros_like(st["lse"])
    at = 0
    for b in range(st["B"]):
        n = int(st["n"][b])
        for h in range(Hkv):
            if st["packed"]:
                q, k, v = (st[x][i, at:at + n].float() for x, i in (("q", slice(h * g, h * g + g)), ("k", h), ("v", h)))
            else:
                q, k, v = (st[x][b, i, :n].float() for x, i in (("q", slice(h * g, h * g + g)), ("k", h), ("v", h)))
            o, s = _plain_causal(q, k, v)
            if st["packed"]:
                out[at:at + n, h * g:h * g + g] = o.transpose(0, 1).bfloat16()
                lse[h * g:h * g + g, at:at + n] = s
            else:
                out[b, h * g:h * g + g, :n] = o.bfloat16()
                lse[b, h * g:h * g + g, :n] = s
        at += n
    return {"out": out, "lse": lse}


def _plain_decode4(st):
    L, B, Hq, Hkv, D = (st[k] for k in ("L", "B", "Hq", "Hkv", "D"))
    g = Hq // Hkv
    off = torch.from_numpy(st["off"]).to(DEV)
    wide = int(st["cap"].max())
    slot = torch.arange(wide, device=DEV)
    n, free = st["len"].long(), st["free"].long()                                   # [B, L, Hkv]
    held = (slot < (n + (free < n))[..., None]) & (slot != free[..., None])           # rows are slots 0 .. len without `free`
    row = (torch.arange(B, device=DEV)[:, None, None] * st["stride"] + off)[..., None] + slot
    row = torch.where(held, row, torch.zeros_like(row))
    heads = B * L * Hkv
    out = torch.empty((B, L, Hkv, g, D), dtype=torch.bfloat16, device=DEV)
    lse = torch.empty((B, L, Hkv, g), dtype=torch.float32, device=DEV)
    step = max(1, (1 << 24) // wide)                                                # heads at a time

    def values(codes, scale, chan, at):
        c = codes[at]
        u = torch.stack([c & 15, c >> 4], dim=-1).flatten(-2).float() - 8.0
        return u * scale[at][..., None] * chan[:, None, :]

    q = st["q"].float().permute(1, 0, 2, 3).reshape(heads, g, D)
    chan = st["chan"].expand(B, L, Hkv, 4, D).reshape(heads, 4, D)
    row, held = row.reshape(heads, wide), held.reshape(heads, wide)
    for i in range(0, heads, step):
        j = slice(i, min(heads, i + step))
        s = torch.bmm(q[j], values(st["k_codes"], st["row_scale"][:, 0], chan[j, 0], row[j]).transpose(1, 2)) / math.sqrt(D)
        s = s.masked_fill(~held[j, None, :], float("-inf"))
        m = s.amax(dim=-1, keepdim=True)
        p = torch.exp(s - m)
        total = p.sum(dim=-1, keepdim=True)
        o = torch.bmm(p, values(st["v_codes"], st["row_scale"][:, 1], chan[j, 2], row[j])) / total
        out.view(heads, g, D)[j] = o.bfloat16()
        lse.view(heads, g)[j] = (m + torch.log(total)).squeeze(-1)
    return {"out": out.permute(1, 0, 2, 3, 4).reshape(L, B, Hq, D), "lse": lse.permute(1, 0, 2, 3).reshape(L, B, Hq)}


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    if case["op"] == "norm_rope":
        n = case["B"] * case["T"]
        elems = n * (case["Hq"] + case["Hkv"]) * case["D"]
        return {"bytes": 4 * elems + 4 * n, "flops": 8 * elems}
    if case["op"] == "prompt":
        n = _lengths(case).astype(np.float64)
        rows = n.sum()
        return {"bytes": float(rows * ((2 * case["Hq"] + 2 * case["Hkv"]) * case["D"] * 2 + 4 * case["Hq"])),
                "flops": float(4 * case["D"] * case["Hq"] * (n * (n + 1) / 2).sum())}
    rows = float(_held(case, _capacities(case)).sum())
    heads = case["L"] * case["B"] * case["Hq"]
    return {"bytes": rows * (2 * 64 + 8) + heads * (2 * 128 * 2 + 4), "flops": 4 * 128 * rows * (case["Hq"] // case["Hkv"])}


# ------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    return {"norm_rope": _exact_norm_rope, "prompt": _exact_prompt, "decode4": _exact_decode4}[case["op"]](st)


def _exact_norm_rope(st):
    rot, D = st["rot"], st["D"]
    angle = st["pos"].double()[..., None] * st["inv_freq"].double()             # [B, T, rot / 2]
    turn = torch.polar(torch.ones_like(angle), angle)[:, None]
    if st["interleaved"]:
        first, second = torch.arange(0, rot, 2), torch.arange(1, rot, 2)
    else:
        first, second = torch.arange(rot // 2), torch.arange(rot // 2, rot)

    def one(x, w):
        y = x.double().clone()
        if w is not None:
            y = y / (y.square().sum(-1, keepdim=True) / D + 1e-6).sqrt() * w.double()
        z = torch.complex(y[..., first], y[..., second]) * turn
        y[..., first], y[..., second] = z.real, z.imag
        return y

    q, k = one(st["q_in"], st["qw"]), one(st["k_in"], st["kw"])
    return {"q": q.squeeze(2) if st["decode"] else q, "k": k.squeeze(2) if st["decode"] else k}


def _exact_prompt(st):
    g, D = st["Hq"] // st["Hkv"], st["D"]
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(st["lse"].shape, dtype=torch.float64, device=DEV)
    ends = np.cumsum(st["n"])
    for b, n in enumerate(st["n"].tolist()):
        at = int(ends[b]) - n
        for h in range(st["Hq"]):
            q, k, v = ((st[x][i, at:at + n] if st["packed"] else st[x][b, i, :n]).double()
                       for x, i in (("q", h), ("k", h // g), ("v", h // g)))
            for r0 in range(0, n, 2048):
                r1 = min(n, r0 + 2048)
                s = torch.mm(q[r0:r1], k[:r1].t()) / D ** 0.5
                s += torch.full((r1 - r0, r1), float("-inf"), dtype=torch.float64, device=DEV).triu(r0 + 1)
                z = torch.logsumexp(s, dim=1)
                o = torch.mm(torch.exp(s - z[:, None]), v[:r1])
                if st["packed"]:
                    out[at + r0:at + r1, h], lse[h, at + r0:at + r1] = o, z
                else:
                    out[b, h, r0:r1], lse[b, h, r0:r1] = o, z
    return {"out": out, "lse": lse}


def _exact_decode4(st):
    L, B, Hkv, D = (st[k] for k in ("L", "B", "Hkv", "D"))
    g = st["Hq"] // Hkv
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(st["lse"].shape, dtype=torch.float64, device=DEV)
    n, free = st["len"].cpu().numpy(), st["free"].cpu().numpy()

    def values(codes, which, rows, l, h):
        c = st[codes][rows].double()
        u = torch.empty((c.shape[0], D), dtype=torch.float64, device=DEV)
        u[:, 1::2] = torch.floor(c / 16)
        u[:, 0::2] = c - 16 * u[:, 1::2]
        return (u - 8) * st["row_scale"][rows, which].double()[:, None] * st["chan"][l, h, 2 * which].double()

    for b in range(B):
        for l in range(L):
            for h in range(Hkv):
                slots = np.delete(np.arange(n[b, l, h] + 1), free[b, l, h])
                rows = torch.from_numpy(b * st["stride"] + st["off"][l, h] + slots).to(DEV)
                s = st["q"][l, b, h * g:h * g + g].double() @ values("k_codes", 0, rows, l, h).t() / D ** 0.5
                z = torch.logsumexp(s, dim=1)
                lse[l, b, h * g:h * g + g] = z
                out[l, b, h * g:h * g + g] = torch.exp(s - z[:, None]) @ values("v_codes", 1, rows, l, h)
    return {"out": out, "lse": lse}
