"""Speculative decoding over budgeted caches as cases to measure: what a serving step calls when a draft model has put
forward a tree of tokens.

  tree     attention of a tree of drafted tokens over the slabs of one layer and over their own ancestors
  verify   which drafted tokens stand, by the target's and the draft's probabilities and given random numbers
  commit   the accepted tokens' rows into the slabs: attention scores, eviction, append

Each has a plain form in elementary torch operations, and the call a user makes of the library (`own`).
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
N_SINK = 4                       # rows of the first four positions are never evicted


# ------------------------------------------------------------------ cases
def listed():
    return [
        # a chain of four drafted tokens over two small caches: latency
        dict(name="tree-chain-small", op="tree", B=1, Hq=4, Hkv=2, D=64, mean=256, sigma=1.0, T=4, spread=1, kv="bf16", varlen=False),
        # one layer of one sequence, 32K context at 30 %, sixteen drafted tokens: what a model's layer loop issues
        dict(name="tree-layer", op="tree", B=1, Hq=32, Hkv=8, D=128, mean=9824, sigma=1.0, T=16, spread=4, kv="bf16", varlen=False),
        # one layer of sixteen sequences at different lengths, 8K context, group of seven, an odd number of nodes
        dict(name="tree-batch-g7", op="tree", B=16, Hq=28, Hkv=4, D=128, mean=2448, sigma=1.5, T=27, spread=6, kv="bf16", varlen=True),
        # one layer of 32 sequences, 32K context at 30 %
        dict(name="tree-batch-32k", op="tree", B=32, Hq=32, Hkv=8, D=128, mean=9824, sigma=1.0, T=16, spread=4, kv="bf16", varlen=False),
        # the largest trees over FP8 slabs
        dict(name="tree-fp8-64", op="tree", B=16, Hq=32, Hkv=8, D=128, mean=9824, sigma=1.0, T=64, spread=8, kv="fp8", varlen=False),
        # a chain of eight over 4-bit slabs
        dict(name="tree-int4-8", op="tree", B=16, Hq=32, Hkv=8, D=128, mean=9824, sigma=1.0, T=8, spread=1, kv="int4", varlen=False),
        # one sequence, a chain of four drafted tokens and the draft's whole distributions
        dict(name="verify-chain", op="verify", B=1, T=5, V=32000, spread=1, draft="drawn", half=False),
        # sixteen trees whose siblings were drawn without replacement
        dict(name="verify-trees", op="verify", B=16, T=32, V=128000, spread=5, draft="distinct", half=False),
        # a large batch of trees of the draft's likeliest tokens (no distribution beside them), bf16 probabilities
        dict(name="verify-batch", op="verify", B=256, T=12, V=152064, spread=3, draft="top", half=True),
        # every layer of one sequence after a verification, 32K context at 30 %: scores, eviction, append
        dict(name="commit-model", op="commit", L=32, B=1, Hq=32, Hkv=8, D=128, mean=9824, sigma=1.0, T=16, spread=4, kv="bf16",
             scored=True, varlen=False),
        # the same under sinks + window, which keeps no scores
        dict(name="commit-window", op="commit", L=32, B=1, Hq=32, Hkv=8, D=128, mean=9824, sigma=1.0, T=16, spread=4, kv="bf16",
             scored=False, varlen=False),
        # sixteen sequences at different lengths over 4-bit slabs, group of seven
        dict(name="commit-batch-int4", op="commit", L=28, B=16, Hq=28, Hkv=4, D=128, mean=2448, sigma=1.5, T=9, spread=2, kv="int4",
             scored=True, varlen=True),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["tree", "tree", "verify", "commit"])
    T = _log_int(rng, 1, 64)
    spread = rng.choice([1, 2, 4, 8])
    if op == "verify":
        V = _log_int(rng, 300, 152064)
        B = max(1, min(_log_int(rng, 1, 256), int(3.1e8 / (T * V))))
        return dict(op=op, B=B, T=T, V=V, spread=spread, draft=rng.choice(["drawn", "distinct", "top"]), half=rng.random() < 0.3)
    hkv, g = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 3, 4, 5, 6, 7, 8])
    kv = rng.choice(["bf16", "bf16", "fp8", "int4"])
    D = rng.choice([64, 128]) if kv == "bf16" else 128
    B = _log_int(rng, 1, 32)
    L = 1 if op == "tree" else _log_int(rng, 1, 32)
    rows = 2400000 if op == "commit" else min(2400000, 1.5e8 / (g * T))
    mean = max(64, min(_log_int(rng, 64, 32768), int(rows / (L * B * hkv))))
    case = dict(op=op, B=B, Hq=hkv * g, Hkv=hkv, D=D, mean=mean, sigma=rng.choice([0.0, 0.5, 1.0, 1.5]), T=T, spread=spread, kv=kv,
                varlen=rng.random() < 0.5)
    if op == "commit":
        case.update(L=L, scored=rng.random() < 0.7)
    return case


# ------------------------------------------------------------------ what a user's program has in hand
def _capacities(case):
    """int32 [L, Hkv] tokens, multiples of 16, unequal the way an importance profile leaves them (a model's profile
    and a batch's lengths belong to the case, like its sizes: they do not change with the inputs)."""
    L = case.get("L", 1)
    rs = np.random.RandomState(L * 7919 + case["mean"])
    w = np.exp(rs.standard_normal((L, case["Hkv"])) * case["sigma"])
    w = np.minimum(w / w.mean(), 3.0)
    return (16 * np.maximum(2, np.round(case["mean"] * w / w.mean() / 16))).astype(np.int32)


def _held(case, cap):
    """Rows each cache holds, [B, L, Hkv]."""
    full = np.broadcast_to(cap[None].astype(np.int64) - 1, (case["B"],) + cap.shape)
    if not case["varlen"]:
        return full.copy()
    share = np.random.RandomState(case["B"]).uniform(0.125, 1.0, (case["B"], 1, 1))
    return np.maximum(1, (full * share).astype(np.int64))


def _accepted(case):
    """Tokens a verification accepts, [B]."""
    return np.random.RandomState(case["B"] * 31 + case["T"]).randint(1, min(case["T"], 6) + 1, case["B"]).astype(np.int32)


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    return {"tree": _prepare_tree, "verify": _prepare_verify, "commit": _prepare_commit}[case["op"]](case, gen)


def _randn(shape, gen, dtype=torch.bfloat16):
    return torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32).to(dtype)


def _trees(case, gen):
    """parent int32 [B, T]: node 0 is the token that is certain, every other hangs on one of the `spread` before it."""
    B, T = case["B"], case["T"]
    i = torch.arange(T, device=DEV)
    back = torch.floor(torch.rand((B, T), generator=gen, device=DEV) * torch.clamp(i, max=case["spread"])).long()
    return torch.clamp(i - 1 - back, min=-1).to(torch.int32)


def _slabs(case, gen):
    """The cache of `case`: slabs, scales, lengths, holes."""
    L, B, Hkv, D, kv = case.get("L", 1), case["B"], case["Hkv"], case["D"], case["kv"]
    cap = _capacities(case)
    flat = cap.reshape(-1).astype(np.int64)
    off = np.concatenate([[0], np.cumsum(flat)[:-1]]).reshape(L, Hkv)
    stride = int(flat.sum())
    st = dict(case, L=L, cap=cap, off=off, stride=stride)
    # one channel of each head sticks out by 8, as keys and values of real models do; the channel scales know it
    chan = 0.5 + torch.rand((2, L, Hkv, D), generator=gen, device=DEV)
    chan.scatter_(3, torch.randint(0, D, (2, L, Hkv, 1), generator=gen, device=DEV), 8.0)
    head_of = torch.repeat_interleave(torch.arange(L * Hkv, device=DEV), torch.from_numpy(flat).to(DEV), output_size=stride)
    slabs, scales = [], []
    for i in range(2):
        c = chan[i].reshape(L * Hkv, D)
        parts = []
        for _ in range(B):
            x = _randn((stride, D), gen).float() * c[head_of]
            if kv == "bf16":
                parts.append((x.bfloat16(), None))
            elif kv == "fp8":
                parts.append(((x * 4.0).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8), None))
            else:
                parts.append(_codes4(x, 1.0 / c[head_of]))
        slabs.append(torch.cat([p[0] for p in parts]))
        if kv == "int4":
            scales.append(torch.cat([p[1] for p in parts]))
    st["k_slab"], st["v_slab"] = slabs
    st["row_scale"] = torch.stack(scales, dim=1).contiguous() if kv == "int4" else None                # [rows, 2] K, V
    st["kv_scale"] = None
    if kv == "fp8":
        st["kv_scale"] = torch.tensor([0.25, 4.0, 0.25, 4.0], device=DEV).expand(L, Hkv, 4).contiguous()
    elif kv == "int4":
        st["kv_scale"] = torch.stack([chan[0], 1.0 / chan[0], chan[1], 1.0 / chan[1]], dim=2).contiguous()   # [L, Hkv, 4, D]
    # a full cache has one freed slot among its rows; a joining sequence is not full yet
    n = _held(case, cap)
    if case["varlen"]:
        free = n.copy()
    else:
        free = np.minimum(n, (torch.rand((B, L, Hkv), generator=gen, device=DEV).cpu().numpy() * (n + 1)).astype(np.int64))
    st["len"] = torch.from_numpy(n.astype(np.int32)).to(DEV)
    st["free"] = torch.from_numpy(free.astype(np.int32)).to(DEV)
    return st


def _codes4(x, inv_chan):
    """Rows [n, D] -> (codes uint8 [n, D / 2], scale fp32 [n]): y = x / channel scale, scale = max |y| / 7,
    code = round(y / scale) + 8, the even channel in the low half of a byte."""
    y = x * inv_chan
    scale = y.abs().amax(dim=-1) / 7.0
    u = (torch.round(y / scale[..., None]).clamp(-7, 7) + 8).to(torch.uint8)
    return u[..., 0::2] | (u[..., 1::2] << 4), scale


def _own_cache(st):
    from paper_2502_13176_b200 import binding as bk
    kinds = {"bf16": bk.KV_BF16, "fp8": bk.KV_FP8_E4M3, "int4": bk.KV_INT4}
    scored = st.get("scored", True)
    st["shape"] = bk.make_shape(st["L"], st["Hq"], st["Hkv"], st["D"], 16, N_SINK, 1, 2 if scored else 1)
    cache = bk.Cache(st["shape"], st["cap"], st["off"], st["stride"], st["B"], kv_dtype=kinds[st["kv"]],
                     kv_scale=None if st["kv_scale"] is None else st["kv_scale"].cpu().numpy())
    cache.k_slab.copy_(st["k_slab"])
    cache.v_slab.copy_(st["v_slab"])
    cache.len.copy_(st["len"])
    cache.free_slot.copy_(st["free"])
    if st["row_scale"] is not None:
        cache.row_scale.copy_(st["row_scale"])
    if "pos" in st:
        cache.pos.copy_(st["pos"])
        cache.score.copy_(st["score"])
    st["cache"] = cache


def _prepare_tree(case, gen):
    st = _slabs(case, gen)
    B, T, Hq, Hkv, D = (case[k] for k in ("B", "T", "Hq", "Hkv", "D"))
    st["q"], st["k"], st["v"] = (_randn((B, h, T, D), gen) for h in (Hq, Hkv, Hkv))
    st["parent"] = _trees(case, gen)
    n = np.full(B, T)
    if case["varlen"]:
        n = np.random.RandomState(B * 17 + T).randint(1, T + 1, B)
        n[0] = T
    st["n_nodes"] = torch.from_numpy(n.astype(np.int32)).to(DEV)
    st["out"] = torch.zeros((B, Hq, T, D), dtype=torch.bfloat16, device=DEV)
    st["lse"] = torch.zeros((B, Hq, T), dtype=torch.float32, device=DEV)
    if own:
        from paper_2502_13176_b200 import binding as bk
        _own_cache(st)
        st["plan"] = bk.baklava_tree_plan(st["shape"], st["cap"], B, 0, T, kv_dtype=st["cache"].kv_dtype).to(DEV)
        st["ws"] = bk.decode_workspace(st["plan"])
    return st


def _prepare_verify(case, gen):
    B, T, V = case["B"], case["T"], case["V"]
    st = dict(case, draft_kind=case["draft"], parent=_trees(case, gen), n_nodes=torch.full((B,), T, dtype=torch.int32, device=DEV))
    logits = 2.5 * torch.randn((B, T, V), generator=gen, device=DEV)
    kind = torch.bfloat16 if case["half"] else torch.float32
    st["target"] = torch.softmax(logits, dim=-1).to(kind)
    logits.add_(torch.randn((B, T, V), generator=gen, device=DEV), alpha=0.7)                # the draft model is another one
    st["draft"] = torch.softmax(logits, dim=-1).to(kind)
    # a node is its parent's first, second ... child
    parent = st["parent"].long()
    same = (parent[:, :, None] == parent[:, None, :]) & (torch.arange(T, device=DEV)[None, None, :] < torch.arange(T, device=DEV)[None, :, None])
    nth = same.sum(dim=-1)
    of = torch.clamp(parent, min=0)
    if case["draft"] == "drawn":
        noise = torch.rand((B, T), generator=gen, device=DEV, dtype=torch.float64)
        tok = torch.empty((B, T), dtype=torch.int64, device=DEV)
        for b in range(B):                                    # (a sequence at a time: the sums need 64 bits a value)
            sums = torch.cumsum(st["draft"][b].double(), dim=-1)[of[b]]
            tok[b] = torch.searchsorted(sums, (noise[b] * sums[:, -1])[:, None], right=True)[:, 0]
    else:
        if case["draft"] == "distinct":                       # the largest of log q + Gumbel noise: draws without replacement
            for b in range(B):
                logits[b] -= torch.log(-torch.log(torch.rand((T, V), generator=gen, device=DEV).clamp(1e-20, 1 - 1e-7)))
        best = torch.topk(logits, min(T, V), dim=-1).indices
        tok = best[torch.arange(B, device=DEV)[:, None], of, torch.clamp(nth, max=best.shape[-1] - 1)]
    st["tokens"] = torch.clamp(tok, max=V - 1).to(torch.int32).contiguous()
    if case["draft"] == "top":
        st["draft"] = None
    st["u_accept"] = torch.rand((B, T), generator=gen, device=DEV)
    st["u_sample"] = torch.rand((B,), generator=gen, device=DEV)
    st["path"] = torch.zeros((B, T), dtype=torch.int32, device=DEV)
    st["n_path"] = torch.zeros((B,), dtype=torch.int32, device=DEV)
    st["next"] = torch.zeros((B,), dtype=torch.int32, device=DEV)
    st["status"] = torch.zeros((1,), dtype=torch.int32, device=DEV)
    return st


def _prepare_commit(case, gen):
    st = _slabs(case, gen)
    L, B, T, Hq, Hkv, D = (st[k] for k in ("L", "B", "T", "Hq", "Hkv", "D"))
    st["q"], st["k"], st["v"] = (_randn((L, B, h, T, D), gen) for h in (Hq, Hkv, Hkv))
    # positions rise with the slots but for the holes; scores as a prompt's attention leaves them, a long tail
    rows = B * st["stride"]
    first = np.repeat(st["off"].reshape(-1), st["cap"].reshape(-1))
    slot = torch.from_numpy(np.tile(np.arange(st["stride"]) - first, B).astype(np.int32)).to(DEV)
    st["pos"] = torch.where(slot < N_SINK, slot, slot * 3 + 7)
    st["score"] = torch.exp(torch.randn((rows,), generator=gen, device=DEV)) if case["scored"] else torch.zeros((rows,), device=DEV)
    st["t_pos"] = torch.full((B,), 1 << 20, dtype=torch.int32, device=DEV)
    st["t_next"] = torch.zeros((B,), dtype=torch.int32, device=DEV)
    # the accepted path of each tree: from the root down to a node that is deep enough, cut to the accepted length
    parent, a = _trees(case, gen).cpu().numpy(), _accepted(case)
    path = np.full((B, T), -1, dtype=np.int32)
    for b in range(B):
        way, i = [], T - 1
        while i >= 0:
            way.append(i)
            i = parent[b, i]
        way = way[::-1][:a[b]]
        a[b] = len(way)
        path[b, :len(way)] = way
    st["path"], st["n_path"] = torch.from_numpy(path).to(DEV), torch.from_numpy(a).to(DEV)
    st["max_path"] = min(T, 6)
    st["lse"] = torch.zeros((L, B, Hq, T), dtype=torch.float32, device=DEV)
    if case["scored"]:                                       # what attention over the tree left behind
        _path_scores(st, lse_only=True)
    if own:
        from paper_2502_13176_b200 import binding as bk
        _own_cache(st)
        st["plan"] = bk.baklava_decode_plan(st["shape"], st["cap"], B, 0, L, st["stride"], kv_dtype=st["cache"].kv_dtype).to(DEV)
        st["ws"] = bk.tree_commit_workspace(st["shape"], st["plan"], st["max_path"])
    return st


# ------------------------------------------------------------------ one pass
def run(st):
    if own:
        return _call(st)
    return {"tree": _plain_tree, "verify": _plain_verify, "commit": _plain_commit}[st["op"]](st)


def _call(st):
    from paper_2502_13176_b200 import binding as bk
    if st["op"] == "tree":
        bk.baklava_tree_attn(st["shape"], st["cache"], st["q"], st["k"], st["v"], st["parent"], st["n_nodes"], st["out"], st["lse"],
                             st["plan"], st["ws"])
        return {"out": st["out"], "lse": st["lse"]}
    if st["op"] == "verify":
        flags = bk.VERIFY_DISTINCT if st["draft"] is not None and st["draft_kind"] == "distinct" else 0
        bk.baklava_tree_verify(st["target"], st["draft"], st["tokens"], st["parent"], st["n_nodes"], st["u_accept"], st["u_sample"],
                               st["path"], st["n_path"], st["next"], st["status"], flags)
        return {"path": st["path"], "n_path": st["n_path"], "next": st["next"]}
    c = st["cache"]
    bk.baklava_tree_commit(st["shape"], c, st["q"], st["k"], st["v"], st["lse"], st["path"], st["n_path"], st["max_path"],
                           st["t_pos"], st["t_next"], 0 if st["scored"] else bk.FLAG_NO_SCORE, st["plan"], st["ws"])
    st["t_pos"], st["t_next"] = st["t_next"], st["t_pos"]
    return {"k_slab": c.k_slab, "v_slab": c.v_slab, "row_scale": c.row_scale, "pos": c.pos, "score": c.score, "len": c.len,
            "free": c.free_slot, "t_pos": st["t_pos"]}


def _rows_of(st):
    """Slab row of every slot [heads, wide] of the heads (b, l, h), and which of them hold a row."""
    B, wide = st["B"], int(st["cap"].max())
    off = torch.from_numpy(st["off"]).to(DEV)
    slot = torch.arange(wide, device=DEV)
    n, free = st["len"].long(), st["free"].long()                                   # [B, L, Hkv]
    held = (slot < (n + (free < n))[..., None]) & (slot != free[..., None])           # rows are slots 0 .. len without `free`
    row = (torch.arange(B, device=DEV)[:, None, None] * st["stride"] + off)[..., None] + slot
    return torch.where(held, row, torch.zeros_like(row)).flatten(0, 2), held.flatten(0, 2)


def _values(st, which, row, heads):
    """What the slab rows `row` [heads, n] stand for, fp32; `heads`: their index among the layers' KV heads."""
    data = (st["k_slab"], st["v_slab"])[which][row]
    if st["kv"] == "bf16":
        return data.float()
    if st["kv"] == "fp8":
        return data.view(torch.float8_e4m3fn).float() * st["kv_scale"].flatten(0, 1)[heads, 2 * which, None, None]
    u = torch.stack([data & 15, data >> 4], dim=-1).flatten(-2).float() - 8.0
    return u * st["row_scale"][row][..., which, None] * st["kv_scale"].flatten(0, 1)[heads, 2 * which, None, :]


def _ancestors(parent):
    """[B, T, T]: whether node j is node i or above it."""
    T = parent.shape[1]
    up = torch.eye(T, device=DEV) + (parent[:, :, None] == torch.arange(T, device=DEV)).float()
    for _ in range(6):                                       # paths of up to 64 steps
        up = (up @ up > 0).float()
    return up > 0


def _plain_tree(st):
    B, T, Hq, Hkv, D = (st[k] for k in ("B", "T", "Hq", "Hkv", "D"))
    g = Hq // Hkv
    row, held = _rows_of(st)
    up = _ancestors(st["parent"])                             # [B, T, T]
    q = st["q"].float().reshape(B * Hkv, g * T, D) / math.sqrt(D)
    k, v = st["k"].float().reshape(B * Hkv, T, D), st["v"].float().reshape(B * Hkv, T, D)
    seq, head = torch.arange(B * Hkv, device=DEV) // Hkv, torch.arange(B * Hkv, device=DEV) % Hkv
    step = max(1, (1 << 20) // row.shape[1])                  # heads at a time: the whole would not fit in 32 bits
    outs, lses = [], []
    for i in range(0, B * Hkv, step):
        j = slice(i, min(B * Hkv, i + step))
        s = torch.bmm(q[j], _values(st, 0, row[j], head[j]).transpose(1, 2)).masked_fill(~held[j, None, :], float("-inf"))
        own_s = torch.bmm(q[j], k[j].transpose(1, 2)).masked_fill(~up[seq[j]].repeat(1, g, 1), float("-inf"))
        m = torch.maximum(s.amax(dim=-1, keepdim=True), own_s.amax(dim=-1, keepdim=True))
        p, own_p = torch.exp(s - m), torch.exp(own_s - m)
        total = p.sum(dim=-1, keepdim=True) + own_p.sum(dim=-1, keepdim=True)
        outs.append((torch.bmm(p, _values(st, 1, row[j], head[j])) + torch.bmm(own_p, v[j])) / total)
        lses.append((m + torch.log(total)).squeeze(-1))
    there = (torch.arange(T, device=DEV) < st["n_nodes"][:, None])[:, None, :]                # nodes behind the last stay as they were
    st["out"] = torch.where(there[..., None], torch.cat(outs).view(B, Hq, T, D).bfloat16(), st["out"])
    st["lse"] = torch.where(there, torch.cat(lses).view(B, Hq, T), st["lse"])
    return {"out": st["out"], "lse": st["lse"]}


def _plain_verify(st):
    """Nodes in ascending order: a node is tried when its turn comes and its parent is the last one that was accepted."""
    B, T, V = st["B"], st["T"], st["V"]
    every = torch.arange(B, device=DEV)
    cur = torch.zeros(B, dtype=torch.int64, device=DEV)
    r = st["target"][:, 0].double()                           # what is left of the target's distribution: 64 bits, sums decide
    gone = torch.zeros((B, V), dtype=torch.bool, device=DEV)   # tokens that were tried at this node
    path = torch.full((B, T), -1, dtype=torch.int64, device=DEV)
    path[:, 0] = 0
    count = torch.ones(B, dtype=torch.int64, device=DEV)
    for c in range(1, T):
        turn = (st["parent"][:, c] == cur) & (c < st["n_nodes"])
        tok = st["tokens"][:, c].long()
        if st["draft"] is None:
            q = torch.zeros((B, V), dtype=torch.float64, device=DEV)
            q[every, tok] = 1.0
        else:
            q = st["draft"][every, cur].double()
            if st["draft_kind"] == "distinct":
                q = torch.where(gone, 0.0, q / (1.0 - torch.where(gone, q, 0.0).sum(dim=-1, keepdim=True)))
        taken = turn & (st["u_accept"][:, c].double() * q[every, tok] < r[every, tok])
        refused = turn & ~taken
        rest = torch.clamp(r - q, min=0.0)
        total = rest.sum(dim=-1, keepdim=True)
        rest = torch.where(total > 0, rest / total, st["target"][every, cur].double())
        gone[every, tok] |= refused
        gone &= ~taken[:, None]
        r = torch.where(refused[:, None], rest, torch.where(taken[:, None], st["target"][:, c].double(), r))
        cur = torch.where(taken, c, cur)
        path[every, torch.clamp(count, max=T - 1)] = torch.where(taken, c, path[every, torch.clamp(count, max=T - 1)])
        count = count + taken
    sums = torch.cumsum(r, dim=-1)
    token = (sums <= st["u_sample"].double()[:, None] * sums[:, -1:]).sum(dim=-1)             # the first whose sum is above
    return {"path": path.int(), "n_path": count.int(), "next": token.int()}


def _path_scores(st, lse_only=False):
    """Attention of the accepted nodes over slab rows [heads, wide] and over themselves [heads, P]: sums over a group's
    queries and the nodes.  With lse_only the rows' normalisers are made instead, as attention over the tree leaves them."""
    L, B, T, Hq, Hkv, D = (st[k] for k in ("L", "B", "T", "Hq", "Hkv", "D"))
    g, P, heads = Hq // Hkv, st["max_path"], B * L * Hkv
    row, held = _rows_of(st)
    path = torch.clamp(st["path"][:, :P].long(), min=0)                                       # [B, P]
    on = torch.arange(P, device=DEV) < st["n_path"][:, None]
    at = path[None, :, None, :].expand(L, B, Hq, P)

    def per_head(x, h):                                       # [L, B, h, T, D] -> [heads, h / Hkv * P, D]
        x = torch.gather(x, 3, path[None, :, None, :, None].expand(L, B, h, P, D)).float()
        return x.permute(1, 0, 2, 3, 4).reshape(heads, h // Hkv * P, D)

    q, k = per_head(st["q"], Hq) / math.sqrt(D), per_head(st["k"], Hkv)
    lse = torch.gather(st["lse"], 3, at).permute(1, 0, 2, 3).reshape(heads, g * P, 1)
    seq, head = torch.arange(heads, device=DEV) // (L * Hkv), torch.arange(heads, device=DEV) % (L * Hkv)
    below = torch.tril(torch.ones((P, P), dtype=torch.bool, device=DEV)).repeat(g, 1)         # a node sees itself and those before it
    below = below & on[:, None, :] & on.repeat(1, g)[:, :, None]                              # [B, g P, P]
    step = max(1, (1 << 20) // row.shape[1])
    old, new, made = [], [], []
    for i in range(0, heads, step):
        j = slice(i, min(heads, i + step))
        live = held[j, None, :] & on[seq[j]].repeat(1, g)[:, :, None]
        s = torch.bmm(q[j], _values(st, 0, row[j], head[j]).transpose(1, 2)).masked_fill(~live, float("-inf"))
        own_s = torch.bmm(q[j], k[j].transpose(1, 2)).masked_fill(~below[seq[j]], float("-inf"))
        if lse_only:
            made.append(torch.logsumexp(torch.cat([s, own_s], dim=-1), dim=-1))
        else:
            old.append(torch.exp(s - lse[j]).sum(dim=1))
            new.append(torch.exp(own_s - lse[j]).sum(dim=1))
    if lse_only:
        wider = torch.zeros((L, B, Hq, T + 1), dtype=torch.float32, device=DEV)               # (one place for what is no node)
        wider.scatter_(3, torch.where(on[None, :, None, :], at, T), torch.cat(made).view(B, L, Hq, P).transpose(0, 1))
        st["lse"] = wider[..., :T].contiguous()
        return None
    return torch.cat(old), torch.cat(new)


def _plain_commit(st):
    L, B, T, Hkv, D, P = (st[k] for k in ("L", "B", "T", "Hkv", "D", "max_path"))
    heads, wide = B * L * Hkv, int(st["cap"].max())
    C = torch.from_numpy(st["cap"].reshape(-1)).to(DEV).long().repeat(B)
    row, held = _rows_of(st)
    slot = torch.arange(wide, device=DEV)
    base = row.new_tensor(st["off"].reshape(-1)).repeat(B) + torch.arange(B, device=DEV).repeat_interleave(L * Hkv) * st["stride"]
    a = st["n_path"].long().repeat_interleave(L * Hkv)
    n = st["len"].flatten().long()
    t_last = (st["t_pos"] + st["n_path"] - 1).long().repeat_interleave(L * Hkv)
    join = torch.arange(P, device=DEV) < a[:, None]                                            # [heads, P]
    new_pos = (st["t_pos"].long().repeat_interleave(L * Hkv)[:, None] + torch.arange(P, device=DEV)).expand(heads, P)
    new_score = torch.zeros((heads, P), device=DEV)
    if st["scored"]:
        add, new_score = _path_scores(st)
        st["score"].index_put_((row[held],), st["score"][row[held]] + add[held])
    # the rows that leave: the first of the order (score, latest first), or the oldest where no scores are kept
    pos, score = st["pos"][row].long(), st["score"][row]
    both_pos, both_score = torch.cat([pos, new_pos], dim=1), torch.cat([score, new_score], dim=1)
    window = (C - 1 - N_SINK) // (2 if st["scored"] else 1)
    may_go = torch.cat([held, join], dim=1) & (both_pos >= N_SINK) & (both_pos <= (t_last - window)[:, None])
    if st["scored"]:
        key = (both_score.view(torch.int32).long() << 32) + ((1 << 32) - 1 - both_pos)
    else:
        key = both_pos
    key = torch.where(may_go, key, torch.full_like(key, (1 << 63) - 1))
    k = torch.clamp(n + a - (C - 1), min=0)
    _, first = torch.topk(key, P + 1, dim=1, largest=False, sorted=True)
    leave = torch.zeros((heads, wide + P), dtype=torch.bool, device=DEV)
    leave.scatter_(1, first, torch.arange(P + 1, device=DEV) < k[:, None])
    # the rows that stay of the new ones take the free slots from the lowest up; the next free slot is the hole
    open_slot = (slot < C[:, None]) & (~held | leave[:, :wide])
    rank = torch.cumsum(open_slot, dim=1) - 1
    table = C[:, None].repeat(1, P + 2)
    table.scatter_(1, torch.where(open_slot & (rank <= P), rank, torch.full_like(rank, P + 1)), slot.expand(heads, wide))
    stay = join & ~leave[:, wide:]
    to = torch.gather(table, 1, torch.clamp(torch.cumsum(stay, dim=1) - 1, min=0))
    at = (base[:, None] + to)[stay]
    path = torch.clamp(st["path"][:, :P].long(), min=0)
    for which, name in ((0, "k"), (1, "v")):
        x = torch.gather(st[name], 3, path[None, :, None, :, None].expand(L, B, Hkv, P, D)).permute(1, 0, 2, 3, 4).reshape(heads, P, D)
        slab = st[name + "_slab"]
        if st["kv"] == "bf16":
            slab[at] = x[stay]
        elif st["kv"] == "fp8":
            inv = st["kv_scale"].flatten(0, 1)[:, 2 * which + 1].repeat(B)
            slab[at] = (x.float() * inv[:, None, None]).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)[stay]
        else:
            codes, scale = _codes4(x.float(), st["kv_scale"].flatten(0, 1)[:, 2 * which + 1].repeat(B, 1)[:, None, :])
            slab[at] = codes[stay]
            st["row_scale"][at, which] = scale[stay]
    st["pos"][at] = new_pos[stay].int()
    st["score"][at] = new_score[stay]
    st["len"] = (n + a - k).int().view(B, L, Hkv)
    st["free"] = torch.gather(table, 1, stay.sum(dim=1, keepdim=True)).int().view(B, L, Hkv)
    st["t_pos"] = st["t_pos"] + st["n_path"]
    return {"k_slab": st["k_slab"], "v_slab": st["v_slab"], "row_scale": st["row_scale"], "pos": st["pos"], "score": st["score"],
            "len": st["len"], "free": st["free"], "t_pos": st["t_pos"]}


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    if case["op"] == "verify":
        size = 2 if case["half"] else 4                       # one row of each distribution, where the walk ends
        return {"bytes": case["B"] * case["V"] * size * (1 if case["draft"] == "top" else 2), "flops": 2 * case["B"] * case["V"]}
    rows = float(_held(case, _capacities(case)).sum())
    D, g, T, B, Hkv = case["D"], case["Hq"] // case["Hkv"], case["T"], case["B"], case["Hkv"]
    one = {"bf16": 2 * D, "fp8": D, "int4": D // 2 + 4}[case["kv"]]                            # a row of K or of V
    if case["op"] == "tree":
        nodes = B * T * Hkv
        return {"bytes": rows * 2 * one + nodes * (g * 4 * D + 4 * D + 4 * g), "flops": 4 * D * rows * g * T}
    a = _accepted(case)
    joined = float(a.sum()) * case["L"] * Hkv
    if not case["scored"]:
        return {"bytes": rows * 4 + joined * (4 * D + 2 * one), "flops": rows}
    mean_a = float(a.mean())
    return {"bytes": rows * (one + 12) + joined * (4 * D + 2 * one + 2 * D * g), "flops": 2 * D * rows * g * mean_a}


# ------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    if case["op"] == "commit" and _capacities(case).size * case["B"] > 400:
        return None                                           # head after head: over twenty seconds
    st = prepare(case, seed)
    return {"tree": _exact_tree, "verify": _exact_verify, "commit": _exact_commit}[case["op"]](st)


def _held_slots(st, b, l, h):
    n, f = int(st["len"][b, l, h]), int(st["free"][b, l, h])
    return torch.tensor([s for s in range(n + 1) if s != f][:n], device=DEV)


def _stored(st, which, rows, l, h):
    data = (st["k_slab"], st["v_slab"])[which][rows]
    if st["kv"] == "bf16":
        return data.double()
    if st["kv"] == "fp8":
        return data.view(torch.float8_e4m3fn).double() * st["kv_scale"][l, h, 2 * which].double()
    x = torch.empty((rows.numel(), st["D"]), dtype=torch.float64, device=DEV)
    x[:, 1::2] = torch.floor(data.double() / 16)
    x[:, 0::2] = data.double() - 16 * x[:, 1::2]
    return (x - 8) * st["row_scale"][rows, which].double()[:, None] * st["kv_scale"][l, h, 2 * which].double()


def _way_up(parent, i):
    way = []
    while i >= 0:
        way.append(i)
        i = int(parent[i])
    return way[::-1]


def _exact_tree(st):
    B, T, Hq, Hkv, D = (st[k] for k in ("B", "T", "Hq", "Hkv", "D"))
    g = Hq // Hkv
    out = torch.zeros((B, Hq, T, D), dtype=torch.float64, device=DEV)
    lse = torch.zeros((B, Hq, T), dtype=torch.float64, device=DEV)
    parents = st["parent"].cpu().numpy()
    for b in range(B):
        nodes = int(st["n_nodes"][b])
        hidden = torch.full((nodes, T), float("-inf"), dtype=torch.float64)
        for i in range(nodes):
            hidden[i, _way_up(parents[b], i)] = 0.0
        hidden = hidden.to(DEV)
        for h in range(Hkv):
            rows = b * st["stride"] + int(st["off"][0, h]) + _held_slots(st, b, 0, h)
            keys = torch.cat([_stored(st, 0, rows, 0, h), st["k"][b, h].double()])
            vals = torch.cat([_stored(st, 1, rows, 0, h), st["v"][b, h].double()])
            for y in range(h * g, h * g + g):
                s = st["q"][b, y, :nodes].double() @ keys.t() / D ** 0.5
                s[:, rows.numel():] += hidden
                z = torch.logsumexp(s, dim=1)
                out[b, y, :nodes], lse[b, y, :nodes] = torch.exp(s - z[:, None]) @ vals, z
    return {"out": out, "lse": lse}


def _exact_verify(st):
    B, T, V = st["B"], st["T"], st["V"]
    parents, tokens, u = st["parent"].cpu().numpy(), st["tokens"].cpu().numpy(), st["u_accept"].cpu().numpy().astype(np.float64)
    path = np.full((B, T), -1, dtype=np.int32)
    count, token = np.zeros(B, dtype=np.int32), np.zeros(B, dtype=np.int32)
    for b in range(B):
        at, way = 0, [0]
        while True:
            left, tried, fell = st["target"][b, at].double(), [], None
            for c in [i for i in range(at + 1, int(st["n_nodes"][b])) if parents[b, i] == at]:
                x = int(tokens[b, c])
                if st["draft"] is None:
                    q = torch.zeros(V, dtype=torch.float64, device=DEV)
                    q[x] = 1.0
                else:
                    q = st["draft"][b, at].double()
                    if st["draft_kind"] == "distinct" and tried:
                        q[sorted(set(tried))] = 0.0
                        q = q / (1.0 - float(st["draft"][b, at].double()[sorted(set(tried))].sum()))
                if u[b, c] * float(q[x]) < float(left[x]):
                    fell = c
                    break
                tried.append(x)
                rest = (left - q) * (left > q)
                mass = float(rest.sum())
                left = rest / mass if mass > 0 else st["target"][b, at].double()
            if fell is None:
                break
            at = fell
            way.append(fell)
        sums = torch.cumsum(left, dim=0)
        token[b] = int(torch.searchsorted(sums, float(st["u_sample"][b]) * sums[-1:], right=True)[0])
        path[b, :len(way)], count[b] = way, len(way)
    return {"path": torch.from_numpy(path).to(DEV), "n_path": torch.from_numpy(count).to(DEV), "next": torch.from_numpy(token).to(DEV)}


def _exact_commit(st):
    L, B, Hq, Hkv, D = (st[k] for k in ("L", "B", "Hq", "Hkv", "D"))
    g = Hq // Hkv
    score = st["score"].double()
    pos, length, hole = st["pos"].clone(), st["len"].clone(), st["free"].clone()
    for b in range(B):
        a = int(st["n_path"][b])
        way = st["path"][b, :a].long()
        t0 = int(st["t_pos"][b])
        for l in range(L):
            for h in range(Hkv):
                C, n = int(st["cap"][l, h]), int(st["len"][b, l, h])
                first = b * st["stride"] + int(st["off"][l, h])
                slots = _held_slots(st, b, l, h)
                rows = first + slots
                fresh = torch.zeros(a, dtype=torch.float64, device=DEV)
                if st["scored"]:
                    keys = torch.cat([_stored(st, 0, rows, l, h), st["k"][l, b, h, way].double()])
                    q = st["q"][l, b, h * g:h * g + g][:, way].double()
                    s = q @ keys.t() / D ** 0.5                                               # [g, a, n + a]
                    s[:, :, n:] += torch.full((a, a), float("-inf"), dtype=torch.float64, device=DEV).triu(1)
                    p = torch.exp(s - st["lse"][l, b, h * g:h * g + g][:, way].double()[..., None]).sum(dim=(0, 1))
                    score[rows] += p[:n]
                    fresh = p[n:]
                places = torch.cat([pos[rows].long(), t0 + torch.arange(a, device=DEV)]).cpu().numpy()
                weights = torch.cat([score[rows], fresh]).cpu().numpy()
                window = (C - 1 - N_SINK) // (2 if st["scored"] else 1)
                loose = [i for i in range(n + a) if N_SINK <= places[i] <= t0 + a - 1 - window]
                loose.sort(key=(lambda i: (weights[i], -places[i])) if st["scored"] else (lambda i: places[i]))
                leave = set(loose[:max(0, n + a - (C - 1))])
                slot = slots.cpu().numpy()
                busy = {int(slot[i]) for i in range(n) if i not in leave}
                spare = [x for x in range(min(C, n + a + 2)) if x not in busy]
                for i in range(a):
                    if n + i not in leave:
                        x = spare.pop(0)
                        pos[first + x], score[first + x] = t0 + i, fresh[i]
                length[b, l, h], hole[b, l, h] = n + a - len(leave), spare[0] if spare else C
    return {"k_slab": None, "v_slab": None, "row_scale": None, "pos": pos, "score": score, "len": length, "free": hole,
            "t_pos": st["t_pos"] + st["n_path"]}
