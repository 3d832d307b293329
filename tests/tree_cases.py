"""Caches and trees for the tests of drafted tokens: random rows in every slab format, NaN and infinities in every slot that
holds no row, and what the held rows stand for in fp64."""
import numpy as np
import torch

from oracle import fp8 as ofp8
from oracle import int4 as o4
from oracle.cache import HeadCache
from paper_2502_13176_b200 import binding as bk

FORMATS = {"bf16": bk.KV_BF16, "fp8": bk.KV_FP8_E4M3, "int4": bk.KV_INT4}


class Held:
    """A device cache and its rows on the host."""

    def __init__(self, shape, caps, B, kv, held, holes, seed, spread=1.0, poison=True, seq_gap=0):
        """held, holes: [B, L, Hkv] rows and free slots (a hole where below `held`)."""
        rng = np.random.default_rng(seed)
        self.shape, self.B, self.kv = shape, B, kv
        caps = np.asarray(caps, dtype=np.int32).reshape(shape.L, shape.Hkv)
        flat = caps.reshape(-1).astype(np.int64)
        off = np.concatenate([[0], np.cumsum(flat)[:-1]]).reshape(caps.shape)
        self.cap, self.off, self.stride = caps, off, int(flat.sum()) + seq_gap
        D, rows = shape.D, B * self.stride
        scale = None
        self.chan = np.exp(rng.normal(0, 0.5, (shape.L, shape.Hkv, 2, D))).astype(np.float32)
        if kv == "fp8":
            s = (2.0 ** rng.integers(-4, 2, (shape.L, shape.Hkv, 2))).astype(np.float32)
            scale = np.stack([s[..., 0], 1 / s[..., 0], s[..., 1], 1 / s[..., 1]], axis=-1)
        elif kv == "int4":
            scale = np.stack([self.chan[:, :, 0], 1 / self.chan[:, :, 0], self.chan[:, :, 1], 1 / self.chan[:, :, 1]], axis=2)
        c = self.cache = bk.Cache(shape, caps, off, self.stride, B, kv_dtype=FORMATS[kv], kv_scale=scale)
        x = torch.from_numpy(rng.normal(0, spread, (2, rows, D)).astype(np.float32))
        if kv == "bf16":
            data = x.bfloat16()
        elif kv == "fp8":
            data = x.to(torch.float8_e4m3fn).view(torch.uint8)
        else:
            data = torch.from_numpy(rng.integers(0, 256, (2, rows, D // 2)).astype(np.uint8))
            low, high = (data & 15).clamp(min=1), (data >> 4).clamp(min=1)           # code 0 is never written
            data = low | (high << 4)
            self.row_scale = np.abs(rng.normal(0.2, 0.1, (rows, 2))).astype(np.float32) * np.float32(spread)
        self.len = np.broadcast_to(np.asarray(held), (B,) + caps.shape).astype(np.int32)
        self.free = np.broadcast_to(np.asarray(holes), (B,) + caps.shape).astype(np.int32)
        self.live = np.zeros(rows, dtype=bool)
        for b in range(B):
            for l in range(shape.L):
                for h in range(shape.Hkv):
                    self.live[self.rows(b, l, h)] = True
        dead = torch.from_numpy(~self.live)
        if poison:
            if kv == "bf16":
                bad = torch.tensor([float("nan"), float("inf"), -float("inf")]).bfloat16()
                data[:, dead] = bad[torch.arange(D) % 3]
            elif kv == "fp8":
                data[:, dead] = 0x7F                          # NaN
            else:
                self.row_scale[~self.live] = np.nan
        self.data = data
        c.k_slab.copy_(data[0])
        c.v_slab.copy_(data[1])
        if kv == "int4":
            c.row_scale.copy_(torch.from_numpy(self.row_scale))
        c.len.copy_(torch.from_numpy(self.len))
        c.free_slot.copy_(torch.from_numpy(self.free))
        self.pos = np.full(rows, -1, dtype=np.int32)
        self.score = np.zeros(rows, dtype=np.float32)
        for b in range(B):
            for l in range(shape.L):
                for h in range(shape.Hkv):
                    r = self.rows(b, l, h)
                    self.pos[r] = rng.permutation(3 * len(r) + 2)[:len(r)]
                    self.score[r] = rng.lognormal(0, 1, len(r)).astype(np.float32)
        c.pos.copy_(torch.from_numpy(self.pos))
        c.score.copy_(torch.from_numpy(self.score))

    def slots(self, b, l, h):
        n, f = int(self.len[b, l, h]), int(self.free[b, l, h])
        return np.array([s for s in range(n + 1) if s != f][:n], dtype=np.int64)

    def rows(self, b, l, h):
        return b * self.stride + int(self.off[l, h]) + self.slots(b, l, h)

    def values(self, which, rows, l, h):
        """fp64 values of slab rows."""
        d = self.data[which][torch.from_numpy(np.asarray(rows))]
        if self.kv == "bf16":
            return d.double().numpy()
        if self.kv == "fp8":
            return ofp8.decode(d.numpy()) * float(self.cache.kv_scale_host[l, h, 2 * which])
        return o4.values(o4.unpack(d.numpy()), self.row_scale[rows, which], self.cache.kv_scale_host[l, h, 2 * which])

    def as_stored(self, x, l, h, which):
        """Values a row x [n, D] (fp64 of bf16) has once it is in the slab."""
        if self.kv == "bf16":
            return x
        four = self.cache.kv_scale_host[l, h]
        if self.kv == "fp8":
            return ofp8.quantise_rows(x, four[2 * which], four[2 * which + 1])[1]
        codes, s = o4.quantise_rows(x, four[2 * which + 1])
        return o4.values(codes, s, four[2 * which])

    def twin(self, b, l, h):
        """The head as an oracle cache."""
        s = self.shape
        hc = HeadCache(int(self.cap[l, h]), s.D, s.n_sink, s.recent_num, s.recent_den)
        slots, rows = self.slots(b, l, h), self.rows(b, l, h)
        hc.K[slots], hc.V[slots] = self.values(0, rows, l, h), self.values(1, rows, l, h)
        hc.pos[slots], hc.score[slots] = self.pos[rows], self.score[rows]
        hc.length, hc.free_slot = int(self.len[b, l, h]), int(self.free[b, l, h])
        return hc


def random_tree(rng, T, kind):
    """parent [T]: a chain, a star, or anything (several roots among it)."""
    if kind == "chain":
        return np.arange(T) - 1
    if kind == "star":
        return np.concatenate([[-1], np.zeros(T - 1)]).astype(np.int64)
    return np.array([int(rng.integers(-1, i)) if i else -1 for i in range(T)])


def bf16_normal(rng, shape, spread=1.0):
    return torch.from_numpy(rng.normal(0, spread, shape).astype(np.float32)).bfloat16()
