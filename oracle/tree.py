"""Drafted tokens: attention of a tree of them over one head's cache, their verification, and the commit of the accepted
ones.  Test infrastructure only.

The paper decodes a token at a time.  Here node i of a tree hangs on node parent[i] < i, or on the cache (-1), and Eq. 7 is
applied per node: it attends to the cache's rows and to its own path.  Verification is speculative sampling: the outcome has
the target's own distribution whatever the draft was.  The commit is Eq. 4 for each accepted node, the accumulated
attention of all of them, and the retention policy once.
"""
import numpy as np

from .attention import decode_attention, log_sum_exp
from .eviction import select_keep


def way(parent, i):
    """Nodes from the root down to node i."""
    out = []
    while i >= 0:
        out.append(int(i))
        i = int(parent[i])
    return out[::-1]


def tree_attention(q, k, v, parent, K, V):
    """q [g, T, D], k, v [T, D] of the nodes, K, V [n, D] the cache's rows -> (out [g, T, D], lse [g, T])."""
    g, T, D = np.asarray(q).shape
    out, lse = np.zeros((g, T, D)), np.zeros((g, T))
    for i in range(T):
        w = way(parent, i)
        keys, vals = np.concatenate([K, np.asarray(k)[w]]), np.concatenate([V, np.asarray(v)[w]])
        out[:, i], _ = decode_attention(np.asarray(q)[:, i], keys, vals)
        lse[:, i] = log_sum_exp(np.asarray(q)[:, i], keys)
    return out, lse


def verify(target, draft, tokens, parent, n, u_accept, u_sample, distinct=False):
    """target, draft [T, V] (draft may be None) -> (path list, next token; -1 where nothing can be drawn)."""
    if n == 0:
        return [], -1
    positive = lambda x: np.where(np.asarray(x, dtype=np.float64) > 0, np.asarray(x, dtype=np.float64), 0.0)   # noqa: E731
    V = np.asarray(target).shape[1]
    at, path = 0, [0]
    while True:
        r, gone, down = positive(target[at]), np.zeros(V, dtype=bool), None
        for c in range(at + 1, n):
            if parent[c] != at:
                continue
            x = int(tokens[c])
            if draft is None:
                q = np.zeros(V)
                q[x] = 1.0
            else:
                q = positive(draft[at])
                if distinct:
                    left = 1.0 - q[gone].sum()
                    q = np.where(gone, 0.0, q / left) if left > 0 else np.zeros(V)
            if float(u_accept[c]) * q[x] < r[x]:
                down = c
                break
            gone[x] = True
            rest = np.maximum(r - q, 0.0)
            r = rest / rest.sum() if rest.sum() > 0 else positive(target[at])
        if down is None:
            break
        at = down
        path.append(down)
    total = r.sum()
    if not total > 0:
        return path, -1
    above = np.nonzero((np.cumsum(r) > float(u_sample) * total) & (r > 0))[0]
    return path, int(above[0]) if len(above) else int(np.nonzero(r > 0)[0][-1])


def commit(hc, q, k, v, lse, path, t0, score=True, evict=True):
    """The accepted nodes `path` into HeadCache `hc` (changed in place): q [g, T, D], k, v [T, D], lse [g, T].

    Rows that stay keep their slots; joining rows that stay take the free slots in ascending order, the next free slot
    becomes free_slot.  Returns False where the path does not fit (evict=False): nothing joins then."""
    q, k, v, lse = (np.asarray(x, dtype=np.float64) for x in (q, k, v, lse))
    a, D = len(path), hc.D
    slots = hc.valid_slots()
    n = len(slots)
    fresh = np.zeros(a)
    if score:
        keys = np.concatenate([hc.K[slots], k[path]])
        for i, node in enumerate(path):
            seen = n + i + 1                                  # the cache's rows and the path up to the node
            p = np.exp(q[:, node] @ keys[:seen].T / np.sqrt(float(D)) - lse[:, node][:, None]).sum(axis=0)
            hc.score[slots] += p[:n]
            fresh[:i + 1] += p[n:]
    if not evict and n + a > hc.C:
        return False
    pos = np.concatenate([hc.pos[slots], t0 + np.arange(a)])
    keep = np.arange(n + a)
    if evict:
        # without scores the rows that are left over go by age: the oldest first
        rank = np.concatenate([hc.score[slots], fresh]) if score else pos.astype(np.float64)
        keep = select_keep(pos, rank, hc.C - 1, hc.n_sink, hc.recent_num, hc.recent_den)
    stays = np.zeros(n + a, dtype=bool)
    stays[keep] = True
    busy = set(int(s) for s, on in zip(slots, stays[:n]) if on)
    spare = [s for s in range(hc.C) if s not in busy]
    for i in range(a):
        if stays[n + i]:
            s = spare.pop(0)
            hc.K[s], hc.V[s], hc.pos[s], hc.score[s] = k[path[i]], v[path[i]], t0 + i, fresh[i]
    hc.length, hc.free_slot = int(stays.sum()), spare[0] if spare else hc.C
    return True
