"""Verification of drafted tokens against the fp64 definition: every number out is an integer and has to be equal."""
import numpy as np
import pytest
import torch

from oracle import tree as ot
from paper_2502_13176_b200 import binding as bk
from tests.tree_cases import random_tree

pytestmark = pytest.mark.gpu


def verify(target, draft, tokens, parent, nodes, ua, us, flags=0):
    B, T, _ = target.shape
    dev = "cuda"
    i32 = lambda x: torch.as_tensor(np.asarray(x), dtype=torch.int32).to(dev)                 # noqa: E731
    f32 = lambda x: torch.as_tensor(np.asarray(x), dtype=torch.float32).to(dev)               # noqa: E731
    path = torch.full((B, T), 99, dtype=torch.int32, device=dev)
    count, token = (torch.full((B,), 99, dtype=torch.int32, device=dev) for _ in range(2))
    status = torch.zeros((1,), dtype=torch.int32, device=dev)
    bk.baklava_tree_verify(target, draft, i32(tokens), i32(parent), None if nodes is None else i32(nodes), f32(ua), f32(us), path, count,
                           token, status, flags)
    torch.cuda.synchronize()
    return path.cpu().numpy(), count.cpu().numpy(), token.cpu().numpy(), int(status.item())


def check(target, draft, tokens, parent, nodes, ua, us, distinct):
    path, count, token, status = verify(target, draft, tokens, parent, nodes, ua, us, bk.VERIFY_DISTINCT if distinct else 0)
    t64 = target.double().cpu().numpy()
    d64 = None if draft is None else draft.double().cpu().numpy()
    B, T, _ = target.shape
    lengths = []
    for b in range(B):
        n = T if nodes is None else int(np.clip(nodes[b], 0, T))
        want, nxt = ot.verify(t64[b], None if d64 is None else d64[b], tokens[b], parent[b], n, np.float32(ua[b]), np.float32(us[b]), distinct)
        assert count[b] == len(want) and path[b].tolist() == want + [-1] * (T - len(want)), (b, path[b], want)
        assert token[b] == nxt, (b, token[b], nxt)
        lengths.append(len(want))
    assert status == 0
    return lengths


def case(seed, B, T, V, kind, dtype=torch.float32, tree="any", like=0.7, sharp=2.0):
    rng = np.random.default_rng(seed)
    logits = rng.normal(0, sharp, (B, T, V))
    soft = lambda x: torch.softmax(torch.from_numpy(x), dim=-1).to(dtype)                     # noqa: E731
    target, draft = soft(logits), soft(logits + rng.normal(0, like, logits.shape))
    parent = np.stack([np.maximum(random_tree(rng, T, tree), -1) for _ in range(B)])
    parent[:, 1:] = np.maximum(parent[:, 1:], 0)              # (nodes that hang on the cache are reached by no walk)
    tokens = np.zeros((B, T), dtype=np.int64)
    d64 = draft.double().numpy()
    for b in range(B):
        for n in range(T):
            kids = [c for c in range(1, T) if parent[b, c] == n]
            p = d64[b, n] / d64[b, n].sum()
            if kids and kind == "drawn":
                tokens[b, kids] = rng.choice(V, len(kids), p=p)
            elif kids and kind == "distinct":
                tokens[b, kids] = rng.choice(V, len(kids), replace=len(kids) > V, p=p)
            elif kids:
                tokens[b, kids] = np.argsort(-p)[np.arange(len(kids)) % V]
    return (target.cuda(), None if kind == "points" else draft.cuda(), tokens, parent, None, rng.random((B, T)), rng.random(B), kind == "distinct")


@pytest.mark.parametrize("kind", ["drawn", "distinct", "points"])
@pytest.mark.parametrize("B,T,V,tree", [(1, 1, 1, "any"), (3, 2, 7, "chain"), (5, 5, 33, "star"), (40, 9, 257, "any"), (7, 64, 1000, "star"),
                                        (4, 64, 131, "chain"), (33, 16, 5003, "any"), (2, 6, 50257, "any")])
def test_matches_the_definition(kind, B, T, V, tree):
    check(*case(B * 1000 + T, B, T, V, kind, tree=tree))


@pytest.mark.parametrize("kind", ["drawn", "distinct", "points"])
def test_bf16_probabilities(kind):
    check(*case(77, 20, 12, 3001, kind, torch.bfloat16))


def test_long_and_short_walks_occur():
    """Drafts that are the target are all taken, others hardly."""
    a = check(*case(5, 16, 12, 400, "drawn", tree="chain", like=0.0))
    b = check(*case(6, 16, 12, 400, "drawn", tree="chain", like=6.0))
    assert min(a) == 12 and max(b) < 12 and 1 in b


def test_node_counts_and_idle_sequences():
    t, d, tok, par, _, ua, us, dist = case(9, 6, 8, 100, "drawn")
    par[3, 5:] = 1000                                         # nobody looks behind the last node
    tok[3, 5:] = -7
    check(t, d, tok, par, [8, 0, 1, 5, -3, 20], ua, us, dist)


def test_strided_rows():
    t, d, tok, par, n, ua, us, dist = case(10, 4, 6, 333, "distinct")
    wide = torch.full((4, 6, 352), float("nan"), device="cuda")
    wide[..., :333] = t
    other = torch.full((4, 6, 341), float("nan"), device="cuda")
    other[..., 8:] = d
    check(wide[..., :333], other[..., 8:], tok, par, n, ua, us, dist)


def test_the_draw_at_its_borders():
    """u = 0 takes the first token with any mass, u just below 1 the last; a token's own border belongs to the next one."""
    V = 4096
    p = torch.zeros((1, 1, V))
    p[0, 0, [5, 100, 4000]] = torch.tensor([0.25, 0.25, 0.5])
    for u, want in [(0.0, 5), (0.2499, 5), (0.25, 100), (0.5, 4000), (1 - 2.0 ** -24, 4000)]:
        _, _, token, _ = verify(p.cuda(), None, [[0]], [[-1]], None, [[0.0]], [u])
        assert token[0] == want, u


def test_zeros_nan_and_nothing_left():
    V = 50
    p = torch.full((2, 2, V), float("nan"))
    p[0, :, 7] = 0.5
    par, tok = [[-1, 0], [-1, 0]], [[0, 7], [0, 7]]
    path, count, token, status = verify(p.cuda(), None, tok, par, None, [[0, 0.6], [0, 0.6]], [0.3, 0.3])
    # sequence 0: refused, then nothing is left of its row: the row itself again; sequence 1: a row without mass
    assert count.tolist() == [1, 1] and token.tolist() == [7, -1] and status == bk.STATUS_BAD_STATE


@pytest.mark.parametrize("tok,par", [([0, 50], [-1, 0]), ([0, -1], [-1, 0]), ([0, 1], [-1, 1]), ([0, 1], [-1, -2]), ([0, 1], [3, 0])])
def test_what_cannot_be_is_skipped(tok, par):
    p = torch.full((2, 2, 50), 0.02).cuda()
    path, count, token, status = verify(p, p, [tok, [0, 1]], [par, [-1, 0]], None, np.zeros((2, 2)), [0.5, 0.5])
    assert status == bk.STATUS_BAD_STATE and count[0] == 0 and token[0] == -1 and path[0].tolist() == [-1, -1]
    assert count[1] == 2 and token[1] >= 0


def test_repeated_and_replayed():
    args = case(12, 24, 20, 4001, "distinct")
    t, d, tok, par, _, ua, us, _ = args
    ref = verify(t, d, tok, par, None, ua, us, bk.VERIFY_DISTINCT)
    dev = [torch.as_tensor(np.asarray(x), dtype=k).cuda() for x, k in ((tok, torch.int32), (par, torch.int32), (ua, torch.float32), (us, torch.float32))]
    outs = [torch.zeros((24, 20), dtype=torch.int32, device="cuda")] + [torch.zeros((24,), dtype=torch.int32, device="cuda") for _ in range(2)]
    status = torch.zeros((1,), dtype=torch.int32, device="cuda")
    call = lambda: bk.baklava_tree_verify(t, d, dev[0], dev[1], None, dev[2], dev[3], *outs, status, bk.VERIFY_DISTINCT)   # noqa: E731
    call()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        call()
    for x in outs:
        x.zero_()
    graph.replay()
    torch.cuda.synchronize()
    for x, r in zip(outs, ref):
        np.testing.assert_array_equal(x.cpu().numpy(), r)


@pytest.mark.parametrize("V", [1, 2, 7, 40])
def test_the_same_token_twice_among_distinct_siblings(V):
    """What should not be there: a token that has left already has nothing of q any more, and nothing of what is left of the target.

    Once all of q has left but for one token, r and q / left are both one there, and every further refusal takes all but a rounding of r.
    What is left is formed as p - K q, to 2^-52 of p: equality can be asked for while it is above 2^-30 of p, as then 22 bits of
    it are right and the comparisons of this test's random numbers (24 bits) are decided by less than one in a million of them."""
    t, d, tok, par, _, ua, us, _ = case(20 + V, 40, 16, V, "drawn", tree="star", like=1.5)
    path, count, token, status = verify(t, d, tok, par, None, ua, us, bk.VERIFY_DISTINCT)
    t64, d64 = t.double().cpu().numpy(), d.double().cpu().numpy()
    sure = 0
    for b in range(40):
        want, nxt = ot.verify(t64[b], d64[b], tok[b], par[b], 16, np.float32(ua[b]), np.float32(us[b]), True)
        got = path[b, :count[b]].tolist(), int(token[b])
        assert got[0][0] == 0 and all(par[b, c] == p for p, c in zip(got[0], got[0][1:])) and 0 <= got[1] < V
        mass = least = 1.0
        r, gone = t64[b, 0], np.zeros(V, dtype=bool)
        for c in range(1, want[1] if len(want) > 1 else 16):  # the refused children of the root
            if par[b, c] == 0:
                left = 1 - d64[b, 0][gone].sum()
                rest = np.maximum(r - np.where(gone, 0, d64[b, 0] / left), 0) if left > 0 else r
                gone[tok[b, c]] = True
                mass *= rest.sum()
                least = min(least, mass)
                r = rest / rest.sum() if rest.sum() > 0 else t64[b, 0]
        if least > 2.0 ** -30:
            sure += 1
            assert got == (want, nxt), b
    assert status == 0 and (V < 7 or sure > 10), sure
