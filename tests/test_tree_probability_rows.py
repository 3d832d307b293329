"""Rows of probabilities that repeat or overlap are refused: the call takes rows at one distance of at least a row."""
import pytest
import torch

from paper_2502_13176_b200 import binding as bk

VOCAB = 100


def call(**bad):
    B, T, V = next(iter(bad.values())).shape
    p = torch.zeros((B, T, V))
    i = lambda *s: torch.zeros(s, dtype=torch.int32)                                          # noqa: E731
    a = dict(target=p, draft=p, tokens=i(B, T), parent=i(B, T), n_nodes=None, u_accept=torch.zeros(B, T), u_sample=torch.zeros(B), path=i(B, T),
             n_path=i(B), next_token=i(B), status=i(1))
    bk.baklava_tree_verify(**dict(a, **bad))


def rows():
    row = torch.zeros(VOCAB)
    return {"one row for all": row.expand(3, 5, VOCAB), "one row for a sequence's nodes": torch.zeros(3, 1, VOCAB).expand(3, 5, VOCAB),
            "one row for the nodes of one sequence": row.expand(1, 5, VOCAB), "one row for sequences of one node": row.expand(3, 1, VOCAB),
            "a sequence's rows for all": torch.zeros(1, 5, VOCAB).expand(3, 5, VOCAB),
            "a window that slides over a row": torch.zeros(2000).as_strided((2, 4, VOCAB), (200, 50, 1)),
            "a window over one sequence's": torch.zeros(2000).as_strided((1, 4, VOCAB), (7, 50, 1)),
            "one value for all rows of a vocabulary of one": torch.zeros(1).expand(3, 5, 1)}


@pytest.mark.parametrize("which", ["target", "draft"])
@pytest.mark.parametrize("name", rows())
def test_refused(monkeypatch, which, name):
    monkeypatch.setattr(bk, "_device", lambda: -1)            # (the CPU: nothing may reach the library)
    monkeypatch.setattr(bk, "_tree_call", lambda *a: pytest.fail("a call was made"))
    with pytest.raises(ValueError, match=which):
        call(**{which: rows()[name]})


@pytest.mark.parametrize("x,want", [(torch.zeros(3, 5, VOCAB), 100), (torch.zeros(1, 1, VOCAB), 100), (torch.zeros(VOCAB).expand(1, 1, VOCAB), 100),
                                    (torch.zeros(3, 5, 2 * VOCAB)[..., :VOCAB], 200), (torch.zeros(3, 5, VOCAB)[:, :1], 500),
                                    (torch.zeros(1, 9, VOCAB)[:, ::2], 200), (torch.zeros(3, 5, 1), 1)])
def test_taken(x, want):
    assert bk._probabilities(x, "target", -1, x.shape, torch.float32) == (x.data_ptr(), want)
