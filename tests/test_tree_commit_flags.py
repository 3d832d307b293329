"""Flags of the commit that are there, and those that are not."""
import pytest

from paper_2502_13176_b200 import binding as bk
from paper_2502_13176_b200 import build as bkbuild
from tests.test_tree_refusals import INVALID, WORKSPACE, commit


@pytest.fixture(scope="module", autouse=True)
def _built():
    bkbuild.build()


@pytest.mark.parametrize("flags,code", [(bk.FLAG_ROW_QUOTIENT, WORKSPACE), (bk.FLAG_ROW_QUOTIENT | bk.FLAG_NO_SCORE | bk.FLAG_NO_EVICT, WORKSPACE),
                                        (32, INVALID), (bk.FLAG_ROW_QUOTIENT | bk.FLAG_OVERLAP_PREV, INVALID)])
def test_flags(flags, code):
    assert commit(flags=flags, ws_bytes=100) == code
