"""Prompts that have no rows between them: an empty tensor has no address, and that is no error (no GPU)."""
import pytest

from paper_2412_20105_amd import binding as st3
from test_block_host import FAKE, INVALID, OK, UNSUPPORTED, cache, packed, rows, shape

NONE = rows(None)


def store(k=NONE, v=NONE, cu=FAKE, total=0, max_len=0, c=None, sh=None):
    return st3.lib().st3_block_store(sh or shape(), k, v, cu, total, max_len, c or cache(), None)


def test_no_rows():
    assert packed(q=NONE, k=NONE, v=NONE, out=NONE, total=0, max_len=0) == OK
    assert packed(q=NONE, k=NONE, v=NONE, out=NONE, total=0, max_len=0, window=0, score=None, ws=None, wb=0) == OK
    assert store() == OK


@pytest.mark.parametrize("bad,want", [(dict(cu=None), INVALID), (dict(total=-1), INVALID), (dict(max_len=1), INVALID), (dict(sh=shape(dim=80)), UNSUPPORTED)])
def test_the_other_arguments_are_looked_at_all_the_same(bad, want):
    assert packed(**{**dict(q=NONE, k=NONE, v=NONE, out=NONE, total=0, max_len=0), **bad}) == want
    assert store(**bad) == want
    assert store(c=cache(n_pages=0)) == INVALID


def test_rows_that_exist_have_an_address():
    for which in ("q", "k", "v", "out"):
        assert packed(**{which: NONE}) == INVALID
    assert packed(q=NONE, max_len=0) == INVALID and store(total=5) == INVALID
