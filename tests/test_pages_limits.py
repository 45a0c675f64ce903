"""Sizes of the page tables whose indices would not fit the kernels' arithmetic are refused on the host."""
import pytest

from test_rollout_refusals import UNSUPPORTED, status

TOO_MANY = [1 << 30, 2 ** 31 - 1]


@pytest.mark.parametrize("n", TOO_MANY)
@pytest.mark.parametrize("name,arg", [("respec_pages_compact", "num_pages"), ("respec_pages_compact", "page_table_len"),
                                      ("respec_pages_compact", "max_moves"), ("respec_pages_fork", "page_table_len"),
                                      ("respec_pages_fork", "num_pages"), ("respec_pages_resize", "num_pages")])
def test_refused(name, arg, n):
    extra = {"workspace_bytes": 1 << 40} if name != "respec_pages_fork" else {}
    got, text = status(name, **{arg: n}, **extra)
    assert got == UNSUPPORTED and "2^30" in text
