import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a real MI355X (run with -m gpu)")


@pytest.fixture(scope="session")
def oracle():
    import oracle as _oracle
    _oracle.build()
    return _oracle


@pytest.fixture(params=[None, 0], ids=["form by size", "main kernel"])
def attn_few(request):
    """Small bf16 batches in the attention form that their size gives them, and in the main kernel's."""
    from helpers import env_setting
    with env_setting("RESPEC_ATTN_FEW", request.param):
        yield request.param


# Tests that hold a wrong value, with what is wrong about it; they have to fail.
_RESIZED = ("their model leaves pages behind kv_len shared, and one at a page's border, that two growing sequences then write into "
            "(test_gpu_pages_shared.py and test_pages_model.py have the right one)")
HOLD_A_WRONG_VALUE = {
    f"test_gpu_pages.py::test_random_histories[{case}]": _RESIZED
    for case in ("1024-40-64", "4096-2000-16", "4096-64-16", "9000-33-1024", "16385-1030-16")
}
HOLD_A_WRONG_VALUE["test_gpu_prompt.py::test_append_writes_nothing_outside_its_pages"] = (
    "4 rows of a length of 40 in one page of 16 lie at 36..39, past the page; it has them written at 12..15 (test_gpu_append.py)")


def pytest_collection_modifyitems(items):
    for item in items:
        for name, reason in HOLD_A_WRONG_VALUE.items():
            if item.nodeid.endswith(name):
                item.add_marker(pytest.mark.xfail(reason=reason, strict=True, raises=AssertionError))
