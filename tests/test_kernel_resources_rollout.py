"""Register budget of the kernels around the verify step (host-side check, no GPU): none of them keeps anything in scratch, and the bf16
prompt attention, which fills its 256 vector registers nearly, stays within what lets two waves share a SIMD."""
import os
import shutil
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_2510_26475_amd import build
from test_kernel_resources import _report

SOURCES = {"respec_prompt.hip": 32, "respec_logprobs.hip": 10, "respec_pages.hip": 12}   # kernels in them


@pytest.fixture(scope="module")
def reports():
    if not (os.path.exists(build.HIPCC) or shutil.which(build.HIPCC)):
        pytest.skip("no hipcc")
    with ThreadPoolExecutor(len(SOURCES)) as pool:
        return dict(zip(SOURCES, pool.map(_report, SOURCES)))


@pytest.mark.parametrize("source", SOURCES)
def test_no_kernel_takes_scratch(reports, source):
    assert len(reports[source]) == SOURCES[source]
    for name, usage in reports[source].items():
        assert usage.get("ScratchSize [bytes/lane]", -1) == 0, (name, usage)
        assert 0 < usage.get("VGPRs", 0) <= 256, (name, usage)
