"""A plan of the attention over shared pages holds for further layers whatever the knobs say by then."""
import pytest
import torch

from plain_cache import Cache
from test_gpu_shared import POOLS, run, workspace
from test_gpu_shared_splits import knobs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,pool", POOLS)
@pytest.mark.parametrize("first,then", [(dict(OWN_HEAD=0, HEAD=0), dict(OWN_HEAD=9, HEAD=20)), (dict(OWN_HEAD=9, HEAD=20), dict(OWN_HEAD=0, HEAD=0)),
                                        (dict(), dict(OWN_HEAD=5, HEAD=1, COST=700, TILES=9, RANGES=3)), (dict(RANGES=5, TILES=1), dict())])
def test_next_layer_under_other_knobs(dtype, pool, first, then):
    """Long sequences in many parts, a group whose shared keys are cut too: the bits of a full call under the first knobs."""
    groups, shared, R = [[0, 1, 2], [3, 4]], [1280, 64], [3, 2, 4, 1, 4, 2]
    lens = [1300, 1700, 1290, 100, 2500, 3000]
    c = Cache(lens, 2, 64, 16, dtype, groups, shared, pool, seed=51)
    ws = workspace(6, sum(R), 2, 4, 3000, 8, 2, 64, dtype)
    with knobs(**first):
        run(c, R, 8, dtype, groups, shared, ws=ws)
        want = run(c, R, 8, dtype, groups, shared, seed=52)
    with knobs(**then):
        got = run(c, R, 8, dtype, groups, shared, ws=ws, seed=52, entry="respec_verify_attention_shared_next_layer")
    assert torch.equal(got[1], want[1]) and torch.equal(got[2], want[2])
