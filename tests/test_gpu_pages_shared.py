"""Shared pages on the GPU: a sequence that grows writes into pages of its own, whatever its fork left it."""
import random

import pytest
import torch

import pages_model
from paper_2510_26475_amd import binding
from test_gpu_pages import Cache, ints

pytestmark = pytest.mark.gpu


def cache(cap, num_pages, ps):
    c = Cache(cap, num_pages, ps)
    c.model = pages_model.Pages(cap, num_pages, ps)
    return c


@pytest.mark.parametrize("num_pages", [40, 5000, 20000])   # one launch, two, three
@pytest.mark.parametrize("kv,pages", [(16, 2), (16, 5), (5, 3), (33, 3), (0, 2), (48, 3), (47, 3)])
def test_children_of_a_parent_with_room_append_into_pages_of_their_own(num_pages, kv, pages):
    ps, Hkv, D, children = 16, 1, 64, 3
    B = 1 + children
    c = cache([8] * B, num_pages, ps)
    c.resize([pages * ps] + [-1] * children)
    prompt = torch.arange(kv, device="cuda").float()[:, None, None].expand(kv, Hkv, D) + 1000
    pools = [torch.zeros((num_pages, ps, Hkv, D), device="cuda") for _ in range(2)]
    for i in range(kv):
        for p in pools:
            p[c.model.table[0][i // ps], i % ps] = prompt[i]
    c.set_len([kv] + [0] * children)
    c.fork([-1] + [0] * children)
    new = [4, 1, 20, 45]
    want = [kv + n for n in new]
    src, dst, missing = c.resize(want)
    assert missing == [0] * B and c.model.written_twice([kv] * B, want) == []
    for b in range(B):   # as the arrays on the GPU have it
        assert all(c.refs[e].item() == 1 for e in c.table[8 * b + kv // ps:8 * b + c.model.count[b]].tolist())
    binding.respec_pages_copy(*pools, c.src, c.dst)
    rows = torch.randn((sum(new), Hkv, D), device="cuda")
    c.set_len(want)
    q_indptr = ints([0] + new).cumsum(0).to(torch.int32)
    binding.respec_append_paged(rows, -rows, *pools, q_indptr, c.indptr, c.table, c.kv, max(new))
    at = 0
    for b in range(B):
        pages_of = torch.tensor(c.model.table[b][:c.model.count[b]], device="cuda")
        for p, sign in zip(pools, (1, -1)):
            held = p[pages_of].flatten(0, 1)
            assert torch.equal(held[:kv], prompt) and torch.equal(held[kv:want[b]], sign * rows[at:at + new[b]])
        at += new[b]


@pytest.mark.parametrize("num_pages,B,ps", [(37, 5, 16), (1024, 40, 64), (1025, 300, 16), (4096, 2000, 16), (4096, 30, 16), (4097, 20, 64), (9000, 33, 1024),
                                              (16385, 1030, 16), (70000, 60, 16)])
def test_histories(num_pages, B, ps):
    """Random steps, with forks of sequences that hold more than their tokens need, against the model."""
    rng = random.Random(num_pages + B)
    cap = [rng.randrange(1, max(2, 3 * num_pages // B + 2)) for _ in range(B)]
    c = cache(cap, num_pages, ps)
    for step in range(20):
        kind = rng.choice(["resize", "resize", "fork", "compact", "lengths"])
        if kind == "resize":
            kv = list(c.model.kv)
            want = [rng.choice([-1, 0, rng.randrange(0, ps * (k + 2)), n + rng.randrange(0, 4 * ps)]) for k, n in zip(cap, kv)]
            missing = c.resize(want)[2]
            assert c.model.written_twice(kv, [-1 if m else w for w, m in zip(want, missing)]) == []
        elif kind == "lengths":
            c.set_len([rng.randrange(0, k * ps + 1) for k in c.model.count])
        elif kind == "fork":
            c.fork([rng.choice([-1, rng.randrange(0, B)]) for _ in range(B)])
        else:
            c.compact(rng.choice([1, 3, num_pages // 2 + 1]), in_place=rng.random() < 0.5)


@pytest.mark.parametrize("num_pages", [3000, 9000, 30000])
@pytest.mark.parametrize("shared", [0, 1, 2, 3, 7, 499, 998, 999, 1000])
def test_a_long_reserve_is_replaced_as_far_as_it_is_shared(num_pages, shared):
    """The parent keeps its first `shared` pages, so a child that holds 1,000 has that many to replace behind its length."""
    ps, n = 16, 1000
    for kv in (0, 5, 2 * ps):
        c = cache([n] * 2, num_pages, ps)
        c.resize([n * ps, -1])
        c.fork([-1, 0])
        c.set_len([shared * ps, kv])
        c.resize([shared * ps, -1])
        assert (c.refs == 2).sum().item() == shared
        c.resize([-1, (n - 1) * ps + 1])
        assert (c.refs == 2).sum().item() == min(shared, kv // ps)


def test_captured_group_with_a_reserve_replays():
    c = cache([6, 6, 6], 24, 16)
    c.resize([80, -1, -1])
    c.set_len([32, 0, 0])
    pools = [torch.randn((24, 16, 2, 64), device="cuda") for _ in range(2)]
    back, parent, want = ints([-1, 0, 0]), ints([-1, 0, 0]), ints([-1, 40, 70])
    for step in (lambda: c.model.resize(back.tolist()), lambda: c.model.fork(parent.tolist()), lambda: c.model.resize(want.tolist())):
        step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.respec_pages_resize(back, *c.state, c.src, c.dst, c.missing, c.ps, c.ws)
        binding.respec_pages_fork(parent, *c.state, c.missing)
        binding.respec_pages_resize(want, *c.state, c.src, c.dst, c.missing, c.ps, c.ws)
        binding.respec_pages_copy(*pools, c.src, c.dst)
    for _ in range(4):
        graph.replay()
        torch.cuda.synchronize()
        c.same()
        assert (c.refs[c.table[2:5].long()] == 1).all()    # the parent's room is its own again
        (torch.ones(1000, device="cuda") * 2).sum().item()
