"""Page tables of the cache on the GPU against the same steps on the host, and the copies of their contents."""
import random

import pytest
import torch

import plain
from paper_2510_26475_amd import binding

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Cache:
    """The state on the GPU beside its model on the host."""

    def __init__(self, cap, num_pages, ps):
        self.model, self.ps = plain.Pages(cap, num_pages, ps), ps
        B = len(cap)
        self.indptr = ints([0] + cap).cumsum(0).to(torch.int32)
        self.table, self.count, self.kv = ints([-1] * sum(cap)), ints([0] * B), ints([0] * B)
        self.refs = ints([0] * num_pages)
        self.src, self.dst, self.missing = (ints([9] * B) for _ in range(3))
        self.ws = torch.empty(binding.respec_pages_workspace_bytes(B, num_pages), dtype=torch.uint8, device="cuda")
        self.state = (self.indptr, self.table, self.count, self.kv, self.refs)

    def same(self):
        m = self.model
        assert self.table.tolist() == [e for row in m.table for e in row]
        assert self.count.tolist() == m.count and self.kv.tolist() == m.kv and self.refs.tolist() == m.refs
        assert min(m.refs) >= 0

    def resize(self, want):
        lists = self.model.resize(want)
        self.ws.fill_(0xff)
        binding.respec_pages_resize(ints(want), *self.state, self.src, self.dst, self.missing, self.ps, self.ws)
        assert (self.src.tolist(), self.dst.tolist(), self.missing.tolist()) == lists
        self.same()
        return lists

    def fork(self, parent):
        missing = self.model.fork(parent)
        binding.respec_pages_fork(ints(parent), *self.state, self.missing)
        assert self.missing.tolist() == missing
        self.same()
        return missing

    def compact(self, moves, in_place):
        want = self.model.compact(moves)
        table, refs = (self.table, self.refs) if in_place else (torch.empty_like(self.table), torch.empty_like(self.refs))
        src, dst, end = ints([9] * moves), ints([9] * moves), ints([9])
        self.ws.fill_(0xff)
        binding.respec_pages_compact(self.table, self.refs, table, refs, src, dst, end, self.ws)
        assert (src.tolist(), dst.tolist(), end.item()) == want
        self.table.copy_(table)
        self.refs.copy_(refs)
        self.same()
        return src, dst

    def set_len(self, lens):
        self.model.kv = list(lens)
        self.kv.copy_(ints(lens))


def test_grow_share_write_and_give_back():
    c = Cache([4, 4, 4, 4], 10, 16)
    c.resize([40, -1, 17, 0])
    c.set_len([40, 0, 17, 0])
    c.fork([-1, 0, -1, 0])
    src, dst, missing = c.resize([48, 49, -1, 40])   # two of the three holders write into the shared page, one of them grows too
    assert [s >= 0 for s in src] == [True, True, False, False] and missing == [0] * 4
    c.resize([0, -1, -1, -1])
    c.resize([-1, 0, 0, 0])
    assert c.refs.tolist() == [0] * 10


def test_a_full_pool_and_a_short_table_leave_the_sequence_as_it_was():
    c = Cache([2, 5, 5, 5], 6, 16)
    c.resize([16, 32, 0, 0])
    assert c.resize([33, 48, 64, 16])[2] == [2, 0, 4, 1]   # too long for its table; served; too many; behind it in the order
    assert c.resize([0, -1, -1, 16])[2] == [0, 0, 0, 0]
    assert c.resize([-1, 0, 96, 32])[2] == [0, 0, 6, 0]    # six pages do not go into a table of five: they are not kept from the next one
    assert c.resize([-1, 16, 0, 80])[2] == [0, 0, 0, 0]
    assert c.resize([16, 0, -1, -1])[2] == [1, 0, 0, 0]    # what the call gives back is free for the next one only
    c.resize([-1, -1, 64, 32])


def test_forks_that_cannot_be():
    c = Cache([3, 2, 3, 3, 3], 12, 16)
    c.resize([48, 0, 0, 16, 0])
    c.set_len([41, 0, 0, 3, 0])
    # table too short; a child's child; holds pages; no such sequence
    assert c.fork([-1, 0, 4, 0, 0]) == [0, -1, -1, -1, 0]
    assert c.fork([0, -1, 99, -1, -1]) == [-1, 0, -1, 0, 0]
    c.fork([-1, -1, 1, -1, -1])                            # of an empty sequence: empty


@pytest.mark.parametrize("num_pages,B,ps", [(1, 1, 16), (37, 5, 16), (1024, 40, 64), (1025, 300, 16), (4096, 2000, 16), (4096, 64, 16), (4097, 20, 64), (9000, 33, 1024),
                                              (16384, 9, 16), (16385, 1030, 16), (70000, 60, 16)])
def test_random_histories(num_pages, B, ps):
    rng = random.Random(num_pages)
    cap = [rng.randrange(1, max(2, 3 * num_pages // B + 2)) for _ in range(B)]
    c = Cache(cap, num_pages, ps)
    for step in range(14):
        kind = rng.choice(["resize", "resize", "fork", "compact", "lengths"])
        if kind == "resize":
            c.resize([rng.choice([-1, 0, rng.randrange(0, ps * (k + 2)), n + rng.randrange(0, 2 * ps)])
                      for k, n in zip(cap, c.model.kv)])
        elif kind == "lengths":
            c.set_len([rng.randrange(0, k * ps + 1) for k in c.model.count])
        elif kind == "fork":
            c.fork([rng.choice([-1, rng.randrange(0, B)]) for _ in range(B)])
        else:
            c.compact(rng.choice([1, 3, num_pages // 2 + 1]), in_place=rng.random() < 0.5)


def test_compact_by_steps_reaches_the_whole():
    c = Cache([1] * 600, 2000, 16)
    c.resize([16] * 600)
    c.resize([0 if b % 3 else -1 for b in range(600)])
    whole = plain.Pages([1], 1, 16)
    for _ in range(5):
        c.compact(40, in_place=True)
    assert c.table[c.table >= 0].max().item() == 199 and sorted(c.table[c.table >= 0].tolist()) == list(range(200))
    c.compact(7, in_place=False)                           # nothing left to move
    c.resize([0] * 600)
    c.compact(3, in_place=True)                            # nothing held at all


@pytest.mark.parametrize("dtype,ps,Hkv,D", [(torch.bfloat16, 16, 4, 128), (torch.float32, 64, 1, 64), (torch.bfloat16, 1024, 8, 128),
                                            (torch.bfloat16, 16, 1, 8), (torch.float32, 32, 3, 68)])
def test_copies(dtype, ps, Hkv, D):
    n = 23
    pools = [torch.randn((n, ps, Hkv, D), device="cuda").to(dtype) for _ in range(2)]
    want = [p.clone() for p in pools]
    src, dst = [3, -1, 5, 22, 4, 9, 7, 40, -3], [0, 2, -1, 1, 4, 23, 8, 2, 2]
    for a, b in [(3, 0), (22, 1), (7, 8)]:
        for w, p in zip(want, pools):
            w[b] = p[a]
    binding.respec_pages_copy(*pools, ints(src), ints(dst))
    for w, p in zip(want, pools):
        assert torch.equal(w, p)


def test_many_copies_and_offsets_past_32_bits():
    ps, Hkv, D = 64, 8, 128                                # 128 KiB a page
    n = (1 << 32) // (ps * Hkv * D * 2) + 50
    k, v = (torch.empty((n, ps, Hkv, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    m = 40
    k[-m:], v[-m:] = torch.randn((m, ps, Hkv, D), device="cuda").bfloat16(), torch.randn((m, ps, Hkv, D), device="cuda").bfloat16()
    src = torch.full((20000,), -1, dtype=torch.int32, device="cuda")
    dst = src.clone()
    at = torch.randperm(20000, device="cuda")[:m]
    src[at] = torch.arange(n - m, n, dtype=torch.int32, device="cuda")
    dst[at] = torch.arange(0, m, dtype=torch.int32, device="cuda")
    binding.respec_pages_copy(k, v, src, dst)
    assert torch.equal(k[:m], k[-m:]) and torch.equal(v[:m], v[-m:])


def test_captured_calls_replay():
    """A group's turn (give back, fork, grow, copy) as one graph, replayed: the same state each time."""
    c = Cache([4, 5, 5, 5], 20, 16)
    c.resize([50, 16, 32, 0])
    c.set_len([50, 10, 20, 0])
    pools = [torch.randn((20, 16, 2, 64), device="cuda") for _ in range(2)]
    back, parent, want = ints([-1, 0, 0, 0]), ints([-1, 0, 0, 0]), ints([-1, 70, 51, 50])
    c.model.resize(back.tolist())
    c.model.fork(parent.tolist())
    src, dst, _ = c.model.resize(want.tolist())
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
        assert c.src.tolist() == src and c.dst.tolist() == dst
        for a, b in zip(src, dst):
            assert a < 0 or all(torch.equal(p[a], p[b]) for p in pools)
        (torch.ones(1000, device="cuda") * 2).sum().item()


def test_states_that_are_not_one_stay_inside_the_buffers():
    """Counts past the table, ids that are no pages, offsets outside the table: nothing outside the arrays is touched."""
    guard = 64
    big = {n: torch.full((guard + k + guard,), 5, dtype=torch.int32, device="cuda") for n, k in (("table", 12), ("refs", 8), ("count", 4), ("kv", 4))}
    v = {n: t[guard:-guard] for n, t in big.items()}
    indptr = ints([0, 3, 99, -7, 12])
    v["table"].copy_(ints([0, 1, 2, 99, -4, 7, 3, 1 << 30, 5, 6, 0, 0]))
    v["refs"].copy_(ints([1, 2, 0, 0, 1, 1, 1, 1]))
    v["count"].copy_(ints([3, 1 << 30, -2, 12]))
    v["kv"].copy_(ints([40, 1 << 30, -9, 100]))
    src, dst, missing = ints([9] * 4), ints([9] * 4), ints([9] * 4)
    ws = torch.empty(binding.respec_pages_workspace_bytes(4, 8), dtype=torch.uint8, device="cuda")
    state = (indptr, v["table"], v["count"], v["kv"], v["refs"])
    for want in ([100, 5, 2000000000, 0], [0, 0, 0, 0], [16, 16, 16, 2147483647]):
        binding.respec_pages_resize(ints(want), *state, src, dst, missing, 16, ws)
        binding.respec_pages_fork(ints([2, 0, -1, 1 << 30]), *state, missing)
        binding.respec_pages_compact(v["table"], v["refs"], v["table"], v["refs"], src, dst, missing[:1], ws)
    torch.cuda.synchronize()
    for t in big.values():
        assert (t[:guard] == 5).all() and (t[-guard:] == 5).all()
