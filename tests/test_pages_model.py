"""The host model of the page tables on its own: shared pages that are about to be written, by hand and over random histories."""
import random

import pytest

from pages_model import Pages


def group(kv, pages, children, ps=16, num_pages=60):
    """A parent of `kv` tokens that holds `pages` pages, and its children."""
    m = Pages([8] * (1 + children), num_pages, ps)
    m.resize([pages * ps] + [-1] * children)
    m.kv[0] = kv
    assert m.fork([-1] + [0] * children) == [0] * (1 + children)
    return m


def test_a_shared_page_at_a_border_is_replaced_and_not_copied():
    m = group(16, 2, 2)
    assert m.resize([-1, 20, 20]) == ([-1] * 3, [-1] * 3, [0] * 3)
    assert m.table[0][:2] == [0, 1] and m.table[1][:2] == [0, 2] and m.table[2][:2] == [0, 3]
    assert m.refs[:4] == [3, 1, 1, 1]


def test_every_shared_page_up_to_the_last_wanted_one_is_replaced():
    m = group(5, 4, 2)
    src, dst, missing = m.resize([40, 10, 70])
    assert m.table[0][:4] == [4, 5, 6, -1] and m.table[1][:2] == [7, -1] and m.table[2][:6] == [8, 9, 10, 11, 12, -1]
    assert (src, dst, missing) == ([0, 0, 0], [4, 7, 8], [0] * 3) and m.refs[:4] == [0] * 4


def test_holders_that_do_not_grow_keep_their_pages():
    m = group(5, 3, 1)
    assert m.resize([5, 0]) == ([-1] * 2, [-1] * 2, [0] * 2)
    assert m.table[0][:2] == [0, -1] and m.refs[:3] == [1, 0, 0]


def test_too_few_pages_for_the_shared_ones():
    m = group(16, 3, 1, num_pages=4)
    assert m.resize([-1, 48])[2] == [0, 2] and m.table[1][:3] == [0, 1, 2] and m.refs == [2, 2, 2, 0]
    assert m.resize([-1, 32])[2] == [0, 0] and m.table[1][:3] == [0, 3, -1] and m.refs == [2, 1, 1, 1]


@pytest.mark.parametrize("seed", range(40))
def test_no_page_is_written_by_two_sequences(seed):
    rng = random.Random(seed)
    B, ps = rng.randrange(2, 12), 16
    m = Pages([rng.randrange(1, 12) for _ in range(B)], rng.randrange(10, 90), ps)
    for _ in range(60):
        kind = rng.choice(["resize", "resize", "fork", "lengths", "compact"])
        if kind == "resize":
            want = [rng.choice([-1, 0, kv, kv + rng.randrange(0, 4 * ps)]) for kv in m.kv]
            kv = list(m.kv)
            missing = m.resize(want)[2]
            assert m.written_twice(kv, [-1 if x else w for w, x in zip(want, missing)]) == []
            for b in range(B):     # and nobody else names them
                if want[b] > kv[b] and not missing[b]:
                    assert all(m.refs[e] == 1 for e in m.table[b][kv[b] // ps:m.count[b]])
        elif kind == "fork":
            m.fork([rng.choice([-1, rng.randrange(0, B)]) for _ in range(B)])
        elif kind == "lengths":
            m.kv = [rng.randrange(0, c * ps + 1) for c in m.count]
        else:
            m.compact(rng.randrange(1, 9))
        names = [e for row, c in zip(m.table, m.count) for e in row[:c]]
        assert all(m.refs[i] == names.count(i) for i in range(len(m.refs)))
