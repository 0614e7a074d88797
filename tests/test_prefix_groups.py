"""kvcache.prefix_groups on the CPU: the groups of a batch's block table against
all ways of cutting it into runs."""

import itertools

import numpy as np
import pytest

from paper_2607_13095_amd.kvcache import prefix_groups


def _saved(table, lens, pg, cu, shared):
    total = 0
    for a, b, s in zip(cu[:-1], cu[1:], shared):
        assert 0 <= s <= min(lens[a:b], default=0) if b - a > 1 else s == 0
        for i in range(a, b):  # what is said to be shared is on the same pages
            n = -(-int(s) // pg)
            assert np.array_equal(table[i, :n], table[a, :n]) and np.all(table[i, :n] >= 0)
        total += (b - a - 1) * int(s)
    return total


def _best(table, lens, pg):
    ns = len(lens)
    best = 0
    for cuts in itertools.product([0, 1], repeat=ns - 1):
        cu = [0] + [i + 1 for i, c in enumerate(cuts) if c] + [ns]
        total = 0
        for a, b in zip(cu[:-1], cu[1:]):
            n = 0
            while n < table.shape[1] and table[a, n] >= 0 and np.all(table[a:b, n] == table[a, n]):
                n += 1
            total += (b - a - 1) * min(n * pg, min(lens[a:b]))
        best = max(best, total)
    return best


@pytest.mark.parametrize("seed", range(40))
def test_prefix_groups(seed):
    r = np.random.default_rng(seed)
    ns, pg = int(r.integers(1, 9)), int(r.choice([16, 64]))
    lens = r.integers(0, 6 * pg, ns).tolist()
    table = np.full((ns, 6), -1, np.int32)
    for b, n in enumerate(lens):
        table[b, :-(-n // pg)] = 100 * b + np.arange(-(-n // pg))
        if b and r.random() < 0.7:  # the first pages of the sequence before it
            m = int(r.integers(0, 7))
            take = min(m, -(-n // pg), -(-lens[b - 1] // pg))
            table[b, :take] = table[b - 1, :take]
    cu, shared = prefix_groups(table, lens, pg)
    assert cu.dtype == shared.dtype == np.int32
    assert cu[0] == 0 and cu[-1] == ns and np.all(np.diff(cu) > 0) and len(shared) == len(cu) - 1
    assert _saved(table, lens, pg, cu, shared) == _best(table, lens, pg)


def test_prefix_groups_empty():
    cu, shared = prefix_groups(np.zeros((0, 4), np.int32), [], 16)
    assert cu.tolist() == [0] and shared.size == 0
