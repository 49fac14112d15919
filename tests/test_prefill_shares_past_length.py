"""How attention of a step's new tokens shares out its work where sequences have more new tokens than their length says: the rows before the first
token see nothing and cost no tiles, and where the capacity is so small that parts are not joined, no item is split.  On the CPU."""
import ctypes
import random

import pytest

from paper_2609_20888_b200 import binding as eb
from paper_2609_20888_b200 import build as ebuild


@pytest.fixture(scope="module")
def lib():
    ebuild.build()
    return eb.load()


def shares(lib, heads, g_shift, d, ctas, n, lens):
    whole = ctypes.c_int(0)
    ints = ctypes.c_int32 * len(n)
    rc = lib.eta_selftest_prefill_shares(len(n), heads, g_shift, d, ctas, ints(*n), ints(*lens), ctypes.byref(whole))
    return rc, whole.value


@pytest.mark.parametrize("n,length,heads,g_shift", [(600, 512, 2, 2), (4096, 512, 8, 2), (5000, 300, 1, 2), (2000, 512, 8, 2), (1000, 64, 2, 2),
                                                    (100000, 512, 8, 3), (100000, 1, 8, 0), (257, 0, 4, 3), (1 << 20, 512, 2, 3)])
@pytest.mark.parametrize("ctas", [148, 160, 20, 1])
def test_nothing_is_split_where_nothing_is_joined(lib, n, length, heads, g_shift, ctas):
    assert shares(lib, heads, g_shift, 128, ctas, [n], [length]) == (0, 1)


def test_any_lengths(lib):
    rng = random.Random(1)
    ways = [0, 0]
    for _ in range(1500):
        most = rng.choice([512, 512, 100, 2000, 100000])
        n = [rng.choice([0, 1, rng.randint(1, 300), int(2 ** rng.uniform(0, 13))]) for _ in range(rng.choice([1, 1, 2, 3, rng.randint(1, 150)]))]
        lens = [min(most, rng.choice([0, 1, most, rng.randint(0, most), max(0, x - rng.randint(-300, 300))])) for x in n]
        rc, whole = shares(lib, rng.choice([1, 2, 3, 8]), rng.randint(0, 3), rng.choice([64, 128]), rng.choice([148, 148, 132, 160, 1, 7]), n, lens)
        assert rc == 0, (rc, n, lens)
        ways[whole] += 1
    assert min(ways) > 100


def test_far_fewer_tokens_than_rows(lib):
    """Some that see a long context beside many rows that see nothing: split items beside ones without tiles."""
    for g_shift in range(4):
        rc, whole = shares(lib, 2, g_shift, 128, 148, [100000, 1, 7, 3000], [50000, 100000, 3, 40])
        assert rc == 0 and not whole


def test_what_the_check_cannot_take(lib):
    """More sequences or CTAs than the kernel has tables for: refused."""
    whole = ctypes.c_int(0)
    ints = ctypes.c_int32 * 1025
    assert lib.eta_selftest_prefill_shares(1025, 1, 0, 64, 148, ints(), ints(), ctypes.byref(whole)) == -1
    assert shares(lib, 1, 0, 64, 161, [1], [1])[0] == -1 and shares(lib, 1, 0, 64, 0, [1], [1])[0] == -1
