"""How the calls on pages are launched, on the CPU: one CTA where there is little to do, else a cluster, if the GPU holds one (a part of a GPU, or groups with
fewer SMs, may not; the launch would be refused there)."""
import ctypes

from paper_2609_20888_b200 import binding as eb
from paper_2609_20888_b200 import build as ebuild


def test_a_cluster_only_where_one_fits():
    ebuild.build()
    lib = eb.load()
    one = lib.eta_selftest_pages_one_cta
    one.argtypes, one.restype = [ctypes.c_int64, ctypes.c_int], ctypes.c_int
    for entries in (1, 1000, 4096):
        assert one(entries, 0) == one(entries, 1) == one(entries, 18) == 1
    for entries in (4097, 100000, 1 << 40):
        assert one(entries, 0) == 1 and one(entries, -1) == 1
        assert one(entries, 1) == one(entries, 18) == 0
