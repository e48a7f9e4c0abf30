"""Arrays without elements in the checks of what overlaps what, without a GPU."""

import ctypes

from paper_2607_01308_amd import _cabi as C

ref = ctypes.byref


def test_arrays_of_nothing_overlap_nothing():
    """An array without elements lies in no other one, whatever its address."""
    cache = C.CmQcache(2, 4, 128, 16, 100, 0x1000000, 0x2000000)
    f = dict(n=3, n_rows=12, table_dev=0x300000, table_width=9, lens_dev=0x310000, rows_dev=0x320000,
             path_dev=0x330000, counts_dev=0x340000, lens_out_dev=0x350000, freed_dev=0x300010, n_freed=0,
             info_dev=0x350000 + 4)
    # (refused for the last of its checks: the earlier ones, that of freed_dev among them, have passed)
    assert C.lib().cm_qcache_keep(ref(cache), ref(C.CmQkeep(**f)), None) == C.CM_EINVAL
    assert C.lib().cm_last_error().decode().startswith("info_dev is")
