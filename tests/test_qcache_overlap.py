"""cm_qcache_tables refuses outputs that lie over its inputs: other workgroups may read these after
the outputs are written. Without a GPU."""

import pytest

from paper_2607_01308_amd import _cabi as C


@pytest.mark.parametrize("over,what", [
    (dict(lens=0x10000), "lens_dev overlaps held_dev"), (dict(lens=0x10004), "lens_dev overlaps held_dev"),
    (dict(lens=0xfffc), "lens_dev overlaps held_dev"), (dict(rows=0x20000), "rows_dev overlaps new_dev"),
    (dict(rows=0x20000 - 4 * 5), "rows_dev overlaps new_dev"), (dict(table=0x30000), "table_dev overlaps free_dev"),
    (dict(table=0x30000 - 4 * 39), "table_dev overlaps free_dev"),
    (dict(slots=0x10000), "slots_dev overlaps held_dev"), (dict(info=0x2fff0), "info_dev overlaps free_dev"),
    # side by side: refused for what is checked after them
    (dict(lens=0x10014, info=None), "info_dev is NULL"),
    (dict(held=0x10000, new=0x10000, info=None), "info_dev is NULL"),
])
def test_outputs_over_inputs(over, what):
    f = dict(pages=10, block=16, n=5, held=0x10000, new=0x20000, free=0x30000, n_free=4, table=0x40000,
             width=8, tokens=3, slots=0x60000, rows=0x70000, lens=0x80000, info=0x90000)
    f.update(over)
    st = C.lib().cm_qcache_tables(f["pages"], f["block"], f["n"], f["held"], f["new"], f["free"],
                                  f["n_free"], f["table"], f["width"], f["tokens"], f["slots"],
                                  f["rows"], f["lens"], f["info"], None)
    assert st == C.CM_EINVAL and C.lib().cm_last_error().decode().startswith(what)
