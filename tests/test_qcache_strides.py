"""Strides of dimensions of size 1, which nobody uses, do not have to be aligned; the others do.
Without a GPU: a call whose strides are taken is refused for what is checked after them."""

import ctypes

import pytest

from paper_2607_01308_amd import _cabi as C
from test_qcache_cabi import cache, step

ref = ctypes.byref


@pytest.mark.parametrize("over,taken", [
    (dict(n=1, n_rows=1, q_row_stride=1025, out_row_stride=3), True),
    (dict(n=2, n_rows=2, q_row_stride=1025), False),
    (dict(n=2, n_rows=2, out_row_stride=3), False),
    (dict(n=1, n_rows=1, q_row_stride=-8), False),
    (dict(n=1, n_rows=1, q_row_stride=2 ** 41), False),
    (dict(q_heads=1, q_head_stride=1, out_head_stride=7), True),
    (dict(q_heads=2, q_head_stride=1), False),
    (dict(q_heads=2, out_head_stride=7), False),
])
def test_queries_and_outputs(over, taken):
    c = cache(H=1)
    st = C.lib().cm_qcache_attention(ref(c), 0, ref(step(**over)), None, 0, None)
    assert st == (C.CM_EWORKSPACE if taken else C.CM_EINVAL)


@pytest.mark.parametrize("layers,tokens,H,strides,taken", [
    (1, 1, 1, (3, 5, 7), True), (2, 1, 1, (3, 5, 7), False), (2, 1, 1, (8, 5, 7), True),
    (1, 2, 1, (3, 5, 7), False), (1, 2, 1, (3, 8, 7), True), (1, 1, 2, (3, 5, 7), False),
    (1, 1, 2, (3, 5, 8), True), (1, 1, 1, (-8, 0, 0), False), (1, 1, 1, (0, 2 ** 41, 0), False)])
def test_rows(layers, tokens, H, strides, taken):
    rows, good = C.CmQrows(0x300000, *strides), C.CmQrows(0x300000, 1024, 512, 128)
    for k, v, name in ((rows, good, "k"), (good, rows, "v")):
        st = C.lib().cm_qcache_write(ref(cache(H=H)), 0, layers, C.CM_BF16, ref(k), ref(v), tokens,
                                     None, None)
        assert st == C.CM_EINVAL
        message = C.lib().cm_last_error().decode()
        assert message.startswith("slots_dev" if taken else name + " has a stride"), message
