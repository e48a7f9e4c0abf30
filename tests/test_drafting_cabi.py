"""The entry points of drafted decoding without a GPU: what they refuse on the host before anything is
enqueued, and what the Python layer refuses by type, shape and device."""

import ctypes

import pytest
import torch

import paper_2607_01308_amd as cm
from paper_2607_01308_amd import _cabi as C

ref = ctypes.byref


@pytest.fixture(scope="module")
def lib():
    return C.lib()


def heads(**over):
    f = dict(in_dev=0x100000, in_token_stride=1024, in_head_stride=128, out_dev=0x200000,
             out_token_stride=1024, out_head_stride=128, weight_dev=0x300000, weight_dtype=C.CM_BF16, heads=8)
    f.update(over)
    return C.CmHeadRows(**f)


def rotate(lib, q=None, k=None, **over):
    f = dict(d=128, dtype=C.CM_BF16, tokens=3, positions=0x400000, base=1e6, style=C.CM_ROPE_HALF,
             reserved=0, eps=1e-6)
    f.update(over)
    rope = C.CmRope(f["base"], f["style"], f["reserved"])
    return lib.cm_norm_rotate(f["d"], f["dtype"], f["tokens"], f["positions"], ref(rope), f["eps"],
                              ref(q or heads()), ref(k or heads()), None)


@pytest.mark.parametrize("over,code", [
    (dict(d=32), C.CM_ESHAPE), (dict(d=96), C.CM_ESHAPE), (dict(d=512), C.CM_ESHAPE), (dict(dtype=2), C.CM_EDTYPE),
    (dict(tokens=-1), C.CM_EINVAL), (dict(tokens=2 ** 31), C.CM_EINVAL), (dict(positions=None), C.CM_EINVAL),
    (dict(positions=0x400002), C.CM_EINVAL), (dict(base=0.0), C.CM_EINVAL), (dict(base=float("nan")), C.CM_EINVAL),
    (dict(base=-2.0), C.CM_EINVAL), (dict(style=2), C.CM_EINVAL), (dict(reserved=1), C.CM_EINVAL),
    (dict(eps=-1e-6), C.CM_EINVAL), (dict(eps=float("nan")), C.CM_EINVAL), (dict(eps=float("inf")), C.CM_EINVAL),
])
def test_rotations_refused(lib, over, code):
    assert rotate(lib, **over) == code
    assert lib.cm_last_error().decode() != ""


@pytest.mark.parametrize("over,code", [
    (dict(in_dev=None), C.CM_EINVAL), (dict(in_dev=0x100008), C.CM_EINVAL), (dict(out_dev=None), C.CM_EINVAL),
    (dict(out_dev=0x200004), C.CM_EINVAL), (dict(in_token_stride=1025), C.CM_EINVAL),
    (dict(in_head_stride=-128), C.CM_EINVAL), (dict(out_token_stride=2 ** 41), C.CM_EINVAL),
    (dict(out_head_stride=4), C.CM_EINVAL), (dict(weight_dtype=3), C.CM_EDTYPE),
    (dict(weight_dev=0x300001), C.CM_EINVAL), (dict(weight_dev=0x300002, weight_dtype=C.CM_F32), C.CM_EINVAL),
    (dict(heads=-1), C.CM_ESHAPE), (dict(heads=65536), C.CM_ESHAPE),
])
def test_heads_refused(lib, over, code):
    assert rotate(lib, q=heads(**over)) == code
    assert rotate(lib, k=heads(**over)) == code
    assert lib.cm_last_error().decode() != ""


def test_rotations_of_nothing(lib):
    assert rotate(lib, tokens=0, positions=None, q=heads(in_dev=None, out_dev=None)) == C.CM_OK
    none = heads(heads=0, in_dev=None, out_dev=None)
    assert rotate(lib, q=none, k=none, positions=None) == C.CM_OK
    rope = C.CmRope(1e4, 0, 0)
    assert lib.cm_norm_rotate(64, C.CM_F32, 5, None, ref(rope), 0.0, None, None, None) == C.CM_OK
    assert lib.cm_norm_rotate(64, C.CM_F32, 5, None, None, 0.0, None, None, None) == C.CM_EINVAL


def drafts(**over):
    f = dict(n=2, dtype=C.CM_F32, n_rows=5, vocabulary=100, probs_dev=0x100000, probs_stride=100,
             draft_probs_dev=0x200000, draft_probs_stride=100, drafts_dev=0x300000, parents_dev=0x400000,
             rows_dev=0x500000, accept_dev=0x600000, sample_dev=0x700000, path_dev=0x800000,
             counts_dev=0x900000, tokens_dev=0xa00000)
    f.update(over)
    return C.CmDrafts(**f)


@pytest.mark.parametrize("over,code", [
    (dict(n=0), C.CM_EINVAL), (dict(n=C.CM_QCACHE_MAX_REQUESTS + 1), C.CM_EINVAL), (dict(dtype=7), C.CM_EDTYPE),
    (dict(n_rows=-1), C.CM_EINVAL), (dict(n_rows=2 ** 31), C.CM_EINVAL), (dict(vocabulary=0), C.CM_EINVAL),
    (dict(vocabulary=2 ** 31), C.CM_EINVAL), (dict(probs_dev=None), C.CM_EINVAL),
    (dict(probs_dev=0x100002), C.CM_EINVAL), (dict(draft_probs_dev=0x200001), C.CM_EINVAL),
    (dict(probs_stride=-1), C.CM_EINVAL), (dict(draft_probs_stride=2 ** 41), C.CM_EINVAL),
    (dict(drafts_dev=None), C.CM_EINVAL), (dict(drafts_dev=0x300004), C.CM_EINVAL),
    (dict(parents_dev=None), C.CM_EINVAL), (dict(parents_dev=0x400001), C.CM_EINVAL),
    (dict(rows_dev=None), C.CM_EINVAL), (dict(rows_dev=0x500002), C.CM_EINVAL),
    (dict(accept_dev=None), C.CM_EINVAL), (dict(accept_dev=0x600002), C.CM_EINVAL),
    (dict(sample_dev=None), C.CM_EINVAL), (dict(sample_dev=0x700003), C.CM_EINVAL),
    (dict(path_dev=None), C.CM_EINVAL), (dict(path_dev=0x800002), C.CM_EINVAL),
    (dict(counts_dev=None), C.CM_EINVAL), (dict(counts_dev=0x900001), C.CM_EINVAL),
    (dict(tokens_dev=None), C.CM_EINVAL), (dict(tokens_dev=0xa00004), C.CM_EINVAL),
])
def test_drafts_refused(lib, over, code):
    assert lib.cm_verify_drafts(ref(drafts(**over)), None) == code
    assert lib.cm_last_error().decode() != ""
    assert lib.cm_verify_drafts(None, None) == C.CM_EINVAL


def test_drafts_workspace(lib):
    def size(**over):
        n = ctypes.c_size_t(7)
        return lib.cm_verify_drafts_size(ref(drafts(**over)), ref(n)), n.value

    assert size(n=1024, vocabulary=200_000) == (C.CM_OK, 0) and size(vocabulary=1000) == (C.CM_OK, 0)
    assert size(n=0)[0] == C.CM_EINVAL and size(dtype=7)[0] == C.CM_EDTYPE and size(vocabulary=0)[0] == C.CM_EINVAL
    assert lib.cm_verify_drafts_size(None, ref(ctypes.c_size_t(0))) == C.CM_EINVAL
    assert lib.cm_verify_drafts_size(ref(drafts()), None) == C.CM_EINVAL
    # misaligned, whatever is needed
    need = size(n=2, vocabulary=200_000)[1]
    if need:
        for at, some in ((0xb00010, need), (0xb00000, need - 1)):
            wrong = drafts(n=2, vocabulary=200_000, probs_stride=200_000, draft_probs_stride=200_000, workspace=at,
                           workspace_bytes=some)
            assert lib.cm_verify_drafts(ref(wrong), None) == C.CM_EWORKSPACE


def cache(**over):
    f = dict(L=2, H=4, d=128, block=16, pages=100, codes_dev=0x100000, scales_dev=0x200000)
    f.update(over)
    return C.CmQcache(**f)


def kept(**over):
    f = dict(n=3, n_rows=12, table_dev=0x300000, table_width=9, lens_dev=0x310000, rows_dev=0x320000,
             path_dev=0x330000, counts_dev=0x340000, lens_out_dev=0x350000, freed_dev=0x360000, n_freed=10,
             info_dev=0x370000)
    f.update(over)
    return C.CmQkeep(**f)


@pytest.mark.parametrize("over,code", [
    (dict(n=0), C.CM_EINVAL), (dict(n=C.CM_QCACHE_MAX_REQUESTS + 1), C.CM_EINVAL), (dict(n_rows=-1), C.CM_EINVAL),
    (dict(n_rows=2 ** 31), C.CM_EINVAL), (dict(table_width=0), C.CM_EINVAL), (dict(table_width=2 ** 27), C.CM_EINVAL),
    (dict(n_freed=-1), C.CM_EINVAL), (dict(n_freed=2 ** 31), C.CM_EINVAL), (dict(table_dev=None), C.CM_EINVAL),
    (dict(lens_dev=0x310002), C.CM_EINVAL), (dict(rows_dev=None), C.CM_EINVAL), (dict(path_dev=None), C.CM_EINVAL),
    (dict(counts_dev=0x340001), C.CM_EINVAL), (dict(lens_out_dev=None), C.CM_EINVAL),
    (dict(freed_dev=None), C.CM_EINVAL), (dict(freed_dev=0x360002), C.CM_EINVAL), (dict(info_dev=None), C.CM_EINVAL),
    (dict(info_dev=0x370004), C.CM_EINVAL),
    # what is written lies over what is read
    (dict(lens_out_dev=0x310000), C.CM_EINVAL), (dict(freed_dev=0x300020), C.CM_EINVAL),
    (dict(info_dev=0x320008), C.CM_EINVAL), (dict(lens_out_dev=0x340008), C.CM_EINVAL),
])
def test_keeps_refused(lib, over, code):
    assert lib.cm_qcache_keep(ref(cache()), ref(kept(**over)), None) == code
    assert lib.cm_last_error().decode() != ""


def test_caches_refused(lib):
    for over, code in ((dict(L=0), C.CM_EINVAL), (dict(d=96), C.CM_ESHAPE), (dict(block=8), C.CM_ESHAPE),
                       (dict(pages=0), C.CM_EINVAL), (dict(codes_dev=None), C.CM_EINVAL)):
        assert lib.cm_qcache_keep(ref(cache(**over)), ref(kept()), None) == code
        assert lib.cm_qcache_copy(ref(cache(**over)), 0, 1, 3, 0x400000, 0x500000, None) == code
    assert lib.cm_qcache_keep(ref(cache()), None, None) == C.CM_EINVAL


@pytest.mark.parametrize("first,layers,n,src,dst,code", [
    (-1, 1, 3, 0x400000, 0x500000, C.CM_EINVAL), (0, 3, 3, 0x400000, 0x500000, C.CM_EINVAL),
    (2, 1, 3, 0x400000, 0x500000, C.CM_EINVAL), (0, -1, 3, 0x400000, 0x500000, C.CM_EINVAL),
    (0, 2, -1, 0x400000, 0x500000, C.CM_EINVAL), (0, 2, 2 ** 31, 0x400000, 0x500000, C.CM_EINVAL),
    (0, 2, 3, None, 0x500000, C.CM_EINVAL), (0, 2, 3, 0x400000, 0x500002, C.CM_EINVAL),
    (0, 2, 0, None, None, C.CM_OK), (2, 0, 3, None, None, C.CM_OK),
])
def test_copies_refused(lib, first, layers, n, src, dst, code):
    assert lib.cm_qcache_copy(ref(cache()), first, layers, n, src, dst, None) == code


def tree(lib, **over):
    f = dict(n=2, n_rows=9, parents=0x100000, rows=0x110000, lens=0x120000, window=0, words=1,
             masks=0x130000, positions=0x140000, info=0x150000)
    f.update(over)
    return lib.cm_qcache_tree(f["n"], f["n_rows"], f["parents"], f["rows"], f["lens"], f["window"],
                              f["words"], f["masks"], f["positions"], f["info"], None)


@pytest.mark.parametrize("over,code", [
    (dict(n=0), C.CM_EINVAL), (dict(n=C.CM_QCACHE_MAX_REQUESTS + 1), C.CM_EINVAL), (dict(n_rows=-1), C.CM_EINVAL),
    (dict(n_rows=2 ** 31), C.CM_EINVAL), (dict(window=-1), C.CM_EINVAL), (dict(words=-1), C.CM_EINVAL),
    (dict(words=0), C.CM_EINVAL), (dict(words=17), C.CM_EINVAL), (dict(masks=None), C.CM_EINVAL),
    (dict(masks=0x130004), C.CM_EINVAL), (dict(parents=0x100002), C.CM_EINVAL), (dict(rows=None), C.CM_EINVAL),
    (dict(rows=0x110001), C.CM_EINVAL), (dict(lens=None), C.CM_EINVAL), (dict(lens=0x120002), C.CM_EINVAL),
    (dict(positions=None), C.CM_EINVAL), (dict(positions=0x140002), C.CM_EINVAL), (dict(info=None), C.CM_EINVAL),
    (dict(info=0x150003), C.CM_EINVAL), (dict(positions=0x100010), C.CM_EINVAL), (dict(info=0x120004), C.CM_EINVAL),
    (dict(masks=0x110000), C.CM_EINVAL),
])
def test_trees_refused(lib, over, code):
    assert tree(lib, **over) == code
    assert lib.cm_last_error().decode() != ""


def step(**over):
    f = dict(n=3, q_heads=8, dtype=C.CM_BF16, window=0, n_rows=12, max_rows=4, scale=0.1,
             q_dev=0x300000, q_row_stride=1024, q_head_stride=128, out_dev=0x400000,
             out_row_stride=1024, out_head_stride=128, lse_dev=0x500000, rows_dev=0x510000,
             lens_dev=0x600000, table_dev=0x700000, table_width=9)
    f.update(over)
    return C.CmQattention(**f)


def attend(lib, c=None, layer=0, ws=0x800000, bytes=1 << 40, tree=(0x900000, 1, 0xa00000), **over):
    t = None if tree is None else ref(C.CmQtree(*tree))
    return lib.cm_qcache_tree_attention(ref(c or cache()), layer, ref(step(**over)), t, ws, bytes, None)


@pytest.mark.parametrize("over,code", [
    (dict(n=0), C.CM_EINVAL), (dict(n=C.CM_QCACHE_MAX_REQUESTS + 1), C.CM_EINVAL), (dict(q_heads=6), C.CM_ESHAPE),
    (dict(q_heads=65 * 4), C.CM_ESHAPE), (dict(dtype=2), C.CM_EDTYPE), (dict(window=-1), C.CM_EINVAL),
    (dict(n_rows=-1), C.CM_EINVAL), (dict(n_rows=2 ** 31), C.CM_EINVAL), (dict(max_rows=-1), C.CM_EINVAL),
    (dict(scale=float("nan")), C.CM_EINVAL), (dict(rows_dev=None), C.CM_EINVAL), (dict(rows_dev=0x510002), C.CM_EINVAL),
    (dict(lens_dev=None), C.CM_EINVAL), (dict(table_dev=0x700002), C.CM_EINVAL), (dict(table_width=0), C.CM_EINVAL),
    (dict(table_width=2 ** 27), C.CM_EINVAL), (dict(q_dev=0x300008), C.CM_EINVAL), (dict(q_row_stride=1025), C.CM_EINVAL),
    (dict(out_dev=None), C.CM_EINVAL), (dict(out_head_stride=4), C.CM_EINVAL), (dict(lse_dev=0x500002), C.CM_EINVAL),
    (dict(layer=-1), C.CM_EINVAL), (dict(layer=2), C.CM_EINVAL), (dict(tree=None), C.CM_EINVAL),
    (dict(tree=(None, 1, 0xa00000)), C.CM_EINVAL), (dict(tree=(0x900004, 1, 0xa00000)), C.CM_EINVAL),
    (dict(tree=(0x900000, 0, 0xa00000)), C.CM_EINVAL), (dict(tree=(0x900000, 17, 0xa00000)), C.CM_EINVAL),
    (dict(window=5, tree=(0x900000, 1, None)), C.CM_EINVAL), (dict(window=5, tree=(0x900000, 1, 0xa00002)), C.CM_EINVAL),
    (dict(ws=None), C.CM_EWORKSPACE), (dict(ws=0x800010), C.CM_EWORKSPACE), (dict(bytes=1000), C.CM_EWORKSPACE),
])
def test_tree_attention_refused(lib, over, code):
    assert attend(lib, **over) == code
    assert lib.cm_last_error().decode() != ""


def test_tree_attention_sizes(lib):
    def size(c, **over):
        out = ctypes.c_size_t(0)
        assert lib.cm_qcache_tree_attention_size(ref(c), ref(step(**over)), ref(out)) == C.CM_OK
        return out.value

    assert attend(lib, n_rows=0, q_dev=None, out_dev=None, ws=None) == C.CM_OK
    assert lib.cm_qcache_tree_attention_size(ref(cache()), ref(step()), None) == C.CM_EINVAL
    assert lib.cm_qcache_tree_attention_size(ref(cache()), None, ref(ctypes.c_size_t())) == C.CM_EINVAL
    need = size(cache())
    assert attend(lib, bytes=need - 1) == C.CM_EWORKSPACE
    # partial results follow from the workgroups that run together, not from rows or lengths
    most = max(size(cache(H=h, L=1), q_heads=h * 4, n_rows=r, max_rows=r, table_width=w)
               for h in (1, 8, 64, 300) for r in (1, 4, 100, 100000) for w in (9, 1 << 20))
    assert need < most < 256 << 20


def test_binding_refusals():
    """By type, shape and device, without a GPU."""
    lens = torch.tensor([3], dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU"):
        cm.qcache_tree(None, torch.tensor([0, 3], dtype=torch.int32), lens, 3, 3)
    q = torch.zeros((3, 4, 64))
    pos = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU"):
        cm.norm_rotate(q, None, pos, 1e4)
    with pytest.raises(TypeError, match="bfloat16 or float32"):
        cm.norm_rotate(q.half(), None, pos, 1e4)
    with pytest.raises(ValueError, match="style"):
        cm.norm_rotate(q, None, pos, 1e4, style="other")
    with pytest.raises(ValueError, match="heads"):
        cm.norm_rotate(q[0], None, pos, 1e4)
    rows = torch.tensor([0, 3], dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU"):
        cm.verify_drafts(torch.zeros((3, 5)), torch.zeros(3, dtype=torch.int64), pos, rows, torch.zeros(3),
                         torch.zeros(1))
    with pytest.raises(ValueError, match="rows"):
        cm.verify_drafts(torch.zeros((3, 5)), torch.zeros(3, dtype=torch.int64), pos, rows[:1], torch.zeros(3),
                         torch.zeros(1))
