"""The 8-bit paged cache's entry points without a GPU: what they refuse on the host
before anything is enqueued, workspace sizes, and (against a build of the host code
under AddressSanitizer and UndefinedBehaviorSanitizer) the same again."""

import ctypes
import os
import subprocess
import sys

import pytest

import paper_2607_01308_amd as cm
from paper_2607_01308_amd import _cabi as C
from paper_2607_01308_amd import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = ctypes.c_void_p


@pytest.fixture(scope="module")
def lib():
    return C.lib()


def cache(**over):
    f = dict(L=2, H=4, d=128, block=16, pages=100, codes_dev=0x100000, scales_dev=0x200000)
    f.update(over)
    return C.CmQcache(**f)


def step(**over):
    f = dict(n=3, q_heads=8, dtype=C.CM_BF16, window=0, n_rows=3, max_rows=1, scale=0.1,
             q_dev=0x300000, q_row_stride=1024, q_head_stride=128, out_dev=0x400000,
             out_row_stride=1024, out_head_stride=128, lse_dev=0x500000, rows_dev=None,
             lens_dev=0x600000, table_dev=0x700000, table_width=9)
    f.update(over)
    return C.CmQattention(**f)


def size(lib, c, s):
    out = ctypes.c_size_t(0)
    st = lib.cm_qcache_attention_size(ctypes.byref(c), ctypes.byref(s), ctypes.byref(out))
    return st, out.value


BAD_CACHES = [
    (dict(L=0), C.CM_EINVAL), (dict(H=0), C.CM_EINVAL), (dict(L=4096, H=8), C.CM_ESHAPE),
    (dict(d=32), C.CM_ESHAPE), (dict(d=96), C.CM_ESHAPE), (dict(d=512), C.CM_ESHAPE),
    (dict(block=8), C.CM_ESHAPE), (dict(block=48), C.CM_ESHAPE), (dict(block=256), C.CM_ESHAPE),
    (dict(pages=0), C.CM_EINVAL), (dict(pages=2 ** 31), C.CM_EINVAL),
    (dict(codes_dev=None), C.CM_EINVAL), (dict(codes_dev=0x100008), C.CM_EINVAL),
    (dict(scales_dev=None), C.CM_EINVAL), (dict(scales_dev=0x200002), C.CM_EINVAL),
]


@pytest.mark.parametrize("over,code", BAD_CACHES)
def test_caches_refused(lib, over, code):
    c = cache(**over)
    k = C.CmQrows(0x300000, 0, 512, 128)
    assert size(lib, c, step())[0] == code
    assert lib.cm_qcache_attention(ctypes.byref(c), 0, ctypes.byref(step()), 0x800000, 1 << 40,
                                   None) == code
    assert lib.cm_qcache_write(ctypes.byref(c), 0, 1, C.CM_BF16, ctypes.byref(k), ctypes.byref(k),
                               3, 0x900000, None) == code
    assert lib.cm_last_error().decode() != ""


@pytest.mark.parametrize("over,code", [
    (dict(n=0), C.CM_EINVAL), (dict(n=C.CM_QCACHE_MAX_REQUESTS + 1), C.CM_EINVAL),
    (dict(q_heads=0), C.CM_ESHAPE), (dict(q_heads=6), C.CM_ESHAPE), (dict(q_heads=65 * 4), C.CM_ESHAPE),
    (dict(dtype=2), C.CM_EDTYPE), (dict(window=-1), C.CM_EINVAL),
    (dict(n_rows=-1), C.CM_EINVAL), (dict(n_rows=2 ** 31), C.CM_EINVAL),
    (dict(max_rows=-1), C.CM_EINVAL), (dict(scale=float("nan")), C.CM_EINVAL),
    (dict(scale=float("inf")), C.CM_EINVAL),
    (dict(n_rows=4), C.CM_EINVAL),                       # without rows: one a request
    (dict(rows_dev=0x111002), C.CM_EINVAL),
    (dict(lens_dev=None), C.CM_EINVAL), (dict(lens_dev=0x111001), C.CM_EINVAL),
    (dict(table_dev=None), C.CM_EINVAL), (dict(table_dev=0x111002), C.CM_EINVAL),
    (dict(table_width=0), C.CM_EINVAL), (dict(table_width=2 ** 27), C.CM_EINVAL),
    (dict(q_dev=None), C.CM_EINVAL), (dict(q_dev=0x300008), C.CM_EINVAL),
    (dict(q_row_stride=1025), C.CM_EINVAL), (dict(q_head_stride=-8), C.CM_EINVAL),
    (dict(q_row_stride=2 ** 41), C.CM_EINVAL),
    (dict(out_dev=None), C.CM_EINVAL), (dict(out_dev=0x400004), C.CM_EINVAL),
    (dict(out_row_stride=1028), C.CM_EINVAL), (dict(out_head_stride=4), C.CM_EINVAL),
    (dict(lse_dev=0x500002), C.CM_EINVAL),
])
def test_attention_steps_refused(lib, over, code):
    assert lib.cm_qcache_attention(ctypes.byref(cache()), 0, ctypes.byref(step(**over)), 0x800000,
                                   1 << 40, None) == code
    assert lib.cm_last_error().decode() != ""


def test_attention_layer_and_workspace(lib):
    c, s = cache(), step()
    st, need = size(lib, c, s)
    assert st == C.CM_OK and need > 0
    f = lib.cm_qcache_attention
    ref = ctypes.byref
    assert f(ref(c), 2, ref(s), 0x800000, need, None) == C.CM_EINVAL
    assert f(ref(c), -1, ref(s), 0x800000, need, None) == C.CM_EINVAL
    assert f(ref(c), 0, ref(s), None, need, None) == C.CM_EWORKSPACE
    assert f(ref(c), 0, ref(s), 0x800010, need, None) == C.CM_EWORKSPACE
    assert f(ref(c), 0, ref(s), 0x800000, need - 1, None) == C.CM_EWORKSPACE
    assert f(ref(c), 0, None, 0x800000, need, None) == C.CM_EINVAL
    assert f(None, 0, ref(s), 0x800000, need, None) == C.CM_EINVAL
    assert lib.cm_qcache_attention_size(ref(c), ref(s), None) == C.CM_EINVAL
    assert lib.cm_qcache_attention_size(ref(c), None, ctypes.byref(ctypes.c_size_t())) == C.CM_EINVAL
    # nothing to do: no pointer is needed and nothing is enqueued
    none = step(n_rows=0, rows_dev=0x111000, q_dev=None, out_dev=None)
    assert f(ref(c), 0, ref(none), None, 0, None) == C.CM_OK
    # more rows, more requests and wider heads need no less
    for more in (dict(n_rows=5000, rows_dev=0x111000, max_rows=5000), dict(n=1000, n_rows=1000)):
        assert size(lib, c, step(**more))[1] >= need


@pytest.mark.parametrize("over,code", [
    (dict(first=2), C.CM_EINVAL), (dict(first=-1), C.CM_EINVAL), (dict(layers=3), C.CM_EINVAL),
    (dict(layers=-1), C.CM_EINVAL), (dict(first=1, layers=2), C.CM_EINVAL),
    (dict(dtype=5), C.CM_EDTYPE), (dict(tokens=-1), C.CM_EINVAL), (dict(tokens=2 ** 31), C.CM_EINVAL),
    (dict(k=None), C.CM_EINVAL), (dict(v=None), C.CM_EINVAL), (dict(slots=None), C.CM_EINVAL),
    (dict(slots=0x900004), C.CM_EINVAL),
    (dict(k=C.CmQrows(0x300004, 0, 512, 128)), C.CM_EINVAL),
    (dict(k=C.CmQrows(None, 0, 512, 128)), C.CM_EINVAL),
    (dict(v=C.CmQrows(0x300000, 0, 513, 128)), C.CM_EINVAL),
    (dict(v=C.CmQrows(0x300000, 0, 512, 4)), C.CM_EINVAL),
    (dict(v=C.CmQrows(0x300000, -8, 512, 128)), C.CM_EINVAL),
])
def test_writes_refused(lib, over, code):
    f = dict(first=0, layers=1, dtype=C.CM_BF16, k=C.CmQrows(0x300000, 0, 512, 128),
             v=C.CmQrows(0x310000, 0, 512, 128), tokens=3, slots=0x900000)
    f.update(over)
    k = ctypes.byref(f["k"]) if f["k"] is not None else None
    v = ctypes.byref(f["v"]) if f["v"] is not None else None
    st = lib.cm_qcache_write(ctypes.byref(cache()), f["first"], f["layers"], f["dtype"], k, v,
                             f["tokens"], f["slots"], None)
    assert st == code and lib.cm_last_error().decode() != ""


def test_writes_of_nothing(lib):
    r = C.CmQrows(None, 0, 0, 0)
    for layers, tokens in ((0, 5), (2, 0)):
        assert lib.cm_qcache_write(ctypes.byref(cache()), 0, layers, C.CM_F32, ctypes.byref(r),
                                   ctypes.byref(r), tokens, None, None) == C.CM_OK


@pytest.mark.parametrize("over,code", [
    (dict(pages=0), C.CM_EINVAL), (dict(block=20), C.CM_ESHAPE), (dict(n=0), C.CM_EINVAL),
    (dict(n=C.CM_QCACHE_MAX_REQUESTS + 1), C.CM_EINVAL), (dict(held=None), C.CM_EINVAL),
    (dict(new=None), C.CM_EINVAL), (dict(new=0x20002), C.CM_EINVAL), (dict(n_free=-1), C.CM_EINVAL),
    (dict(n_free=2 ** 31), C.CM_EINVAL), (dict(free=None), C.CM_EINVAL), (dict(table=None), C.CM_EINVAL),
    (dict(width=0), C.CM_EINVAL), (dict(width=2 ** 27), C.CM_EINVAL), (dict(tokens=-1), C.CM_EINVAL),
    (dict(tokens=2 ** 31), C.CM_EINVAL), (dict(slots=None), C.CM_EINVAL), (dict(slots=0x60004), C.CM_EINVAL),
    (dict(rows=None), C.CM_EINVAL), (dict(lens=0x80001), C.CM_EINVAL), (dict(info=None), C.CM_EINVAL),
    (dict(info=0x90004), C.CM_EINVAL),
])
def test_tables_refused(lib, over, code):
    f = dict(pages=10, block=16, n=2, held=0x10000, new=0x20000, free=0x30000, n_free=4, table=0x40000,
             width=8, tokens=3, slots=0x60000, rows=0x70000, lens=0x80000, info=0x90000)
    f.update(over)
    assert lib.cm_qcache_tables(f["pages"], f["block"], f["n"], f["held"], f["new"], f["free"],
                                f["n_free"], f["table"], f["width"], f["tokens"], f["slots"], f["rows"],
                                f["lens"], f["info"], None) == code
    assert lib.cm_last_error().decode() != ""


def test_binding_refusals():
    """What the Python layer refuses by type and shape (no GPU is touched)."""
    import torch
    codes = torch.zeros((1, 2, 3, 2, 16, 64), dtype=torch.uint8)
    scales = torch.zeros((1, 2, 3, 2))
    for c, s, kind in ((codes[0], scales, ValueError), (codes.float(), scales, TypeError),
                       (codes, scales.double(), TypeError), (codes, scales[..., :1], ValueError),
                       (codes.transpose(2, 3), scales, ValueError),
                       (codes[:, :1], scales, ValueError), (codes, scales, ValueError)):
        with pytest.raises(kind):
            cm.QCache(c, s)


CHILD = """
import ctypes, sys
sys.path.insert(0, sys.argv[3])
import paper_2607_01308_amd._cabi as C
C.LIB_PATH = sys.argv[1]
assert C.lib()._name == sys.argv[1]
assert hasattr(ctypes.CDLL(None), "__asan_init"), "sanitizer runtime not loaded"
import pytest
sys.exit(pytest.main(["-q", "-p", "no:cacheprovider", sys.argv[2], "-k", "not sanitizers"]))
"""


@pytest.mark.skipif(bool(os.environ.get("LD_PRELOAD")),
                    reason="this process already preloads a library; the sanitizer runtime "
                           "must come first")
def test_refusals_under_sanitizers():
    lib = build.SAN_LIB
    sources = [os.path.join(build.CSRC, f) for f in ("api.cpp", "internal.h", "qcache.h")]
    if not os.path.exists(lib) or os.path.getmtime(lib) < max(os.path.getmtime(s) for s in sources):
        build.build_sanitized()
    env = dict(os.environ, LD_PRELOAD=build.sanitizer_runtime(),
               ASAN_OPTIONS="detect_leaks=0:halt_on_error=1:abort_on_error=0",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = subprocess.run([sys.executable, "-c", CHILD, lib, os.path.abspath(__file__), ROOT], env=env,
                       capture_output=True, text=True, timeout=600, cwd=ROOT)
    out = r.stdout[-4000:] + r.stderr[-4000:]
    assert r.returncode == 0, out
    assert "AddressSanitizer" not in r.stderr and "runtime error" not in r.stderr, out
    assert " passed" in r.stdout, out


@pytest.mark.parametrize("H,d,G,dtype", [(8, 128, 4, C.CM_BF16), (8, 256, 4, C.CM_BF16), (1, 128, 8, C.CM_F32),
                                         (64, 64, 1, C.CM_BF16), (300, 128, 1, C.CM_F32)])
def test_workspace_does_not_grow_with_the_rows(lib, H, d, G, dtype):
    """Partial results are of cut tiles alone, whose items are as many as the GPU runs together, not as
    many as there are rows."""
    def need(n, rows):
        return size(lib, cache(H=H, d=d, L=1), step(n=n, q_heads=H * G, dtype=dtype, n_rows=rows,
                                                    rows_dev=0x111000, max_rows=rows))

    sizes = []
    for n, rows in ((1, 1), (3, 60), (1, 4096), (1, 16384), (1, 250000), (1024, 200), (1024, 200000)):
        st, bytes = need(n, rows)
        assert st == C.CM_OK
        sizes.append(bytes)
    assert sizes[3] == sizes[4] == sizes[6] and max(sizes) == sizes[3]
    assert max(sizes) < 160 << 20
