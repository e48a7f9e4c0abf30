"""Verification shared by several workgroups that do not wait for one another, or not long: what has not come is
summed by the request's first workgroup, with the same results, and the workspace ends up zero. The waits of the
library are set from here; with 0 nobody looks, so every helper ends at once, or every helper's sums are
missing."""

import ctypes

import numpy as np
import pytest
import torch

from paper_2607_01308_amd import _cabi as C
from test_gpu_verify import case

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture
def waits():
    """Sets (for a pass, for the helpers' sums) in ticks of 10 ns; as they were, afterwards."""
    words = (ctypes.c_uint64 * 2).in_dll(C.lib(), "_ZN2cm12verify_waitsE")
    were = list(words)
    assert min(were) > 0

    def set_to(helper, sums):
        words[0], words[1] = [w if x is None else x for x, w in zip((helper, sums), were)]

    yield set_to
    set_to(None, None)


@pytest.mark.parametrize("sampled", [True, False])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,V", [(1, 200_003), (3, 100_001), (30, 40_000), (1, 600_000)])
def test_helpers_that_are_not_waited_for(waits, n, V, dtype, sampled):
    c = case([int(x) for x in np.random.default_rng(V).integers(6, 14, size=n)], V, 4, dtype, sampled, seed=V + 1)
    if not sampled:
        c["probs"][:, :4] *= V / 8
    i32 = dict(dtype=torch.int32, device="cuda")
    T, q = len(c["parents"]), c["draft_probs"]
    parents, rows = torch.tensor(c["parents"], **i32), torch.tensor(c["rows"], **i32)
    u, s = torch.tensor(c["accept"], device="cuda"), torch.tensor(c["sample"], device="cuda")
    path, counts, tokens = torch.empty(T, **i32), torch.empty(n, **i32), torch.empty(n, dtype=torch.int64, device="cuda")
    step = C.CmDrafts(n, C.CM_BF16 if dtype is BF16 else C.CM_F32, T, V, c["probs"].data_ptr(), V,
                      None if q is None else q.data_ptr(), V, c["drafts"].data_ptr(), parents.data_ptr(),
                      rows.data_ptr(), u.data_ptr(), s.data_ptr(), path.data_ptr(), counts.data_ptr(),
                      tokens.data_ptr())
    stream = torch.cuda.current_stream().cuda_stream

    def run():
        for x in (path, counts, tokens):
            x.fill_(-7)
        assert C.lib().cm_verify_drafts(ctypes.byref(step), stream) == C.CM_OK
        return path.tolist(), counts.tolist(), tokens.tolist()

    want = run()                                             # one workgroup for each request
    need = ctypes.c_size_t(0)
    assert C.lib().cm_verify_drafts_size(ctypes.byref(step), ctypes.byref(need)) == C.CM_OK and need.value > 0
    ws = torch.zeros(need.value, dtype=torch.uint8, device="cuda")
    step.workspace, step.workspace_bytes = ws.data_ptr(), need.value
    # nobody looks; no helper; no sums; both again in turn with the waits of the library; and waits that end in
    # the middle of a pass
    for helper, sums in ((0, 0), (0, None), (None, 0), (None, None), (0, 0), (None, None), (None, 0), (None, 30),
                         (200, None), (20, 20), (None, 100), (None, None)):
        waits(helper, sums)
        assert run() == want, f"waits of {helper}, {sums}"
        assert not bool(ws.any()), f"waits of {helper}, {sums}"
