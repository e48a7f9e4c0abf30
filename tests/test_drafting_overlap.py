"""Memory that a verification writes and that something else of the same call lies in: refused on the host.
Several workgroups take a request, so what one writes another may still have to read."""

import ctypes

import pytest

from paper_2607_01308_amd import _cabi as C

ref = ctypes.byref
N, ROWS, V = 2, 5, 100
# the arrays of a call, with the bytes that each takes
BYTES = dict(probs_dev=((ROWS - 1) * 128 + V) * 4, draft_probs_dev=((ROWS - 1) * 104 + V) * 4, drafts_dev=8 * ROWS,
             parents_dev=4 * ROWS, rows_dev=4 * (N + 1), accept_dev=4 * ROWS, sample_dev=4 * N, path_dev=4 * ROWS,
             counts_dev=4 * N, tokens_dev=8 * N)
WRITTEN = ("path_dev", "counts_dev", "tokens_dev")
AT = {name: 0x100000 * (i + 1) for i, name in enumerate(BYTES)}


def call(**over):
    f = dict(AT, n=N, dtype=C.CM_F32, n_rows=ROWS, vocabulary=V, probs_stride=128, draft_probs_stride=104)
    f.update(over)
    status = C.lib().cm_verify_drafts(ref(C.CmDrafts(**f)), None)
    return status, C.lib().cm_last_error().decode()


@pytest.mark.parametrize("written", WRITTEN)
@pytest.mark.parametrize("other", [name for name in BYTES])
def test_outputs_over_what_else_there_is(written, other):
    if written == other:
        return
    # the output over the first and the last bytes of the other one, and begun before it
    unit = 8 if "tokens_dev" in (written, other) or other == "drafts_dev" else 4
    for at in (AT[other], AT[other] + (BYTES[other] - 1) // unit * unit, AT[other] - BYTES[written] + unit):
        status, message = call(**{written: at})
        assert status == C.CM_EINVAL
        assert "overlaps" in message and written in message and other in message


def test_workspace_over_what_else_there_is():
    need = ctypes.c_size_t(0)
    wide = dict(vocabulary=200_000, probs_stride=200_000, draft_probs_stride=200_000,
                **{name: 0x10000000 * (i + 1) for i, name in enumerate(BYTES)})
    step = C.CmDrafts(n=N, dtype=C.CM_F32, **wide)
    assert C.lib().cm_verify_drafts_size(ref(step), ref(need)) == C.CM_OK
    if need.value == 0:
        pytest.skip("one workgroup for each request on this machine")
    for name in BYTES:
        status, message = call(**wide, workspace=wide[name], workspace_bytes=need.value)
        assert status == C.CM_EINVAL and "workspace" in message and name in message


def test_strides_that_no_memory_holds():
    """Extents beyond 64 bits are not taken for small ones."""
    status, message = call(n_rows=2 ** 31 - 1, probs_stride=2 ** 40, draft_probs_stride=2 ** 40)
    assert status == C.CM_EINVAL and "overlaps" in message
