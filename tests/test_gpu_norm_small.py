"""norm_rotate of rows whose squares leave the range of fp32 downwards, with an eps that does not cover
them: as far off as any other row (tests/draft_ref.py)."""

import pytest
import torch

import paper_2607_01308_amd as cm
from test_gpu_norm_rotate import check, values

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
POWERS = [0, -20, -47, -48, -49, -60, -64, -70, -80, -100, -120, -126]


@pytest.mark.parametrize("eps", [0.0, 2.0 ** -149, 2.0 ** -126, 2.0 ** -100, 2.0 ** -68, 2.0 ** -66, 2.0 ** -64,
                                 2.0 ** -20])
@pytest.mark.parametrize("dtype,d,style", [(F32, 64, "half"), (F32, 128, "interleaved"), (F32, 256, "half"),
                                           (BF16, 64, "interleaved"), (BF16, 128, "half"), (BF16, 256, "half")])
def test_small_rows(dtype, d, style, eps):
    """Rows of one size, and of both, side by side in a wave."""
    T = len(POWERS)
    scale = torch.exp2(torch.tensor(POWERS, dtype=torch.float64, device="cuda"))
    x = values(T, 5, d, seed=d, dtype=F32).double()
    x[:, :2] *= scale[:, None, None]
    x[:, 2] *= scale.flip(0)[:, None]
    x[:, 3, ::2] *= scale[:, None]
    x[:, 4] = 0
    x[:, 4, 3] = scale
    x = x.to(dtype)
    w = values(d, seed=2, dtype=dtype)
    positions = [3 * i for i in range(T)]
    pos = torch.tensor(positions, dtype=torch.int32, device="cuda")
    got, _ = cm.norm_rotate(x, None, pos, 1e4, style=style, q_weight=w, eps=eps)
    check(x, got, positions, 1e4, style, w, eps)


def test_zeros_with_and_without_eps():
    """Rows of zeros are zeros for any eps above 0, and 0 / 0 without."""
    x = torch.zeros((2, 3, 64), device="cuda")
    pos = torch.zeros(2, dtype=torch.int32, device="cuda")
    w = torch.ones(64, device="cuda")
    for eps in (2.0 ** -149, 2.0 ** -100, 1e-6):
        assert bool((cm.norm_rotate(x, None, pos, 1e4, q_weight=w, eps=eps)[0] == 0).all())
    assert bool(torch.isnan(cm.norm_rotate(x, None, pos, 1e4, q_weight=w, eps=0.0)[0]).all())
