"""ServingCache.accept on the GPU: a path that is not as verify_drafts gives it is told by what accept
returns."""

import pytest
import torch

import paper_2607_01308_amd as cm

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("path,bad", [([0, 2, 4, -1, -1, 0, 1], False), ([0, 4, 2, -1, -1, 0, 1], True),
                                      ([0, 2, 5, -1, -1, 0, 1], True), ([0, 0, 1, -1, -1, 0, 1], True),
                                      ([0, -1, -1, -1, -1, 0, 1], True)])
def test_paths_that_are_not_ascending_are_told(path, bad):
    """Place 0's path, of which three nodes are to stay; place 1's is always right."""
    H, d, B = 2, 64, 16
    sc = cm.ServingCache(cm.QCache.empty(2, H, d, 12, B), 2, 100)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x = torch.randn((2, 40, H, d), generator=g, device="cuda")
    step = sc.extend([14, 5])
    sc.write(0, x[:, :19], x[:, :19], step)
    step = sc.draft([[-1, 0, 0, 1, 2], [-1, 0]])
    sc.write(0, x[:, 19:26], x[:, 19:26], step)
    codes = sc.cache.codes.view(torch.uint8).clone()
    kept = sc.accept(step, torch.tensor(path, dtype=torch.int32, device="cuda"), [3, 2])
    assert sc.lengths == [17, 7] == kept.lens.tolist() == sc._held.tolist()
    if bad:
        with pytest.raises(cm.CmError, match="path"):
            kept.check()
        assert torch.equal(sc.cache.codes.view(torch.uint8), codes)
    else:
        assert kept.check() is kept and kept.info.tolist() == [0, 0]
        assert not torch.equal(sc.cache.codes.view(torch.uint8), codes)
