"""The quantizer of the 4-bit products (lcsm_q4_quantize) where weights are not
what they should be, and its bounds (needs an MI355X)."""
import numpy as np
import pytest
import torch

from gpu_harness import dev, lcsm_mod

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.mark.parametrize("sdtype", TYPES)
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("K,group", [(256, 64), (129, 128), (700, 256)])
def test_weights_that_are_not_finite_are_not_made_finite(K, group, value, sdtype):
    """One such weight: its group's scale and every output of its row show it, whatever
    the inputs; all else is as without it."""
    r = np.random.default_rng(K)
    w = torch.from_numpy(r.standard_normal((1, 6, K)).astype(np.float32)).to(dev())
    codes0, scales0 = lcsm_mod().Q4.quantize(w, group, TYPES[sdtype])
    for at in (0, K - 1, K // 2):
        bad = w.clone()
        bad[0, 4, at] = value
        codes, scales = lcsm_mod().Q4.quantize(bad, group, TYPES[sdtype])
        mine = torch.zeros_like(scales, dtype=torch.bool)
        mine[0, 4, at // group] = True
        assert not torch.isfinite(scales[mine]).any() and torch.equal(scales[~mine], scales0[~mine])
        rest = torch.tensor([0, 1, 2, 3, 5], device=dev())
        assert torch.equal(codes[0, rest], codes0[0, rest])
        q = lcsm_mod().Q4(codes, scales, K, group)
        x = torch.from_numpy(r.standard_normal((3, K)).astype(np.float32)).to(dev())
        x[2] = 0.0
        for dtype in TYPES.values():
            y = q.matvec(0, x.to(dtype))
            assert not torch.isfinite(y[:, 4]).any() and torch.isfinite(y[:, rest]).all()


def test_scales_beyond_their_type():
    w = torch.full((2, 32), 1e6, device=dev())
    w[1] = 1e5
    codes, scales = lcsm_mod().Q4.quantize(w, 32, torch.float16)
    assert not torch.isfinite(scales[0]).any() and torch.isfinite(scales[1]).all()
    assert bool((codes[0] == 0x88).all()) and bool((codes[1] == 0xFF).all())


def test_more_groups_than_one_grid_has_waves():
    """2^26 + 3 groups of 32, what lies past the first rows different from them."""
    rows = 2 ** 26 + 3
    w = torch.zeros((rows, 32), device=dev())
    w[:2, 0], w[-3:, 31], w[2 ** 25, 5] = 7.0, -14.0, 3.5
    codes, scales = lcsm_mod().Q4.quantize(w, 32, torch.float32)
    want = torch.zeros((rows, 1), device=dev())
    want[:2], want[-3:], want[2 ** 25] = 1.0, 2.0, 0.5
    assert torch.equal(scales, want)
    got = codes[[0, 1, 2, 2 ** 25, rows - 4, rows - 3, rows - 1]].cpu()
    plain = torch.full((16,), 0x88, dtype=torch.uint8)
    first, last, middle = plain.clone(), plain.clone(), plain.clone()
    first[0], last[15], middle[2] = 0x8F, 0x18, 0xF8
    assert torch.equal(got, torch.stack([first, first, plain, middle, plain, last, last]))
