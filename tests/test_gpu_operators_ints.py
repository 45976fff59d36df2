"""Sizes and layers that a C int does not hold are refused by the binding of the
gated layer's operators, not taken modulo 2^32 (needs an MI355X)."""
import pytest
import torch

from gpu_harness import dev, lcsm_mod

pytestmark = pytest.mark.gpu
FAR = 2 ** 32


def test_layers_beyond_an_int():
    lcsm = lcsm_mod()
    x = torch.zeros((2, 32), device=dev())
    q = lcsm.Q4(*lcsm.Q4.quantize(torch.ones((1, 8, 32), device=dev()), 32), 32, 32)
    norm = lcsm.Norm(32, dtype=torch.float32)
    ssm = lcsm.Ssm(torch.ones((1, 32, 1), device=dev()), -torch.ones((1, 4), device=dev()), slots=2, groups=2, states=4,
                   dtype=torch.float32, max_tokens=8)
    calls = [lambda m: q.matvec(m, x), lambda m: norm.block(m, x, x), lambda m: ssm.step(m, x, x[:, :4]),
             lambda m: ssm.prompt(m, x, x[:, :4])]
    for call in calls:
        call(0)
        for layer in (FAR, FAR - 1, -FAR, 1, -1):
            with pytest.raises(lcsm.LcsmError) as e:
                call(layer)
            assert e.value.code == lcsm.LCSM_EINVAL


def test_sizes_beyond_an_int():
    lcsm = lcsm_mod()
    w, A = torch.ones((1, 32, 1), device=dev()), -torch.ones((1, 4), device=dev())
    good = dict(slots=2, groups=2, states=4, max_tokens=8)
    for k, v in good.items():
        with pytest.raises(ValueError):
            lcsm.Ssm(w, A, **{**good, k: v + FAR})
    for args in (dict(D=32 + FAR), dict(D=32, groups=1 + FAR), dict(D=32, layers=1 + FAR)):
        with pytest.raises(ValueError):
            lcsm.Norm(**args)
    codes, scales = lcsm.Q4.quantize(torch.ones((1, 8, 32), device=dev()), 32)
    for K, group in ((32 + FAR, 32), (32, 32 + FAR)):
        with pytest.raises(ValueError):
            lcsm.Q4(codes, scales, K, group)
    with pytest.raises(ValueError):
        lcsm.Q4.quantize(torch.ones((1, 8, 32), device=dev()), 32 + FAR)
