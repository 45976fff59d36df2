"""Norms of more rows than one axis of a launch has workgroups for (needs an
MI355X); tolerances are those of test_gpu_norm.py, and derived there."""
import numpy as np
import pytest
import torch

from gpu_harness import dev, lcsm_mod
from oracle import ssm as oracle
from test_gpu_norm import SUMS, ULP, close

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("R,D,groups", [(2 ** 26 + 5, 1, 1), (2 ** 26 + 5, 2, 2), (2 ** 20 * 4 + 1, 8, 1), (2 ** 20 + 3, 600, 6)])
def test_many_rows(R, D, groups):
    """Rows that repeat with a period that no launch shape has."""
    period = 61
    r = np.random.default_rng(D)
    o, res = (r.standard_normal((period, D)).astype(np.float32) for _ in range(2))
    many = lambda v: (torch.from_numpy(v).to(dev()).bfloat16().repeat(R // period + 1, 1)[:R]).contiguous()  # noqa: E731
    a, b = many(o), many(res)
    ctx = lcsm_mod().Norm(D, post="rms", pre="rms", groups=groups, eps=1e-2)
    got = ctx.block(0, a, b)
    torch.cuda.synchronize()
    want = oracle.block_norm(a[:period].double().cpu().numpy(), None, b[:period].double().cpu().numpy(), "rms", "rms", "none", groups,
                             1.0, 1e-2, None, None, None, None, None)
    for g, w in zip(got, want):
        close(g[:period], w, SUMS + ULP["bf16"])
        whole = R // period * period
        assert bool((g[:whole].view(-1, period, D) == g[:period]).all()) and torch.equal(g[whole:], g[:R - whole])
