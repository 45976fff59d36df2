"""A prompt call of so many sequences and heads that its workgroups are more than
one axis of a launch takes (needs an MI355X).  Tolerances are those of
test_gpu_ssm.py, and derived there."""
import numpy as np
import pytest
import torch

from gpu_harness import dev, lcsm_mod
from oracle import ssm as oracle
from test_gpu_ssm import SUMS, close

pytestmark = pytest.mark.gpu


def test_many_sequences_of_many_heads():
    """8201 slots of 64 heads x 4096, of which some sequences have a token or two."""
    H, P, N, n, T = 64, 4096, 1, 8201, 300
    D = H * P
    r = np.random.default_rng(1)
    w = r.standard_normal((D + 2, 1)).astype(np.float32)
    A, bias = -(1 + r.random(H)).astype(np.float32), r.standard_normal(D + 2).astype(np.float32)
    up = lambda v: torch.from_numpy(v[None]).to(dev())  # noqa: E731
    ctx = lcsm_mod().Ssm(up(w), up(A), slots=n, groups=1, states=N, conv_bias=up(bias), dtype=torch.float32, max_tokens=T)
    lens = np.zeros(n, np.int64)
    lens[[0, 1, 100, 4095, 4096, n - 2, n - 1]] = [70, 1, 64, 65, 2, 31, 67]
    assert lens.sum() == T
    offs = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    x, dt = torch.randn((T, D + 2), device=dev()), torch.randn((T, H), device=dev())
    y = ctx.prompt(0, x, dt, offsets=torch.from_numpy(offs).to(dev()))
    torch.cuda.synchronize()
    for i in np.flatnonzero(lens):
        rows = slice(offs[i], offs[i + 1])
        want, S, _ = oracle.scan(x[rows].double().cpu().numpy(), dt[rows].double().cpu().numpy(), None, w, bias, A, np.zeros(H),
                                 np.zeros(H), 1, N, np.zeros((H, P, N)), np.zeros((0, D + 2)))
        close(y[rows].cpu().numpy(), want, SUMS, f"sequence {i}")
        close(ctx.state(0)[i].cpu().numpy(), S, SUMS, f"state {i}")
    assert float(ctx.state(0)[5:99].abs().max()) == 0.0
