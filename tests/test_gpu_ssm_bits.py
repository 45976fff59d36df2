"""The state space mixer's sums where their terms cancel (needs an MI355X): what
is left of them has to be good to the output's type, by itself.

Two states of a channel are alike and C takes them with opposite signs, all but
2^-9 of the term.  Sums as good as fp32's (six roundings of 2^-24 on the way to C
and to the state: 4e-7, 1e-6 allowed) then leave 2^9 1e-6 of the output, beside
its own rounding (2^-24, 2^-8, 2^-11)."""
import numpy as np
import pytest
import torch

from gpu_harness import dev, lcsm_mod
from oracle import ssm as oracle

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}


def raw_of(u, guess):
    """v with silu(v) = u (u > -0.27), in fp64."""
    v = guess
    for _ in range(60):
        s = 1 / (1 + np.exp(-v))
        v -= (v * s - u) / (s * (1 + v * (1 - s)))
    return v


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T", [40, 190, 300, 1500])
@pytest.mark.parametrize("N", [2, 50, 100, 200])
def test_outputs_of_terms_that_cancel(N, T, dtype):
    H, P = 2, 33
    D = H * P
    C = D + 2 * N
    r = np.random.default_rng(N + T)
    xbc = np.zeros((T, C), np.float32)
    xbc[:, :D] = r.uniform(16.0, 64.0, (T, D))  # (no output is below what fp16 holds in full)
    at = sorted(r.choice(N, 2, replace=False).tolist())
    conv_b = np.zeros(C, np.float32)
    xbc[:, D + at[0]] = xbc[:, D + at[1]] = 1.0
    for k, u in ((at[0], 0.25 * (1 + 2.0 ** -9)), (at[1], -0.25)):
        xbc[:, D + N + k] = 0.5 if u > 0 else -0.75
        conv_b[D + N + k] = raw_of(u, 0.5 if u > 0 else -0.6) - xbc[0, D + N + k]
    conv_w, A = np.ones((C, 1), np.float32), np.full(H, -0.01, np.float32)
    rows = torch.from_numpy(xbc).to(TYPES[dtype])
    dt = torch.from_numpy(r.uniform(-2, 0, (T, H)).astype(np.float32)).to(TYPES[dtype])
    up = lambda v: torch.from_numpy(v[None]).to(dev())  # noqa: E731
    ctx = lcsm_mod().Ssm(up(conv_w), up(A), slots=1, groups=1, states=N, conv_bias=up(conv_b), dtype=TYPES[dtype], max_tokens=T)
    got = ctx.prompt(0, rows.to(dev()), dt.to(dev())).double().cpu().numpy()
    want, _, _ = oracle.scan(rows.double().numpy(), dt.double().numpy(), None, conv_w, conv_b, A, np.zeros(H), np.zeros(H), 1, N,
                             np.zeros((H, P, N)), np.zeros((0, C)))
    assert (want > 0).all()
    err = (np.abs(got - want) / want).max()
    assert err <= ULP[dtype] + 2.0 ** 9 * 1e-6, err
