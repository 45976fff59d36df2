"""Every form of the 4-bit product that the rule on sizes can choose, against the
fp64 oracle (needs an MI355X, but for the check that the cases reach every form).

Tolerances: y is rounded once to its type (2^-24, 2^-8, 2^-11 of itself), and the
sums before that are fp32's over at most 2100 exact products: 130 roundings in a
row (one for the products of 32 inputs, one for their scale), each of 2^-24 of what
is summed up to there, which in a random order leave sqrt(130) 2^-24 < 2^-20 of the
terms' magnitudes."""
import itertools

import numpy as np
import pytest
import torch

from gpu_harness import dev, lcsm_mod, say
from oracle import ssm as oracle
from q4_rule import form

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}

# rows, outputs, inputs: tails in all three
SIZES = [(1, 8209, 1300), (16, 8209, 333), (3, 8209, 2100), (5, 333, 1300), (20, 8185, 333), (31, 8185, 1300), (31, 4090, 1300),
         (18, 100, 1300), (130, 4112, 333), (513, 4105, 1300), (61, 4081, 1300), (40, 1543, 333), (100, 77, 1300)]
GROUPS = [32, 64, 128, 384]


def test_the_cases_reach_every_form():
    sweep = itertools.product([1, 2, 16, 17, 32, 33, 64, 65, 200, 513, 4096], [1, 100, 2000, 4081, 4112, 8176, 8177, 8512, 16384, 65000],
                              [1, 128, 773, 2048, 2049, 8192, 16384], [32, 64, 128], [2, 4])
    want = {form(R, N, K, g, size) for R, N, K, g, size in sweep}
    have = {form(R, N, K, g, size) for (R, N, K), g, size in itertools.product(SIZES, GROUPS, [2, 4])}
    assert have == want and len(want) >= 30


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("group", GROUPS)
@pytest.mark.parametrize("R,N,K", SIZES)
def test_forms(R, N, K, group, dtype):
    r = np.random.default_rng(R + N + K + group)
    ng = -(-K // group)
    zeros = r.integers(0, 256, (1, N, ng), dtype=np.uint8) if (R + group) % 3 else None
    bias = r.standard_normal((1, N)).astype(np.float32) if R % 2 else None
    codes = r.integers(0, 256, (1, N, (K + 1) // 2), dtype=np.uint8)
    scales = torch.from_numpy(((0.5 + r.random((1, N, ng))) / np.sqrt(K)).astype(np.float32)).to(TYPES[dtype])
    up = lambda v: None if v is None else torch.from_numpy(v).to(dev())  # noqa: E731
    ctx = lcsm_mod().Q4(up(codes), scales.to(dev()), K, group, zeros=up(zeros), bias=up(bias))
    x = torch.from_numpy(r.standard_normal((R, K + 3)).astype(np.float32)).to(TYPES[dtype])
    wide = torch.full((R, N + 5), 7.0, dtype=TYPES[dtype], device=dev())
    say(f"[q4] {form(R, N, K, group, TYPES[dtype].itemsize)}: {R} rows x {N} x {K} group {group} {dtype}")
    y = ctx.matvec(0, x.to(dev())[:, 1:1 + K], wide[:, 2:2 + N])
    torch.cuda.synchronize()
    w = oracle.q4_weights(codes[0].astype(np.int64), scales[0].double().numpy(), None if zeros is None else zeros[0], K, group)
    xs = x[:, 1:1 + K].double().numpy()
    want, terms = xs @ w.T, np.abs(xs) @ np.abs(w.T)
    if bias is not None:
        want, terms = want + bias[0], terms + np.abs(bias[0])
    err = np.abs(y.double().cpu().numpy() - want)
    assert (err <= ULP[dtype] * np.abs(want) + 2.0 ** -20 * terms).all(), (err / terms).max()
    assert bool((wide[:, :2] == 7.0).all()) and bool((wide[:, 2 + N:] == 7.0).all())
