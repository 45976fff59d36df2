"""Prompts that are cut into segments, with up to 64 states, again and again
(needs an MI355X): the same bits every time and the oracle's values.  Between the
calls the LDS of every compute unit is left with other values, so that factors
read before they are there would not be the last call's.  Tolerances are those
of test_gpu_ssm.py, and derived there."""
import pytest
import torch

from test_gpu_ssm import TYPES, Layer, ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(3, 64, 16, 1, 4), (4, 32, 64, 2, 4), (5, 33, 64, 1, 3), (3, 41, 23, 3, 2)], ids=str)
def test_cut_prompts_repeat(shape, dtype):
    lay = Layer(*shape, dtype=dtype, slots=2, max_tokens=2600, seed=31 + sum(shape), decay=4.0)
    other = Layer(8, 64, 64, 1, 4, dtype=dtype, slots=1, max_tokens=4096, seed=32, decay=300.0)
    x, xr = lay.inputs(2600)
    offs = [0, 1900, 2600]
    fill, _ = other.inputs(4096)
    got = []
    for _ in range(4):
        y = lay.ctx.prompt(0, x[0], x[1], z=x[2], offsets=ints(offs), src=ints([-1, -1]), dst=ints([0, 1]))
        got.append((y.clone(), lay.ctx.state(0).clone()))
        other.ctx.prompt(0, fill[0], fill[1], z=fill[2])
    torch.cuda.synchronize()
    lay.check(got[0][0], lay.want(xr, offs, src=[-1, -1]))
    for y, s in got[1:]:
        assert torch.equal(y, got[0][0]) and torch.equal(s, got[0][1])
