"""Linear attention at the ends of its ranges (needs an MI355X): batches of as many
sequences as leave a call uncut, of very unequal lengths, and states that grow.

Tolerances are those of tests/test_gpu_lin.py.  A state that grows adds to an
exponent of up to E bits two roundings of 2^-24 of it, E 1.4 2^-24 of the factor:
1e-5 for the 120 bits here, within the 2e-5 of the magnitudes' sums."""
import numpy as np
import pytest
import torch

from gpu_harness import say
from test_gpu_lin import TYPES, Layer, ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [7, 8, 9, 20])
@pytest.mark.parametrize("where", ["first", "last"])
def test_one_long_sequence_among_short_ones(n, where, dtype):
    """64 states of one block of values: calls of fewer than eight sequences are cut into segments, others are not."""
    lay = Layer(64, 64, 24, 32, dtype=dtype, slots=n, max_tokens=1000, seed=n)
    lens = lay.rng.integers(0, 5, n)
    lens[0 if where == "first" else -1] = 700
    offs = [0] + np.cumsum(lens).tolist()
    lay.set_states()
    x = lay.inputs(offs[-1])
    say(f"[lin] {n} sequences, one of 700 {where} {dtype}")
    lay.check(lay.ctx.prompt(0, *x, offsets=ints(offs)), lay.want(x, offs))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("g,lens", [(1.3, [1, 5, 33]), (0.1, [1, 700, 64, 65])], ids=str)
def test_states_that_grow(g, lens, dtype):
    """Where e^(g n) of a call's tokens comes near 2^127: 2^120 of a chunk's 64, of which 33 are there, and 2^101 of 704 of a
    cut call."""
    lay = Layer(2, 1, 16, 20, dtype=dtype, slots=4, max_tokens=900, seed=14, decay=g)
    lay.set_states()
    offs = [0] + np.cumsum(lens).tolist()
    x = lay.inputs(offs[-1])
    say(f"[lin] growth {g} {lens} {dtype}")
    y = lay.ctx.prompt(0, *x, offsets=ints(offs))
    lay.check(y, lay.want(x, offs))
    assert torch.isfinite(y).all()
