"""Many rows against 8-bit weights without a bias (needs an MI355X): pieces of each
size, more of them than there are workgroups and in several columns, so that a
workgroup goes from one piece to the next.  Every column and three rows of every 64
are compared with the oracle, by the bounds of tests/test_gpu_q8.py."""
import numpy as np
import pytest
import torch

from gpu_harness import dev, say
from test_gpu_q8 import TYPES, Matrix

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("K", [70, 300])
# pieces of 256 x 256 (512 on 256 workgroups), 128 x 128 (588 on 512), 128 x 64 (576 on 512), 64 x 64 (544 on 512), each with whole
# pieces only, then with rows and outputs that end inside one
@pytest.mark.parametrize("R,N", [(8192, 4096), (2688, 3584), (2304, 2048), (1088, 2048), (8150, 4112), (2650, 3600), (2290, 2064),
                                 (1080, 2064)])
def test_workgroups_of_several_pieces(R, N, K, dtype):
    m = Matrix(N, K, R, bias=False, seed=R + K)
    x = m.rows(R, dtype)
    # outputs into a wider tensor, aligned to 16 bytes
    wide = torch.full((R, N + 16), 7.0, dtype=TYPES[dtype], device=dev())
    say(f"[q8] pieces {R} x {K} -> {N} {dtype}")
    y = m.ctx.matmul(0, x, y=wide[:, 8:8 + N])
    torch.cuda.synchronize()
    assert bool((wide[:, :8] == 7).all()) and bool((wide[:, 8 + N:] == 7).all())
    some = (np.arange(0, R, 64)[:, None] + m.rng.integers(0, 64, (len(range(0, R, 64)), 3))).reshape(-1)
    some = torch.from_numpy(np.unique(np.append(some[some < R], [0, R - 1]))).to(dev())
    m.check(y[some], x[some], dtype)
    assert torch.equal(m.ctx.matmul(0, x), y)
