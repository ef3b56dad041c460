"""Pages and sampling rules on the GPU at the borders of what the calls take."""
import numpy as np
import pytest
import torch

import workloads as W
from test_gpu_requests import Rules

pytestmark = pytest.mark.gpu
i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,V", [(5, 600), (5, 40000), (132, 3001), (132, 600)])
def test_no_temperature_is_too_high_for_infinities(dtype, rows, V):
    """At an infinite temperature finite values share a row equally, and infinite ones the whole; at very high ones a row whose values
    span more than float32 has the weights of the formula."""
    inf = float("inf")
    c = Rules(51, dtype, [1] * rows, V, 0, 2, temps=(inf, inf, 3.0e38, inf, 1.0e38), path=False)
    c.rules[:, 1:] = [1, 0, 0]
    c.counts[:] = 0
    c.mask[:] = 0xffffffff
    c.mask[1, ::2] = 0
    c.mask_row = np.resize([0, 0, 0, 1, 0], rows)
    c.logits[0::5, 7] = c.logits[0::5, V - 2] = inf     # infinities share the whole
    c.logits[0::5, 9] = -inf
    c.logits[1::5, 5] = 3.0e38                          # the largest less the least is beyond float32
    c.logits[1::5, V - 1] = -3.0e38
    c.logits[2::5, 3], c.logits[2::5, V - 1] = 3.0e38, -3.0e38
    c.logits[4::5, 3], c.logits[4::5, V - 1] = 3.0e38, -3.0e38
    c.biases = [[(11, inf)] if b % 5 == 3 else [] for b in range(rows)]
    z, p = c.run()
    z = W.widen(z)
    p = W.widen(p)
    assert np.isfinite(p).all()
    for t in range(rows):
        want = np.zeros(V)
        T = float(c.rules[t, 0])
        top, left = z[t].max(), z[t] > -inf
        if top == inf:
            want[z[t] == inf] = 1
        elif T == inf:
            want[left] = 1
        else:
            want[left] = np.exp((z[t][left] - top) / T)
        want /= want.sum()
        # (z - max) / T of at most 6, in float32 with a factor of 2^-126 and less: 2^-20; a sum of V numbers
        assert (np.abs(p[t] - want) <= 1e-4 * want + 1e-37).all(), (t, np.abs(p[t] - want).max())
