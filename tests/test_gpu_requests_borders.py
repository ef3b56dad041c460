"""Pages and sampling rules on the GPU at the borders of what the calls take."""
import numpy as np
import pytest
import torch

import workloads as W
from oracle import rules_probs_ref
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


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,V", [(4, 700), (130, 700)])
def test_tokens_that_were_never_there_have_no_penalty(dtype, rows, V):
    """Penalties that are infinite, or no numbers, fall on what a request has had and on nothing else."""
    inf, nan = float("inf"), float("nan")
    c = Rules(52, dtype, [1] * rows, V, 0, 0, temps=(1.0,), path=False)
    c.rules[:, 1:] = np.resize([[1, 0, inf], [1, inf, 0], [1, 0, nan], [1, 0.5, 0.25]], (rows, 3))
    c.counts[:] = 0
    c.counts[:, 20], c.counts[:, 21] = 3, 1 << 30
    c.biases = [[(21, 1.5), (30, 2.0), (31, -1.0)] for _ in range(rows)]
    z, p = c.run()
    z, x = W.widen(z), W.widen(c.logits)
    half = 2.0 ** -23 if dtype == "f32" else 2.0 ** -8  # one rounding of the sum, and one of the type
    for token, more in ((21, 1.5), (30, 2.0), (31, -1.0), (40, 0.0)):
        assert (np.abs(z[:, token] - x[:, token] - more) <= half * (np.abs(x[:, token]) + 2)).all(), token
    for t in range(rows):
        assert z[t, 20] == -inf if t % 4 < 3 else np.abs(z[t, 20] - (x[t, 20] - 1.25)) <= half * 10
    want = rules_probs_ref(z, np.arange(rows + 1), c.rules)
    assert dtype != "f32" or (np.abs(W.widen(p) - want) <= 1e-5 * want + 1e-37).all()
