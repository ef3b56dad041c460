"""Attention over the 4-bit cache where scores are so large that a unit in their last place is more than an exponent: the largest score's keys
share the weight, and the log-sum-exp is that score.  One element of a query is not zero, so that scores are single products and ties are ties."""
import numpy as np
import pytest
import torch

import workloads as W
from kv4 import mixed_case
from oracle import kv4_values_ref
from test_gpu_kv4 import _attend, hb, step  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,Hq,D,nodes", [("bf16", 4, 128, 1), ("bf16", 14, 128, 4), ("bf16", 8, 64, 2), ("bf16", 14, 128, 40), ("bf16", 8, 64, 40),
                                              ("f32", 6, 128, 3), ("f32", 4, 64, 20), ("f32", 4, 96, 3)])
@pytest.mark.parametrize("sign", [1, -1])
def test_scores_of_any_size(hb, step, dtype, Hq, D, nodes, sign):
    """sign -1: every score is far below zero."""
    rng = np.random.default_rng(91)
    for e in (8, 20, 25, 28, 30, 32, 36, 60, 100):
        case = mixed_case(91, dtype, Hq, 2, D, 16, [0, 70, 1500], [nodes] * 3)
        i = case.inp
        case.pool[0][..., 3] = (case.pool[0][..., 3] & 0xf0) | rng.integers(1, 8, case.pool[0].shape[:-1])  # element 6, above zero
        live = case.pool[1][..., 0] != 255
        case.pool[1][..., 0] = np.where(live, 126 + rng.integers(0, 3, live.shape), 255)
        case.k = kv4_values_ref(*case.pool[:2])
        i.q[:] = 0
        i.q[:, :, 6] = sign * 2.0 ** e
        i.k_tree[:, :, 6] = torch.from_numpy(2.0 ** rng.integers(-2, 3, tuple(i.k_tree.shape[:2])).astype(np.float32)).to(i.k_tree.dtype)
        ref, ref_lse = case.attend()
        mass, _ = case.attend(v=np.abs(case.v), v_tree=np.abs(W.widen(i.v_tree)))
        for splits in (0, 1):
            out, lse = _attend(hb, step, case, num_splits=splits)
            # ties are exact and what is not tied weighs nothing or, for the smallest scores, has a score that is good to 2^-22 of itself
            worst = 2.0 ** -22 * np.abs(ref_lse)[..., None] if e < 20 else 0.0
            unit = 2.0 ** -8 if dtype == "bf16" else 1e-5
            far = np.abs(W.widen(out) - ref) / (unit * (np.abs(ref) + mass) + 2 * worst * mass + 1e-30)
            assert (far <= 1).all(), f"2^{e}, splits={splits}: {far.max():.3g} of the tolerance"
            lse_far = np.abs(W.widen(lse) - ref_lse) / (2.0 ** -21 * np.abs(ref_lse) + 4e-6)
            assert (lse_far <= 1).all(), f"2^{e}, splits={splits}: lse {lse_far.max():.3g} of the tolerance"
