"""How close the 4-bit cache's attention comes: log-sum-exps row by row to float32's error, and results to the bf16 cache's with the same
values, relative to what they are sums of."""
import math

import numpy as np
import pytest
import torch

import workloads as W
from kv4 import mixed_case
from test_gpu_kv4 import _attend, hb, step  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu


def _score_sums(case):
    """Of every row, over the keys that it sees: the largest softmax_scale * sum_d |q_d k_d|; [total nodes, Hq]."""
    i, G = case.inp, case.inp.Hq // case.inp.Hkv
    q, kt, best = np.abs(W.widen(i.q)), np.abs(W.widen(i.k_tree)), np.zeros((i.total_nodes, i.Hq))
    for b in range(i.B):
        n0, n1, p = int(i.node_offset[b]), int(i.node_offset[b + 1]), np.arange(int(i.prefix_len[b]))
        k = np.abs(case.k[i.block_table.numpy()[b, p // i.page], :, p % i.page])
        for g in range(i.Hkv):
            rows = q[n0:n1, g * G:(g + 1) * G]
            cached = (rows @ k[:, g].T).max(-1) if len(p) else np.zeros(rows.shape[:2])
            own = rows @ kt[n0:n1, g].T
            for r in range(n1 - n0):
                path, up = [], r
                while up >= 0:
                    path.append(up)
                    up = int(i.parent[n0 + up])
                best[n0 + r, g * G:(g + 1) * G] = np.maximum(cached[r], own[r][:, path].max(-1))
    return abs(i.softmax_scale) * best


@pytest.mark.parametrize("dtype,Hq,D,nodes", [("bf16", 28, 128, 1), ("bf16", 14, 128, 4), ("bf16", 14, 128, 30), ("bf16", 8, 64, 2), ("bf16", 8, 64, 40),
                                              ("bf16", 4, 96, 3), ("f32", 6, 128, 20), ("f32", 4, 64, 4)])
@pytest.mark.parametrize("peaked", [False, True])
def test_log_sum_exp_row_by_row(hb, step, dtype, Hq, D, nodes, peaked):
    case = mixed_case(81, dtype, Hq, 2, D, 16, [0, 3, 700, 2500], [nodes] * 4, peaked=peaked)
    _, ref = case.attend()
    # products of bf16 numbers are exact in float32: what is left is a sum of D of them, scaled, exponentials and their sum
    tol = 4 * 2.0 ** -24 * math.sqrt(D) * _score_sums(case) + 4e-6 * (1 + np.abs(ref))
    for splits in (0, 1, 3):
        _, lse = _attend(hb, step, case, num_splits=splits)
        far = np.abs(W.widen(lse) - ref) / tol
        assert (far <= 1).all(), f"splits={splits}: {far.max():.3g} of the tolerance"


@pytest.mark.parametrize("nodes", [1, 8, 60])
def test_the_bf16_cache_with_the_same_values(hb, step, nodes):
    case = mixed_case(82, "bf16", 28, 4, 128, 16, [700, 90, 3000], [nodes] * 3)
    i = case.inp
    ref, ref_lse = case.attend()
    mass, _ = case.attend(v=np.abs(case.v), v_tree=np.abs(W.widen(i.v_tree)))
    out, lse = _attend(hb, step, case)
    i.k_pool, i.v_pool = torch.from_numpy(case.k).bfloat16(), torch.from_numpy(case.v).bfloat16()
    other, other_lse = step.tree_verify_attn(case.desc(), step.to_device(i))
    torch.cuda.synchronize()
    # each side rounds its probabilities and its result to bf16, half a unit being at most 2^-8 of them
    tol = 2.0 ** -7 * (np.abs(ref) + mass)
    far = np.abs(W.widen(out) - W.widen(other)) / tol
    assert (far <= 1).all(), far.max()
    # the sum of the bf16 cache's probabilities may be that of the rounded ones
    far = np.abs(W.widen(lse) - W.widen(other_lse)) / (2.0 ** -8 + 1e-5 * (1 + np.abs(ref_lse)))
    assert (far <= 1).all(), far.max()
