"""The 4-bit cache's attention and attention weights with numbers up to the type's largest, and infinities: off a row's path they
do not matter; where they are seen, results are the definition's (float64 oracle)."""
import math

import numpy as np
import pytest
import torch

import workloads as W
from kv4 import mixed_case
from oracle import kv4_attn_weight_ref, kv4_values_ref
from test_gpu_kv4 import _attend, hb, step  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu

LARGEST = {"f32": [torch.finfo(torch.float32).max, torch.finfo(torch.float32).min, 3.3961776e38, -3.3961776e38, 3.39e38],
           "bf16": [torch.finfo(torch.bfloat16).max, torch.finfo(torch.bfloat16).min]}
LAYOUTS = [("f32", 6, 128, 3), ("f32", 6, 128, 12), ("f32", 6, 128, 60), ("f32", 4, 64, 5), ("f32", 4, 96, 12),
           ("bf16", 14, 128, 3), ("bf16", 14, 128, 60), ("bf16", 4, 64, 12)]


@pytest.mark.parametrize("dtype,Hq,D,nodes", LAYOUTS)
def test_off_the_path_they_do_not_matter(hb, step, dtype, Hq, D, nodes):
    case = mixed_case(8, dtype, Hq, 2, D, 16, [33, 100], [nodes, nodes])
    i = case.inp
    want = _attend(hb, step, case)
    leaf = int(i.node_offset[1]) + nodes - 1  # nobody's ancestor
    others = [r for r in range(i.total_nodes) if r != leaf]
    for bad in LARGEST[dtype] + [math.inf, -math.inf, math.nan]:
        i.k_tree[leaf], i.v_tree[leaf] = bad, bad
        got = _attend(hb, step, case)
        assert all(torch.equal(g[others], w[others]) for g, w in zip(got, want)), bad


@pytest.mark.parametrize("dtype,Hq,D,nodes", LAYOUTS + [("bf16", 14, 64, 40), ("bf16", 28, 128, 64)])
@pytest.mark.parametrize("lens", [[33, 100], [0, 3000]])
def test_values_that_are_seen(hb, step, dtype, Hq, D, nodes, lens):
    """One node's value in an element: sums in float32 hold it.  Elements beside it are as they would be without."""
    for turn, x in enumerate(LARGEST[dtype]):
        case = mixed_case(9 + turn, dtype, Hq, 2, D, 16, lens, [nodes, nodes])
        i = case.inp
        i.v_tree[int(i.node_offset[1]) + nodes // 2, turn % 2, 5] = x
        i.v_tree[nodes - 1, 1, D - 1 - turn] = x
        out, lse = _attend(hb, step, case)
        case.check_attention(out, lse, label=str(x))


@pytest.mark.parametrize("dtype,D", [("f32", 64), ("f32", 128), ("f32", 96), ("bf16", 64), ("bf16", 128)])
def test_rows_that_see_one_key_return_its_value(hb, step, dtype, D):
    for x in LARGEST[dtype]:
        case = mixed_case(12, dtype, 4, 2, D, 16, [0, 0], [1, 1])
        case.inp.v_tree[:] = x
        out, _ = _attend(hb, step, case)
        # a weight, its product with the value, a reciprocal and the product with it: 2^-24 each
        assert (np.abs(W.widen(out) - W.widen(case.inp.v_tree[:1, :1])) <= 2.0 ** -22 * abs(x)).all(), x


@pytest.mark.parametrize("dtype,Hq,D,nodes", LAYOUTS)
def test_keys_and_queries_that_are_seen(hb, step, dtype, Hq, D, nodes):
    """Times the smallest normal number, so that a score is an ordinary one."""
    tiny = 2.0 ** -126
    for turn, x in enumerate(LARGEST[dtype]):
        case = mixed_case(9 + turn, dtype, Hq, 2, D, 16, [33, 200], [nodes, nodes])
        i = case.inp
        i.k_tree[int(i.node_offset[1]) + nodes // 2, :, 6] = x
        i.q[:, :, 6] = tiny
        out, lse = _attend(hb, step, case)
        case.check_attention(out, lse, label=f"key {x}")
        case = mixed_case(9 + turn, dtype, Hq, 2, D, 16, [33, 200], [nodes, nodes])
        i = case.inp
        i.q[nodes // 2, :, 6] = x
        i.k_tree[:, :, 6] = tiny
        case.pool[0][..., 3] &= 0xf0  # cached keys are zero there
        case.k = kv4_values_ref(*case.pool[:2])
        out, lse = _attend(hb, step, case)
        case.check_attention(out, lse, label=f"query {x}")


@pytest.mark.parametrize("dtype,Hq,D,nodes", LAYOUTS)
def test_a_seen_key_whose_score_is_minus_infinity_weighs_nothing(hb, step, dtype, Hq, D, nodes):
    case = mixed_case(9, dtype, Hq, 2, D, 16, [33, 200], [nodes, nodes])
    i = case.inp
    node = int(i.node_offset[1]) + max(1, nodes // 2)
    largest = case.largest_sum()
    i.q[:, :, 6] = i.q[:, :, 6].abs() + 0.25
    i.k_tree[node, :, 6] = 0.0
    largest = max(largest, case.largest_sum())
    i.k_tree[node, :, 6] = -1e30  # as good as: its weight is zero in 64 bits too
    ref = case.attend()
    i.k_tree[node, :, 6] = -math.inf
    out, lse = _attend(hb, step, case)
    i.k_tree[node, :, 6] = -1e30
    case.largest_sum = lambda: largest
    case.check_attention(out, lse, ref)


@pytest.mark.parametrize("D", [64, 128, 96])
def test_weights_of_queries_up_to_the_largest(hb, D):
    """Queries at the type's largest in a block whose cached keys lie about the smallest normal number."""
    case = mixed_case(31, "f32", 4, 2, D, 16, [17, 300], [3, 12])
    i, rng = case.inp, np.random.default_rng(5)
    case.pool[1][..., 1] = 1  # the block's scale: 2^-126
    case.k = kv4_values_ref(*case.pool[:2])
    i.k_tree[:, :, 32:64] *= 2.0 ** -126
    for turn, x in enumerate(LARGEST["f32"]):
        i.q[:, :, 40 + turn] = x * torch.from_numpy(rng.choice([-1.0, 1.0], tuple(i.q.shape[:2])).astype(np.float32))
    _, lse = case.attend()
    weight = rng.random((2, 2, case.cap)).astype(np.float32)
    lse32 = torch.from_numpy(lse).float()
    want = kv4_attn_weight_ref(W.widen(i.q), case.k, i.block_table.numpy(), i.prefix_len.numpy(), [range(0, 3), range(3, 15)], W.widen(lse32),
                               i.softmax_scale, 0.5, weight)
    pool, t = case.device()
    w = torch.from_numpy(weight).cuda()
    hb.hb_kv4_attn_weight(case.desc(), t["q"], pool[0], pool[1], t["block_table"], t["prefix_len"], t["node_offset"], None, None, 1, lse32.cuda(), 0.5, w)
    torch.cuda.synchronize()
    # a score's sum of D products in float32, then an exponential and a sum of the rows: relative to the weight
    tol = want * (4 * 2.0 ** -24 * math.sqrt(D) * (case.largest_sum() + 4) + 4e-6)
    assert (np.abs(W.widen(w) - want) <= tol).all(), (np.abs(W.widen(w) - want) / tol).max()


@pytest.mark.parametrize("dtype,D", [("f32", 128), ("f32", 96), ("bf16", 64), ("bf16", 96)])
def test_a_block_of_keys_that_is_no_number_reaches_its_head_alone(hb, step, dtype, D):
    case = mixed_case(14, dtype, 4, 2, D, 16, [256, 90], [1, 1])
    clean = _attend(hb, step, case)
    case.pool[1][int(case.inp.block_table[0, 3]), 1, 7, 1] = 255
    out, lse = _attend(hb, step, case)
    assert torch.isnan(out[0, 2:].float()).all() and torch.isnan(lse[0, 2:]).all()
    assert torch.equal(out[0, :2], clean[0][0, :2]) and torch.equal(out[1], clean[0][1]) and torch.equal(lse[1], clean[1][1])
