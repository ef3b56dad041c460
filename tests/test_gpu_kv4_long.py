"""Long prefixes of the 4-bit cache on the paths that only they reach: chunks of more than 1024 keys, whose pages a wavefront asks for again
and again, and weights of several rounds to a workgroup."""
import math

import numpy as np
import pytest
import torch

import workloads as W
from kv4 import mixed_case
from oracle import kv4_attn_weight_ref
from test_gpu_kv4 import _attend, hb, step  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,Hq,D,nodes", [("bf16", 4, 128, 1), ("bf16", 14, 128, 2), ("bf16", 14, 64, 5), ("bf16", 14, 128, 9), ("bf16", 14, 128, 10),
                                              ("bf16", 14, 64, 33), ("bf16", 28, 128, 40), ("f32", 4, 128, 3), ("f32", 6, 64, 20)])
@pytest.mark.parametrize("page", [16, 48])
def test_attention_without_a_cut(hb, step, dtype, Hq, D, nodes, page):
    """Lengths on both sides of where the 64, 128, 192 sixteens of keys that a wavefront knows the pages of end."""
    case = mixed_case(71, dtype, Hq, 2, D, page, [1025, 2049, 3333, 1024, 2047, 40], [nodes] * 6)
    ref = case.attend()
    for splits in (1, 2):
        out, lse = _attend(hb, step, case, num_splits=splits)
        case.check_attention(out, lse, ref, f"splits={splits}")


@pytest.mark.parametrize("dtype,Hq,D", [("bf16", 32, 128), ("bf16", 16, 64), ("f32", 16, 128), ("f32", 8, 64)])
@pytest.mark.parametrize("cap,nodes", [(4096, 3), (8192, 3), (8192, 20), (32768, 3), (32768, 33)])
def test_weights_of_several_rounds(hb, dtype, Hq, D, cap, nodes):
    """16 sequences of eight heads under tables of `cap` positions: two, four and eight rounds of 256 keys to a workgroup, with rows of one batch in
    LDS and of several; lengths in every round, most of them off a multiple of 16."""
    lens = [0, 1, 17, 255, 256, 257, 300, 511, 513, 767, 1000, 1023, 1025, 1300, 2049, 2500]
    case = mixed_case(72, dtype, Hq, 8, D, 16, lens, [nodes] * 16)
    i = case.inp
    table = torch.zeros((16, cap // 16), dtype=torch.int32)
    table[:, :i.max_blocks] = i.block_table
    i.block_table, i.max_blocks, case.cap = table, cap // 16, cap
    _, lse = case.attend()
    weight = np.random.default_rng(73).random((16, 8, cap)).astype(np.float32)
    lse32 = torch.from_numpy(lse).float()
    took = [range(int(i.node_offset[b]), int(i.node_offset[b + 1])) for b in range(16)]
    want = kv4_attn_weight_ref(W.widen(i.q), case.k, table.numpy(), i.prefix_len.numpy(), took, W.widen(lse32), i.softmax_scale, 0.75, weight)
    pool, t = case.device()
    w = torch.from_numpy(weight).cuda()
    hb.hb_kv4_attn_weight(case.desc(), t["q"], pool[0], pool[1], t["block_table"], t["prefix_len"], t["node_offset"], None, None, 1, lse32.cuda(), 0.75, w)
    torch.cuda.synchronize()
    # a score's sum of D products in float32, an exponential, and a sum of the rows: relative to the weight
    tol = want * (4 * 2.0 ** -24 * math.sqrt(D) * (case.largest_sum() + 4) + 4e-6 + nodes * Hq // 8 * 2.0 ** -24)
    assert (np.abs(W.widen(w) - want) <= tol).all(), (np.abs(W.widen(w) - want) / tol).max()
    for b in range(16):
        assert np.array_equal(w[b, :, lens[b]:].cpu().numpy(), weight[b, :, lens[b]:])
