"""The host's bound on prefix lengths sizes the launches of the 4-bit cache's calls: prefixes beyond it are taken whole."""
import math

import numpy as np
import pytest
import torch

import workloads as W
from kv4 import mixed_case
from oracle import kv4_attn_weight_ref, kv4_evict_ref
from test_gpu_kv4 import _attend, _cache, hb, step  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,Hq,D,page,nodes", [("bf16", 14, 128, 16, 3), ("bf16", 14, 128, 16, 40), ("f32", 6, 64, 16, 5), ("bf16", 4, 96, 16, 4),
                                                   ("f32", 4, 32, 5, 3)])
@pytest.mark.parametrize("hint", [1, 100, 1500])
def test_attention(hb, step, dtype, Hq, D, page, nodes, hint):
    case = mixed_case(61, dtype, Hq, 2, D, page, [0, 99, 101, 2000], [nodes] * 4)
    ref = case.attend()
    for splits in (0, 1, 3):
        out, lse = _attend(hb, step, case, hint=hint, num_splits=splits)
        case.check_attention(out, lse, ref, f"hint={hint} splits={splits}")


@pytest.mark.parametrize("dtype,Hq,Hkv,D,page,nodes", [("bf16", 28, 4, 128, 16, 3), ("bf16", 28, 4, 128, 16, 40), ("f32", 4, 2, 64, 16, 12), ("bf16", 4, 2, 96, 16, 5)])
@pytest.mark.parametrize("hint", [1, 300, 1500])
def test_attention_weights(hb, dtype, Hq, Hkv, D, page, nodes, hint):
    case = mixed_case(62, dtype, Hq, Hkv, D, page, [0, 299, 301, 2050], [nodes] * 4)
    i = case.inp
    _, lse = case.attend()
    weight = np.random.default_rng(63).random((4, Hkv, case.cap)).astype(np.float32)
    lse32 = torch.from_numpy(lse).float()
    took = [range(int(i.node_offset[b]), int(i.node_offset[b + 1])) for b in range(4)]
    want = kv4_attn_weight_ref(W.widen(i.q), case.k, i.block_table.numpy(), i.prefix_len.numpy(), took, W.widen(lse32), i.softmax_scale, 0.75, weight)
    pool, t = case.device()
    w = torch.from_numpy(weight).cuda()
    hb.hb_kv4_attn_weight(case.desc(hint=hint), t["q"], pool[0], pool[1], t["block_table"], t["prefix_len"], t["node_offset"], None, None, 1,
                          lse32.cuda(), 0.75, w)
    torch.cuda.synchronize()
    # a score's sum of D products in float32, an exponential, and a sum of the rows: relative to the weight
    tol = want * (4 * 2.0 ** -24 * math.sqrt(D) * (case.largest_sum() + 4) + 4e-6 + nodes * Hq // Hkv * 2.0 ** -24)
    assert (np.abs(W.widen(w) - want) <= tol).all(), (np.abs(W.widen(w) - want) / tol).max()
    for b in range(4):
        n = int(i.prefix_len[b])
        assert np.array_equal(w[b, :, n:].cpu().numpy(), weight[b, :, n:])


@pytest.mark.parametrize("hint", [1, 250, 1100])
@pytest.mark.parametrize("budget", [40, 260, 2000, 6000])
def test_eviction(hb, step, hint, budget):
    """Lengths on both sides of the bound, the protected positions behind it; rows bit for bit."""
    lens = [0, 200, 251, 1101, 2600]
    case = mixed_case(64, "bf16", 4, 2, 64, 16, lens, [1] * 5)
    i, rng, recent, sinks = case.inp, np.random.default_rng(budget), 30, 3
    pool, weight, pos = _cache(case, rng)
    weight = (np.round(weight * 50) / 50).astype(np.float32)
    pos[:] = np.arange(case.cap)
    dev = [torch.from_numpy(p).cuda() for p in pool]
    i32 = lambda v: torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")
    w, p = torch.from_numpy(weight).cuda(), torch.from_numpy(pos).cuda()
    kept, new = i32(np.full((5, 2, budget), -9)), i32([-1] * 5)
    d = case.desc(hint=hint)
    ws = step.alloc_workspace(hb.hb_kv4_evict_workspace_bytes(d, budget))
    hb.hb_kv4_evict(d, budget, recent, sinks, *dev, i.block_table.cuda(), i.prefix_len.cuda(), i.prefix_len.cuda(), w, p, w, p, kept, new, ws)
    torch.cuda.synchronize()
    assert new.tolist() == [min(n, budget) for n in lens]
    table, want, want_w, want_p = i.block_table.numpy(), [x.copy() for x in pool], weight.copy(), pos.copy()
    for b, n in enumerate(lens):
        for h in range(2):
            ref = kv4_evict_ref(n, budget, recent, sinks, n, weight[b, h], pos[b, h])
            assert kept[b, h].tolist() == ref + [-1] * (budget - len(ref)), (b, h)
            for s, src in enumerate(ref):
                want_w[b, h, s], want_p[b, h, s] = weight[b, h, src], pos[b, h, src]
                for x, y in zip(want, pool):
                    x[table[b, s // 16], h, s % 16] = y[table[b, src // 16], h, src % 16]
    assert np.array_equal(w.cpu().numpy(), want_w) and np.array_equal(p.cpu().numpy(), want_p)
    for got, ref in zip(dev, want):
        assert np.array_equal(got.cpu().numpy(), ref)


def test_steps_that_pass_the_bound(hb, step):
    """Kv4VerifyStep under a descriptor whose bound was true when it was built: the newest positions gather weight and, protected by
    `recent`, survive an eviction."""
    rng, V, max_path, budget, recent = np.random.default_rng(3), 300, 4, 40, 8
    case = mixed_case(65, "bf16", 4, 2, 128, 16, [60, 33], [6, 6])
    i = case.inp
    pages, blocks = 6, i.num_blocks + 12
    pools = step.kv4_pool(blocks, 2, 16, 128)
    old, _ = case.device()
    for new, x in zip(pools, old):
        new.zero_()
        new[:i.num_blocks].copy_(x)
    table = torch.arange(i.num_blocks, blocks, dtype=torch.int32).view(2, pages)
    for b in range(2):
        mapped = -(-int(i.prefix_len[b]) // 16)
        table[b, :mapped] = i.block_table[b, :mapped]
    i.block_table, i.max_blocks, i.num_blocks = table, pages, blocks
    dev = step.to_device(i)
    weight = (torch.randn((V, 4 * 128), generator=torch.Generator().manual_seed(1)) * 0.05).bfloat16().cuda()
    draft = torch.zeros(i.total_nodes, dtype=torch.int32, device="cuda")
    s = step.Kv4VerifyStep(case.desc(hint=60), dev, pools, weight, draft, max_path, budget, recent, 0)
    for turn in range(6):
        s.run()
        torch.cuda.synchronize()
        draft.copy_(torch.from_numpy(np.asarray(W.plant_draft_ids(70 + turn, i.trees(), s.target_ids.cpu().numpy(), V, want_depth=[3, 3])[0]).astype(np.int32)))
        s.run()
        torch.cuda.synchronize()
        s.advance()
    torch.cuda.synchronize()
    length, seq = dev.prefix_len.tolist(), s.seq_len.tolist()
    assert length == seq and length[0] > 60 + 8
    s.run()  # from here on every position has been seen by a committed node
    torch.cuda.synchronize()
    for b in range(2):
        assert (s.slot_weight[b, :, :length[b]] > 0).all()
    s.evict()
    torch.cuda.synchronize()
    for b in range(2):
        for h in range(2):
            have = s.slot_pos[b, h, :int(dev.prefix_len[b])].tolist()
            assert len(have) == min(length[b], budget) and set(have) >= set(range(seq[b] - recent, seq[b]))
