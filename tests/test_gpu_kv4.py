"""GPU parity of the 4-bit cache's calls: rows in and out bit for bit, attention and attention weights element by element, evictions
exactly, against the float64 oracle."""
import math

import numpy as np
import pytest
import torch

import workloads as W
from kv4 import Kv4Case, mixed_case
from oracle import kv4_append_ref, kv4_attn_weight_ref, kv4_evict_ref, kv4_quantise_ref, kv4_values_ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hb():
    import paper_2509_18824_amd as m
    return m


@pytest.fixture(scope="module")
def step():
    import paper_2509_18824_amd.step as s
    return s


def _attend(hb, step, case, stream=None, **kw):
    pool, t = case.device()
    desc = case.desc(**kw)
    out, lse = torch.full_like(t["q"], float("nan")), torch.full(t["q"].shape[:2], float("nan"), device="cuda")
    ws = step.alloc_workspace(hb.hb_tree_verify_attn_kv4_workspace_bytes(desc))
    if ws is not None:
        ws.fill_(255)  # what a workspace held does not matter
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())
    hb.hb_tree_verify_attn_kv4(desc, t["q"], t["k_tree"], t["v_tree"], *pool, t["block_table"], t["prefix_len"], t["node_offset"], t["parent"],
                               out, lse, ws, stream=stream)
    torch.cuda.synchronize()
    return out, lse


LENS = [0, 1, 5, 16, 63, 64, 65, 200, 1000]
NODES = [1, 3, 64, 8, 60, 2, 17, 1, 33]


@pytest.mark.parametrize("dtype,Hq,Hkv,D,page", [
    ("bf16", 28, 4, 128, 16), ("bf16", 8, 8, 128, 16), ("bf16", 8, 1, 128, 32), ("bf16", 8, 4, 64, 16), ("bf16", 28, 4, 64, 48),
    ("bf16", 6, 2, 96, 16), ("bf16", 4, 2, 256, 16), ("bf16", 10, 2, 128, 4), ("bf16", 2, 2, 32, 16), ("bf16", 40, 2, 128, 16),
    ("f32", 4, 1, 64, 16), ("f32", 6, 2, 128, 16), ("f32", 4, 4, 128, 5), ("f32", 2, 1, 256, 16), ("f32", 3, 3, 32, 8)])
def test_attention_of_every_layout(hb, step, dtype, Hq, Hkv, D, page):
    case = mixed_case(5, dtype, Hq, Hkv, D, page, LENS, NODES)
    ref = case.attend()
    for splits in (1, 3, 0):
        out, lse = _attend(hb, step, case, num_splits=splits)
        case.check_attention(out, lse, ref, f"splits={splits}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nodes", [1, 2, 4, 9, 10, 18, 37, 64])
def test_attention_of_every_number_of_rows(hb, step, dtype, nodes):
    """Row tiles full and not, one sequence alone and several, peaked scores, a bound on the lengths that is given."""
    for B, L in ((1, 777), (3, 300)):
        case = mixed_case(nodes, dtype, 14, 2, 128, 16, [L - 7 * b for b in range(B)], [nodes] * B, peaked=True)
        ref = case.attend()
        for hint in (0, L):
            out, lse = _attend(hb, step, case, hint=hint)
            case.check_attention(out, lse, ref, f"B={B} hint={hint}")


@pytest.mark.parametrize("B", [1, 70])
def test_single_tokens(hb, step, B):
    lens = [4000] if B == 1 else [(37 * b) % 600 for b in range(B)]
    case = mixed_case(3, "bf16", 28, 4, 128, 16, lens, [1] * B)
    out, lse = _attend(hb, step, case)
    case.check_attention(out, lse)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_that_rise_all_the_way(hb, step, dtype):
    """Every block of keys moves the running maximum far up; then every one lies far below it."""
    case = mixed_case(4, dtype, 4, 2, 128, 16, [500, 500], [3, 20])
    i = case.inp
    for b, up in ((0, True), (1, False)):
        q = W.widen(i.q)[int(i.node_offset[b])]
        for p in range(500):
            for g in range(2):
                x = np.sign(q[2 * g]) * 2.0 ** ((p if up else 500 - p) // 80)
                for t, y in zip(case.pool[:2], kv4_quantise_ref(x)):
                    t[int(i.block_table[b, p // 16]), g, p % 16] = y
    case.k = kv4_values_ref(*case.pool[:2])
    out, lse = _attend(hb, step, case)
    case.check_attention(out, lse)


@pytest.mark.parametrize("nodes", [2, 30])
def test_scale_signs_and_extremes(hb, step, nodes):
    """A scale of zero or less than zero, scores without spread, scales of the format's ends."""
    for scale in (0.0, -0.1, 1e-3):
        case = mixed_case(6, "bf16", 4, 2, 128, 16, [70, 300], [nodes, nodes])
        case.inp.softmax_scale = scale
        out, lse = _attend(hb, step, case)
        case.check_attention(out, lse, label=str(scale))
    case = mixed_case(7, "bf16", 4, 2, 128, 16, [70, 300], [nodes, nodes])
    case.pool[1][case.pool[1] != 255] -= 100  # keys of 2^-100
    case.pool[3][case.pool[3] != 255] += 100  # values of 2^100
    case.k, case.v = kv4_values_ref(*case.pool[:2]), kv4_values_ref(*case.pool[2:])
    out, lse = _attend(hb, step, case)
    case.check_attention(out, lse, label="extremes")


def test_what_is_masked_does_not_matter(hb, step):
    """Slots past a length hold NaN everywhere in these tests; here nodes off a row's path do too, and infinities."""
    for nodes in (3, 12, 60):
        case = mixed_case(8, "bf16", 14, 2, 128, 16, [33, 100], [nodes, nodes])
        i = case.inp
        want = _attend(hb, step, case)
        leaf = int(i.node_offset[1]) + nodes - 1  # nobody's ancestor
        for bad in (float("nan"), float("inf"), -float("inf")):
            i.k_tree[leaf], i.v_tree[leaf] = bad, bad
            got = _attend(hb, step, case)
            others = [r for r in range(i.total_nodes) if r != leaf]
            assert all(torch.equal(g[others], w[others]) for g, w in zip(got, want)), (nodes, bad)


@pytest.mark.parametrize("nodes", [1, 40])
def test_nan_in_a_query_or_a_seen_key_stays_in_its_rows(hb, step, nodes):
    case = mixed_case(9, "bf16", 8, 2, 128, 16, [90, 200], [nodes, nodes])
    want = _attend(hb, step, case)
    case.inp.q[0, 3, 5] = float("nan")
    out, lse = _attend(hb, step, case)
    assert torch.isnan(out[0, 3]).all() and torch.isnan(lse[0, 3])
    keep = torch.ones(out.shape[:2], dtype=torch.bool)
    keep[0, 3] = False
    assert torch.equal(out[keep], want[0][keep]) and torch.equal(lse[keep], want[1][keep])
    case = mixed_case(9, "bf16", 8, 2, 128, 16, [90, 200], [nodes, nodes])
    i = case.inp
    case.pool[1][int(i.block_table[1, 3]), 1, 2, 0] = 255  # a key block of sequence 1, head 1
    out, lse = _attend(hb, step, case)
    n1 = int(i.node_offset[1])
    assert torch.isnan(out[n1:, 4:].float()).all()
    assert torch.equal(out[:n1], want[0][:n1]) and torch.equal(out[n1:, :4], want[0][n1:, :4])


def test_empty_trees_malformed_tables_and_another_stream(hb, step):
    case = mixed_case(10, "bf16", 8, 2, 128, 16, [90, 200, 30], [5, 7, 9])
    want = _attend(hb, step, case)
    s = torch.cuda.Stream()
    got = _attend(hb, step, case, stream=s)
    assert all(torch.equal(g, w) for g, w in zip(got, want))
    i = case.inp
    i.block_table[:, -1] = 1 << 30  # past every length: clamped into the pool, and not used
    got = _attend(hb, step, case)
    assert all(torch.equal(g, w) for g, w in zip(got, want))
    # a sequence without nodes
    i.node_offset[1] = 0
    i.node_offset[2] = 7
    i.node_offset[3] = 7
    got = _attend(hb, step, case)
    assert torch.isfinite(got[0][:7].float()).all()


def test_attention_in_a_graph(hb, step):
    case = mixed_case(11, "bf16", 28, 4, 128, 16, [900, 300], [8, 8])
    pool, t = case.device()
    desc = case.desc()
    ws = step.alloc_workspace(hb.hb_tree_verify_attn_kv4_workspace_bytes(desc))
    out, lse = torch.empty_like(t["q"]), torch.empty(t["q"].shape[:2], device="cuda")
    call = lambda: hb.hb_tree_verify_attn_kv4(desc, t["q"], t["k_tree"], t["v_tree"], *pool, t["block_table"], t["prefix_len"],
                                              t["node_offset"], t["parent"], out, lse, ws)
    call()
    torch.cuda.synchronize()
    want = out.clone(), lse.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(4):
        out.fill_(float("nan"))
        lse.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


def test_long_cache_offsets_beyond_31_bits(hb, step):
    """Codes of one pool beyond 2^31 bytes: the pages that are read lie at its end."""
    blocks, Hkv, page, D = (1 << 31) // (4 * 16 * 64) + 600, 4, 16, 128
    small = mixed_case(12, "bf16", 28, Hkv, D, page, [777, 100], [1, 9])
    i = small.inp
    pool, t = small.device()
    want = small.attend()
    big = step.kv4_pool(blocks, Hkv, page, D)
    shift = blocks - i.num_blocks
    for b, s in zip(big, pool):
        b[shift:].copy_(s)
    desc = small.desc()
    desc.num_blocks = blocks
    table = t["block_table"] + shift
    out, lse = torch.empty_like(t["q"]), torch.empty(t["q"].shape[:2], device="cuda")
    ws = step.alloc_workspace(hb.hb_tree_verify_attn_kv4_workspace_bytes(desc))
    hb.hb_tree_verify_attn_kv4(desc, t["q"], t["k_tree"], t["v_tree"], *big, table, t["prefix_len"], t["node_offset"], t["parent"], out, lse, ws)
    torch.cuda.synchronize()
    small.check_attention(out, lse, want)


# ---- rows in and out --------------------------------------------------------------------------------

def _cache(case, rng):
    """Pool of any bytes, weights and positions, as numpy."""
    i = case.inp
    pool = [rng.integers(0, 256, x.shape).astype(np.uint8) for x in case.pool]
    weight = rng.random((i.B, i.Hkv, case.cap)).astype(np.float32)
    pos = rng.integers(0, 1 << 20, (i.B, i.Hkv, case.cap)).astype(np.int32)
    return pool, weight, pos


@pytest.mark.parametrize("dtype,Hkv,D,page", [("bf16", 4, 128, 16), ("bf16", 1, 64, 16), ("f32", 2, 32, 5), ("bf16", 3, 256, 32), ("f32", 2, 96, 16)])
@pytest.mark.parametrize("extras", [True, False])
def test_append_and_read(hb, dtype, Hkv, D, page, extras):
    """Rows of every size class, blocks with infinities and NaN, ties, zeros and subnormal numbers; a sequence that runs past its
    table; one without rows."""
    rng = np.random.default_rng(21)
    counts, lens = [40, 0, 1, 130, 7], [0, 3, 15, 33, 10]
    inp = W.make_verify_inputs(22, dtype, Hkv, Hkv, D, [L + n for L, n in zip(lens, counts)], [W.chain_tree(1)] * 5, page=page)
    case = Kv4Case(inp)
    lens[4] = case.cap - 4  # three of seven rows find no place
    pool, weight, pos = _cache(case, rng)
    n = sum(counts)
    x = [torch.from_numpy(rng.standard_normal((n, Hkv, D)) * np.exp2(rng.integers(-140, 120, (n, Hkv, 1)).astype(float))).to(inp.q.dtype) for _ in (0, 1)]
    levels = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, -0.0, 0.0, 6.5, -5.0])
    x[0][3, 0, :12] = levels.to(inp.q.dtype)
    x[0][3, 0, 12:32] = 0
    x[0][4] = 0
    x[0][5, 0, 1], x[1][6, 0, D - 1], x[1][7, 0, 0] = float("inf"), float("nan"), -float("inf")
    x[0][8, 0, :] = torch.finfo(inp.q.dtype).max
    offset = np.concatenate([[0], np.cumsum(counts)])
    seq = [L + 100 * b for b, L in enumerate(lens)]
    want = [p.copy() for p in pool], weight.copy(), pos.copy()
    _, new_len = kv4_append_ref(want[0], [W.widen(t) for t in x], inp.block_table.numpy(), lens, [range(offset[b], offset[b + 1]) for b in range(5)],
                                want[1] if extras else None, want[2] if extras else None, seq)
    dev = [torch.from_numpy(p).cuda() for p in pool]
    i32 = lambda v: torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")
    w, p, new, first = torch.from_numpy(weight).cuda(), torch.from_numpy(pos).cuda(), i32([-1] * 5), i32(lens)
    desc, table = case.desc(), inp.block_table.cuda()
    kw = dict(seq_len=i32(seq), weight=w, pos=p, new_len=new) if extras else {}
    hb.hb_kv4_append(desc, x[0].cuda(), x[1].cuda(), *dev, table, first, i32(offset), **kw)
    torch.cuda.synchronize()
    for got, ref in zip(dev, want[0]):
        assert np.array_equal(got.cpu().numpy(), ref)
    assert np.array_equal(w.cpu().numpy(), want[1]) and np.array_equal(p.cpu().numpy(), want[2])
    assert not extras or np.array_equal(new.cpu().numpy(), new_len)
    out = [torch.full((n, Hkv, D), 5.0, dtype=inp.q.dtype, device="cuda") for _ in (0, 1)]
    hb.hb_kv4_read(desc, *dev, table, first, i32(offset), *out)
    torch.cuda.synchronize()
    for t, o, src in zip((0, 2), out, x):
        ref = kv4_values_ref(*kv4_quantise_ref(W.widen(src)))
        ref[offset[4] + 4:offset[5]] = 0  # past the table
        assert np.array_equal(W.widen(o), ref, equal_nan=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_compact(hb, dtype):
    rng = np.random.default_rng(23)
    case = mixed_case(24, dtype, 4, 2, 128, 16, [0, 31, 100, 12], [8, 60, 5, 12])
    i, max_path = case.inp, 6
    pool, weight, pos = _cache(case, rng)
    accept = [3, 6, 0, 1]
    path = np.full((4, max_path), -1)
    for b, n in enumerate(accept):
        nodes = int(i.node_offset[b + 1] - i.node_offset[b])
        path[b, :n] = np.sort(rng.choice(nodes, n, replace=False))
    took = [[int(i.node_offset[b]) + x for x in path[b, :accept[b]]] for b in range(4)]
    want = [p.copy() for p in pool], weight.copy(), pos.copy()
    slots, new_len = kv4_append_ref(want[0], [W.widen(i.k_tree), W.widen(i.v_tree)], i.block_table.numpy(), i.prefix_len.numpy(), took, want[1], want[2])
    dev, t = case.device()
    dev = [torch.from_numpy(p).cuda() for p in pool]
    i32 = lambda v: torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")
    w, p, new, out_slots = torch.from_numpy(weight).cuda(), torch.from_numpy(pos).cuda(), i32([-1] * 4), i32(np.full((4, max_path), -7))
    hb.hb_kv4_compact(case.desc(), t["k_tree"], t["v_tree"], *dev, t["block_table"], t["prefix_len"], t["node_offset"], i32(accept), i32(path), max_path,
                      None, w, p, out_slots, new)
    torch.cuda.synchronize()
    for got, ref in zip(dev, want[0]):
        assert np.array_equal(got.cpu().numpy(), ref)
    assert np.array_equal(w.cpu().numpy(), want[1]) and np.array_equal(p.cpu().numpy(), want[2])
    assert np.array_equal(new.cpu().numpy(), new_len)
    assert out_slots.tolist() == [s + [-1] * (max_path - len(s)) for s in slots]


# ---- attention weights ------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,Hq,Hkv,D,page", [("bf16", 28, 4, 128, 16), ("bf16", 8, 8, 64, 32), ("f32", 4, 1, 64, 16), ("bf16", 40, 2, 128, 16),
                                                 ("bf16", 4, 2, 256, 16), ("f32", 6, 2, 96, 5), ("bf16", 16, 2, 128, 4)])
@pytest.mark.parametrize("paths", [True, False])
def test_attention_weights(hb, dtype, Hq, Hkv, D, page, paths):
    case = mixed_case(31, dtype, Hq, Hkv, D, page, [0, 1, 17, 64, 300, 1100], [3, 1, 12, 64, 5, 2])
    i, max_path = case.inp, 6
    rng = np.random.default_rng(32)
    _, lse = case.attend()
    accept, path, took = [2, 1, 6, 5, 0, 1], np.full((6, max_path), -1), []
    for b, n in enumerate(accept):
        n0, n1 = int(i.node_offset[b]), int(i.node_offset[b + 1])
        path[b, :n] = np.sort(rng.choice(n1 - n0, n, replace=False))
        took.append([n0 + x for x in path[b, :n]] if paths else range(n0, n1))
    weight = rng.random((i.B, Hkv, case.cap)).astype(np.float32)
    lse32 = torch.from_numpy(lse).float()
    want = kv4_attn_weight_ref(W.widen(i.q), case.k, i.block_table.numpy(), i.prefix_len.numpy(), took, W.widen(lse32), i.softmax_scale, 0.75, weight)
    pool, t = case.device()
    w = torch.from_numpy(weight).cuda()
    i32 = lambda v: torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")
    hb.hb_kv4_attn_weight(case.desc(), t["q"], pool[0], pool[1], t["block_table"], t["prefix_len"], t["node_offset"],
                          i32(accept) if paths else None, i32(path) if paths else None, max_path, lse32.cuda(), 0.75, w)
    torch.cuda.synchronize()
    got = W.widen(w)
    # a score's sum of D products in float32, then an exponential and a sum of the rows: relative to the weight
    tol = want * (4 * 2.0 ** -24 * math.sqrt(D) * (case.largest_sum() + 4) + 4e-6)
    assert (np.abs(got - want) <= tol).all(), (np.abs(got - want) / tol).max()
    for b in range(i.B):
        assert np.array_equal(got[b, :, int(i.prefix_len[b]):], weight[b, :, int(i.prefix_len[b]):])


# ---- eviction ---------------------------------------------------------------------------------------

@pytest.mark.parametrize("budget,recent,sinks", [(1, 0, 0), (1, 1, 0), (16, 3, 4), (100, 20, 4), (300, 0, 0), (300, 296, 4), (5000, 64, 4)])
@pytest.mark.parametrize("in_place", [True, False])
def test_eviction(hb, step, budget, recent, sinks, in_place):
    """Lengths below, at and above the budget; weights with many ties, infinities and NaN; rows bit for bit."""
    lens = [0, 1, budget if budget < 1000 else 700, 301, 299, 1100, 2500]
    case = mixed_case(41, "bf16", 4, 2, 64, 16, lens, [1] * 7)
    i, rng = case.inp, np.random.default_rng(budget)
    pool, weight, _ = _cache(case, rng)
    weight = np.round(weight * 20) / 20
    weight[3], weight[4, 0] = 0.5, -0.0
    weight[4, 0, ::2] = 0.0
    weight[5, :, 10:30], weight[5, :, 30:40], weight[6, :, 5:700] = np.nan, np.inf, -np.inf
    weight[6, 1, 100:2000] *= 1e-30
    weight = weight.astype(np.float32)
    seq = np.array(lens) + 13
    pos = np.stack([[np.sort(rng.choice(n + 13, case.cap, replace=True)) for _ in range(2)] for n in lens]).astype(np.int32)
    for b, n in enumerate(lens):
        for h in range(2):  # distinct positions, in no order
            pos[b, h, :n] = rng.permutation(n + 13)[:n]
    dev = [torch.from_numpy(p).cuda() for p in pool]
    i32 = lambda v: torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")
    w, p = torch.from_numpy(weight).cuda(), torch.from_numpy(pos).cuda()
    w_out, p_out = (w, p) if in_place else (torch.full_like(w, 7.0), torch.full_like(p, 7))
    kept, new = i32(np.full((7, 2, budget), -9)), i32([-1] * 7)
    ws = step.alloc_workspace(hb.hb_kv4_evict_workspace_bytes(case.desc(), budget))
    hb.hb_kv4_evict(case.desc(), budget, recent, sinks, *dev, i.block_table.cuda(), i.prefix_len.cuda(), i32(seq), w, p, w_out, p_out, kept, new, ws)
    torch.cuda.synchronize()
    assert new.tolist() == [min(n, budget) for n in lens]
    table, want = i.block_table.numpy(), [x.copy() for x in pool]
    want_w, want_p = (weight.copy(), pos.copy()) if in_place else (np.full_like(weight, 7), np.full_like(pos, 7))
    for b, n in enumerate(lens):
        for h in range(2):
            ref = kv4_evict_ref(n, budget, recent, sinks, seq[b], weight[b, h], pos[b, h])
            assert kept[b, h].tolist() == ref + [-1] * (budget - len(ref)), (b, h)
            for s, src in enumerate(ref):
                want_w[b, h, s], want_p[b, h, s] = weight[b, h, src], pos[b, h, src]
                for x, y in zip(want, pool):
                    x[table[b, s // 16], h, s % 16] = y[table[b, src // 16], h, src % 16]
    assert np.array_equal(w_out.cpu().numpy(), want_w, equal_nan=True) and np.array_equal(p_out.cpu().numpy(), want_p)
    for got, ref in zip(dev, want):
        assert np.array_equal(got.cpu().numpy(), ref)


@pytest.mark.parametrize("length", [300, 40000])
def test_eviction_keeps_protected_positions_in_front_of_infinite_weights(hb, step, length):
    """As many infinite weights as the budget holds, in front of what is protected."""
    cap, budget, recent, sinks = (length + 15) // 16 * 16, 64, 5, 3
    d = step.make_desc(dtype="bf16", B=1, Hq=1, Hkv=1, D=32, page=16, max_blocks=cap // 16, num_blocks=cap // 16, total_nodes=0, max_nodes=1, softmax_scale=1.0)
    weight = np.full((1, 1, cap), np.inf, dtype=np.float32)
    pos = np.zeros((1, 1, cap), dtype=np.int32)
    pos[0, 0, :length] = np.arange(length)[::-1]  # the recent ones in front, the first ones last
    weight[0, 0, :30] = 0.25
    cuda = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    pool = [torch.zeros(s, dtype=torch.uint8, device="cuda") for s in ((cap // 16, 1, 16, 16), (cap // 16, 1, 16, 1)) * 2]
    kept, new = i32([[[-9] * budget]]), i32([-1])
    w, p = cuda(weight), cuda(pos)
    hb.hb_kv4_evict(d, budget, recent, sinks, *pool, i32([list(range(cap // 16))]), i32([length]), i32([length]), w, p, w, p, kept, new,
                    step.alloc_workspace(hb.hb_kv4_evict_workspace_bytes(d, budget)))
    torch.cuda.synchronize()
    assert kept[0, 0].tolist() == kv4_evict_ref(length, budget, recent, sinks, length, weight[0, 0], pos[0, 0])
    assert set(p[0, 0, :budget].tolist()) >= set(range(sinks)) | set(range(length - recent, length))


def test_a_tree_without_nodes_has_no_path(hb, step):
    """accept_len that names nodes of an empty tree, for one sequence and for all: nothing is written, lengths stay."""
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    for offsets in ([0, 0, 2], [0, 0, 0]):
        n = offsets[-1]
        d = step.make_desc(dtype="bf16", B=2, Hq=2, Hkv=1, D=64, page=16, max_blocks=2, num_blocks=4, total_nodes=n, max_nodes=2, softmax_scale=1.0)
        rows = torch.ones((max(n, 1), 1, 64), dtype=torch.bfloat16, device="cuda")[:n]
        pool = [torch.full(s, 9, dtype=torch.uint8, device="cuda") for s in ((4, 1, 16, 32), (4, 1, 16, 2)) * 2]
        slots, new = i32([[7, 7], [7, 7]]), i32([-1, -1])
        hb.hb_kv4_compact(d, rows, rows, *pool, i32([[0, 1], [2, 3]]), i32([3, 4]), i32(offsets), i32([2, 1]), i32([[0, 1], [1, 0]]), 2,
                          None, None, None, slots, new)
        torch.cuda.synchronize()
        assert new.tolist() == [3, 5 if n else 4] and slots.tolist() == [[-1, -1], [36 if n else -1, -1]]
        assert all((p[:2] == 9).all() for p in pool) and (n or all((p == 9).all() for p in pool))


@pytest.mark.parametrize("dtype,Hq,D,nodes,lens", [("bf16", 14, 128, 3, [33, 5000]), ("bf16", 14, 128, 12, [0, 300]), ("bf16", 14, 128, 60, [100, 5000]),
                                                   ("bf16", 4, 64, 40, [7, 90]), ("bf16", 16, 64, 60, [0, 3000]), ("bf16", 14, 128, 61, [33, 0]),
                                                   ("f32", 6, 128, 50, [33, 2000]), ("f32", 2, 64, 5, [0, 100]), ("bf16", 4, 96, 12, [33, 2000])])
def test_values_of_nodes_that_are_not_finite_reach_the_rows_that_see_them(hb, step, dtype, Hq, D, nodes, lens):
    """Infinities and NaN in elements of an inner node, of the last one and of the root: the rows whose path they lie on have them in
    these elements, and nothing else of any result changes by a bit."""
    case = mixed_case(9, dtype, Hq, 2, D, 16, lens, [nodes, nodes])
    i, G = case.inp, Hq // 2
    n1, parent = int(i.node_offset[1]), i.parent.tolist()
    clean = _attend(hb, step, case)
    bad = {(0, 1, 5): float("inf"), (nodes // 2, 0, D - 1): -float("inf"), (nodes - 1, 1, 40): float("nan"), (nodes // 2, 1, 17): float("inf"),
           (0, 0, 2): float("-inf")}
    want = clean[0].float()
    for (node, h, e), x in bad.items():
        i.v_tree[n1 + node, h, e] = x
        for row in range(nodes):
            up = row
            while up > node:
                up = parent[n1 + up]
            if up == node:
                want[n1 + row, h * G:(h + 1) * G, e] = x
    zeroed = mixed_case(9, dtype, Hq, 2, D, 16, lens, [nodes, nodes])
    for node, h, e in bad:
        zeroed.inp.v_tree[n1 + node, h, e] = 0
    base = _attend(hb, step, zeroed)
    got = _attend(hb, step, case)
    odd = ~torch.isfinite(want)
    assert odd.any() and torch.equal(torch.nan_to_num(got[0].float()[odd], nan=7.0), torch.nan_to_num(want[odd], nan=7.0))
    assert torch.equal(got[0][~odd], base[0][~odd]) and torch.equal(got[1], base[1])


@pytest.mark.parametrize("B", [2, 64, 65, 130])
def test_append_and_read_of_many_sequences(hb, B):
    """Prompts of none to a few rows each, several sequences to a wavefront's rows."""
    rng = np.random.default_rng(B)
    counts, lens = rng.integers(0, 6, B), rng.integers(0, 30, B)
    counts[B // 2:B // 2 + 3] = 0
    counts[-1] = 21
    inp = W.make_verify_inputs(23, "bf16", 2, 2, 64, [int(x) for x in lens + counts], [W.chain_tree(1)] * B, page=16)
    case = Kv4Case(inp)
    pool, _, _ = _cache(case, rng)
    n, offset = int(counts.sum()), np.concatenate([[0], np.cumsum(counts)])
    x = [torch.from_numpy(rng.standard_normal((n, 2, 64))).to(torch.bfloat16) for _ in (0, 1)]
    want = [p.copy() for p in pool]
    kv4_append_ref(want, [W.widen(t) for t in x], inp.block_table.numpy(), lens, [range(offset[b], offset[b + 1]) for b in range(B)], None, None, None)
    dev = [torch.from_numpy(p).cuda() for p in pool]
    i32 = lambda v: torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")
    new, table, first = i32([-1] * B), inp.block_table.cuda(), i32(lens)
    hb.hb_kv4_append(case.desc(), x[0].cuda(), x[1].cuda(), *dev, table, first, i32(offset), new_len=new)
    out = [torch.full((n, 2, 64), 5.0, dtype=torch.bfloat16, device="cuda") for _ in (0, 1)]
    hb.hb_kv4_read(case.desc(), *dev, table, first, i32(offset), *out)
    torch.cuda.synchronize()
    assert new.tolist() == (lens + counts).tolist()
    for got, ref in zip(dev, want):
        assert np.array_equal(got.cpu().numpy(), ref)
    for o, src in zip(out, x):
        assert np.array_equal(W.widen(o), kv4_values_ref(*kv4_quantise_ref(W.widen(src))))


@pytest.mark.parametrize("B,nodes,longest", [(1, 1, 768), (1, 1, 769), (1, 8, 1025), (8, 4, 1024), (8, 4, 1025), (2, 60, 256), (2, 60, 257), (6, 60, 1153)])
def test_where_prefixes_begin_to_be_cut(hb, step, B, nodes, longest):
    """The longest prefix at the bound that the call is given, the others anywhere below; and a bound that leaves room."""
    lens = [longest] + [longest * (b + 1) % 700 for b in range(B - 1)]
    case = mixed_case(51, "bf16", 28, 4, 64, 16, lens, [nodes] * B, peaked=True)
    ref = case.attend()
    for hint in (longest, longest + 300):
        out, lse = _attend(hb, step, case, hint=hint)
        case.check_attention(out, lse, ref, f"hint={hint}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_weights_of_paths_of_any_bound(hb, dtype):
    """Bounds on a path's length beyond a wavefront; a path that names a node twice, and ids outside the tree, which are clamped."""
    case = mixed_case(32, dtype, 14, 2, 128, 16, [70, 600], [64, 20])
    i, max_path = case.inp, 100
    _, lse = case.attend()
    path = np.full((2, max_path), -5)
    path[0, :64] = np.arange(64)[::-1]
    path[1, :7] = [3, 3, 19, 0, 25, -2, 8]
    accept = [64, 7]
    took = [list(path[0, :64]), [64 + x for x in (3, 3, 19, 0, 19, 0, 8)]]
    weight = np.random.default_rng(1).random((2, 2, case.cap)).astype(np.float32)
    lse32 = torch.from_numpy(lse).float()
    want = kv4_attn_weight_ref(W.widen(i.q), case.k, i.block_table.numpy(), i.prefix_len.numpy(), took, W.widen(lse32), i.softmax_scale, 0.5, weight)
    pool, t = case.device()
    w, i32 = torch.from_numpy(weight).cuda(), lambda v: torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")
    hb.hb_kv4_attn_weight(case.desc(), t["q"], pool[0], pool[1], t["block_table"], t["prefix_len"], t["node_offset"], i32(accept), i32(path),
                          max_path, lse32.cuda(), 0.5, w)
    torch.cuda.synchronize()
    # as in test_attention_weights; 64 nodes of seven heads are 448 float32 additions on top
    tol = want * (4 * 2.0 ** -24 * math.sqrt(128) * (case.largest_sum() + 4) + 4e-6 + 448 * 2.0 ** -24)
    assert (np.abs(W.widen(w) - want) <= tol).all(), (np.abs(W.widen(w) - want) / tol).max()
