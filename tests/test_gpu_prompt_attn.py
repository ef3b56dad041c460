"""hb_prompt_attn on the GPU against the oracle."""
import numpy as np
import pytest
import torch

import workloads as W
from prompts import Prompts

pytestmark = pytest.mark.gpu


def _algos(dtype, D, page):
    import paper_2509_18824_amd as hb
    both = dtype == "bf16" and D in (64, 128) and page & (page - 1) == 0
    return (hb.HB_ATTN_AUTO, hb.HB_ATTN_SCALAR) if both else (hb.HB_ATTN_AUTO,)


SHAPES = [
    # dtype, Hq, Hkv, D, page, cached, rows
    ("f32", 4, 1, 64, 16, [0], [1]),
    ("f32", 4, 1, 64, 16, [0, 256], [255, 3]),
    ("f32", 6, 2, 128, 32, [33, 0, 7], [0, 65, 64]),
    ("f32", 3, 3, 8, 1, [5], [40]),
    ("f32", 2, 1, 72, 48, [100, 1], [17, 1]),
    ("f32", 2, 2, 256, 16, [19], [33]),
    ("bf16", 28, 4, 128, 16, [0], [1]),
    ("bf16", 28, 4, 128, 16, [0], [37]),
    ("bf16", 28, 4, 128, 16, [100, 0, 63, 1], [5, 0, 64, 130]),
    ("bf16", 28, 4, 128, 16, [0, 0], [300, 1]),
    ("bf16", 8, 8, 128, 16, [0, 17], [257, 31]),
    ("bf16", 32, 8, 64, 64, [65, 0, 128], [33, 200, 1]),
    ("bf16", 8, 1, 64, 1, [9], [100]),
    ("bf16", 5, 1, 128, 2, [64], [129]),
    ("bf16", 2, 1, 80, 48, [50], [70]),
    ("bf16", 2, 1, 256, 16, [50], [20]),
    ("bf16", 40, 10, 128, 32, [31], [64]),
]


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s)))
@pytest.mark.parametrize("splits", [0, 1, 5])
def test_against_the_oracle(shape, splits):
    c = Prompts(sum(shape[1:5]) + len(shape[6]), *shape, sharp=1.5)
    for algo in _algos(shape[0], shape[3], shape[4]):
        out, lse = c.run(algo=algo, num_splits=splits)
        c.check(out, lse, label=f"{shape} splits {splits} algo {algo}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_one_token_over_a_long_prefix(dtype):
    c = Prompts(5, dtype, 4, 2, 64, 16, [3000, 1, 0, 1500], [1, 1, 1, 2])
    for algo in _algos(dtype, 64, 16):
        for splits in (0, 7):
            out, lse = c.run(algo=algo, num_splits=splits)
            c.check(out, lse)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [8, 64, 72, 128, 136, 256])
def test_many_parts(dtype, D):
    """More parts than a thread of the join has under way, and than its lanes have groups; some rows see nothing of some."""
    c = Prompts(21, dtype, 6, 2, D, 16, [5000, 30, 4700], [3, 40, 1])
    for algo in _algos(dtype, D, 16):
        for splits in (18, 70):
            out, lse = c.run(algo=algo, num_splits=splits)
            c.check(out, lse)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_sequences(dtype):
    """More of them than a wavefront has lanes, most of one row or none."""
    rng = np.random.default_rng(8)
    rows = rng.integers(0, 3, 150).tolist()
    c = Prompts(9, dtype, 4, 2, 64, 8, rng.integers(0, 20, 150).tolist(), rows)
    for algo in _algos(dtype, 64, 8):
        out, lse = c.run(algo=algo)
        c.check(out, lse)


@pytest.mark.parametrize("scale", [0.0, -0.2, 3.0])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_any_scale(dtype, scale):
    c = Prompts(6, dtype, 4, 2, 64, 16, [20], [50], scale=scale)
    out, lse = c.run()
    c.check(out, lse)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
def test_what_a_row_does_not_see_has_no_influence(dtype, D):
    """Bits of later rows, of slots behind the prefix (NaN in every case here) and of rows that nobody has."""
    c = Prompts(7, dtype, 4, 2, D, 16, [21, 40], [90, 100], spare=2)
    at = int(c.offset[1]) + 60
    bad = [torch.inf, -torch.inf, torch.nan]
    for algo in _algos(dtype, D, 16):
        for splits in (1, 4):
            want, want_lse = c.run(algo=algo, num_splits=splits)
            d = c.device()
            for i, x in enumerate(bad):
                d["k"][at + i], d["v"][at + i] = x, bad[i - 1]
            got, got_lse = c.run(dev=d, algo=algo, num_splits=splits)
            clean = [*range(at), ]
            assert torch.equal(got[clean], want[clean]) and torch.equal(got_lse[clean], want_lse[clean])
            assert not torch.isfinite(got[at + 2:].float()).any()  # NaN keys reach whoever sees them


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_values_that_are_not_finite_reach_those_who_see_them(dtype):
    c = Prompts(11, dtype, 4, 2, 64, 16, [10], [80])
    ref, ref_lse = c.reference()
    for algo in _algos(dtype, 64, 16):
        for splits in (1, 3):
            d = c.device()
            d["v"][30, 0, 5] = torch.inf
            d["v"][40, 1, 6] = torch.nan
            d["v"][50, 0, 7] = -torch.inf
            d["v"][60, 0, 7] = torch.inf
            out, lse = c.run(dev=d, algo=algo, num_splits=splits)
            o = W.widen(out)
            assert (o[30:, :2, 5] == np.inf).all() and np.isnan(o[40:, 2:, 6]).all() and (o[50:60, :2, 7] == -np.inf).all() and np.isnan(o[60:, :2, 7]).all()
            o[30:, :2, 5], o[40:, 2:, 6], o[50:, :2, 7] = ref[30:, :2, 5], ref[40:, 2:, 6], ref[50:, :2, 7]
            c.check(torch.from_numpy(o), lse, label="the others")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_keys_whose_scores_are_minus_infinity(dtype):
    """The first 70 keys, prefix and prompt, have none but such scores, and those behind are about -600: weights are relative to
    what a row has seen.  Rows that see nothing else have no result."""
    c = Prompts(16, dtype, 4, 2, 64, 16, [40], [90])
    c.q[:, :, 0] = 8.0
    c.q[:, :, 1:] *= 0.25
    c.k[:, :, 0], c.k_pool[:, :, :, 0] = -600.0, -torch.inf
    c.k[:30, :, 0] = -torch.inf
    ref, ref_lse = c.reference()
    seen = np.arange(90) >= 30
    for algo in _algos(dtype, 64, 16):
        for splits in (1, 2, 3):
            out, lse = c.run(algo=algo, num_splits=splits)
            o = W.widen(out)
            assert np.isnan(o[~seen]).all()
            assert np.abs(o[seen] - ref[seen]).max() <= (1e-3 if dtype == "f32" else 2.0 ** -6) * (4 + np.abs(ref[seen]).max())
            assert np.abs(W.widen(lse)[seen] - ref_lse[seen]).max() <= 600 * 2.0 ** -14


def test_largest_scores_and_values():
    """Scores near float32's exponents' middle: weights of one key alone, and sums of the type's largest values."""
    c = Prompts(12, "bf16", 4, 2, 128, 16, [30], [70], scale=50.0)
    for algo in _algos("bf16", 128, 16):
        out, lse = c.run(algo=algo)
        assert torch.isfinite(out.float()).all() and torch.isfinite(lse).all()
        ref, ref_lse = c.reference()
        assert np.abs(W.widen(lse) - ref_lse).max() <= 2e-4 * np.abs(ref_lse).max()
    c = Prompts(13, "bf16", 4, 2, 128, 16, [30], [70])
    c.v.fill_(3.0e38)
    c.v_pool = torch.where(torch.isnan(c.v_pool), c.v_pool, 3.0e38)
    for algo in _algos("bf16", 128, 16):
        out, _ = c.run(algo=algo, num_splits=1)
        assert torch.isinf(out.float()).any() or (out.float() - 3.0e38).abs().max() <= 2.0 ** -7 * 3.0e38


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_behind_the_last_sequence_stay(dtype):
    c = Prompts(14, dtype, 4, 2, 64, 16, [3, 5], [10, 0])
    keep = [c.q, c.k, c.v]
    pad = lambda t: torch.cat((t, torch.full((9, *t.shape[1:]), float("nan"), dtype=t.dtype)))
    c.q, c.k, c.v = map(pad, keep)
    for algo in _algos(dtype, 64, 16):
        out, lse = c.run(desc=c.desc(total=19, algo=algo))
        assert (out[10:] == 7).all() and (lse[10:] == 7).all()
        ref = [np.concatenate([x, np.zeros((9, *x.shape[1:]))]) for x in Prompts(14, dtype, 4, 2, 64, 16, [3, 5], [10, 0]).reference()]
        assert np.abs(W.widen(out[:10]) - ref[0][:10]).max() <= (1e-4 if dtype == "f32" else 4e-2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_nothing_cached_and_no_cache(dtype):
    c = Prompts(15, dtype, 4, 2, 64, 16, [0, 0], [33, 12])
    for algo in _algos(dtype, 64, 16):
        a, b = c.run(algo=algo), c.run(algo=algo, prefix=False)
        c.check(*a)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        assert torch.equal(c.run(algo=algo, lse=False)[0], a[0])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_longer_prefix_than_the_hint_is_taken_whole(dtype):
    c = Prompts(16, dtype, 4, 2, 64, 16, [900, 300], [3, 20])
    for algo in _algos(dtype, 64, 16):
        out, lse = c.run(algo=algo, hint=16)
        c.check(out, lse)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_malformed_lengths_and_tables_stay_inside(dtype):
    """Page ids outside the pool, lengths beyond the table, offsets that fall or leave the rows: defined nowhere, and they end."""
    c = Prompts(17, dtype, 4, 2, 64, 16, [40, 9], [30, 5])
    for algo in _algos(dtype, 64, 16):
        for name, value in (("table", 1 << 30), ("table", -5), ("lens", 1 << 30), ("lens", -7)):
            d = c.device()
            d[name].fill_(value)
            c.run(dev=d, algo=algo)
        for offset in ([0, 30, 10], [-3, 5, 9], [0, 50, 60]):
            d = c.device()
            d["offset"] = torch.tensor(offset, dtype=torch.int32, device="cuda")
            out, _ = c.run(dev=d, algo=algo)
            assert out.shape[0] == 35
        torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_same_bits_again_and_on_another_stream(dtype):
    c = Prompts(18, dtype, 8, 2, 128, 16, [700, 0, 50], [40, 130, 1])
    want = c.run()
    dev = c.device()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        got = [c.run(dev=dev) for _ in range(3)]
    stream.synchronize()
    for g in got:
        assert torch.equal(g[0], want[0]) and torch.equal(g[1], want[1])


def test_two_graphs_that_share_a_workspace_and_lengths_that_change():
    import paper_2509_18824_amd as hb
    import paper_2509_18824_amd.step as S
    cases = [Prompts(19, "bf16", 8, 2, 128, 16, [600, 30], [3, 50]), Prompts(20, "bf16", 8, 2, 64, 16, [0, 900], [64, 1])]
    ws = S.alloc_workspace(max(hb.hb_prompt_attn_workspace_bytes(c.desc()) for c in cases))
    devs = [c.device() for c in cases]
    outs = [torch.zeros_like(d["q"]) for d in devs]
    lses = [torch.zeros(d["q"].shape[:2], device="cuda") for d in devs]

    def call(i):
        c, d = cases[i], devs[i]
        hb.hb_prompt_attn(c.desc(), d["q"], d["k"], d["v"], d["k_pool"], d["v_pool"], d["table"], d["lens"], d["offset"], outs[i], lses[i], ws)

    graphs = []
    for i in range(2):
        call(i)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(i)
        graphs.append(g)
    for shrink in (0, 1, 7):
        for i, c in enumerate(cases):
            devs[i]["lens"].copy_(torch.tensor([max(0, n - shrink) for n in c.lens], dtype=torch.int32))
        want = []
        for i in range(2):
            call(i)
            want.append((outs[i].clone(), lses[i].clone()))
        torch.cuda.synchronize()
        for o in outs:
            o.zero_()
        for i in (0, 1, 0):
            graphs[i].replay()
        torch.cuda.synchronize()
        for i in range(2):
            assert torch.equal(outs[i], want[i][0]) and torch.equal(lses[i], want[i][1])


def test_a_long_cache_whose_offsets_pass_32_bits():
    """A pool of more than 2^31 elements, the pages in use behind them."""
    import paper_2509_18824_amd as hb
    c = Prompts(21, "bf16", 8, 8, 128, 16, [200], [20])
    blocks = (1 << 31) // (8 * 16 * 128) + 40
    d = c.device()
    for name in ("k_pool", "v_pool"):
        big = torch.zeros((blocks, 8, 16, 128), dtype=torch.bfloat16, device="cuda")
        big[blocks - c.num_blocks:] = d[name]
        d[name] = big
    d["table"] += blocks - c.num_blocks
    for algo in (hb.HB_ATTN_AUTO, hb.HB_ATTN_SCALAR):
        desc = c.desc(algo=algo)
        desc.num_blocks = blocks
        out, lse = c.run(dev=d, desc=desc)
        c.check(out, lse)


@pytest.mark.parametrize("seed", range(6))
def test_long_prompts_row_by_row(seed):
    """Prompts of thousands of rows, against the definition in float64 on the GPU."""
    Hq, Hkv, D, page, lens, rows = [(28, 4, 128, 16, [0], [2500]), (8, 8, 64, 32, [1000, 0], [1300, 700]), (16, 2, 128, 64, [3000], [515]),
                                    (8, 1, 128, 16, [0, 700, 5], [1, 1200, 1025]), (28, 4, 64, 16, [4100], [257]), (4, 4, 128, 16, [0], [3333])][seed]
    gen = torch.Generator(device="cuda").manual_seed(seed)
    c = Prompts(seed, "bf16", Hq, Hkv, D, page, [0] * len(lens), [1] * len(lens))  # pools, made on the GPU instead
    used = [-(-n // page) for n in lens]
    r = lambda *s: torch.randn(s, generator=gen, device="cuda").bfloat16()
    T = sum(rows)
    c.lens, c.rows, c.T, c.max_blocks, c.num_blocks = lens, rows, T, max(max(used), 1), sum(used) + 1
    c.offset = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    table = np.full((len(lens), c.max_blocks), c.num_blocks - 1)
    perm, at = np.random.default_rng(seed).permutation(sum(used)), 0
    for b, n in enumerate(used):
        table[b, :n] = perm[at:at + n]
        at += n
    i32 = lambda x: torch.from_numpy(np.asarray(x, dtype=np.int32)).cuda()
    d = dict(q=r(T, Hq, D) * torch.linspace(0.3, 3, Hq, device="cuda")[:, None].bfloat16(), k=r(T, Hkv, D), v=r(T, Hkv, D),
             k_pool=r(c.num_blocks, Hkv, page, D), v_pool=r(c.num_blocks, Hkv, page, D), table=i32(table), lens=i32(lens), offset=i32(c.offset))
    out, lse = c.run(dev=d)
    for b, n in enumerate(lens):
        lo, hi = c.offset[b], c.offset[b + 1]
        ids = torch.from_numpy(table[b, :used[b]]).cuda().long()
        for h in range(Hq):
            g = h // (Hq // Hkv)
            k, v = (torch.cat((p[ids, g].reshape(-1, D)[:n], x[lo:hi, g])).double() for p, x in ((d["k_pool"], d["k"]), (d["v_pool"], d["v"])))
            s = (d["q"][lo:hi, h].double() @ k.T) * c.scale
            s.masked_fill_(~torch.ones_like(s, dtype=torch.bool).tril(n), -torch.inf)
            p = torch.softmax(s, 1)
            want, mass = p @ v, p @ v.abs()
            tol = 2.0 ** -8 * (mass + want.abs()) + 2e-3 * mass  # scores of up to some twenty, sums of thousands: as in Prompts.check
            assert ((out[lo:hi, h].double() - want).abs() <= tol).all(), (b, h)
            assert ((lse[lo:hi, h].double() - torch.logsumexp(s, 1)).abs() <= 1e-3).all(), (b, h)
