"""Pages and sampling rules on the GPU at the borders of what the calls take."""
import ctypes as C

import numpy as np
import pytest
import torch

import workloads as W
from oracle import pages_take_ref, rules_probs_ref, tree_accept_sample_ref
from test_gpu_requests import Rules, _pages, _take

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


# ---- pages ------------------------------------------------------------------------------------------

def test_rows_that_the_slots_cannot_hold_are_not_served():
    """Offsets beyond the rows, or falling: such a sequence keeps what it has, and bars nobody."""
    import paper_2509_18824_amd as hb
    lens, have, blocks = [5, 0, 17, 3], [1, 0, 2, 1], 30
    table = np.full((4, 8), -1)
    table[0, 0], table[2, :2], table[3, 0] = 20, [21, 22], 23
    for offset, bad in (([0, 4, 4, 30, 33], (2, 3)), ([0, 20, 10, 12, 14], (1,)), ([-2, 3, 5, 7, 9], (0,))):
        got = dict(table=i32(table), slots=i32([-2] * 25), new_len=i32([-9] * 4), have=i32([-9] * 4), granted=i32([-9] * 4), left=i32([-9]))
        hb.hb_pages_take(16, 3, i32(lens), i32(offset), i32(have), i32(list(range(20)) + [-1] * 10), i32([20]), got["table"], got["slots"],
                         got["new_len"], got["have"], got["granted"], got["left"])
        rows = np.diff(offset)
        for b in range(4):
            if b in bad:
                assert got["granted"][b] == 0 and got["new_len"][b] == lens[b] and got["have"][b] == have[b]
                assert np.array_equal(got["table"][b].cpu().numpy(), table[b])
            else:
                assert got["granted"][b] == 1 and got["new_len"][b] == lens[b] + rows[b]
                assert got["have"][b] == max(have[b], -(-(lens[b] + rows[b] + 3) // 16))
                assert (got["slots"][offset[b]:offset[b + 1]] >= 0).all()
        assert got["left"] == 20 - int((got["have"].cpu() - torch.tensor(have)).sum())


def test_pages_without_slots_by_the_c_call():
    """Without slots no number of rows bounds the offsets."""
    import paper_2509_18824_amd as hb
    c = _pages(3, 20, 16, 50, 60, 0, 2)
    want = _take(c)
    got = dict(table=i32(c["table"]), new_len=i32([-9] * 20), have=i32([-9] * 20), granted=i32([-9] * 20), left=i32([-9]))
    lens, offset, have, free, count = i32(c["lens"]), i32(c["offset"]), i32(c["have"]), i32(c["free"]), i32([c["n_free"]])
    at = lambda t: C.c_void_p(t.data_ptr())
    stream = C.c_void_p(torch.cuda.current_stream().cuda_stream)
    assert hb.lib.hb_pages_take(20, 16, c["max_blocks"], c["blocks"], 0, 2, at(lens), at(offset), at(have), at(free), at(count), at(got["table"]), None,
                                at(got["new_len"]), at(got["have"]), at(got["granted"]), at(got["left"]), stream) == 0
    torch.cuda.synchronize()
    for name in got:
        assert torch.equal(got[name], want[name]), name


def test_tables_of_many_entries_without_slots():
    """A row of pages longer than a workgroup has threads, and several of them."""
    import paper_2509_18824_amd as hb
    B, page, n = 3, 1, 5000
    blocks = B * n + 9
    table, have, left = i32(np.full((B, n + 3), -1)), i32([0] * B), i32([0])
    free = np.random.default_rng(5).permutation(blocks)
    hb.hb_pages_take(page, 0, i32([0] * B), i32(np.arange(B + 1) * n), i32([0] * B), i32(free), i32([blocks]), table, None, None, have, None, left)
    want, _, _, kept, _, rest = pages_take_ref(page, n + 3, blocks, 0, [0] * B, np.arange(B + 1) * n, [0] * B, free, np.full((B, n + 3), -1),
                                               np.zeros(B * n, int))
    assert np.array_equal(table.cpu().numpy(), want) and have.tolist() == kept.tolist() and left.tolist() == [rest]


@pytest.mark.parametrize("short", [False, True])
def test_empty_places_take_no_pages(short):
    """A negative length: nobody is there, nothing is reserved, and nobody behind waits for it."""
    import paper_2509_18824_amd as hb
    B, page, reserve, max_blocks, blocks = 6, 16, 8, 5, 40
    lens, rows, have = np.array([-1, 20, -1, 0, -7, 3]), np.array([0, 5, 0, 30, 4, 2]), np.array([0, 2, 1, 0, 0, 1])
    offset = np.concatenate([[0], np.cumsum(rows)])
    table = np.full((B, max_blocks), -1)
    table[1, :2], table[2, 0], table[5, 0] = [30, 31], 32, 33
    there = lens >= 0
    free = list(range(3 if short else 20))
    got = dict(table=i32(table), slots=i32([-2] * int(offset[-1])), new_len=i32([-9] * B), have=i32([-9] * B), granted=i32([-9] * B), left=i32([-9]))
    hb.hb_pages_take(page, reserve, i32(lens), i32(offset), i32(have), i32(free + [-1] * (blocks - len(free))), i32([len(free)]), got["table"], got["slots"],
                     got["new_len"], got["have"], got["granted"], got["left"])
    # as if they were not in the batch
    want_table, want_slots = table.copy(), np.full(offset[-1], -1)
    packed = np.concatenate([[0], np.cumsum(rows[there])])
    t, s, n, h, g, left = pages_take_ref(page, max_blocks, blocks, reserve, lens[there], packed, have[there], free, table[there], np.full(packed[-1], -2))
    want_table[there] = t
    want_slots[np.repeat(there, rows)] = s
    assert np.array_equal(got["table"].cpu().numpy(), want_table) and np.array_equal(got["slots"].cpu().numpy(), want_slots)
    for name, x, empty in (("new_len", n, lens), ("have", h, have), ("granted", g, 0 * lens)):
        want = np.array(empty)
        want[there] = x
        assert got[name].tolist() == want.tolist(), name
    assert got["left"].tolist() == [left]


def test_a_place_that_a_request_has_left():
    """Its pages are the others' until somebody comes, also where pages run short."""
    import paper_2509_18824_amd.step as S
    pages = S.PagePool(3, 16, 6, 7, 64, reserve=8)
    step = lambda *rows: (pages.take(i32(np.concatenate([[0], np.cumsum(rows)]))), pages.advance())
    step(30, 20, 1)
    assert pages.pages.tolist() == [3, 2, 1] and pages.free_count.tolist() == [1]
    pages.length[0] = -1
    pages.give(pages.length)
    for _ in range(2):
        step(0, 1, 1)
        assert pages.pages.tolist() == [0, 2, 1] and pages.free_count.tolist() == [4] and pages.length[0] == -1
    step(0, 60, 1)
    assert pages.granted.tolist() == [0, 1, 1] and pages.pages.tolist() == [0, 6, 1] and pages.free_count.tolist() == [0]
    step(0, 0, 12)  # no page is left: the last one waits for those of sequence 1, not for the empty place
    assert pages.granted.tolist() == [0, 1, 0] and pages.length.tolist() == [-1, 82, 4]
    pages.length[1] = -1
    pages.give(pages.length)
    pages.length[0] = 0
    step(40, 0, 12)
    assert pages.granted.tolist() == [1, 0, 1] and pages.length.tolist() == [40, -1, 16] and pages.pages.tolist() == [3, 0, 2]


# ---- in place ---------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("nodes,V,biases,masks", [([8], 1000, 3, 5), ([60, 0, 1], 1001, 40, 9), ([3, 2], 33, 5, 2), ([5, 9], 40000, 1500, 3),
                                                  ([1, 1], 100003, 7, 1), ([1] * 130, 4001, 3, 5), ([7], 9000, 900, 0)])
def test_rules_in_place(dtype, nodes, V, biases, masks):
    """Logits over themselves, with counts, paths, biases and masks: the bits of the call beside it."""
    import paper_2509_18824_amd as hb
    c = Rules(61 + V, dtype, nodes, V, biases, masks)
    c.logits[0, ::3] = float("nan")
    c.counts[:, :40] = 1
    z, _ = c.run()
    x = c.logits.cuda()
    hb.hb_rules_logits(x, max(nodes), *c.args(), x)
    assert torch.equal(x.view(torch.int32 if dtype == "f32" else torch.int16), z.view(torch.int32 if dtype == "f32" else torch.int16))


# ---- a sampled step ---------------------------------------------------------------------------------

@pytest.mark.parametrize("seed", range(4))
def test_every_token_of_a_sampled_step(seed):
    """Drafts drawn from what the target thinks, so that many are accepted; a sequence whose grammar leaves nothing.  Acceptance is in exact
    integers: of the step's own probabilities the oracle makes the same paths, tokens and last tokens, and these are counted."""
    import paper_2509_18824_amd.step as S
    from test_gpu_request_steps import _sampled
    inp, step, rng, vocab = _sampled(S, 70 + seed)
    off, parent = inp.node_offset.numpy(), inp.parent.numpy()
    r = step.rules
    r.mask[4].zero_()
    r.mask_row[off[1]:off[2]] = 4
    r.rules[:, 0] = torch.tensor(np.resize([1.5, 0.0, 2.5], inp.B), dtype=torch.float32)
    had = r.counts.clone()
    pools = [p.clone() for p in (step.dev.k_pool, step.dev.v_pool)]
    step.run()
    p = step.probs.double().cpu().numpy()
    draft = step.draft_ids.cpu().numpy().copy()
    q = np.full((inp.total_nodes, vocab), 1.0 / vocab)
    for b in range(inp.B):
        for n in range(off[b], off[b + 1]):
            q[n] = 0.9 * p[n] / max(p[n].sum(), 1e-30) + 0.1 / vocab
            if n > off[b]:
                draft[n] = rng.choice(vocab, p=q[off[b] + parent[n]] / q[off[b] + parent[n]].sum())
    step.draft_ids.copy_(torch.from_numpy(draft))
    step.q_draft.copy_(torch.from_numpy(q.astype(np.float32)))
    r.counts.copy_(had)
    step.dev.k_pool.copy_(pools[0])
    step.dev.v_pool.copy_(pools[1])
    step.run()
    got = step.probs.cpu().numpy()
    u = lambda t: t.cpu().numpy().view(np.uint32)
    want = tree_accept_sample_ref(off, parent, draft, got, step.q_draft.cpu().numpy(), u(step.u_accept), u(step.u_bonus), inp.max_path)
    for name, x in zip(("accept_len", "accept_path", "out_tokens", "bonus"), want):
        assert np.array_equal(getattr(step, name).cpu().numpy(), x), name
    alen, _, tokens, bonus = want
    assert alen.max() >= 3 and alen[1] == 1 and bonus[1] == -1 and not got[off[1]:off[2]].any()
    for b in range(inp.B):
        assert tokens[b, alen[b] - 1] == bonus[b]  # -1 where a mask has left nothing
        for t in tokens[b][tokens[b] >= 0]:
            had[b, t] += 1
    assert torch.equal(had, r.counts)
