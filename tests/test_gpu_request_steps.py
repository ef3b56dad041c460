"""A request's whole way on the GPU: pages for its prompt, the prompt through the layers in parts, verification steps over the same
cache with tokens sampled by the request's rules, and its pages back; eagerly and from HIP graphs."""
import numpy as np
import pytest
import torch

import workloads as W
from oracle import (linear_ref, pages_give_ref, pages_take_ref, prompt_attn_ref, qkv_rope_project_ref, rmsnorm_ref, rules_logits_ref,
                    rules_probs_ref, swiglu_ref, tree_accept_sample_ref)
from oracle.toy_decoder import round_bf16

pytestmark = pytest.mark.gpu
HQ, HKV, D, PAGE, F, V = 4, 2, 128, 16, 1024, 4096
K = HQ * D
wide = lambda t: W.widen(t.cpu())
i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


@pytest.fixture(scope="module")
def S():
    import paper_2509_18824_amd.step as s
    return s


class Model:
    def __init__(self, n_layers, whole=True, seed=17):
        g = torch.Generator(device="cuda").manual_seed(seed)
        mk = self.mk = lambda *shape, std: (torch.randn(shape, generator=g, device="cuda") * std).to(torch.bfloat16)
        n = range(n_layers)
        self.w_qkv = [mk((HQ + 2 * HKV) * D, K, std=K ** -0.5) for _ in n]
        self.w_o = [mk(K, K, std=0.3 * K ** -0.5) for _ in n]
        self.mlp = dict(norm1=[mk(K, std=0.2) + 1 for _ in n], norm2=[mk(K, std=0.2) + 1 for _ in n],
                        w_gate_up=[mk(2 * F, K, std=K ** -0.5) for _ in n], w_down=[mk(K, F, std=0.3 * F ** -0.5) for _ in n],
                        norm_f=mk(K, std=0.2) + 1, eps=1e-6) if whole else None
        self.lm, self.embedding = mk(V, K, std=0.1), mk(V, K, std=1.0)

    def pools(self, num_blocks):
        return [tuple(torch.full((num_blocks, HKV, PAGE, D), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in "kv") for _ in self.w_qkv]

    def hidden_ref(self, x):
        """A whole prompt's final hidden states in float64, rounded to bf16 where the kernels hand a bf16 tensor on."""
        x, T = wide(x), x.shape[0]
        for l in range(len(self.w_qkv)):
            a = x if self.mlp is None else round_bf16(rmsnorm_ref(x, wide(self.mlp["norm1"][l]), 1e-6))
            q, k, v = (round_bf16(t) for t in qkv_rope_project_ref(a, wide(self.w_qkv[l]), None, np.arange(T), HQ, HKV, D, 1e6))
            o, _ = prompt_attn_ref(q, k, v, None, None, None, None, [0, T], D ** -0.5)
            y = x = round_bf16(linear_ref(round_bf16(o).reshape(T, -1), wide(self.w_o[l]), x))
            if self.mlp is not None:
                m = round_bf16(rmsnorm_ref(y, wide(self.mlp["norm2"][l]), 1e-6))
                x = round_bf16(linear_ref(round_bf16(swiglu_ref(m, wide(self.mlp["w_gate_up"][l]))), wide(self.mlp["w_down"][l]), y))
        return x if self.mlp is None else rmsnorm_ref(x, wide(self.mlp["norm_f"]), 1e-6)


def _stack(S, model, pages, pools, B, T, max_blocks, num_blocks):
    desc = S.make_desc("bf16", B, HQ, HKV, D, PAGE, max_blocks, num_blocks, T, 1, D ** -0.5, hint=max_blocks * PAGE)
    return S.PromptLayerStack(desc, pages, pools, model.w_qkv, model.w_o, model.lm, i32([0] * (B + 1)), model.mk(T, K, std=1.0), mlp=model.mlp)


def _load(stack, model, parts):
    """parts: each sequence's next tokens."""
    offset = np.concatenate([[0], np.cumsum([len(p) for p in parts])])
    stack.row_offset.copy_(i32(offset))
    stack.hidden0[:offset[-1]].copy_(model.embedding[np.concatenate(parts).astype(int)])
    return offset


def _near(got, ref):
    """Two layers of bf16 hand-overs."""
    assert np.linalg.norm(got - ref) <= 1e-2 * np.linalg.norm(ref) and np.abs(got - ref).max() <= 0.1 * (1 + np.abs(ref).max())


@pytest.mark.parametrize("whole", [True, False])
def test_prompts_in_parts_against_the_oracle(S, whole):
    """Three prompts in two calls and some padding: hidden states, first tokens, and the rows in the pools."""
    rng, model, B, T, blocks = np.random.default_rng(3), Model(2, whole), 3, 80, 40
    pages, pools = S.PagePool(B, PAGE, 12, blocks, T), None
    pages.free_pages.copy_(i32(rng.permutation(blocks)))
    pools = model.pools(blocks)
    stack = _stack(S, model, pages, pools, B, T, 12, blocks)
    prompts = [rng.integers(0, V, n) for n in (65, 30, 17)]
    refs = [model.hidden_ref(model.embedding[p]) for p in prompts]
    at = [0, 0, 0]
    for sizes in ([40, 0, 17], [25, 30, 0]):
        offset = _load(stack, model, [p[a:a + n] for p, a, n in zip(prompts, at, sizes)])
        stack.run()
        first, hidden = stack.first_ids.cpu().numpy(), wide(stack.final_hidden)
        for b, n in enumerate(sizes):
            if not n:
                assert first[b] == -1
                continue
            _near(hidden[offset[b]:offset[b + 1]], refs[b][at[b]:at[b] + n])
            logits = hidden[offset[b + 1] - 1] @ wide(model.lm).T
            assert logits[first[b]] >= logits.max() - 1e-4 * np.abs(logits).max()
            at[b] += n
            # the last layer's rows, where the tables say
            table = pages.block_table[b].cpu().numpy()
            for j in range(n):
                p = at[b] - n + j
                for rows, pool in zip((stack.k, stack.v), pools[1]):
                    assert torch.equal(pool[table[p // PAGE], :, p % PAGE], rows[offset[b] + j])
    assert pages.length.tolist() == [65, 30, 17] and pages.pages.tolist() == [5, 2, 2] and pages.free_count.tolist() == [blocks - 9]


def test_a_prompt_that_gets_no_pages_waits(S):
    """Of three prompts the second is refused: it has no first token and no rows in the cache, the others are as if alone, and it goes on
    when another's pages are given back."""
    rng, model, B, T, blocks = np.random.default_rng(13), Model(2), 3, 160, 6
    pages, pools = S.PagePool(B, PAGE, 12, blocks, T), None
    pools = model.pools(blocks)
    stack = _stack(S, model, pages, pools, B, T, 12, blocks)
    prompts = [rng.integers(0, V, n) for n in (40, 70, 0)]
    offset = _load(stack, model, prompts)
    stack.run()
    assert pages.granted.tolist() == [1, 0, 1] and pages.length.tolist() == [40, 0, 0] and stack.first_ids.tolist()[1:] == [-1, -1]
    assert (pages.slots[40:].cpu() == -1).all() and pages.free_count.item() == 3
    _near(wide(stack.final_hidden)[:40], model.hidden_ref(model.embedding[prompts[0]]))
    pages.length[0] = 0
    pages.give(pages.length)
    assert pages.free_count.item() == blocks
    _load(stack, model, [prompts[0][:0], prompts[1], prompts[0][:0]])
    stack.run()
    assert pages.granted.tolist() == [1, 1, 1] and pages.length.tolist() == [0, 70, 0]
    ref = model.hidden_ref(model.embedding[prompts[1]])
    _near(wide(stack.final_hidden)[:70], ref)
    logits = wide(stack.final_hidden)[69] @ wide(model.lm).T
    assert logits[stack.first_ids[1].item()] >= logits.max() - 1e-4 * np.abs(logits).max()


def test_a_prompt_and_then_verification_steps_over_its_cache(S):
    """Prompt, tree, prompt again: what a verification step sees of a prompt is what the prompt's own rows saw.  The nodes of a chain
    have the hidden states of the prompt that goes on with them (both within 1e-2 of the exact ones, two layers of bf16), the
    accepted ones are appended, and a later part of a prompt goes on behind them."""
    rng, model, B, blocks = np.random.default_rng(5), Model(2), 2, 40
    pages, pools = S.PagePool(B, PAGE, 12, blocks, 64, reserve=8), model.pools(blocks)
    prompts = [rng.integers(0, V, n) for n in (37, 16)]
    stack = _stack(S, model, pages, pools, B, 64, 12, blocks)
    _load(stack, model, prompts)
    stack.run()
    first = stack.first_ids.tolist()
    chain = [np.concatenate([[first[b]], rng.integers(0, V, 5)]) for b in range(B)]
    trees = [W.chain_tree(6)] * B
    inp = W.make_verify_inputs(3, "bf16", HQ, HKV, D, [37, 16], trees, page=PAGE, poison=False)
    dev = S.to_device(inp)
    dev.block_table, dev.prefix_len = pages.block_table, pages.length
    desc = S.make_desc("bf16", B, HQ, HKV, D, PAGE, 12, blocks, 12, 6, D ** -0.5, hint=192)
    draft = i32(np.concatenate(chain))
    verify = S.VerifyLayerStack(desc, dev, pools, model.w_qkv, model.w_o, model.lm, draft, inp.max_path, model.embedding[draft.long()], mlp=model.mlp)
    verify.run(compact=False)
    target = verify.target_ids.cpu().numpy().reshape(B, 6)
    hidden = wide(verify.final_hidden).reshape(B, 6, K)
    for b in range(B):
        _near(hidden[b], model.hidden_ref(model.embedding[np.concatenate([prompts[b], chain[b]])])[-6:])
    # the target's own tokens, where the chain goes on with them: sequence 0 accepts two nodes and sequence 1 all that are right
    for b, n in enumerate((2, 3)):
        for i in range(n - 1):
            chain[b][i + 1] = target[b][i]
            draft.copy_(i32(np.concatenate(chain)))
            verify.hidden[0].copy_(model.embedding[draft.long()])
            verify.run(compact=False)
            target = verify.target_ids.cpu().numpy().reshape(B, 6)
    verify.run()
    n = verify.accept_len.tolist()
    assert n[0] >= 2 and n[1] >= 3
    pages.length.copy_(verify.new_len)
    assert pages.length.tolist() == [37 + n[0], 16 + n[1]]
    more = [np.concatenate([[verify.bonus[b].item()], rng.integers(0, V, 9)]) for b in range(B)]
    offset = _load(stack, model, more)
    stack.run()
    hidden = wide(stack.final_hidden)
    for b in range(B):
        _near(hidden[offset[b]:offset[b + 1]], model.hidden_ref(model.embedding[np.concatenate([prompts[b], chain[b][:n[b]], more[b]])])[-10:])


def test_prompts_from_a_hip_graph(S):
    """A part of each prompt a replay, lengths and rows changing between them, against the eager run: the same bits everywhere."""
    rng, model, B, T, blocks = np.random.default_rng(8), Model(2), 3, 96, 60
    pages, pools = S.PagePool(B, PAGE, 16, blocks, T), model.pools(blocks)
    stack = _stack(S, model, pages, pools, B, T, 16, blocks)
    state = [pages.block_table, pages.length, pages.pages, pages.free_pages, pages.free_count] + [t for kv in pools for t in kv]
    _load(stack, model, [rng.integers(0, V, 5)] * B)
    pristine = [t.clone() for t in state]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        stack.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        stack.run()
    for t, t0 in zip(state, pristine):
        t.copy_(t0)
    for sizes in ([30, 1, 65], [20, 17, 0], [0, 0, 0], [16, 33, 40], [1, 1, 1]):
        offset = _load(stack, model, [rng.integers(0, V, n) for n in sizes])
        before = [t.clone() for t in state]
        stack.run()
        torch.cuda.synchronize()
        eager = [t.clone() for t in state + [stack.final_hidden[:offset[-1]], stack.first_ids, pages.slots]]
        for t, t0 in zip(state, before):
            t.copy_(t0)
        stack.first_ids.fill_(-7)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager, state + [stack.final_hidden[:offset[-1]], stack.first_ids, pages.slots]):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_pages_over_many_steps_of_a_graph(S):
    """Requests that come, grow, run out of pages and end, taken, advanced and given by one graph, against the oracle in step."""
    rng, B, blocks, max_blocks, reserve, most = np.random.default_rng(4), 9, 60, 14, 3, 200
    pages = S.PagePool(B, PAGE, max_blocks, blocks, most, reserve)
    offset, keep = i32([0] * (B + 1)), i32([0] * B)

    def step():
        pages.take(offset)
        pages.advance()
        torch.minimum(pages.length, keep, out=pages.length)
        pages.give(pages.length)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    length, have, table = np.zeros(B, int), np.zeros(B, int), pages.block_table.cpu().numpy()
    free = list(pages.free_pages[:pages.free_count.item()].cpu().numpy())
    assert sorted(free) == list(range(blocks))
    short = 0
    for i in range(25):
        rows = rng.integers(0, 50, B) * (rng.random(B) < 0.5)
        off = np.concatenate([[0], np.cumsum(rows)])
        if off[-1] > most:
            continue
        kept = np.where(rng.random(B) < 0.15, 0, 10 ** 6)
        offset.copy_(i32(off))
        keep.copy_(i32(kept))
        graph.replay()
        torch.cuda.synchronize()
        table, slots, length, have, granted, left = pages_take_ref(PAGE, max_blocks, blocks, reserve, length, off, have, np.asarray(free, int), table,
                                                                   np.full(most, -1))
        short += int((granted == 0).sum())
        free = free[:left]
        length = np.minimum(length, kept)
        assert np.array_equal(pages.slots.cpu().numpy(), slots) and np.array_equal(pages.granted.cpu().numpy(), granted)
        free, have = pages_give_ref(PAGE, length, have, table, list(free))
        n = len(free)
        assert pages.length.tolist() == list(length) and pages.pages.tolist() == list(have) and pages.free_count.tolist() == [n]
        assert np.array_equal(pages.block_table.cpu().numpy(), table) and pages.free_pages[:n].tolist() == free
        assert sorted(free + [t for b in range(B) for t in table[b, :have[b]]]) == list(range(blocks))  # nothing lost or given twice
    assert short > 0


def _sampled(S, seed=6):
    rng = np.random.default_rng(seed)
    inp = W.make_config(4, scale_down=8)
    B, T, vocab = inp.B, inp.total_nodes, 2048
    _, weight = W.make_lmhead_inputs(44, 1, inp.Hq * inp.D, vocab, dtype="bf16")
    dev, desc = S.to_device(inp), S.desc_for(inp)
    f32 = lambda x: torch.from_numpy(np.asarray(x, dtype=np.float32)).cuda()
    q = rng.random((T, vocab)) ** 6
    bits = lambda n: torch.from_numpy(rng.integers(-2 ** 31, 2 ** 31, n, dtype=np.int64).astype(np.int32)).cuda()
    had = np.where(rng.random((B, vocab)) < 0.05, rng.integers(1, 4, (B, vocab)), 0) + (rng.random((B, vocab)) < 0.1) * (1 << 30)
    temps = np.resize([0.7, 0.0, 1.1], B)
    rules = S.SamplingRules(i32(had), f32(np.stack([temps, rng.uniform(0.9, 1.3, B), rng.uniform(0, 0.5, B), rng.uniform(0, 0.5, B)], 1)),
                            i32(np.arange(B + 1) * 3), i32(rng.integers(0, vocab, 3 * B)), f32(rng.choice([-np.inf, 1.5], 3 * B)),
                            i32(rng.integers(-2 ** 31, 2 ** 31, (5, vocab // 32))), i32(rng.integers(-1, 5, T)))
    draft = i32(rng.integers(0, vocab, T))
    step = S.SampledVerifyStep(desc, dev, weight.cuda(), draft, f32(q / q.sum(1, keepdims=True)), bits(T), bits(B), inp.max_path, rules)
    return inp, step, rng, vocab


def test_a_sampled_step_against_the_oracle(S):
    """Its logits by the rules, its probabilities, what acceptance makes of them, and what is counted."""
    inp, step, rng, vocab = _sampled(S)
    r, had = step.rules, step.rules.counts.cpu().numpy().astype(np.int64)
    step.run()
    off, parent, draft = inp.node_offset.numpy(), inp.parent.numpy(), step.draft_ids.cpu().numpy()
    bias = [[(int(t), float(v)) for t, v in zip(r.bias_id[3 * b:3 * b + 3].tolist(), r.bias_value[3 * b:3 * b + 3].tolist())] for b in range(inp.B)]
    z = rules_logits_ref(W.widen(step.logits.cpu()), off, parent, draft, had, r.rules.cpu().numpy(), bias, r.mask.cpu().numpy().view(np.uint32),
                         r.mask_row.cpu().numpy())
    p = rules_probs_ref(z.astype(np.float32).astype(np.float64), off, r.rules.cpu().numpy())
    got = step.probs.cpu().numpy()
    # |z| < 64 here; five float32 operations and the division by T >= 0.7: 2^-24 * 64 * 12 / 0.7, and a sum of 2048
    assert np.abs(np.where(np.isfinite(z), z, 0)).max() < 64
    assert (np.abs(got - p) <= 1e-4 * p + 1e-37).all()
    u = lambda t: t.cpu().numpy().view(np.uint32)
    alen, path, toks, bonus = tree_accept_sample_ref(off, parent, draft, got, step.q_draft.cpu().numpy(), u(step.u_accept), u(step.u_bonus),
                                                     inp.max_path)
    same = step.accept_len.cpu().numpy() == alen
    assert same.mean() >= 0.9  # float32 sums of 2048 turn a draw that lies this close to a border
    for b in np.nonzero(same)[0]:
        assert np.array_equal(step.accept_path[b].cpu().numpy(), path[b]) and np.array_equal(step.out_tokens[b].cpu().numpy()[:alen[b] - 1], toks[b][:alen[b] - 1])
    for b, row in enumerate(step.out_tokens.cpu().numpy()):
        for t in row[row >= 0]:
            had[b, t] += 1
    assert np.array_equal(step.rules.counts.cpu().numpy(), had)


def test_sampled_steps_from_a_hip_graph(S):
    """Other random bits, rules, drafts and counts at each replay: the eager step's bits."""
    inp, step, rng, vocab = _sampled(S, 7)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step.run()
    outs = [step.logits, step.probs, step.accept_len, step.accept_path, step.out_tokens, step.bonus, step.new_len, step.rules.counts, step.dev.k_pool]
    for _ in range(4):
        step.u_accept.random_(-2 ** 31, 2 ** 31 - 1)
        step.u_bonus.random_(-2 ** 31, 2 ** 31 - 1)
        step.draft_ids.random_(0, vocab)
        step.rules.rules[:, 0].uniform_(0, 1.5)
        step.rules.mask_row.random_(-1, 5)
        counts, pool = step.rules.counts.clone(), step.dev.k_pool.clone()
        step.run()
        torch.cuda.synchronize()
        eager = [t.clone() for t in outs]
        step.rules.counts.copy_(counts)
        step.dev.k_pool.copy_(pool)
        step.probs.fill_(5)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager, outs):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_calls_on_two_streams_at_once(S):
    """Every call beside another of its kind, each with buffers of its own, handed the stream or found on the current one."""
    import paper_2509_18824_amd as hb
    from prompts import Prompts
    from test_gpu_requests import Rules, _pages, _take
    cases = [Prompts(31, "bf16", 8, 2, 128, 16, [900, 40], [200, 33]), Prompts(32, "f32", 4, 2, 64, 16, [700, 3], [50, 90])]
    rules = [Rules(33, "bf16", [60, 60, 40], 5000, 9, 5), Rules(34, "f32", [3, 8], 30000, 700, 5)]
    want = [(c.run(), r.run(), _take(_pages(9 + i, 12, 16, 90, 300, 0, 2))) for i, (c, r) in enumerate(zip(cases, rules))]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(4):
        made = []
        for i, (c, r, stream) in enumerate(zip(cases, rules, streams)):
            with torch.cuda.stream(stream):
                made.append((c.run(), r.run(), _take(_pages(9 + i, 12, 16, 90, 300, 0, 2))))
        torch.cuda.synchronize()
        for w, m in zip(want, made):
            for a, b in zip((*w[0], *w[1], *w[2].values()), (*m[0], *m[1], *m[2].values())):
                assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    # the stream as an argument: behind what fills the rows there, not behind the current stream
    k = torch.zeros((64, 4, 128), dtype=torch.bfloat16, device="cuda")
    pools = [torch.zeros((8, 4, 16, 128), dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    slots = i32(np.arange(64))
    torch.cuda.synchronize()
    with torch.cuda.stream(streams[0]):
        for _ in range(50):
            k.add_(1.0)
    hb.hb_kv_append(S.make_desc("bf16", 1, 4, 4, 128, 16, 1, 8, 0, 1, 1.0), k, k, slots, *pools, stream=streams[0])
    torch.cuda.synchronize()
    assert (pools[0][:4] == 50.0).all() and (pools[1][:4] == 50.0).all() and (pools[0][4:] == 0).all()
