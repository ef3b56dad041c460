"""Pins of the oracle of pages, prompts and sampling rules (no GPU)."""
import numpy as np
import pytest
import torch

from oracle import pages_give_ref, pages_take_ref, prompt_attn_ref, rules_logits_ref, rules_probs_ref, tree_attn_ref


def _prompt_inputs(seed, lens, rows, Hq=4, Hkv=2, D=8, page=4):
    rng = np.random.default_rng(seed)
    used = [-(-n // page) for n in lens]
    order = rng.permutation(sum(used) + 1)
    table = np.full((len(lens), max(max(used), 1)), -1)
    at = 0
    for b, n in enumerate(used):
        table[b, :n] = order[at:at + n]
        at += n
    off = np.concatenate([[0], np.cumsum(rows)])
    r = lambda *s: rng.standard_normal(s)
    return r(off[-1], Hq, D), r(off[-1], Hkv, D), r(off[-1], Hkv, D), r(len(order), Hkv, page, D), r(len(order), Hkv, page, D), table, lens, off


def test_prompt_attention_is_causal_attention_of_the_library():
    q, k, v, *_ , off = _prompt_inputs(1, [0], [9])
    out, lse = prompt_attn_ref(q, k, v, None, None, None, None, off, 0.3)
    t = lambda x: torch.from_numpy(x).transpose(0, 1)
    want = torch.nn.functional.scaled_dot_product_attention(t(q), t(k).repeat_interleave(2, 0), t(v).repeat_interleave(2, 0), is_causal=True, scale=0.3)
    np.testing.assert_allclose(out, want.transpose(0, 1).numpy(), atol=1e-12)
    np.testing.assert_allclose(lse[0], 0.3 * np.einsum("hd,hd->h", q[0], k[0].repeat(2, 0)), atol=1e-12)  # one key


def test_a_prompt_is_a_chain():
    x = _prompt_inputs(2, [5, 0, 11], [3, 0, 6])
    q, k, v, kp, vp, table, lens, off = x
    parent = np.concatenate([np.arange(n) - 1 for n in (3, 0, 6)])
    want = tree_attn_ref(q, k, v, kp, vp, table, lens, off, parent, 0.4)
    got = prompt_attn_ref(q, k, v, kp, vp, table, lens, off, 0.4)
    for a, b in zip(got, want):
        np.testing.assert_allclose(a, b, atol=1e-12)


def test_a_part_of_a_prompt_over_what_is_cached_is_the_whole_prompt():
    q, k, v, *_, off = _prompt_inputs(3, [0], [12])
    whole, _ = prompt_attn_ref(q, k, v, None, None, None, None, off, 0.5)
    pool = [np.full((3, 2, 4, 8), np.nan) for _ in range(2)]
    for p in range(7):
        pool[0][2 - p // 4, :, p % 4], pool[1][2 - p // 4, :, p % 4] = k[p], v[p]
    part, _ = prompt_attn_ref(q[7:], k[7:], v[7:], *pool, [[2, 1]], [7], [0, 5], 0.5)
    np.testing.assert_allclose(part, whole[7:], atol=1e-12)


def test_pages_are_taken_in_order_and_given_back():
    table = np.full((4, 3), -1)
    table[1, 0] = 9
    got = pages_take_ref(4, 3, 10, 1, [0, 3, 0, 8], [0, 5, 6, 6, 12], [0, 1, 0, 0], [1, 2, 3, 4, 5], table, np.full(12, -2))
    t, slots, new_len, have, granted, left = got
    # 5 + 1 positions: two pages; 3 + 1 + 1: two, one is there; 0 + 0 + 1: one; the last wants four pages, of three at most
    assert t.tolist() == [[5, 4, -1], [9, 3, -1], [2, -1, -1], [-1, -1, -1]]
    assert slots.tolist() == [20, 21, 22, 23, 16, 39] + [-1] * 6
    assert new_len.tolist() == [5, 4, 0, 8] and have.tolist() == [2, 2, 1, 0] and granted.tolist() == [1, 1, 1, 0] and left == 1
    free, keep = pages_give_ref(4, [0, 3, 0, 0], have, t, [1])
    assert free == [1, 2, 3, 4, 5] and keep.tolist() == [0, 1, 0, 0]


def test_when_pages_run_out_only_those_go_on_that_need_none():
    table = np.full((4, 4), -1)
    table[3, 0] = 7
    _, slots, new_len, have, granted, left = pages_take_ref(4, 4, 8, 0, [0, 0, 0, 2], [0, 4, 16, 20, 22], [0, 0, 0, 1], [1, 2, 3], table, np.zeros(22))
    assert granted.tolist() == [1, 0, 0, 1] and left == 2 and new_len.tolist() == [4, 0, 0, 4] and have.tolist() == [1, 0, 0, 1]
    assert slots[20:].tolist() == [30, 31] and (slots[4:20] == -1).all()


def test_rules_by_hand():
    # tokens 0 .. 4; the output had token 1 twice, the prompt token 2; the path (below the root) holds 1 and 4
    counts = np.array([[0, 2, 1 << 30, 0, 0]])
    logits = np.array([[1.0, 2.0, -3.0, 0.5, 4.0]] * 3)
    rules = [[0.5, 2.0, 0.25, 0.125]]
    mask = np.array([[0b10111]], dtype=np.uint32)
    z = rules_logits_ref(logits, [0, 3], [-1, 0, 1], [3, 1, 4], counts, rules, [[(0, 0.5), (0, 0.25)]], mask, [-1, 0, 7])
    np.testing.assert_allclose(z[0], [1.75, 1.0 - 0.5, -6.0, 0.5, 4.0])                 # the root's own token is counted already
    np.testing.assert_allclose(z[1], [1.75, 1.0 - 0.625, -6.0, -np.inf, 4.0])           # token 1 three times, 3 forbidden
    np.testing.assert_allclose(z[2], [1.75, 1.0 - 0.625, -6.0, 0.5, 2.0 - 0.375])       # and 4 once; mask 7 is none
    p = rules_probs_ref(z, [0, 3], rules)
    np.testing.assert_allclose(p[0], torch.softmax(torch.tensor(z[0]) / 0.5, 0).numpy())
    assert p[1, 3] == 0


def test_probabilities_at_the_borders():
    z = np.array([[1.0, 3.0, 3.0], [-np.inf] * 3, [np.inf, 0.0, np.inf]])
    p = rules_probs_ref(z, [0, 1, 2, 3], [[0.0, 1, 0, 0]] + [[1.0, 1, 0, 0]] * 2)
    assert p.tolist() == [[0, 1, 0], [0, 0, 0], [0.5, 0, 0.5]]
    assert rules_logits_ref([[np.nan, 1.0]], [0, 1], None, None, None, None, None, None, None).tolist() == [[-np.inf, 1.0]]


@pytest.mark.parametrize("seed", range(3))
def test_without_rules_probabilities_are_the_softmax(seed):
    x = np.random.default_rng(seed).standard_normal((4, 33))
    z = rules_logits_ref(x, [0, 4], [-1, 0, 1, 0], [1, 2, 3, 4], None, None, None, None, None)
    np.testing.assert_allclose(rules_probs_ref(z, [0, 4], None), torch.softmax(torch.from_numpy(x), 1).numpy(), atol=1e-15)
