"""The library calls that the request classes make, recorded in place of the library (no GPU)."""
import pytest
import torch

import workloads as W
import paper_2509_18824_amd.step as S
from test_step_calls import calls  # noqa: F401  (the fixture that records)


def _prompts(n_layers, whole, norm_f=True):
    t = lambda *shape: torch.zeros(shape, dtype=torch.bfloat16)
    K, F, T = 256, 64, 20
    desc = S.make_desc("bf16", 3, 2, 1, 128, 16, 4, 9, T, 1, 0.1)
    pools = [(t(9, 1, 16, 128), t(9, 1, 16, 128))] * n_layers
    mlp = dict(norm1=[t(K)] * n_layers, norm2=[t(K)] * n_layers, w_gate_up=[t(2 * F, K)] * n_layers, w_down=[t(K, F)] * max(n_layers, 1),
               eps=1e-6) if whole else None
    if whole and norm_f:
        mlp["norm_f"] = t(K)
    pages = S.PagePool(3, 16, 4, 9, T, device="cpu")
    return S.PromptLayerStack(desc, pages, pools, [t(4 * 128, K)] * max(n_layers, 1), [t(K, K)] * max(n_layers, 1), t(50, K),
                              torch.tensor([0, 7, 7, 11], dtype=torch.int32), t(T, K), mlp=mlp)


@pytest.mark.parametrize("n_layers,whole,norm_f", [(2, True, True), (2, True, False), (3, False, False), (0, True, True), (0, True, False), (0, False, False)])
def test_a_prompt_stack(calls, n_layers, whole, norm_f):
    stack = _prompts(n_layers, whole, norm_f)
    stack.pages.length.copy_(torch.tensor([4, 9, 30]))
    stack.run()
    layer = ["qkv_rope_project_ws", "prompt_attn", "kv_append"] + (["out_project_norm_ws", "swiglu_project"] if whole else ["out_project_ws"])
    names = ["pages_take", "rope_table"] + (["rmsnorm"] if whole and (n_layers or norm_f) else [])
    for l in range(n_layers):
        names += layer + ([("out_project_norm_ws" if l + 1 < n_layers or norm_f else "out_project_ws")] if whole else [])
    assert [c for c, _ in calls] == names + ["lmhead_argmax"]
    # positions behind what is cached; rows behind the last sequence have any
    assert calls[1][1][2].tolist()[:11] == [4, 5, 6, 7, 8, 9, 10, 30, 31, 32, 33] and calls[1][1][2].dtype is torch.int32
    assert stack.first_ids[1] == -1


def test_a_page_pool(calls):
    pages = S.PagePool(3, 16, 4, 9, 20, reserve=5, device="cpu")
    offset = torch.tensor([0, 1, 2, 3], dtype=torch.int32)
    pages.slots.fill_(7)
    pages.take(offset)
    pages.give(pages.length)
    assert [c for c, _ in calls] == ["pages_take", "pages_give"] and calls[0][1][:2] == (16, 5)
    assert pages.slots.tolist() == [-1] * 20 and sorted(pages.free_pages.tolist()) == list(range(9))


@pytest.mark.parametrize("compact,counts", [(True, True), (False, True), (True, False)])
def test_a_sampled_step(calls, compact, counts):
    inp = W.make_verify_inputs(3, "bf16", 4, 2, 128, [20, 9], [W.chain_tree(3), W.seeded_tree(1, n_nodes=12, levels=3)], poison=False)
    dev, desc, T = S.to_device(inp, "cpu"), S.desc_for(inp), inp.total_nodes
    i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32)
    step = S.SampledVerifyStep(desc, dev, torch.empty(50, 512, dtype=torch.bfloat16), i32(T), torch.zeros(T, 50), i32(T), i32(2), inp.max_path,
                               S.SamplingRules(counts=i32(2, 50) if counts else None))
    step.run(compact=compact)
    assert [c for c, _ in calls] == (["tree_verify_attn", "out_project_ws", "rules_probs", "tree_accept_sample"]
                                     + (["kv_compact"] if compact else []) + (["rules_count"] if counts else []))
