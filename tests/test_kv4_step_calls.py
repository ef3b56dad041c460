"""The calls that the 4-bit cache's step class makes, recorded in place of the library (no GPU)."""
import torch

import workloads as W
import paper_2509_18824_amd.step as S


def test_calls_of_a_step_and_an_eviction(monkeypatch):
    made = []
    for name in dir(S.hb):
        if name.startswith("hb_") and not name.endswith(("_bytes", "_splits", "_rows", "_error", "_version")):
            monkeypatch.setattr(S.hb, name, lambda *args, _name=name, **kwargs: made.append((_name[3:], args)))
    inp = W.make_verify_inputs(3, "bf16", 4, 2, 128, [20, 9], [W.chain_tree(3), W.seeded_tree(1, n_nodes=12, levels=3)], poison=False)
    dev, desc = S.to_device(inp, "cpu"), S.desc_for(inp)
    step = S.Kv4VerifyStep(desc, dev, S.kv4_pool(inp.num_blocks, 2, 16, 128, "cpu"), torch.empty(50, 512, dtype=torch.bfloat16),
                           torch.zeros(inp.total_nodes, dtype=torch.int32), 4, 16, 4, 2)
    step.run()
    assert [c for c, _ in made] == ["tree_verify_attn_kv4", "lmhead_accept", "kv4_attn_weight", "kv4_compact"]
    # the weights are those of the prefix that the nodes saw: they are taken before the append, and nobody appends in 16 bits
    assert len(made[1][1]) == 13
    step.new_len.copy_(torch.tensor([22, 12], dtype=torch.int32))
    step.accept_len.copy_(torch.tensor([2, 3], dtype=torch.int32))
    step.advance()
    assert dev.prefix_len.tolist() == [22, 12] and step.seq_len.tolist() == [22, 12]
    del made[:]
    step.evict()
    (name, args), = made
    assert name == "kv4_evict" and args[1:4] == (16, 4, 2) and args[11] is args[13] and args[12] is args[14]
    assert dev.prefix_len is not step.new_len
