"""What the Python binding of the 4-bit cache's calls refuses before the library sees it (no GPU)."""
import pytest
import torch

import paper_2509_18824_amd as hb
import paper_2509_18824_amd.step as S

B, HQ, HKV, D, PAGE, BLOCKS, PER_SEQ, NODES, MAX_PATH, BUDGET, ROWS = 3, 4, 2, 64, 16, 9, 4, 7, 5, 10, 6


def _i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def _desc():
    return S.make_desc(dtype="bf16", B=B, Hq=HQ, Hkv=HKV, D=D, page=PAGE, max_blocks=PER_SEQ, num_blocks=BLOCKS, total_nodes=NODES, max_nodes=4,
                       softmax_scale=0.1)


def _calls():
    """name -> (call, its integer arguments as they have to be at least)"""
    u8 = lambda n: torch.zeros((BLOCKS, HKV, PAGE, n), dtype=torch.uint8)
    pool = [u8(D // 2), u8(D // 32), u8(D // 2), u8(D // 32)]
    rows, nodes = torch.zeros((ROWS, HKV, D), dtype=torch.bfloat16), torch.zeros((NODES, HKV, D), dtype=torch.bfloat16)
    q, lse = torch.zeros((NODES, HQ, D), dtype=torch.bfloat16), torch.zeros(NODES, HQ)
    weight, pos = torch.zeros(B, HKV, PER_SEQ * PAGE), _i32(B, HKV, PER_SEQ * PAGE)
    base = {"block_table": _i32(B, PER_SEQ), "prefix_len": _i32(B)}
    path = {"accept_len": _i32(B), "accept_path": _i32(B, MAX_PATH)}
    ws = torch.zeros(1 << 20, dtype=torch.uint8)
    d = _desc()
    return {
        "append": (lambda a: hb.hb_kv4_append(d, rows, rows, *pool, a["block_table"], a["prefix_len"], a["row_offset"], a["seq_len"], weight, pos, a["new_len"]),
                   {**base, "row_offset": _i32(B + 1), "seq_len": _i32(B), "new_len": _i32(B)}),
        "compact": (lambda a: hb.hb_kv4_compact(d, nodes, nodes, *pool, a["block_table"], a["prefix_len"], a["node_offset"], a["accept_len"], a["accept_path"],
                                                MAX_PATH, a["seq_len"], weight, pos, a["out_slots"], a["new_len"]),
                    {**base, **path, "node_offset": _i32(B + 1), "seq_len": _i32(B), "out_slots": _i32(B, MAX_PATH), "new_len": _i32(B)}),
        "read": (lambda a: hb.hb_kv4_read(d, *pool, a["block_table"], a["first"], a["row_offset"], rows, rows),
                 {"block_table": _i32(B, PER_SEQ), "first": _i32(B), "row_offset": _i32(B + 1)}),
        "attention": (lambda a: hb.hb_tree_verify_attn_kv4(d, q, nodes, nodes, *pool, a["block_table"], a["prefix_len"], a["node_offset"], a["parent"], q, lse, ws),
                      {**base, "node_offset": _i32(B + 1), "parent": _i32(NODES)}),
        "weight": (lambda a: hb.hb_kv4_attn_weight(d, q, pool[0], pool[1], a["block_table"], a["prefix_len"], a["node_offset"], a["accept_len"], a["accept_path"],
                                                   MAX_PATH, lse, 1.0, weight),
                   {**base, **path, "node_offset": _i32(B + 1)}),
        "evict": (lambda a: hb.hb_kv4_evict(d, BUDGET, 1, 1, *pool, a["block_table"], a["prefix_len"], a["seq_len"], weight, pos, weight, pos,
                                            _i32(B, HKV, BUDGET), a["new_len"], ws),
                  {**base, "seq_len": _i32(B), "new_len": _i32(B)}),
    }


EACH = [(name, arg) for name, (_, args) in _calls().items() for arg in args]


@pytest.fixture
def reached(monkeypatch):
    """The library's calls are recorded in place of being made."""
    made = []

    class Recorder:
        def __getattr__(self, name):
            return lambda *args: made.append(name) or 0
    monkeypatch.setattr(hb.binding, "lib", Recorder())
    monkeypatch.setattr(hb.binding, "_stream", lambda stream: None)
    return made


@pytest.mark.parametrize("name,arg", EACH)
def test_integers_of_another_type(reached, name, arg):
    call, args = _calls()[name]
    call(args)
    assert len(reached) == 1
    for other in (args[arg].long(), args[arg].float(), args[arg].short()):
        with pytest.raises(ValueError):
            call({**args, arg: other})
    assert len(reached) == 1


@pytest.mark.parametrize("name,arg", EACH)
def test_integers_that_are_too_few(reached, name, arg):
    """What the kernels would read or write behind."""
    call, args = _calls()[name]
    flat = args[arg].reshape(-1)
    call({**args, arg: flat})
    call({**args, arg: torch.cat((flat, flat))})  # more than the call needs
    assert len(reached) == 2
    for few in (flat[:-1], flat[:0]):
        with pytest.raises(ValueError):
            call({**args, arg: few})
    assert len(reached) == 2
