"""What the calls for pages, prompts and sampling rules refuse, on the host (no GPU)."""
import ctypes as C

import pytest
import torch

import paper_2509_18824_amd as hb
import paper_2509_18824_amd.step as S

L, ODD = hb.lib, C.c_void_p(0x1008)
P = [C.c_void_p(0x100000 * (i + 1)) for i in range(16)]  # far apart


def _desc(**kw):
    base = dict(dtype="bf16", B=2, Hq=28, Hkv=4, D=128, page=16, max_blocks=64, num_blocks=200, total_nodes=120, max_nodes=60, softmax_scale=0.1)
    base.update(kw)
    return S.make_desc(**base)


def _take(B=2, page=16, max_blocks=8, blocks=20, rows=10, reserve=0, **at):
    names = ("prefix_len", "row_offset", "pages", "free_pages", "free_count", "block_table", "slots", "new_len", "pages_out", "granted", "left")
    return L.hb_pages_take(B, page, max_blocks, blocks, rows, reserve, *[at.get(n, P[i]) for i, n in enumerate(names)], None)


def _give(B=2, page=16, max_blocks=8, blocks=20, **at):
    names = ("keep_len", "pages", "block_table", "free_pages", "free_count", "pages_out", "free_now")
    return L.hb_pages_give(B, page, max_blocks, blocks, *[at.get(n, P[i]) for i, n in enumerate(names)], None)


@pytest.mark.parametrize("call", [_take, _give])
def test_pages(call):
    assert call(B=-1) == 1 and call(page=0) == 1 and call(max_blocks=0) == 1 and call(blocks=0) == 1
    assert call(B=8193) == 2 and call(max_blocks=1 << 28) == 2 and call(page=1 << 10, blocks=1 << 22) == 2
    assert call(B=0, free_pages=None) == 0
    for name in ("pages", "free_pages", "free_count", "block_table", "pages_out"):
        assert call(**{name: None}) == 1, name
    # what is written apart from what is read
    assert call(pages_out=P[1] if call is _give else P[2]) == 1 and "pages_out" in hb.hb_last_error()


def test_pages_that_are_taken():
    assert _take(rows=-1) == 1 and _take(reserve=-1) == 1
    assert _take(left=P[4]) == 1 and "free_left" in hb.hb_last_error()
    assert _take(new_len=P[0]) == 1 and _take(slots=P[5]) == 1
    assert _take(granted=P[8]) == 1 and "granted" in hb.hb_last_error()
    assert _take(block_table=C.c_void_p(P[3].value + 4 * 19)) == 1
    assert _give(free_now=P[4]) == 1 and _give(free_pages=P[2]) == 1


def _append(d, n=8, rows=P[0], slots=P[1], pool=P[2]):
    return L.hb_kv_append(C.byref(d), n, rows, rows, slots, pool, pool, None)


def _attn(d, q=P[0], kv=P[1], pool=P[2], ints=P[3], prefix=P[4], out=P[5], ws=P[6], ws_bytes=1 << 40):
    return L.hb_prompt_attn(C.byref(d), q, kv, kv, pool, pool, ints, prefix, ints, out, None, ws, ws_bytes, None)


@pytest.mark.parametrize("call", [_append, _attn])
def test_shapes_that_no_call_takes(call):
    assert call(_desc(D=100)) == 2 and call(_desc(D=264)) == 2 and call(_desc(Hq=30)) == 1 and call(_desc(page=0)) == 1
    assert call(_desc(Hq=65536 * 2, Hkv=65536)) == 2
    d = _desc()
    d.dtype = 4
    assert call(d) == 2
    assert call(_desc(), pool=None) == 1 and call(_desc(), pool=ODD) == 1 and "aligned" in hb.hb_last_error()


def test_append():
    assert _append(_desc(), n=-1) == 1 and _append(_desc(), n=0, rows=None) == 0
    assert _append(_desc(), rows=None) == 1 and _append(_desc(), slots=None) == 1 and _append(_desc(), rows=ODD) == 1
    assert _append(_desc(page=1 << 20, max_blocks=1, num_blocks=1 << 12)) == 2


def test_prompt_attention():
    assert _attn(_desc(B=0, total_nodes=0), q=None) == 0 and _attn(_desc(B=0), q=None) == 0
    for name in ("q", "kv", "out"):
        assert _attn(_desc(), **{name: None}) == 1 and _attn(_desc(), **{name: ODD}) == 1, name
    assert _attn(_desc(total_nodes=1 << 27)) == 2
    assert _attn(_desc(algo=hb.HB_ATTN_MFMA, dtype="f32")) == 2 and _attn(_desc(algo=hb.HB_ATTN_MFMA, D=72)) == 2
    assert _attn(_desc(algo=hb.HB_ATTN_MFMA, page=48)) == 2 and _attn(_desc(algo=hb.HB_ATTN_MFMA, softmax_scale=-1.0)) == 2
    d = _desc(num_splits=4)
    need = hb.hb_prompt_attn_workspace_bytes(d)
    assert need >= 120 * 28 * 4 * 130 * 4
    assert _attn(d, ws=None, ws_bytes=0) == 3 and _attn(d, ws_bytes=need - 1) == 3 and _attn(d, ws=ODD) == 3
    assert hb.hb_prompt_attn_workspace_bytes(_desc(num_splits=1)) == 0 and hb.hb_prompt_attn_workspace_bytes(_desc(D=100)) == 0
    # the most that a descriptor may ask for stays bounded
    for rows in (0, 1, 7, 1000, 1 << 20, 1 << 25):
        for B in (1, 16, 4096):
            n = hb.hb_prompt_attn_workspace_bytes(_desc(B=B, total_nodes=rows, max_blocks=1 << 20, num_blocks=1 << 20))
            assert n < 1 << 30, (rows, B, n)


def _rules(call=L.hb_rules_probs, dtype=1, B=2, nodes=8, T=16, V=1000, n_bias=3, masks=4, **at):
    names = ("logits", "node_offset", "parent", "draft_ids", "counts", "rules", "bias_offset", "bias_id", "bias_value", "mask", "mask_row", "out", "ws")
    a = {n: at.get(n, P[i]) for i, n in enumerate(names)}
    head = [dtype, B, nodes, T, V] + [a[n] for n in names[:7]] + [n_bias, a["bias_id"], a["bias_value"], masks, a["mask"], a["mask_row"], a["out"]]
    return call(*head, a["ws"], at.get("ws_bytes", 1 << 30), None) if call is L.hb_rules_probs else call(*head, None)


@pytest.mark.parametrize("call", [L.hb_rules_probs, L.hb_rules_logits])
def test_rules(call):
    r = lambda **kw: _rules(call, **kw)
    assert r(dtype=2) == 2 and r(B=-1) == 1 and r(T=-1) == 1 and r(V=0) == 1 and r(nodes=0) == 1 and r(nodes=65) == 2 and r(V=(1 << 30) + 1) == 2
    assert r(T=0, logits=None) == 0 and r(B=0, logits=None) == 0
    for name in ("logits", "out"):
        assert r(**{name: None}) == 1, name
    for name in ("logits", "out", "counts", "rules", "mask"):
        assert r(**{name: ODD}) == 1 and "aligned" in hb.hb_last_error(), name
    assert r(parent=None) == 1 and r(draft_ids=None) == 1 and r(node_offset=None) == 1
    assert r(node_offset=None, parent=None, draft_ids=None) == 1 and "one row" in hb.hb_last_error()  # 16 rows of 2 sequences
    assert r(bias_offset=None) == 1 and r(bias_id=None) == 1 and r(bias_value=None) == 1 and r(n_bias=-1) == 1
    assert r(mask=None) == 1 and r(mask_row=None) == 1 and r(masks=-1) == 1


def test_probabilities_have_a_workspace_and_a_place_of_their_own():
    need = hb.hb_rules_probs_workspace_bytes(16, 1000)
    assert need >= 16 * 16 and hb.hb_rules_probs_workspace_bytes(0, 1000) == 0 and hb.hb_rules_probs_workspace_bytes(3, 0) == 0
    assert _rules(ws=None) == 3 and _rules(ws_bytes=need - 1) == 3 and _rules(ws=ODD) == 3
    assert _rules(dtype=0, out=P[0]) == 1 and "probs" in hb.hb_last_error()


def test_counting():
    c = lambda B=2, V=100, n=10, off=P[0], tokens=P[1], prompt=0, counts=P[2]: L.hb_rules_count(B, V, n, off, tokens, prompt, counts, None)
    assert c(B=-1) == 1 and c(n=-1) == 1 and c(V=0) == 1 and c(prompt=2) == 1 and c(tokens=None) == 1 and c(counts=None) == 1
    assert c(n=0, tokens=None) == 0 and c(B=0, tokens=None) == 0 and c(n=11, off=None) == 1


def test_the_binding_refuses_other_types_and_shapes():
    i, f = (lambda *s: torch.zeros(s, dtype=torch.int32)), (lambda *s: torch.zeros(s))
    table, free = i(2, 8), i(20)
    with pytest.raises(ValueError):
        hb.hb_pages_take(16, 0, i(2).long(), i(3), i(2), free, i(1), table, i(4), i(2), i(2), i(2), i(1))
    with pytest.raises(ValueError):
        hb.hb_pages_take(16, 0, i(2), i(2), i(2), free, i(1), table, i(4), i(2), i(2), i(2), i(1))
    with pytest.raises(ValueError):
        hb.hb_pages_give(16, i(2), i(2), i(8, 2).T, free, i(1), i(2), i(1))
    d = _desc(dtype="f32", B=1, Hq=4, Hkv=2, D=8, page=4, max_blocks=2, num_blocks=3, total_nodes=5)
    rows, pool = f(5, 2, 8), f(3, 2, 4, 8)
    for bad in (f(5, 2, 4), rows.bfloat16()):
        with pytest.raises((ValueError, hb.HbError)):
            hb.hb_kv_append(d, bad, bad, i(5), pool, pool.clone())
    with pytest.raises(ValueError):
        hb.hb_kv_append(d, rows, rows, i(4), pool, pool.clone())
    with pytest.raises(ValueError):
        hb.hb_kv_append(d, rows, rows, i(5), f(2, 2, 4, 8), pool)
    q = f(5, 4, 8)
    for bad in (dict(q=f(4, 4, 8)), dict(k=f(4, 2, 8)), dict(pool=f(1)), dict(lens=i(0)), dict(off=i(1)), dict(lse=f(3)), dict(out=q.bfloat16())):
        a = dict(q=q, k=rows, pool=pool, lens=i(1), off=i(2), lse=None, out=q.clone()) | bad
        with pytest.raises((ValueError, hb.HbError)):
            hb.hb_prompt_attn(d, a["q"], a["k"], a["k"], a["pool"], a["pool"], i(1, 2), a["lens"], a["off"], a["out"], a["lse"])
    z = f(4, 33)
    ok = dict(node_offset=i(3), parent=i(4), draft_ids=i(4), counts=i(2, 33), rules=f(2, 4), bias_offset=i(3), bias_id=i(1), bias_value=f(1),
              mask=i(4, 2), mask_row=i(4))
    for bad in (dict(rules=f(2, 3)), dict(counts=i(2, 32)), dict(bias_value=f(2)), dict(mask=i(4, 1)), dict(mask_row=i(3)), dict(parent=i(3)),
                dict(node_offset=i(3).long())):
        with pytest.raises(ValueError):
            hb.hb_rules_logits(z, 4, **(ok | bad), out=z.clone())
    with pytest.raises(ValueError):
        hb.hb_rules_logits(z, 4, **ok, out=z.bfloat16())
    with pytest.raises(ValueError):
        hb.hb_rules_probs(z.bfloat16(), 4, **ok, probs=z.bfloat16(), workspace=None)


def test_what_is_written_has_a_place_of_its_own():
    assert _attn(_desc(), out=P[0]) == 1 and "out" in hb.hb_last_error()
    d = _desc()
    lse = lambda at: L.hb_prompt_attn(C.byref(d), P[0], P[1], P[1], P[2], P[2], P[3], P[4], P[3], P[5], at, P[6], 1 << 40, None)
    assert lse(P[0]) == 1 and "lse" in hb.hb_last_error()
    assert lse(P[5]) == 1 and "overlap" in hb.hb_last_error()
    assert _attn(_desc(num_splits=4), ws=P[0]) == 1 and "workspace" in hb.hb_last_error()
    assert _rules(L.hb_rules_logits, out=C.c_void_p(P[0].value + 16)) == 1 and "out" in hb.hb_last_error()  # neither in place nor apart
    assert _rules(ws=P[0]) == 1 and "workspace" in hb.hb_last_error()
