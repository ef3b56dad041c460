"""What the 4-bit cache's calls refuse, on the host (no GPU)."""
import ctypes as C

import pytest
import torch

import paper_2509_18824_amd as hb
import paper_2509_18824_amd.step as S

L, P, ODD = hb.lib, C.c_void_p(0x1000), C.c_void_p(0x1008)


def _desc(**kw):
    base = dict(dtype="bf16", B=2, Hq=28, Hkv=4, D=128, page=16, max_blocks=64, num_blocks=200, total_nodes=120, max_nodes=60, softmax_scale=0.1)
    base.update(kw)
    return S.make_desc(**base)


def _attn(d, ptr=P, pool=P, ws=C.c_void_p(0x1000), ws_bytes=1 << 40):
    return L.hb_tree_verify_attn_kv4(C.byref(d), ptr, ptr, ptr, pool, pool, pool, pool, ptr, ptr, ptr, ptr, ptr, None, ws, ws_bytes, None)


def _append(d, n=8, rows=P, pool=P, ints=P):
    return L.hb_kv4_append(C.byref(d), n, rows, rows, pool, pool, pool, pool, ints, ints, ints, None, None, None, None, None)


def _compact(d, rows=P, pool=P, ints=P, max_path=6):
    return L.hb_kv4_compact(C.byref(d), rows, rows, pool, pool, pool, pool, ints, ints, ints, ints, ints, max_path, None, None, None, None, None, None)


def _read(d, n=8, rows=P, pool=P, ints=P):
    return L.hb_kv4_read(C.byref(d), n, pool, pool, pool, pool, ints, ints, ints, rows, rows, None)


def _weight(d, q=P, pool=P, path=P, max_path=6, decay=1.0, accept=P):
    return L.hb_kv4_attn_weight(C.byref(d), q, pool, pool, P, P, P, accept, path, max_path, P, decay, P, None)


def _evict(d, budget=100, recent=10, sinks=4, pool=P, ints=P, ws=P, ws_bytes=1 << 40):
    return L.hb_kv4_evict(C.byref(d), budget, recent, sinks, pool, pool, pool, pool, ints, ints, ints, P, P, P, P, P, None, ws, ws_bytes, None)


CALLS = [_attn, _append, _compact, _read, _weight, _evict]


@pytest.mark.parametrize("call", CALLS)
def test_shapes_that_no_call_takes(call):
    assert call(_desc(D=72)) == 2 and "multiple of 32" in hb.hb_last_error()
    assert call(_desc(D=288)) == 2
    assert call(_desc(Hq=30)) == 1
    assert call(_desc(page=0)) == 1
    assert call(_desc(B=20000)) == 2
    assert call(_desc(total_nodes=1 << 20)) == 2
    d = _desc()
    d.dtype = 5
    assert call(d) == 2
    assert call(_desc(), pool=None) == 1
    assert call(_desc(), pool=ODD) == 1 and "aligned" in hb.hb_last_error()
    assert call(_desc(B=0, total_nodes=0), pool=None) == 0


def test_attention():
    assert _attn(_desc(), ptr=None) == 1 and _attn(_desc(), ptr=ODD) == 1
    assert _attn(_desc(max_nodes=65)) == 2
    d = _desc(num_splits=4)
    need = hb.hb_tree_verify_attn_kv4_workspace_bytes(d)
    assert hb.hb_tree_verify_attn_kv4_num_splits(d) == 4 and need >= 120 * 28 * 4 * 130 * 4
    assert _attn(d, ws=None, ws_bytes=0) == 3 and _attn(d, ws_bytes=need - 1) == 3
    assert _attn(d, ws=C.c_void_p(0x1010)) == 3
    assert hb.hb_tree_verify_attn_kv4_workspace_bytes(_desc(D=72)) == 0 and hb.hb_tree_verify_attn_kv4_num_splits(_desc(D=72)) == 0
    assert hb.hb_tree_verify_attn_kv4_workspace_bytes(_desc(num_splits=1)) == 0


def test_rows():
    assert _append(_desc(), n=-1) == 1 and _append(_desc(), rows=None) == 1 and _append(_desc(), rows=ODD) == 1 and _append(_desc(), ints=None) == 1
    assert _append(_desc(), n=1 << 28) == 2
    # a prompt's rows are no tree's nodes
    assert _append(_desc(max_nodes=4096), rows=None) == 1
    assert _read(_desc(), n=-1) == 1 and _read(_desc(), rows=None) == 1 and _read(_desc(), rows=ODD) == 1 and _read(_desc(), ints=None) == 1
    assert _read(_desc(), n=0, rows=None, pool=None) == 0
    assert _compact(_desc(), max_path=0) == 1 and _compact(_desc(), rows=None) == 1 and _compact(_desc(), rows=ODD) == 1
    assert _compact(_desc(), ints=None) == 1 and _compact(_desc(), max_path=1 << 28) == 2


def test_weights():
    assert _weight(_desc(), decay=1.5) == 1 and _weight(_desc(), decay=-0.5) == 1 and _weight(_desc(), decay=float("nan")) == 1
    assert _weight(_desc(), path=None) == 1 and "together" in hb.hb_last_error()
    assert _weight(_desc(), max_path=0) == 1 and _weight(_desc(), q=None) == 1 and _weight(_desc(), q=ODD) == 1


def test_eviction():
    assert _evict(_desc(), budget=0) == 1 and _evict(_desc(), recent=-1) == 1 and _evict(_desc(), sinks=-1) == 1
    assert _evict(_desc(), budget=13) == 1 and "recent" in hb.hb_last_error()
    assert _evict(_desc(), budget=2147483647, recent=2147483647, sinks=2147483647) == 1
    assert _evict(_desc(), ints=None) == 1
    need = hb.hb_kv4_evict_workspace_bytes(_desc(), 100)
    assert need >= 8 * (2 * 100 + 1) * 4
    assert _evict(_desc(), ws_bytes=need - 1) == 3 and _evict(_desc(), ws=None) == 3 and _evict(_desc(), ws=C.c_void_p(0x1010)) == 3
    assert hb.hb_kv4_evict_workspace_bytes(_desc(), 0) == 0 and hb.hb_kv4_evict_workspace_bytes(_desc(D=72), 10) == 0


def test_the_binding_checks_types_and_shapes():
    d = _desc(Hq=4, Hkv=2, D=64, num_blocks=9, total_nodes=5, max_nodes=5)
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8)
    pool = [u8(9, 2, 16, 32), u8(9, 2, 16, 2), u8(9, 2, 16, 32), u8(9, 2, 16, 2)]
    rows, ints = torch.zeros((5, 2, 64), dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    table = torch.zeros((2, 64), dtype=torch.int32)
    slots, pos = torch.zeros(2, 2, 1024), torch.zeros((2, 2, 1024), dtype=torch.int32)
    with pytest.raises(ValueError):
        hb.hb_kv4_append(d, rows, rows[:4], *pool, table, ints, ints)
    with pytest.raises(hb.HbError):
        hb.hb_kv4_append(d, rows.half(), rows.half(), *pool, table, ints, ints)
    with pytest.raises(ValueError):
        hb.hb_kv4_append(d, rows.float(), rows.float(), *pool, table, ints, ints)
    with pytest.raises(ValueError):
        hb.hb_kv4_append(d, rows, rows, pool[0].int(), *pool[1:], table, ints, ints)
    with pytest.raises(ValueError):
        hb.hb_kv4_append(d, rows, rows, pool[1], pool[0], *pool[2:], table, ints, ints)
    with pytest.raises(ValueError):
        hb.hb_kv4_append(d, rows, rows, *pool, table.long(), ints, ints)
    with pytest.raises(ValueError):
        hb.hb_kv4_append(d, rows, rows, *pool, table, ints, ints, weight=slots[:, :, :5])
    with pytest.raises(ValueError):
        hb.hb_kv4_append(d, rows, rows, *pool, table, ints, ints, pos=slots)
    with pytest.raises(ValueError):
        hb.hb_kv4_compact(d, rows[:3], rows[:3], *pool, table, ints, ints, ints, table, 6)
    with pytest.raises(ValueError):
        hb.hb_kv4_append(d, rows, rows, *[x.transpose(0, 1).contiguous().transpose(0, 1) for x in pool], table, ints, ints)  # not dense
    with pytest.raises(ValueError):
        hb.hb_kv4_evict(d, 100, 1, 1, *pool, table, ints, ints, slots, pos, slots, pos, pos, None, None)


def test_the_binding_checks_what_weights_are_made_from():
    d = _desc(Hq=4, Hkv=2, D=64, num_blocks=9, total_nodes=5, max_nodes=5)
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8)
    codes, scales, table = u8(9, 2, 16, 32), u8(9, 2, 16, 2), torch.zeros((2, 64), dtype=torch.int32)
    q, lse, ints, slots = torch.zeros((5, 4, 64), dtype=torch.bfloat16), torch.zeros(5, 4), torch.zeros(3, dtype=torch.int32), torch.zeros(2, 2, 1024)
    call = lambda q, lse: hb.hb_kv4_attn_weight(d, q, codes, scales, table, ints, ints, ints, ints, 1, lse, 1.0, slots)
    for bad in (q.float(), q[:4]):
        with pytest.raises(ValueError):
            call(bad, lse)
    for bad in (lse.double(), lse[:4]):
        with pytest.raises(ValueError):
            call(q, bad)
