"""Lengths and slots that a call of the 4-bit cache writes while it reads its lengths, offsets and paths: memory in common is refused,
on the host (no GPU: every call here ends in the checks)."""
import ctypes as C

import pytest

import paper_2509_18824_amd as hb
import paper_2509_18824_amd.step as S

L, P, ODD = hb.lib, C.c_void_p(0x1000), C.c_void_p(0x1008)
B, MAX_PATH = 2, 6
# where the integer arguments of a call lie: apart, unless a test moves one
AT = {"prefix_len": 0x20000, "seq_len": 0x21000, "offset": 0x22000, "accept_len": 0x23000, "accept_path": 0x24000, "new_len": 0x25000, "out_slots": 0x26000}
BYTES = {"prefix_len": 4 * B, "seq_len": 4 * B, "offset": 4 * (B + 1), "accept_len": 4 * B, "accept_path": 4 * B * MAX_PATH, "new_len": 4 * B,
         "out_slots": 4 * B * MAX_PATH}


def _desc():
    return S.make_desc(dtype="bf16", B=B, Hq=28, Hkv=4, D=128, page=16, max_blocks=64, num_blocks=200, total_nodes=120, max_nodes=60, softmax_scale=0.1)


def _call(name, at, d=None):
    """Ends with what comes behind the check of overlaps: rows that are not aligned, a workspace that is too small."""
    p, d = {k: C.c_void_p(v) for k, v in at.items()}, d or _desc()
    if name == "append":
        return L.hb_kv4_append(C.byref(d), 8, ODD, ODD, P, P, P, P, P, p["prefix_len"], p["offset"], p["seq_len"], None, None, p["new_len"], None)
    if name == "compact":
        return L.hb_kv4_compact(C.byref(d), ODD, ODD, P, P, P, P, P, p["prefix_len"], p["offset"], p["accept_len"], p["accept_path"], MAX_PATH,
                                p["seq_len"], None, None, p["out_slots"], p["new_len"], None)
    return L.hb_kv4_evict(C.byref(d), 100, 10, 4, P, P, P, P, P, p["prefix_len"], p["seq_len"], P, P, P, P, P, p["new_len"], P, 8, None)


READS = {"append": ["prefix_len", "seq_len", "offset"], "compact": ["prefix_len", "seq_len", "offset", "accept_len", "accept_path"],
         "evict": ["prefix_len", "seq_len"]}


@pytest.mark.parametrize("name,read,wrote", [(n, r, "new_len") for n in READS for r in READS[n]] + [("compact", r, "out_slots") for r in READS["compact"]])
def test_memory_in_common_is_refused(name, read, wrote):
    for at in (AT[read], AT[read] + BYTES[read] - 4, AT[read] - BYTES[wrote] + 4):
        assert _call(name, {**AT, wrote: at}) == 1 and "overlap" in hb.hb_last_error()
    for at in (AT[read] + BYTES[read], AT[read] - BYTES[wrote]):  # next to it
        assert _call(name, {**AT, wrote: at}) == (3 if name == "evict" else 1) and "overlap" not in hb.hb_last_error()


@pytest.mark.parametrize("name", READS)
def test_arguments_that_are_not_given_overlap_nothing(name):
    for left_out in ({"new_len": None, "out_slots": None}, {"seq_len": None} if name != "evict" else {"new_len": None}):
        assert _call(name, {**AT, **left_out}) == (3 if name == "evict" else 1) and "overlap" not in hb.hb_last_error()
