"""What the calls for requests write has to lie apart from everything that they read (no GPU)."""
import ctypes as C

import pytest

import paper_2509_18824_amd as hb
import paper_2509_18824_amd.step as S

L = hb.lib
P = [C.c_void_p((i + 1) << 32) for i in range(16)]  # far apart
off = lambda p, n: C.c_void_p(p.value + n)


def _desc(**kw):
    base = dict(dtype="bf16", B=2, Hq=28, Hkv=4, D=128, page=16, max_blocks=64, num_blocks=200, total_nodes=120, max_nodes=60, softmax_scale=0.1)
    return S.make_desc(**(base | kw))


POOL = 200 * 4 * 16 * 128 * 2  # bytes of one of these descriptors' pools


def _refused(rc, name):
    assert rc == 1 and hb.hb_last_error().startswith(f"{name} must not overlap"), (rc, hb.hb_last_error())


def test_append():
    def call(k=P[0], v=P[1], slots=P[2], k_pool=P[3], v_pool=P[4], n=8, **kw):
        return L.hb_kv_append(C.byref(_desc(**kw)), n, k, v, slots, k_pool, v_pool, None)
    _refused(call(v_pool=P[3]), "k_pool")
    _refused(call(v_pool=off(P[3], POOL - 16)), "k_pool")
    _refused(call(k=off(P[3], POOL - 16)), "k_pool")
    _refused(call(v=P[3], k=P[4]), "k_pool")
    _refused(call(slots=off(P[3], 64)), "k_pool")
    _refused(call(k=off(P[4], 1024)), "v_pool")
    _refused(call(slots=off(P[4], -4)), "v_pool")  # its last seven
    # sizes at the ends of their types
    _refused(call(page=1 << 20, max_blocks=1, num_blocks=2047, Hq=65535, Hkv=65535, D=256, dtype="f32", n=2 ** 31 - 1), "k_pool")


NAMES = ("q", "k", "v", "k_pool", "v_pool", "table", "prefix", "offset", "out", "lse", "ws")


def _attn(splits=4, **at):
    a = {n: at.get(n, P[i]) for i, n in enumerate(NAMES)}
    return L.hb_prompt_attn(C.byref(_desc(num_splits=splits)), *[a[n] for n in NAMES[:10]], a["ws"], 1 << 40, None)


@pytest.mark.parametrize("out", ["out", "lse", "ws"])
@pytest.mark.parametrize("read", NAMES[:8])
def test_prompt_attention(out, read):
    at = P[NAMES.index(read)]
    ends = {"k_pool": POOL, "v_pool": POOL, "table": 2 * 64 * 4, "prefix": 8, "offset": 12}
    name = "workspace" if out == "ws" else out
    _refused(_attn(**{out: at}), name)
    _refused(_attn(**{read: off(P[NAMES.index(out)], 256)}), name)
    if read in ends and ends[read] > 256:  # into the last bytes
        _refused(_attn(**{out: off(at, ends[read] - 256)}), name)


RULES = ("logits", "node_offset", "parent", "draft_ids", "counts", "rules", "bias_offset", "bias_id", "bias_value", "mask", "mask_row", "out", "ws")


def _rules(call, B=2, T=16, V=1000, n_bias=3, masks=4, dtype=1, **at):
    a = {n: at.get(n, P[i]) for i, n in enumerate(RULES)}
    head = [dtype, B, 8, T, V] + [a[n] for n in RULES[:7]] + [n_bias, a["bias_id"], a["bias_value"], masks, a["mask"], a["mask_row"], a["out"]]
    return call(*head, a["ws"], 1 << 30, None) if call is L.hb_rules_probs else call(*head, None)


@pytest.mark.parametrize("read", RULES[1:11])
def test_rules(read):
    at = P[RULES.index(read)]
    _refused(_rules(L.hb_rules_logits, out=at), "out")
    _refused(_rules(L.hb_rules_logits, out=at, logits=at), "out")  # in place, and over something else
    _refused(_rules(L.hb_rules_probs, out=at), "probs")
    _refused(_rules(L.hb_rules_probs, ws=at), "workspace")
    _refused(_rules(L.hb_rules_probs, **{read: off(P[11], 64)}), "probs")


def test_rules_to_the_last_byte():
    for read, size in (("counts", 2 * 1000 * 4), ("mask", 4 * 32 * 4), ("rules", 32)):
        _refused(_rules(L.hb_rules_logits, out=off(P[RULES.index(read)], size - 16)), "out")
    _refused(_rules(L.hb_rules_logits, B=2 ** 31 - 1, T=2 ** 31 - 1, V=1 << 30, out=off(P[4], 1 << 60)), "out")


def test_counting():
    call = lambda tokens=P[0], offset=P[1], counts=P[2]: L.hb_rules_count(2, 100, 10, offset, tokens, 0, counts, None)
    _refused(call(counts=P[0]), "counts")
    _refused(call(tokens=off(P[2], 796)), "counts")
    _refused(call(offset=off(P[2], 400)), "counts")
