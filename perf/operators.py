"""The operators of the 4-bit KV cache, one pass of each through the public calls.

A long prefix is held as 4-bit floating point numbers (one sign bit, two exponent bits, one mantissa
bit) in blocks of 32 along the head dimension with a power of two as scale.  Four operators work on it:

  attn    attention of drafted trees, chains and single tokens over the 4-bit prefix and their own nodes
  append  new rows quantised into the pages (a prompt's, or the accepted path of a tree), and the rows
          as the cache now holds them, which is what a prompt's own attention reads
  weight  attention weight that every cached position received from the committed nodes, accumulated
  evict   the positions of lowest weight dropped, what is kept packed into the first pages

Shapes are those of the repository's workloads (28 query and 4 key/value heads of 128, 60-node trees,
8-node chains, contexts up to 32768; a unit-sized float32 model) and generic head layouts.  Inputs are
made on the GPU from the seed alone.  Scores of a head are as sharp as the head's place says; slots at
or past a sequence's length and the pages that no sequence owns hold NaN.
"""
import math
import random

import numpy as np
import torch

own = False

_MODEL = {"Hq": 28, "Hkv": 4, "D": 128, "page": 16}
_DECAY = 0.96875


def listed():
    bf = {"dtype": "bf16", **_MODEL}
    f32 = {"dtype": "f32", "Hq": 4, "Hkv": 1, "D": 64, "page": 16}
    return [
        # one user, one token at a time: what a call costs when little is read
        {"name": "attn_token_b1_2k", "op": "attn", "B": 1, "tree": "chain", "nodes": 1, "L_min": 2048, "L_max": 2048, **bf},
        # a unit-sized model in float32 with a chain of four
        {"name": "attn_chain4_f32", "op": "attn", "B": 1, "tree": "chain", "nodes": 4, "L_min": 256, "L_max": 256, **f32},
        # a serving batch of long contexts without drafts: reading the cache is all there is
        {"name": "attn_token_b16_32k", "op": "attn", "B": 16, "tree": "chain", "nodes": 1, "L_min": 16384, "L_max": 32768, **bf},
        # a serving batch with chain drafts
        {"name": "attn_chain8_b16", "op": "attn", "B": 16, "tree": "chain", "nodes": 8, "L_min": 1024, "L_max": 4096, **bf},
        # a ragged serving batch with drafted trees
        {"name": "attn_tree60_b16", "op": "attn", "B": 16, "tree": "tree", "nodes": 60, "L_min": 1024, "L_max": 8192, **bf},
        # two long interleaved contexts with drafted trees: the most arithmetic
        {"name": "attn_tree60_b2_32k", "op": "attn", "B": 2, "tree": "tree", "nodes": 60, "L_min": 32768, "L_max": 32768, **bf},
        # the accepted paths of a verification step join the cache
        {"name": "append_path6_b16", "op": "append", "B": 16, "path": 6, "L_min": 1024, "L_max": 4096, **bf},
        # two prompts join the cache
        {"name": "append_prompt_b2", "op": "append", "B": 2, "path": 0, "rows_min": 4096, "rows_max": 8192, "L_min": 0,
         "L_max": 100, **bf},
        # weights after one token of one user
        {"name": "weight_token_b1_2k", "op": "weight", "B": 1, "path": 1, "L_min": 2048, "L_max": 2048, **bf},
        # weights after the accepted paths of a serving batch
        {"name": "weight_path6_b16", "op": "weight", "B": 16, "path": 6, "L_min": 1024, "L_max": 8192, **bf},
        # one user's cache goes back to half
        {"name": "evict_b1_2k", "op": "evict", "B": 1, "L_min": 2048, "L_max": 2048, "keep": 1024, "recent": 128, "sinks": 4, **bf},
        # two long contexts are cut to a quarter
        {"name": "evict_b2_32k", "op": "evict", "B": 2, "L_min": 32768, "L_max": 32768, "keep": 8192, "recent": 1024, "sinks": 4, **bf},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["attn", "attn", "attn", "append", "weight", "evict"])
    if rng.random() < 0.2:
        dtype, D, longest = "f32", rng.choice([64, 128]), 4096
        Hq, Hkv = rng.choice([(4, 1), (6, 2), (8, 4), (4, 4)])
    else:
        dtype, D, longest = "bf16", rng.choice([64, 128, 128, 128]), 32768
        Hq, Hkv = rng.choice([(28, 4), (28, 4), (32, 8), (16, 2), (8, 8), (8, 1), (40, 10)])
    case = {"op": op, "dtype": dtype, "Hq": Hq, "Hkv": Hkv, "D": D, "page": rng.choice([16, 16, 16, 32])}
    L = _log_int(rng, 1, longest)
    B = _log_int(rng, 1, 16)
    while B > 1 and B * L * Hkv * D > 16 * 24576 * 4 * 128:
        B -= 1
    case |= {"B": B, "L_min": max(0, L - rng.randrange(0, L + 1)), "L_max": L}
    if op == "attn":
        tree = rng.choice(["chain", "tree"])
        nodes = 1 if rng.random() < 0.2 else _log_int(rng, 1, 64 if tree == "tree" else 16)
        # no more arithmetic than two 60-node trees of 28 heads of 128 over 32768 positions
        while nodes > 1 and nodes * B * L * Hq * D > 60 * 2 * 32768 * 28 * 128:
            nodes -= 1
        case |= {"tree": tree, "nodes": nodes}
    elif op == "append":
        if rng.random() < 0.5:
            case |= {"path": rng.randrange(1, 9)}
        else:
            rows = _log_int(rng, 1, 8192)
            while B > 2 and B * rows * Hkv * D > 2 * 6144 * 4 * 128:
                B -= 1
            case |= {"B": min(B, 2) if rows > 2048 else B, "path": 0, "rows_min": rng.randrange(0, rows + 1), "rows_max": rows}
    elif op == "weight":
        case |= {"path": rng.randrange(1, 9)}
    else:
        keep = _log_int(rng, 1, L)
        recent = rng.randrange(0, keep + 1)
        case |= {"keep": keep, "recent": recent, "sinks": min(4, keep - recent)}
        while case["B"] > 1 and case["B"] * L * Hkv * D > 2 * 32768 * 4 * 128:
            case["B"] -= 1
    return case


# ---- the 4-bit format ------------------------------------------------------------------------------
# element: sign, two bits of exponent, one of mantissa; 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives
# scale byte s: 2^(s - 127), 255: not a number; the smallest power of two under which the largest of the
# block's magnitudes is at most 7 (what lies above 6 becomes 6), within bytes 1 to 252

def _quantise(x):
    """float32 [..., D] -> codes uint8 [..., D / 2] (even element in the low half), scales uint8 [..., D / 32]."""
    x = x.unflatten(-1, (-1, 32))
    top = x.abs().amax(-1)
    bits = top.view(torch.int32)
    s = ((bits >> 23) - 2 + ((bits & 0x7fffff) > 0x600000).int()).clamp(1, 252)
    fine = torch.isfinite(top)
    s = torch.where(fine, s, 255)
    unit = torch.where(fine, (254 - s.clamp(max=252)) << 23, 0).view(torch.float32)  # 1 / scale
    a = torch.where(fine[..., None], x.abs() * unit[..., None], 0.0)
    # to the nearest, ties to the even code
    code = (a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5)
    code = (code | ((torch.signbit(x) & fine[..., None]).to(torch.uint8) << 3)).flatten(-2).unflatten(-1, (-1, 2))
    return code[..., 0] | (code[..., 1] << 4), s.to(torch.uint8)


_MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _values(codes, scales):
    """The float32 numbers that codes [..., D / 2] and scales [..., D / 32] stand for, [..., D]."""
    table = torch.tensor([*_MAGNITUDES, *(-m for m in _MAGNITUDES)], device=codes.device)
    c = table[torch.stack((codes & 15, codes >> 4), -1).flatten(-2).int()]
    s = scales.int()
    s = torch.where(s == 255, 0x7fc00000, torch.where(s == 0, 0x00400000, s << 23)).view(torch.float32)
    return (c.unflatten(-1, (-1, 32)) * s[..., None]).flatten(-2)


# ---- inputs ----------------------------------------------------------------------------------------

def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _parents(rng, kind, n):
    if kind == "chain":
        return [i - 1 for i in range(n)]
    return [-1] + [0 if i <= 10 else rng.randrange(1, i) for i in range(1, n)]


def prepare(case, seed):
    rng, dev, dt = random.Random(seed), "cuda", _dtype(case)
    gen = torch.Generator(device=dev).manual_seed(seed)
    randn = lambda *shape: torch.randn(shape, generator=gen, device=dev)  # noqa: E731
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)  # noqa: E731
    op, B, Hq, Hkv, D, page = (case[k] for k in ("op", "B", "Hq", "Hkv", "D", "page"))
    lens = [rng.randint(case["L_min"], case["L_max"]) for _ in range(B)]
    sizes = random.Random(B * 1000003 + case["L_max"])  # how many new rows a sequence has goes by the case alone
    s = {"case": case, "op": op, "scale": 1.0 / math.sqrt(D)}

    # new rows of each sequence: tree nodes, an accepted path's tree, or a prompt
    path = case.get("path", 0)
    if op == "attn":
        full = case["tree"] == "chain"
        trees = [_parents(rng, case["tree"], case["nodes"] if full else sizes.randint((case["nodes"] + 1) // 2, case["nodes"])) for _ in range(B)]
    elif path:
        trees = [_parents(rng, "tree", min(60, 1 + 11 * (path - 1))) for _ in range(B)]
    elif op == "append":
        trees = [[-1] * sizes.randint(case["rows_min"], case["rows_max"]) for _ in range(B)]
    else:
        trees = [[] for _ in range(B)]
    counts = [len(t) for t in trees]
    offsets = np.concatenate(([0], np.cumsum(counts))).tolist()
    rows = offsets[-1]

    # pages: of all sequences in one shuffled pool, with a few that nobody owns
    pages = [-(-(n + c) // page) for n, c in zip(lens, counts)]
    most = -(-(case["L_max"] + max(counts)) // page)
    max_blocks, blocks = max(most, 1) + 1, B * most + 3
    order = list(range(blocks))
    rng.shuffle(order)
    table, at = [], 0
    for n in pages:
        table.append(order[at:at + n] + [order[-1]] * (max_blocks - n))
        at += n
    cap = max_blocks * page
    s |= {"block_table": ints(table), "prefix_len": ints(lens), "node_offset": ints(offsets), "parent": ints([p for t in trees for p in t] or [0]),
          "blocks": blocks, "max_blocks": max_blocks, "rows": rows, "longest": case["L_max"], "max_nodes": max(max(counts), 1)}
    if op == "append":  # the prefix is there already; what it holds does not matter to the call
        pool = torch.randint(0, 256, (2, blocks, Hkv, page, D // 2), generator=gen, device=dev, dtype=torch.uint8)
        scale = torch.full((2, blocks, Hkv, page, D // 32), 255, device=dev, dtype=torch.uint8)
        s["codes"], s["scales"] = [pool[0], pool[1]], [scale[0], scale[1]]
    else:
        owner = torch.zeros(blocks, dtype=torch.int64, device=dev)
        first = torch.full((blocks,), cap, dtype=torch.int64, device=dev)  # position of a page's first slot
        length = torch.zeros(blocks, dtype=torch.int64, device=dev)
        at = 0
        for b, n in enumerate(pages):
            ids = torch.tensor(order[at:at + n], dtype=torch.int64, device=dev)
            owner[ids], length[ids], first[ids] = b, lens[b], torch.arange(n, device=dev) * page
            at += n
        valid = (first[:, None] + torch.arange(page, device=dev) < length[:, None])[:, None, :, None]
        s["codes"], s["scales"] = [], []
        for _ in range(2):
            codes, scales = _quantise(randn(blocks, Hkv, page, D).to(dt).float())
            s["codes"].append(codes)
            s["scales"].append(torch.where(valid, scales, 255).to(torch.uint8))

    # sharpness of the heads' scores: from near-uniform to a handful of keys
    sharp = torch.linspace(0.3, 3.0, Hq, device=dev)[:, None]
    if op in ("attn", "weight"):
        s["q"] = (randn(rows, Hq, D) * sharp).to(dt)
    if op in ("attn", "append"):
        s["k_new"], s["v_new"] = randn(rows, Hkv, D).to(dt), randn(rows, Hkv, D).to(dt)
    if op in ("append", "weight"):
        s["accept_len"] = ints([rng.randint(1, path) if path else 0 for _ in range(B)])
        s["accept_path"] = ints([[0, *sorted(rng.sample(range(1, len(t)), path - 1))] for t in trees]) if path else None
    if op != "attn":
        s["pos"] = torch.arange(cap, dtype=torch.int32, device=dev).expand(B, Hkv, cap).contiguous()
        s["seq_len"] = s["prefix_len"] + 0
        w = torch.rand((B, Hkv, cap), generator=gen, device=dev)
        s["weight"] = 0.01 * w / (1.001 - w)  # a few positions gather most of it
    if op == "weight":
        # the log-sum-exp that attention left for these rows: over the prefix, as near as makes the weights sum to about one
        spread = sharp.squeeze(1) ** 2 / 2
        n = torch.tensor([max(x, 1) for x, c in zip(lens, counts) for _ in range(c)], dtype=torch.float32, device=dev)
        s["lse"] = (n.log()[:, None] + spread + 0.05 * randn(rows, Hq)).contiguous()
    if op == "append":
        s["read_offset"] = ints([b * path for b in range(B + 1)]) if path else s["node_offset"]
        n = B * path if path else rows
        s["k_read"], s["v_read"] = torch.empty((n, Hkv, D), dtype=dt, device=dev), torch.empty((n, Hkv, D), dtype=dt, device=dev)
    if op == "evict":
        s["seq_len"] += rng.randrange(0, 50)  # positions that are gone already
        s["weight_out"], s["pos_out"] = torch.zeros_like(s["weight"]), torch.zeros_like(s["pos"])
        s["kept"] = torch.empty((B, Hkv, case["keep"]), dtype=torch.int32, device=dev)
    if op in ("append", "evict"):
        s["new_len"] = torch.empty(B, dtype=torch.int32, device=dev)
    if op == "attn":
        s["out"], s["lse"] = torch.empty_like(s["q"]), torch.empty((rows, Hq), dtype=torch.float32, device=dev)
    if own:  # the descriptor, and the workspace of the size that the library names for it
        import paper_2509_18824_amd as hb
        import paper_2509_18824_amd.step as S
        desc = S.make_desc(dt, B, Hq, Hkv, D, page, max_blocks, blocks, rows, min(s["max_nodes"], 64), s["scale"], hint=s["longest"])
        s["desc"] = desc
        s["pool"] = S.Kv4Pool(s["codes"][0], s["scales"][0], s["codes"][1], s["scales"][1])
        if op == "attn":
            s["workspace"] = S.alloc_workspace(hb.hb_tree_verify_attn_kv4_workspace_bytes(desc))
        if op == "evict":
            s["workspace"] = S.alloc_workspace(hb.hb_kv4_evict_workspace_bytes(desc, case["keep"]))
    return s


# ---- one pass --------------------------------------------------------------------------------------

def run(s):
    return (_run_own if own else _run_plain)[s["op"]](s)


def _own_attn(s):
    import paper_2509_18824_amd as hb
    hb.hb_tree_verify_attn_kv4(s["desc"], s["q"], s["k_new"], s["v_new"], *s["pool"], s["block_table"], s["prefix_len"],
                               s["node_offset"], s["parent"], s["out"], s["lse"], s["workspace"])
    return s["out"], s["lse"]


def _own_append(s):
    import paper_2509_18824_amd as hb
    if s["accept_path"] is not None:
        hb.hb_kv4_compact(s["desc"], s["k_new"], s["v_new"], *s["pool"], s["block_table"], s["prefix_len"], s["node_offset"],
                          s["accept_len"], s["accept_path"], s["case"]["path"], s["seq_len"], s["weight"], s["pos"], None, s["new_len"])
    else:
        hb.hb_kv4_append(s["desc"], s["k_new"], s["v_new"], *s["pool"], s["block_table"], s["prefix_len"], s["node_offset"],
                         s["seq_len"], s["weight"], s["pos"], s["new_len"])
    hb.hb_kv4_read(s["desc"], *s["pool"], s["block_table"], s["prefix_len"], s["read_offset"], s["k_read"], s["v_read"])
    return s["k_read"], s["v_read"], s["weight"], s["pos"], s["new_len"]


def _own_weight(s):
    import paper_2509_18824_amd as hb
    hb.hb_kv4_attn_weight(s["desc"], s["q"], s["pool"].k_codes, s["pool"].k_scales, s["block_table"], s["prefix_len"],
                          s["node_offset"], s["accept_len"], s["accept_path"], s["case"]["path"], s["lse"], _DECAY, s["weight"])
    return s["weight"]


def _own_evict(s):
    import paper_2509_18824_amd as hb
    c = s["case"]
    hb.hb_kv4_evict(s["desc"], c["keep"], c["recent"], c["sinks"], *s["pool"], s["block_table"], s["prefix_len"], s["seq_len"],
                    s["weight"], s["pos"], s["weight_out"], s["pos_out"], s["kept"], s["new_len"], s["workspace"])
    return s["kept"], s["weight_out"], s["pos_out"], s["new_len"], s["codes"], s["scales"]


_run_own = {"attn": _own_attn, "append": _own_append, "weight": _own_weight, "evict": _own_evict}


def _prefix(s, which):
    """float32 [B, Hkv, n, D]: the cached keys (0) or values (1) of positions 0 .. n - 1, zeros past a sequence's length."""
    page = s["case"]["page"]
    at = s["block_table"][:, :max(1, -(-s["longest"] // page))].long()
    x = _values(s["codes"][which][at], s["scales"][which][at]).transpose(1, 2).flatten(2, 3)
    there = torch.arange(x.shape[2], device=x.device) < s["prefix_len"][:, None]
    return torch.where(there[:, None, :, None], x, 0.0), there


def _per_sequence(s, x, n):
    """[rows, ...] -> [B, n, ...] with the rows of each sequence first, and which of them exist."""
    at = s["node_offset"][:-1, None] + torch.arange(n, device=x.device)
    there = at < s["node_offset"][1:, None]
    return x[at.clamp(max=x.shape[0] - 1).long()], there


def _plain_attn(s):
    c, n = s["case"], s["max_nodes"]
    Hkv, G, D = c["Hkv"], c["Hq"] // c["Hkv"], c["D"]
    q, is_node = _per_sequence(s, s["q"].float(), n)
    B = q.shape[0]
    q = q.view(B, n, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, n * G, D) * s["scale"]
    kt, vt = (_per_sequence(s, s[k].float(), n)[0].transpose(1, 2).contiguous() for k in ("k_new", "v_new"))
    # who is on whose path: the closure of the parent relation
    par, _ = _per_sequence(s, s["parent"], n)
    step = torch.eye(n, device=q.device) + (par[:, :, None] == torch.arange(n, device=q.device)).float()
    seen = (torch.matrix_power(step, n) > 0) & is_node[:, None, :]
    k, there = _prefix(s, 0)
    sp = torch.where(there[:, None, None, :], q @ k.transpose(2, 3).contiguous(), -math.inf)
    st = (q @ kt.transpose(2, 3).contiguous()).view(B, Hkv, n, G, n)
    st = torch.where(seen[:, None, :, None, :], st, -math.inf).view(B, Hkv, n * G, n)
    m = torch.maximum(sp.amax(-1, keepdim=True), st.amax(-1, keepdim=True))
    sp, st = torch.exp(sp - m), torch.exp(st - m)
    total = sp.sum(-1, keepdim=True) + st.sum(-1, keepdim=True)
    o = (sp @ _prefix(s, 1)[0] + st @ torch.where(is_node[:, None, :, None], vt, 0.0)) / total
    row = torch.arange(s["rows"], device=q.device)
    b = torch.searchsorted(s["node_offset"][1:].contiguous(), row, right=True)
    i = row - s["node_offset"][b]
    out = o.view(B, Hkv, n, G, D)[b, :, i].flatten(1, 2)
    lse = (m + total.log()).view(B, Hkv, n, G)[b, :, i].flatten(1, 2)
    return out.to(s["q"].dtype), lse


def _slots(s, b, position):
    page = s["case"]["page"]
    return s["block_table"][b, position // page].long(), position % page


def _plain_append(s):
    c = s["case"]
    if s["accept_path"] is not None:
        b, j = torch.nonzero(torch.arange(c["path"], device="cuda") < s["accept_len"][:, None], as_tuple=True)
        src, new = s["node_offset"][b] + s["accept_path"][b, j], s["accept_len"]
    else:
        src = torch.arange(s["rows"], device="cuda")
        b = torch.searchsorted(s["node_offset"][1:].contiguous(), src, right=True)
        j, new = src - s["node_offset"][b], s["node_offset"].diff()
    p = s["prefix_len"][b] + j
    block, slot = _slots(s, b, p)
    for which, x in enumerate((s["k_new"], s["v_new"])):
        codes, scales = _quantise(x[src].float())
        s["codes"][which][block, :, slot] = codes
        s["scales"][which][block, :, slot] = scales
    s["weight"][b, :, p] = 0.0
    s["pos"][b, :, p] = (s["seq_len"][b] + j).to(torch.int32)[:, None]
    # the rows as the cache holds them
    row = torch.arange(s["k_read"].shape[0], device="cuda")
    b = torch.searchsorted(s["read_offset"][1:].contiguous(), row, right=True)
    block, slot = _slots(s, b, s["prefix_len"][b] + row - s["read_offset"][b])
    k, v = (_values(s["codes"][i][block, :, slot], s["scales"][i][block, :, slot]).to(s["k_new"].dtype) for i in (0, 1))
    return k, v, s["weight"], s["pos"], s["prefix_len"] + new


def _plain_weight(s):
    c = s["case"]
    Hkv, G, D, n = c["Hkv"], c["Hq"] // c["Hkv"], c["D"], c["path"]
    B = s["prefix_len"].shape[0]
    row = (s["node_offset"][:-1, None] + s["accept_path"]).long()
    committed = torch.arange(n, device="cuda") < s["accept_len"][:, None]
    q = s["q"][row].float().view(B, n, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, n * G, D) * s["scale"]
    lse = torch.where(committed[:, :, None], s["lse"][row], math.inf).view(B, n, Hkv, G).permute(0, 2, 1, 3).reshape(B, Hkv, n * G, 1)
    k, there = _prefix(s, 0)
    got = torch.exp(q @ k.transpose(2, 3).contiguous() - lse).sum(2)
    w = s["weight"][:, :, :got.shape[2]]
    w.copy_(torch.where(there[:, None], _DECAY * w + got, w))
    return s["weight"]


def _plain_evict(s):
    c = s["case"]
    keep, cap = c["keep"], s["weight"].shape[2]
    slot = torch.arange(cap, device="cuda")
    L = s["prefix_len"][:, None, None]
    stays = L.clamp(max=keep)
    safe = (s["pos"] >= s["seq_len"][:, None, None] - c["recent"]) | (s["pos"] < c["sinks"])
    key = torch.where(safe, math.inf, torch.nan_to_num(s["weight"], nan=-math.inf))
    order = torch.sort(torch.where(slot < L, key, -math.inf), dim=2, descending=True, stable=True).indices
    kept = torch.zeros_like(safe).scatter(2, order, (slot < stays).expand_as(safe))
    # the k-th free slot below takes the k-th kept one from above
    above = torch.where(kept & (slot >= stays), slot, cap).sort(2).values
    rank = ((~kept) & (slot < stays)).long().cumsum(2) - 1
    source = torch.where(kept, slot, above.gather(2, rank.clamp(min=0)))[:, :, :keep]
    live = slot[:keep] < stays
    source = torch.where(live, source, slot[:keep])
    s["weight_out"][:, :, :keep] = torch.where(live, s["weight"].gather(2, source), s["weight_out"][:, :, :keep])
    s["pos_out"][:, :, :keep] = torch.where(live, s["pos"].gather(2, source), s["pos_out"][:, :, :keep])
    b = torch.arange(source.shape[0], device="cuda")[:, None, None].expand_as(source)
    h = torch.arange(source.shape[1], device="cuda")[None, :, None].expand_as(source)
    to, to_slot = _slots(s, b, slot[:keep].expand_as(source))
    at, at_slot = _slots(s, b, source)
    for pool in (*s["codes"], *s["scales"]):
        pool[to, h, to_slot] = pool[at, h, at_slot]
    s["kept"].copy_(torch.where(live, source, -1))
    return s["kept"], s["weight_out"], s["pos_out"], stays[:, 0, 0].to(torch.int32), s["codes"], s["scales"]


_run_plain = {"attn": _plain_attn, "append": _plain_append, "weight": _plain_weight, "evict": _plain_evict}


def work(case):
    B, Hq, Hkv, D = (case[k] for k in ("B", "Hq", "Hkv", "D"))
    L = (case["L_min"] + case["L_max"]) / 2
    wide = 4 if case["dtype"] == "f32" else 2
    row = D / 2 + D / 32  # a position's key or value of one head in the cache
    if case["op"] == "attn":
        n = case["nodes"] if case["tree"] == "chain" else ((case["nodes"] + 1) // 2 + case["nodes"]) / 2
        return {"bytes": B * (2 * L * Hkv * row + n * (2 * Hq + 2 * Hkv) * D * wide + n * Hq * 4), "flops": 4 * D * Hq * B * n * (L + (n + 1) / 2)}
    if case["op"] == "append":
        n = (case["path"] + 1) / 2 if case["path"] else (case["rows_min"] + case["rows_max"]) / 2
        return {"bytes": B * n * Hkv * (2 * D * wide + 2 * row + 8) + B * (case["path"] or n) * Hkv * 2 * (row + D * wide), "flops": 0}
    if case["op"] == "weight":
        n = (case["path"] + 1) / 2
        return {"bytes": B * (L * Hkv * (row + 8) + n * Hq * (D * wide + 4)), "flops": 2 * D * Hq * B * n * L}
    # on average a kept position lies in the part that is kept with probability keep / L
    keep = min(case["keep"], L)
    moved = keep * max(0.0, 1 - keep / max(L, 1))
    return {"bytes": B * Hkv * (8 * L + 12 * keep + 4 * row * moved), "flops": 0}


# ---- the definitions in 64 bits --------------------------------------------------------------------

def _exact_rows(s, which, b, positions):
    """float64 [positions, Hkv, D] of sequence b, element by element from the format's definition."""
    page = s["case"]["page"]
    block = s["block_table"][b].long()[positions // page]
    codes, scales = s["codes"][which][block, :, positions % page], s["scales"][which][block, :, positions % page]
    nibble = torch.empty((*codes.shape[:-1], codes.shape[-1] * 2), dtype=torch.int16, device=codes.device)
    nibble[..., 0::2], nibble[..., 1::2] = (codes % 16).short(), (codes // 16).short()
    exponent, mantissa = (nibble // 2) % 4, (nibble % 2).double()
    magnitude = torch.where(exponent == 0, mantissa / 2, torch.exp2(exponent.double() - 1) * (1 + mantissa / 2))
    value = torch.where(nibble >= 8, -magnitude, magnitude)
    scale = torch.where(scales == 255, math.nan, torch.exp2(scales.double() - 127))
    return value * torch.repeat_interleave(scale, 32, dim=-1)


def exact(case, seed):
    s = prepare(case, seed)
    c = case
    B, Hq, Hkv, D = (c[k] for k in ("B", "Hq", "Hkv", "D"))
    G = Hq // Hkv
    lens, offsets = s["prefix_len"].tolist(), s["node_offset"].tolist()
    if c["op"] == "evict":
        w, pos = s["weight"].double().cpu().numpy(), s["pos"].cpu().numpy()
        got = s["weight_out"].double().cpu().numpy()
        for b in range(B):
            stays, end = min(lens[b], c["keep"]), int(s["seq_len"][b])
            for h in range(Hkv):
                x, p = w[b, h, :lens[b]], pos[b, h, :lens[b]]
                rank = np.lexsort((np.arange(lens[b]), -x, ~((p >= end - c["recent"]) | (p < c["sinks"]))))
                chosen = np.sort(rank[:stays])
                low, high = chosen[chosen < stays], chosen[chosen >= stays]
                source = np.arange(stays)
                source[np.setdiff1d(np.arange(stays), low)] = high
                got[b, h, :stays] = x[source]
        return None, torch.from_numpy(got), None, None, None, None
    if c["op"] == "append":
        got = []
        for x in (s["k_new"], s["v_new"]):
            x = x.double().cpu().numpy().reshape(-1, Hkv, D // 32, 32)
            top = np.abs(x).max(-1, keepdims=True)
            # the smallest power of two that brings the largest down to 7 or less
            unit = np.exp2(np.clip(np.ceil(np.log2(np.maximum(top, 1e-300) / 7)), -126, 125))
            levels = np.array(_MAGNITUDES)
            a = np.minimum(np.abs(x) / unit, 6.0)
            low = np.clip(np.searchsorted(levels, a, side="right") - 1, 0, 6)
            down, up = a - levels[low], levels[low + 1] - a
            code = np.where((up < down) | ((up == down) & (low % 2 == 1)), low + 1, low)
            got.append((np.copysign(levels[code], x) * unit).reshape(-1, Hkv, D))
        weight = s["weight"].double().cpu().numpy()
        n = s["k_read"].shape[0]
        k, v = np.full((n, Hkv, D), math.nan), np.full((n, Hkv, D), math.nan)
        for b in range(B):
            if c["path"]:
                took = [offsets[b] + int(i) for i in s["accept_path"][b].tolist()[:int(s["accept_len"][b])]]
            else:
                took = list(range(offsets[b], offsets[b + 1]))
            at = int(s["read_offset"][b])
            k[at:at + len(took)], v[at:at + len(took)] = got[0][took], got[1][took]
            weight[b, :, lens[b]:lens[b] + len(took)] = 0
        return torch.from_numpy(k), torch.from_numpy(v), torch.from_numpy(weight), None, None
    if c["op"] == "weight":
        got = s["weight"].double()
        for b in range(B):
            k = _exact_rows(s, 0, b, torch.arange(lens[b], device="cuda"))
            rows = [offsets[b] + i for i in s["accept_path"][b].tolist()[:int(s["accept_len"][b])]]
            total = torch.zeros((Hkv, lens[b]), dtype=torch.float64, device="cuda")
            for r in rows:
                score = torch.matmul(s["q"][r].double().view(Hkv, G, D), k.permute(1, 2, 0).contiguous()) / math.sqrt(D)
                total += torch.exp(score - s["lse"][r].double().view(Hkv, G, 1)).sum(1)
            got[b, :, :lens[b]] = _DECAY * got[b, :, :lens[b]] + total
        return got
    out = torch.empty((s["rows"], Hq, D), dtype=torch.float64, device="cuda")
    lse = torch.empty((s["rows"], Hq), dtype=torch.float64, device="cuda")
    for b in range(B):
        n0, n = offsets[b], offsets[b + 1] - offsets[b]
        at = torch.arange(lens[b], device="cuda")
        k = torch.cat((_exact_rows(s, 0, b, at), s["k_new"][n0:n0 + n].double()))
        v = torch.cat((_exact_rows(s, 1, b, at), s["v_new"][n0:n0 + n].double()))
        parent, mask = s["parent"][n0:n0 + n].tolist(), torch.zeros((n, n), dtype=torch.bool)
        for i in range(n):
            x = i
            while x >= 0:
                mask[i, x] = True
                x = parent[x]
        mask = torch.cat((torch.ones((n, lens[b]), dtype=torch.bool, device="cuda"), mask.cuda()), 1)
        for h in range(Hkv):
            heads = slice(h * G, (h + 1) * G)
            q = s["q"][n0:n0 + n, heads].double().reshape(n * G, D)
            score = (q @ k[:, h].t().contiguous()).view(n, G, -1) / math.sqrt(D)
            score = score.masked_fill(~mask[:, None], -math.inf)
            lse[n0:n0 + n, heads] = torch.logsumexp(score, -1)
            p = torch.softmax(score, -1).view(n * G, -1)
            out[n0:n0 + n, heads] = (p @ v[:, h].contiguous()).view(n, G, D)
    return out, lse
