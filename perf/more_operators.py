"""What a request needs before its first verification step, and its own sampling rules in every step.

  pages   page tables and slot maps from the requests' lengths: pages taken from a list of free ones (take),
          and given back (give)
  append  rows of K and V written to their slots of the paged cache
  attn    attention of whole prompts, or parts of them, packed one behind the other: causal among their own
          rows, over what the paged cache holds of their sequence already
  rules   penalties for tokens that a request has had, biases and grammar masks on the logits of drafted
          trees, chains and single tokens, to adjusted logits or to the probabilities that sampling
          acceptance takes; the step's new tokens are counted first

Shapes are those of the repository's workloads (28 query and 4 key/value heads of 128, 60-node trees,
8-node chains, contexts up to 32768, 152064 tokens; a unit-sized float32 model) and generic ones.  Inputs
are made on the GPU from the seed alone; slots that no sequence owns hold NaN.
"""
import math
import random

import torch

own = False

_MODEL = {"Hq": 28, "Hkv": 4, "D": 128, "page": 16}


def listed():
    bf = {"dtype": "bf16", **_MODEL}
    f32 = {"dtype": "f32", "Hq": 4, "Hkv": 1, "D": 64, "page": 16}
    return [
        # room for the next verification step's nodes, a serving batch of chains
        {"name": "pages_take_step_b16", "op": "pages", "way": "take", "B": 16, "rows_min": 8, "rows_max": 8, "L_min": 1024, "L_max": 4096,
         "reserve": 8, "page": 16, "short": False},
        # many prompts come in at once, more than there are pages for
        {"name": "pages_take_prompts_b256", "op": "pages", "way": "take", "B": 256, "rows_min": 1, "rows_max": 1024, "L_min": 0,
         "L_max": 0, "reserve": 8, "page": 16, "short": True},
        # a batch of finished requests, and of such as were cut back
        {"name": "pages_give_b64", "op": "pages", "way": "give", "B": 64, "L_min": 1, "L_max": 8192, "page": 16},
        # one token of every request of a batch
        {"name": "append_token_b16", "op": "append", "rows": 16, **bf},
        # two prompts
        {"name": "append_prompt_16k", "op": "append", "rows": 16384, **bf},
        # a unit-sized model in float32, prompts and their log-sum-exp
        {"name": "attn_f32_b2", "op": "attn", "B": 2, "rows_min": 200, "rows_max": 256, "L_min": 0, "L_max": 0, "lse": True, **f32},
        # part of a long prompt over what the cache holds of it
        {"name": "attn_part_512_of_32k", "op": "attn", "B": 1, "rows_min": 512, "rows_max": 512, "L_min": 32256, "L_max": 32256,
         "lse": False, **bf},
        # ragged prompts of a serving batch, some behind a cached beginning
        {"name": "attn_ragged_b8", "op": "attn", "B": 8, "rows_min": 1, "rows_max": 2048, "L_min": 0, "L_max": 1500, "lse": False, **bf},
        # one long prompt: the most arithmetic
        {"name": "attn_prompt_8k", "op": "attn", "B": 1, "rows_min": 8192, "rows_max": 8192, "L_min": 0, "L_max": 0, "lse": False, **bf},
        # one user's chain of eight
        {"name": "probs_chain8_b1", "op": "rules", "way": "probs", "dtype": "bf16", "B": 1, "nodes": 8, "V": 152064, "bias": 20,
         "grammar": 1.0},
        # a serving batch with drafted trees, half of it under a grammar
        {"name": "probs_tree60_b16", "op": "rules", "way": "probs", "dtype": "bf16", "B": 16, "nodes": 60, "V": 152064, "bias": 100,
         "grammar": 0.5},
        # adjusted logits of single tokens in float32
        {"name": "logits_token_b64", "op": "rules", "way": "logits", "dtype": "f32", "B": 64, "nodes": 1, "V": 152064, "bias": 20,
         "grammar": 0.25},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["pages", "append", "attn", "attn", "attn", "rules", "rules"])
    page = rng.choice([16, 16, 16, 32, 64])
    if op == "pages":
        B = _log_int(rng, 1, 256)
        rows = _log_int(rng, 1, 1024)
        L = rng.choice([0, _log_int(rng, 1, 8192)])
        if rng.random() < 0.3:
            return {"op": op, "way": "give", "B": B, "L_min": rng.randrange(0, L + 1), "L_max": L, "page": page}
        return {"op": op, "way": "take", "B": B, "rows_min": rng.randrange(0, rows + 1), "rows_max": rows, "L_min": rng.randrange(0, L + 1),
                "L_max": L, "reserve": rng.randrange(0, 9), "page": page, "short": rng.random() < 0.3}
    if op == "rules":
        nodes, V = rng.choice([1, _log_int(rng, 2, 16), _log_int(rng, 2, 64)]), rng.choice([152064, _log_int(rng, 1000, 152064)])
        B = _log_int(rng, 1, 64)
        while B > 1 and B * nodes * V > 16 * 60 * 152064:
            B -= 1
        return {"op": op, "way": rng.choice(["probs", "probs", "logits"]), "dtype": rng.choice(["bf16", "bf16", "f32"]), "B": B, "nodes": nodes,
                "V": V, "bias": rng.randrange(0, 300), "grammar": rng.choice([0.0, 0.5, 1.0])}
    if rng.random() < 0.2:
        dtype, D, longest = "f32", rng.choice([64, 128]), 1024
        Hq, Hkv = rng.choice([(4, 1), (6, 2), (8, 4), (4, 4)])
    else:
        dtype, D, longest = "bf16", rng.choice([64, 128, 128, 128]), 8192
        Hq, Hkv = rng.choice([(28, 4), (28, 4), (32, 8), (16, 2), (8, 8), (8, 1), (40, 10)])
    heads = {"dtype": dtype, "Hq": Hq, "Hkv": Hkv, "D": D, "page": page}
    if op == "append":
        return {"op": op, "rows": _log_int(rng, 1, 16384 * 512 // max(512, Hkv * D)), **heads}
    rows = _log_int(rng, 1, longest)
    L = rng.choice([0, 0, _log_int(rng, 1, 4 * longest)])
    B = rng.choice([1, _log_int(rng, 1, 16)])
    # no more scores than one prompt of 8192 has (all of them, as if it were not causal)
    while B > 1 and B * rows * (rows + L) * Hq * D > 28 * 128 * 8192 * 8192:
        B -= 1
    while rows * (rows + L) * Hq * D > 28 * 128 * 8192 * 4096:
        rows, L = (rows * 3 + 3) // 4, L // 2
    return {"op": op, "B": B, "rows_min": rng.choice([rows, rng.randrange(0, rows + 1)]), "rows_max": rows, "L_min": rng.randrange(0, L + 1),
            "L_max": L, "lse": rng.random() < 0.3, **heads}


# ---- inputs ----------------------------------------------------------------------------------------

def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _offsets(counts):
    at = [0]
    for n in counts:
        at.append(at[-1] + n)
    return at


def prepare(case, seed):
    rng = random.Random(seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    # how many new rows a sequence has goes by the case alone
    sizes = random.Random(case.get("rows_max", 1) * 1000003 + case.get("B", 1))
    return {"pages": _prepare_pages, "append": _prepare_append, "attn": _prepare_attn, "rules": _prepare_rules}[case["op"]](case, rng, gen, sizes)


def _prepare_pages(case, rng, gen, sizes):
    B, page = case["B"], case["page"]
    take = case["way"] == "take"
    lens = [rng.randint(case["L_min"], case["L_max"]) for _ in range(B)]
    rows = [sizes.randint(case["rows_min"], case["rows_max"]) if take else 0 for _ in range(B)]
    reserve = case.get("reserve", 0)
    have = [-(-n // page) for n in lens]
    want = [-(-(n + r + reserve) // page) for n, r in zip(lens, rows)]
    need = sum(max(0, w - h) for w, h in zip(want, have))
    free = int(need * 0.8) if case.get("short") else need + 40
    max_blocks = -(-(case["L_max"] + case.get("rows_max", 0) + reserve) // page) + 1
    blocks = B * max_blocks + 43
    order = list(range(blocks))
    rng.shuffle(order)
    table, at = [], 0
    for n in have:
        table.append(order[at:at + n] + [-1] * (max_blocks - n))
        at += n
    s = {"case": case, "op": "pages", "blocks": blocks, "max_blocks": max_blocks, "rows": sum(rows), "block_table": _ints(table), "have": _ints(have),
         "free_pages": _ints(order[at:at + free] + [-1] * (blocks - free)), "free_count": _ints([free]), "have_out": _ints([0] * B), "left": _ints([0])}
    if take:
        s |= {"prefix_len": _ints(lens), "row_offset": _ints(_offsets(rows)), "slots": _ints([-2] * sum(rows)), "new_len": _ints([0] * B),
              "granted": _ints([0] * B)}
    else:  # a third is done, the others are cut back
        s["keep_len"] = _ints([0 if rng.random() < 0.33 else rng.randint(0, n) for n in lens])
    return s


def _prepare_append(case, rng, gen, sizes):
    n, Hkv, D, page, dt = case["rows"], case["Hkv"], case["D"], case["page"], _dtype(case)
    randn = lambda *shape: torch.randn(shape, generator=gen, device="cuda").to(dt)  # noqa: E731
    blocks = 2 * -(-n // page) + 2
    slots = torch.randperm(blocks, generator=gen, device="cuda")[:, None] * page + torch.arange(page, device="cuda")
    slots = slots.flatten()[:n].to(torch.int32)
    if n > 8:
        slots[n // 3] = -1  # a row that has no place
    s = {"case": case, "op": "append", "slots": slots, "k": randn(n, Hkv, D), "v": randn(n, Hkv, D), "k_pool": randn(blocks, Hkv, page, D),
         "v_pool": randn(blocks, Hkv, page, D)}
    if own:
        import paper_2509_18824_amd.step as S
        s["desc"] = S.make_desc(dt, 1, Hkv, Hkv, D, page, blocks, blocks, n, 1, 1.0)
    return s


def _prepare_attn(case, rng, gen, sizes):
    B, Hq, Hkv, D, page, dt = (case[k] for k in ("B", "Hq", "Hkv", "D", "page", "dtype"))
    dt = _dtype(case)
    randn = lambda *shape: torch.randn(shape, generator=gen, device="cuda")  # noqa: E731
    lens = [rng.randint(case["L_min"], case["L_max"]) for _ in range(B)]
    counts = [sizes.randint(case["rows_min"], case["rows_max"]) for _ in range(B)]
    if not any(counts):
        counts[0] = 1
    rows = sum(counts)
    used = [-(-n // page) for n in lens]
    blocks = sum(-(-case["L_max"] // page) for _ in range(B)) + 2
    max_blocks = max(1, -(-case["L_max"] // page))
    order = list(range(blocks))
    rng.shuffle(order)
    table, at = [], 0
    owner = torch.full((blocks,), 0, dtype=torch.int64)
    for n, used_b in zip(lens, used):
        ids = order[at:at + used_b]
        table.append(ids + [order[-1]] * (max_blocks - used_b))
        owner[ids] = torch.tensor([min(page, n - i * page) for i in range(used_b)], dtype=torch.int64)
        at += used_b
    there = (torch.arange(page, device="cuda") < owner.cuda()[:, None])[:, None, :, None]
    pools = [torch.where(there, randn(blocks, Hkv, page, D), float("nan")).to(dt) for _ in range(2)]
    # sharpness of the heads' scores: from near-uniform to a handful of keys
    sharp = torch.linspace(0.3, 3.0, Hq, device="cuda")[:, None]
    s = {"case": case, "op": "attn", "scale": 1.0 / math.sqrt(D), "rows": rows, "most_rows": max(counts), "longest": case["L_max"],
         "q": (randn(rows, Hq, D) * sharp).to(dt), "k": randn(rows, Hkv, D).to(dt), "v": randn(rows, Hkv, D).to(dt), "k_pool": pools[0],
         "v_pool": pools[1], "block_table": _ints(table), "prefix_len": _ints(lens), "row_offset": _ints(_offsets(counts))}
    if own:
        import paper_2509_18824_amd as hb
        import paper_2509_18824_amd.step as S
        s["desc"] = S.make_desc(dt, B, Hq, Hkv, D, page, max_blocks, blocks, rows, 1, s["scale"], hint=s["longest"])
        s["workspace"] = S.alloc_workspace(hb.hb_prompt_attn_workspace_bytes(s["desc"]))
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((rows, Hq), dtype=torch.float32, device="cuda") if case["lse"] else None
    return s


def _prepare_rules(case, rng, gen, sizes):
    B, V, nodes, dt = case["B"], case["V"], case["nodes"], _dtype(case)
    randint = lambda hi, *shape: torch.randint(0, hi, shape, generator=gen, device="cuda", dtype=torch.int32)  # noqa: E731
    # a tree has a root, up to ten children of it, and deeper nodes; up to sixteen nodes are a chain
    parents = [[i - 1 if nodes <= 16 else -1 if i == 0 else 0 if i <= 10 else rng.randrange(1, i) for i in range(nodes)] for _ in range(B)]
    T = B * nodes
    # a handful of tokens stand out of the rest
    logits = torch.randn((T, V), generator=gen, device="cuda").mul_(1.5)
    at = randint(V, T, 8).long()
    logits.scatter_(1, at, 4 + 12 * torch.rand((T, 8), generator=gen, device="cuda"))
    # what a request has had: some prompt tokens and some of its own, few of them often
    counts = torch.zeros((B, V), dtype=torch.int32, device="cuda")
    counts.scatter_(1, randint(V, B, min(V, 600)).long(), 1 << 30)
    often = (V * torch.rand((B, 400), generator=gen, device="cuda") ** 3).long().clamp(max=V - 1)
    counts.scatter_add_(1, often, torch.ones_like(often, dtype=torch.int32))
    draft = at[:, 0].to(torch.int32).contiguous()
    rules = [[0.0 if rng.random() < 0.25 else rng.uniform(0.6, 1.3), rng.choice([1.0, rng.uniform(1.0, 1.3)]), rng.uniform(0, 0.5), rng.uniform(0, 0.3)]
             for _ in range(B)]
    ids = [rng.sample(range(V), rng.randint(0, min(V, case["bias"]))) for _ in range(B)]
    values = [[rng.choice([-math.inf, rng.uniform(-5, 5), rng.uniform(0, 5)]) for _ in x] for x in ids]
    words = -(-V // 32)
    bound = [rng.random() < case["grammar"] for _ in range(B)]
    rows = [n if bound[b] else -1 for n, b in zip(range(T), (b for b in range(B) for _ in range(nodes)))]
    order = {t: i for i, t in enumerate(t for t in rows if t >= 0)}
    masks = len(order)
    # a grammar allows nearly everything, or next to nothing; now and then it leaves nothing at all
    dense = (torch.rand((masks, 1), generator=gen, device="cuda") < 0.5).to(torch.int32)
    loose = randint(1 << 31, masks, words) | randint(1 << 31, masks, words) | randint(1 << 31, masks, words)
    tight = randint(1 << 31, masks, words) & randint(1 << 31, masks, words) & randint(1 << 31, masks, words) & randint(1 << 31, masks, words)
    mask = torch.where(dense > 0, loose, tight)
    if masks > 5:
        mask[5] = 0
    new = [[rng.randrange(V) for _ in range(rng.randint(1, 6))] for _ in range(B)]
    s = {"case": case, "op": "rules", "logits": logits.to(dt), "counts": counts, "rules": torch.tensor(rules, device="cuda"), "draft_ids": draft,
         "parent": _ints([p for t in parents for p in t]), "node_offset": _ints([b * nodes for b in range(B + 1)]),
         "bias_offset": _ints(_offsets([len(x) for x in ids])), "bias_id": _ints([i for x in ids for i in x]),
         "bias_value": torch.tensor([v for x in values for v in x], dtype=torch.float32, device="cuda"), "mask": mask if masks else None,
         "mask_row": _ints([order.get(t, -1) for t in rows]) if masks else None,
         "tokens": _ints([x + [-1] * (6 - len(x)) for x in new])}
    if own:
        import paper_2509_18824_amd as hb
        import paper_2509_18824_amd.step as S
        if case["way"] == "probs":
            s["workspace"] = S.alloc_workspace(hb.hb_rules_probs_workspace_bytes(T, V))
        s["out"] = torch.empty((T, V), dtype=torch.float32 if case["way"] == "probs" else dt, device="cuda")
    return s


# ---- one pass --------------------------------------------------------------------------------------

def run(s):
    return (_run_own if own else _run_plain)[s["op"]](s)


def _own_pages(s):
    import paper_2509_18824_amd as hb
    c = s["case"]
    if c["way"] == "give":
        hb.hb_pages_give(c["page"], s["keep_len"], s["have"], s["block_table"], s["free_pages"], s["free_count"], s["have_out"], s["left"])
        return s["free_pages"], s["have_out"], s["left"]
    hb.hb_pages_take(c["page"], c["reserve"], s["prefix_len"], s["row_offset"], s["have"], s["free_pages"], s["free_count"], s["block_table"],
                     s["slots"], s["new_len"], s["have_out"], s["granted"], s["left"])
    return s["block_table"], s["slots"], s["new_len"], s["have_out"], s["granted"], s["left"]


def _own_append(s):
    import paper_2509_18824_amd as hb
    hb.hb_kv_append(s["desc"], s["k"], s["v"], s["slots"], s["k_pool"], s["v_pool"])
    return s["k_pool"], s["v_pool"]


def _own_attn(s):
    import paper_2509_18824_amd as hb
    hb.hb_prompt_attn(s["desc"], s["q"], s["k"], s["v"], s["k_pool"], s["v_pool"], s["block_table"], s["prefix_len"], s["row_offset"], s["out"],
                      s["lse"], s["workspace"])
    return (s["out"], s["lse"]) if s["case"]["lse"] else s["out"]


def _own_rules(s):
    import paper_2509_18824_amd as hb
    hb.hb_rules_count(s["tokens"], s["counts"])
    rules = (s["node_offset"], s["parent"], s["draft_ids"], s["counts"], s["rules"], s["bias_offset"], s["bias_id"], s["bias_value"], s["mask"],
             s["mask_row"])
    if s["case"]["way"] == "probs":
        hb.hb_rules_probs(s["logits"], s["case"]["nodes"], *rules, s["out"], s["workspace"])
    else:
        hb.hb_rules_logits(s["logits"], s["case"]["nodes"], *rules, s["out"])
    return s["out"], s["counts"]


_run_own = {"pages": _own_pages, "append": _own_append, "attn": _own_attn, "rules": _own_rules}


def _plain_pages(s):
    c = s["case"]
    page, have, count = c["page"], s["have"], s["free_count"]
    table = s["block_table"]
    entry = torch.arange(s["max_blocks"], device=table.device, dtype=torch.int32)[None, :]
    if c["way"] == "give":
        keep = torch.minimum(have, (s["keep_len"] + page - 1) // page)
        n = have - keep
        total = n.sum()
        first = n.cumsum(0) - n
        to = count + total - 1 - (first[:, None] + entry - keep[:, None])
        goes = (entry >= keep[:, None]) & (entry < have[:, None])
        free = torch.cat((s["free_pages"], torch.zeros_like(s["free_pages"][:1])))
        free.scatter_(0, torch.where(goes, to, s["blocks"]).flatten().long(), table.flatten())  # the last one is nobody's
        return free[:-1], keep, (count + total).to(torch.int32)
    offset, lens = s["row_offset"], s["prefix_len"]
    rows = offset[1:] - offset[:-1]
    want = (lens + rows + c["reserve"] + page - 1) // page
    fits = want <= s["max_blocks"]
    need = torch.where(fits, (want - have).clamp(min=0), 0)
    cum = need.cumsum(0)
    granted = fits & ((need == 0) | (cum <= count))
    have_out = torch.where(granted, torch.maximum(have, want), have)
    at = count - 1 - ((cum - need)[:, None] + entry - have[:, None])
    new = (entry >= have[:, None]) & (entry < have_out[:, None])
    table = torch.where(new, s["free_pages"][at.clamp(0, s["blocks"] - 1).long()], table)
    r = torch.arange(s["rows"], device=table.device)
    b = torch.searchsorted(offset[1:], r, right=True)
    p = lens[b] + r - offset[b]
    slot = table[b, (p // page).clamp(max=s["max_blocks"] - 1)] * page + p % page
    slots = torch.where(granted[b], slot, -1).to(torch.int32)
    left = count - torch.where(granted, need, 0).sum()
    return table, slots, torch.where(granted, lens + rows, lens), have_out, granted.to(torch.int32), left.to(torch.int32)


def _plain_append(s):
    page = s["case"]["page"]
    fine = s["slots"] >= 0
    at = s["slots"][fine].long()
    s["k_pool"][at // page, :, at % page] = s["k"][fine]
    s["v_pool"][at // page, :, at % page] = s["v"][fine]
    return s["k_pool"], s["v_pool"]


def _keys(s, pool, new, pos, b):
    """float32 [B, Hkv, n, D]: the cached rows of a sequence and then its own, zeros past them."""
    page, lens, offset = s["case"]["page"], s["prefix_len"][:, None], s["row_offset"]
    table = s["block_table"]
    cached = pos < lens
    old = pool[table[b, (pos // page).clamp(max=table.shape[1] - 1)], :, pos % page]
    at = (pos - lens + offset[:-1, None]).clamp(0, s["rows"] - 1)
    there = pos < lens + (offset[1:] - offset[:-1])[:, None]
    x = torch.where(cached[..., None, None], old, new[at])
    return torch.where(there[..., None, None], x, 0).float().transpose(1, 2)


def _plain_attn(s):
    c = s["case"]
    B, Hkv, G = c["B"], c["Hkv"], c["Hq"] // c["Hkv"]
    offset, lens = s["row_offset"], s["prefix_len"]
    b = torch.arange(B, device="cuda")[:, None]
    n, most = s["most_rows"], s["most_rows"] + s["longest"]
    pos = torch.arange(most, device="cuda")[None, :].expand(B, most)
    k, v = _keys(s, s["k_pool"], s["k"], pos, b), _keys(s, s["v_pool"], s["v"], pos, b)
    i = torch.arange(n, device="cuda")
    q = s["q"][(offset[:-1, None] + i).clamp(max=s["rows"] - 1)].float()  # [B, n, Hq, D]
    q = q.permute(0, 2, 1, 3).reshape(B, Hkv, G * n, c["D"])
    score = torch.matmul(q, k.transpose(2, 3)).mul_(s["scale"]).view(B, Hkv, G, n, most)
    score.masked_fill_((pos[:, None, :] > (lens[:, None] + i)[:, :, None])[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = score.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.view(B, Hkv, G * n, most), v).view(B, Hkv, G, n, c["D"]) / total
    lse = (top + total.log()).squeeze(-1)
    # back to the packed rows
    r = torch.arange(s["rows"], device="cuda")
    at = torch.searchsorted(offset[1:].long(), r, right=True)
    out = out.permute(0, 3, 1, 2, 4)[at, r - offset[at]].reshape(s["rows"], c["Hq"], c["D"]).to(s["q"].dtype)
    if not c["lse"]:
        return out
    return out, lse.permute(0, 3, 1, 2)[at, r - offset[at]].reshape(s["rows"], c["Hq"])


def _plain_rules(s):
    c = s["case"]
    B, V, N = c["B"], c["V"], c["nodes"]
    T = B * N
    tokens = s["tokens"]
    s["counts"].scatter_add_(1, tokens.clamp(min=0).long(), (tokens >= 0).int())
    b = torch.arange(B, device="cuda").repeat_interleave(N)
    # ancestors, the node itself among them and the root not
    i = torch.arange(N, device="cuda")
    path = ((s["parent"].view(B, N, 1) == i) | (i[:, None] == i)).float()
    for _ in range(6):  # paths of up to 64 steps
        path = torch.matmul(path, path).clamp(max=1)
    path[:, :, 0] = 0
    had = s["counts"][b]
    count = (had & 0x3fffffff).scatter_add_(1, s["draft_ids"].view(B, 1, N).expand(B, N, N).reshape(T, N).long(), path.view(T, N).int())
    rule = s["rules"][b]
    temperature, repetition, presence, frequency = (rule[:, k:k + 1] for k in range(4))
    z = s["logits"].float()
    z = torch.where(z != z, -math.inf, z)
    z = torch.where((count > 0) | (had >= 1 << 30), torch.where(z > 0, z / repetition, z * repetition), z)
    z = z - (presence * (count > 0) + frequency * count)
    n = s["bias_id"].numel()
    if n:
        owner = torch.searchsorted(s["bias_offset"][1:].contiguous(), torch.arange(n, device="cuda"), right=True)
        bias = torch.zeros((B, V), device="cuda")
        bias[owner, s["bias_id"].long()] = s["bias_value"]
        z = z + bias[b]
    if s["mask"] is not None:
        v = torch.arange(V, device="cuda")
        row = s["mask_row"].long()
        allowed = (s["mask"][row.clamp(min=0)][:, v >> 5] >> (v & 31)) & 1
        z = torch.where((allowed > 0) | (row < 0)[:, None], z, -math.inf)
    if c["way"] == "logits":
        return z.to(s["logits"].dtype), s["counts"]
    top, first = z.max(1, keepdim=True)
    first = torch.where(z == top, torch.arange(V, device="cuda"), V).amin(1, keepdim=True)
    left = top > -math.inf
    p = torch.where(left, ((z - top) / torch.where(temperature > 0, temperature, 1.0)).exp(), 0.0)
    p = p / torch.where(left, p.sum(1, keepdim=True), 1.0)
    one = (torch.arange(V, device="cuda") == first) & left
    return torch.where(temperature > 0, p, one.float()), s["counts"]


_run_plain = {"pages": _plain_pages, "append": _plain_append, "attn": _plain_attn, "rules": _plain_rules}


# ---- the definitions in 64 bits, one sequence and one row at a time ----------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"pages": lambda s: None, "append": _exact_append, "attn": _exact_attn, "rules": _exact_rules}[case["op"]](s)


def _exact_append(s):
    page, out = s["case"]["page"], []
    for pool, rows in ((s["k_pool"], s["k"]), (s["v_pool"], s["v"])):
        flat = pool.double().transpose(1, 2).flatten(0, 1)  # by slots
        source = torch.full((flat.shape[0],), -1, dtype=torch.int64, device=flat.device)
        kept = (s["slots"] >= 0).nonzero().squeeze(1)
        source[s["slots"][kept].long()] = kept
        flat = torch.where((source >= 0)[:, None, None], rows.double()[source.clamp(min=0)], flat)
        out.append(flat.unflatten(0, (-1, page)).transpose(1, 2).contiguous())
    return tuple(out)


def _exact_attn(s):
    c = s["case"]
    G, page = c["Hq"] // c["Hkv"], c["page"]
    offset, lens = s["row_offset"].tolist(), s["prefix_len"].tolist()
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    for b, L in enumerate(lens):
        lo, hi = offset[b], offset[b + 1]
        if lo == hi:
            continue
        pages = s["block_table"][b, :-(-L // page)].long()
        for h in range(c["Hkv"]):
            k, v = (torch.cat((pool[pages, h].reshape(-1, c["D"])[:L], rows[lo:hi, h])).double()
                    for pool, rows in ((s["k_pool"], s["k"]), (s["v_pool"], s["v"])))
            seen = torch.ones((hi - lo, L + hi - lo), dtype=torch.bool, device="cuda").tril(L)
            for g in range(h * G, h * G + G):
                a = (s["q"][lo:hi, g].double() @ k.T * s["scale"]).masked_fill(~seen, -math.inf)
                lse[lo:hi, g] = torch.logsumexp(a, 1)
                out[lo:hi, g] = torch.softmax(a, 1) @ v
    return (out, lse) if c["lse"] else out


def _exact_rules(s):
    c = s["case"]
    V, N = c["V"], c["nodes"]
    counts, parent, draft = s["counts"].clone(), s["parent"].tolist(), s["draft_ids"].tolist()
    at, rules = s["bias_offset"].tolist(), s["rules"].tolist()
    rows = s["mask_row"].tolist() if s["mask"] is not None else [-1] * (c["B"] * N)
    bit = torch.arange(32, device="cuda", dtype=torch.int32)
    out = torch.zeros((c["B"] * N, V), dtype=torch.float64, device="cuda")
    for b, tokens in enumerate(s["tokens"].tolist()):
        for x in tokens:
            if x >= 0:
                counts[b, x] += 1
        temperature, repetition, presence, frequency = s["rules"][b].double().tolist()
        for i in range(N):
            t = b * N + i
            own_count, j = (counts[b] & 0x3fffffff).double(), i
            while j > 0:
                own_count[draft[b * N + j]] += 1
                j = parent[b * N + j]
            z = s["logits"][t].double()
            z = torch.where(torch.isnan(z), -math.inf, z)
            seen = (own_count > 0) | (counts[b] >= 1 << 30)
            z = torch.where(seen, torch.where(z > 0, z / repetition, z * repetition), z)
            z = z - presence * (own_count > 0) - frequency * own_count
            z[s["bias_id"][at[b]:at[b + 1]].long()] += s["bias_value"][at[b]:at[b + 1]].double()
            if rows[t] >= 0:
                z[((s["mask"][rows[t]][:, None] >> bit) & 1).flatten()[:V] == 0] = -math.inf
            if c["way"] == "logits":
                out[t] = z
            elif not torch.isneginf(z).all():
                if temperature > 0:
                    out[t] = torch.softmax(z / temperature, 0)
                else:  # where 32 bits make two of them equal, the lower token is the largest in 32 bits
                    z = z.float()
                    out[t, (z == z.max()).nonzero()[0]] = 1
    return out, None


# ---- what a pass cannot do without -----------------------------------------------------------------

def work(case):
    op = case["op"]
    if op == "pages":
        rows = (case.get("rows_min", 0) + case.get("rows_max", 0)) / 2
        L = (case["L_min"] + case["L_max"]) / 2
        entries = case["B"] * ((L / 2 if case["way"] == "give" else rows + case["reserve"]) / case["page"] + 1)
        # lengths, offsets and counts; a page is read and written; a slot is written for each row
        return {"bytes": 4 * (6 * case["B"] + 2 * entries + case["B"] * rows), "flops": 0}
    if op == "rules":
        T, V, el = case["B"] * case["nodes"], case["V"], 2 if case["dtype"] == "bf16" else 4
        grammar = case["grammar"] * T * V / 8
        return {"bytes": T * V * (el + (4 if case["way"] == "probs" else el)) + case["B"] * V * 4 + grammar, "flops": 8 * T * V}
    el = 2 if case["dtype"] == "bf16" else 4
    if op == "append":
        return {"bytes": 4 * case["rows"] * case["Hkv"] * case["D"] * el, "flops": 0}
    rng = random.Random(case["rows_max"] * 1000003 + case["B"])
    counts = [rng.randint(case["rows_min"], case["rows_max"]) for _ in range(case["B"])]
    L = (case["L_min"] + case["L_max"]) / 2
    rows = sum(counts)
    pairs = sum(n * L + n * (n + 1) / 2 for n in counts)
    size = case["D"] * el
    return {"bytes": 2 * rows * (case["Hq"] + case["Hkv"]) * size + 2 * case["B"] * L * case["Hkv"] * size,
            "flops": 4 * pairs * case["Hq"] * case["D"]}
