"""What brings a request in, and its sampling rules (oracle, float64 and Python integers).

TEST INFRASTRUCTURE ONLY (see oracle/__init__.py).

Pages are taken one after the other in the order of the batch, which is the rule itself; prompts are attended row by row over the
keys that the row may see; sampling rules are applied to one row at a time, with the node's path walked to the root.
"""
from __future__ import annotations

import numpy as np

from .tree_attention import ancestors

PROMPT_FLAG = 1 << 30


def pages_take_ref(page, max_blocks, num_blocks, reserve, prefix_len, row_offset, pages, free_pages, block_table, slots):
    """``free_pages``: the free ones, the next at the end.  Returns (block_table, slots, new_len, pages_out, granted, free_left)."""
    free, table, slots = list(free_pages), np.array(block_table), np.array(slots)
    new_len, have_out, granted, full = [], [], [], False
    for b, (n, have) in enumerate(zip(prefix_len, pages)):
        lo, hi = int(row_offset[b]), int(row_offset[b + 1])
        want = -(-(int(n) + hi - lo + reserve) // page)
        need = max(0, want - int(have))
        ok = want <= max_blocks
        if ok and need:
            full = full or need > len(free)
            ok = not full
        if ok:
            for e in range(int(have), want):
                table[b, e] = free.pop()
        for j in range(hi - lo):
            p = int(n) + j
            e = table[b, p // page] if ok else -1
            slots[lo + j] = e * page + p % page if 0 <= e < num_blocks else -1
        new_len.append(int(n) + (hi - lo if ok else 0))
        have_out.append(max(int(have), want) if ok else int(have))
        granted.append(int(ok))
    return table, slots, np.array(new_len), np.array(have_out), np.array(granted), len(free)


def pages_give_ref(page, keep_len, pages, block_table, free_pages):
    """Returns (free pages, pages_out)."""
    keep = [min(int(h), -(-max(int(n), 0) // page)) for n, h in zip(keep_len, pages)]
    back = [int(block_table[b, e]) for b, h in enumerate(pages) for e in range(keep[b], int(h))]
    return list(free_pages) + back[::-1], np.array(keep)


def prompt_attn_ref(q, k, v, k_pool, v_pool, block_table, prefix_len, row_offset, softmax_scale):
    """(out [T, Hq, D], lse [T, Hq]); rows that no sequence has are zero."""
    q, k, v = (np.asarray(x, dtype=np.float64) for x in (q, k, v))
    T, Hq, D = q.shape
    Hkv = k.shape[1]
    G = Hq // Hkv
    out, lse = np.zeros((T, Hq, D)), np.zeros((T, Hq))
    for b in range(len(row_offset) - 1):
        lo, hi = int(row_offset[b]), int(row_offset[b + 1])
        n = 0 if prefix_len is None else int(prefix_len[b])
        pos = np.arange(n)
        if n:
            page = k_pool.shape[2]
            at = np.asarray(block_table)[b, pos // page]
            kp, vp = (np.asarray(x)[at, :, pos % page, :].astype(np.float64) for x in (k_pool, v_pool))
        else:
            kp = vp = np.zeros((0, Hkv, D))
        for i in range(lo, hi):
            keys, values = np.concatenate([kp, k[lo:i + 1]]), np.concatenate([vp, v[lo:i + 1]])
            for h in range(Hq):
                s = softmax_scale * (keys[:, h // G] @ q[i, h])
                m = s.max()
                e = np.exp(s - m)
                lse[i, h] = m + np.log(e.sum())
                out[i, h] = e @ values[:, h // G] / e.sum()
    return out, lse


def rules_logits_ref(logits, node_offset, parent, draft_ids, counts, rules, biases, mask, mask_row):
    """Adjusted logits [T, V].  ``biases``: for each sequence a list of (token, value); ``mask`` uint32 [masks, words]."""
    logits = np.asarray(logits, dtype=np.float64)
    T, V = logits.shape
    out = np.full((T, V), np.nan)
    for b in range(len(node_offset) - 1):
        n0, n1 = int(node_offset[b]), int(node_offset[b + 1])
        _, repetition, presence, frequency = (1.0, 1.0, 0.0, 0.0) if rules is None else (float(x) for x in rules[b])
        had = np.zeros(V, dtype=np.int64) if counts is None else np.asarray(counts[b], dtype=np.int64)
        for t in range(n0, n1):
            c = had % PROMPT_FLAG
            if parent is not None:
                for a in ancestors(parent[n0:n1], t - n0)[1:]:
                    c[int(draft_ids[n0 + a])] += 1
            seen = (c > 0) | (had >= PROMPT_FLAG)
            with np.errstate(invalid="ignore"):
                z = logits[t].copy()
                z = np.where(seen, np.where(z > 0, z / repetition, z * repetition), z)
                z = z - np.where(c > 0, presence + frequency * c, 0.0)
                for token, value in (biases[b] if biases else []):
                    z[token] += value
            z[np.isnan(z)] = -np.inf
            m = -1 if mask is None else t if mask_row is None else int(mask_row[t])
            if mask is not None and 0 <= m < len(mask):
                v = np.arange(V)
                z[(mask[m][v // 32].astype(np.int64) >> (v % 32)) & 1 == 0] = -np.inf
            out[t] = z
    return out


def rules_probs_ref(z, node_offset, rules):
    """Probabilities [T, V] of adjusted logits."""
    p = np.full(z.shape, np.nan)
    for b in range(len(node_offset) - 1):
        temperature = 1.0 if rules is None else float(rules[b][0])
        for t in range(int(node_offset[b]), int(node_offset[b + 1])):
            top, p[t] = z[t].max(), 0.0
            if top == -np.inf:
                continue
            if not temperature > 0:
                p[t, int(np.argmax(z[t]))] = 1.0
            elif top == np.inf:
                p[t] = (z[t] == top) / (z[t] == top).sum()
            else:
                e = np.exp((z[t] - top) / temperature)
                p[t] = e / e.sum()
    return p
