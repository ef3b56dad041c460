"""The 4-bit KV cache (oracle, float64): its number format, rows into it, attention weights, eviction.

Elements are E2M1 in blocks of 32 with a power of two as scale, the block format of the OCP microscaling
specification; scale = the smallest power of two under which the block's largest magnitude is at most 7.
"""
from __future__ import annotations

import numpy as np

BLOCK = 32
NAN_SCALE = 255
LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def kv4_quantise_ref(x):
    """x [..., D] -> codes uint8 [..., D / 2], scales uint8 [..., D / 32]."""
    x = np.asarray(x, dtype=np.float64)
    blocks = x.reshape(*x.shape[:-1], -1, BLOCK)
    scales = np.full(blocks.shape[:-1], NAN_SCALE, dtype=np.uint8)
    codes = np.zeros(blocks.shape, dtype=np.uint8)
    fine = np.isfinite(blocks).all(-1)
    # exponents from -126 to 125, tried from below: the first that brings the largest down to 7 or less, else the last
    top = np.abs(blocks[fine]).max(-1) if fine.any() else np.zeros(0)
    fits = top[:, None] <= 7 * np.exp2(np.arange(-126, 126, dtype=np.float64))
    first = np.where(fits.any(1), fits.argmax(1), 251)
    scales[fine] = (first + 1).astype(np.uint8)
    mag = np.minimum(np.abs(blocks[fine]) / np.exp2(first - 126.0)[:, None], 6.0)
    far = np.abs(mag[..., None] - LEVELS)
    nearest = far.min(-1, keepdims=True)
    # a tie is between neighbours: the even code of the two
    tied = far == nearest
    code = np.where(tied.sum(-1) == 1, tied.argmax(-1), np.where(tied.argmax(-1) % 2 == 0, tied.argmax(-1), tied.argmax(-1) + 1))
    codes[fine] = code + 8 * np.signbit(blocks[fine])
    codes = codes.reshape(x.shape)
    return codes[..., 0::2] | (codes[..., 1::2] << 4), scales


def kv4_values_ref(codes, scales):
    """float64 [..., D]."""
    codes, scales = np.asarray(codes, dtype=np.int64), np.asarray(scales, dtype=np.int64)
    nibbles = np.stack([codes % 16, codes // 16], -1).reshape(*codes.shape[:-1], -1)
    x = np.where(nibbles >= 8, -1.0, 1.0) * LEVELS[nibbles % 8]
    s = np.where(scales == NAN_SCALE, np.nan, np.exp2(scales - 127.0))
    return (x.reshape(*scales.shape, BLOCK) * s[..., None]).reshape(x.shape)


def kv4_append_ref(pool, rows, block_table, prefix_len, took, weight=None, pos=None, seq_len=None):
    """``pool``: [k_codes, k_scales, v_codes, v_scales], changed in place; ``rows``: (k, v) [n, Hkv, D];
    ``took[b]``: indices of the rows that join sequence b, in order.  Returns (slots per sequence, new_len)."""
    page, cap = pool[0].shape[2], block_table.shape[1] * pool[0].shape[2]
    slots, new_len = [], []
    for b, idx in enumerate(took):
        L = max(int(prefix_len[b]), 0)
        mine = []
        for j, r in enumerate(idx):
            p = L + j
            if p >= cap:
                mine.append(-1)
                continue
            blk, off = int(block_table[b, p // page]), p % page
            for i, x in enumerate(rows):
                pool[2 * i][blk, :, off], pool[2 * i + 1][blk, :, off] = kv4_quantise_ref(x[r])
            if weight is not None:
                weight[b, :, p] = 0
            if pos is not None:
                pos[b, :, p] = (L if seq_len is None else int(seq_len[b])) + j
            mine.append(blk * page + off)
        slots.append(mine)
        new_len.append(L + len(idx))
    return slots, np.array(new_len)


def kv4_attn_weight_ref(q, k_values, block_table, prefix_len, took, lse, softmax_scale, decay, weight):
    """``took[b]``: the committed rows of q [T, Hq, D]; k_values [blocks, Hkv, page, D].  Returns the new weights."""
    out = np.array(weight, dtype=np.float64)
    Hq, page, Hkv = q.shape[1], k_values.shape[2], k_values.shape[1]
    G = Hq // Hkv
    for b, idx in enumerate(took):
        p = np.arange(max(int(prefix_len[b]), 0))
        k = k_values[block_table[b, p // page], :, p % page, :]  # [L, Hkv, D]
        for g in range(Hkv):
            got = np.zeros(len(p))
            for r in idx:
                for h in range(g * G, (g + 1) * G):
                    got += np.exp(softmax_scale * (k[:, g] @ q[r, h]) - lse[r, h])
            out[b, g, :len(p)] = decay * out[b, g, :len(p)] + got
    return out


def kv4_evict_ref(length, budget, recent, sinks, seq_len, weight, pos):
    """One head: the slot whose position is afterwards in slot 0, 1, ..."""
    w = [-np.inf if np.isnan(x) else float(x) for x in weight[:length]]
    safe = [p >= seq_len - recent or p < sinks for p in pos[:length]]
    ranking = sorted(range(length), key=lambda s: (not safe[s], 0.0 if safe[s] else -w[s], s))
    stays = min(length, budget)
    chosen = set(ranking[:stays])
    arrivals = iter(sorted(s for s in chosen if s >= stays))
    return [s if s in chosen else next(arrivals) for s in range(stays)]
