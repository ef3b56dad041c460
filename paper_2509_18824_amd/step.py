"""Convenience wrappers that allocate outputs/workspaces as torch tensors and call the C ABI.

Nothing here computes: each function sizes buffers, fills an ``AttnDesc`` and forwards to the
library.  ``VerifyStep`` chains the calls of one verification step on the current stream.
"""
from __future__ import annotations

from dataclasses import dataclass
from typing import NamedTuple, Optional

import torch

from . import binding as hb


def make_desc(dtype, B, Hq, Hkv, D, page, max_blocks, num_blocks, total_nodes, max_nodes,
              softmax_scale, num_splits=0, hint=0, algo=hb.HB_ATTN_AUTO) -> hb.AttnDesc:
    code = hb.HB_F32 if dtype in ("f32", torch.float32) else hb.HB_BF16
    return hb.AttnDesc(dtype=code, batch=B, num_q_heads=Hq, num_kv_heads=Hkv, head_dim=D,
                       page_size=page, max_blocks_per_seq=max_blocks, num_blocks=num_blocks,
                       total_nodes=total_nodes, max_nodes_per_tree=max_nodes, num_splits=num_splits,
                       max_prefix_len_hint=hint, algo=algo, softmax_scale=float(softmax_scale))


@dataclass
class DeviceInputs:
    """Device copies of one batch (field names as in the C ABI)."""

    q: torch.Tensor
    k_tree: torch.Tensor
    v_tree: torch.Tensor
    k_pool: torch.Tensor
    v_pool: torch.Tensor
    block_table: torch.Tensor
    prefix_len: torch.Tensor
    node_offset: torch.Tensor
    parent: torch.Tensor


def to_device(inp, device="cuda") -> DeviceInputs:
    f = lambda t: t.to(device).contiguous()
    return DeviceInputs(f(inp.q), f(inp.k_tree), f(inp.v_tree), f(inp.k_pool), f(inp.v_pool),
                        f(inp.block_table), f(inp.prefix_len), f(inp.node_offset), f(inp.parent))


def desc_for(inp, num_splits=0, hint=0, algo=hb.HB_ATTN_AUTO) -> hb.AttnDesc:
    max_nodes = int((inp.node_offset[1:] - inp.node_offset[:-1]).max()) if inp.B else 1
    return make_desc(inp.dtype, inp.B, inp.Hq, inp.Hkv, inp.D, inp.page, inp.max_blocks,
                     inp.num_blocks, inp.total_nodes, max_nodes, inp.softmax_scale, num_splits,
                     hint, algo)


def alloc_workspace(nbytes: int, device="cuda") -> Optional[torch.Tensor]:
    if nbytes == 0:
        return None
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


def tree_verify_attn(desc: hb.AttnDesc, dev: DeviceInputs, want_lse=True, workspace=None, out=None):
    """Returns (out, lse).  Allocates what is not passed in."""
    if out is None:
        out = torch.empty_like(dev.q)
    lse = torch.empty(dev.q.shape[:2], dtype=torch.float32, device=dev.q.device) if want_lse else None
    if workspace is None:
        workspace = alloc_workspace(hb.hb_tree_verify_attn_workspace_bytes(desc), dev.q.device)
    hb.hb_tree_verify_attn(desc, dev.q, dev.k_tree, dev.v_tree, dev.k_pool, dev.v_pool, dev.block_table,
                           dev.prefix_len, dev.node_offset, dev.parent, out, lse, workspace)
    return out, lse


def lmhead_argmax(hidden, weight, want_max=True, workspace=None):
    M = hidden.shape[0]
    ids = torch.empty(M, dtype=torch.int32, device=hidden.device)
    mx = torch.empty(M, dtype=torch.float32, device=hidden.device) if want_max else None
    if workspace is None:
        workspace = alloc_workspace(max(8, hb.hb_lmhead_argmax_workspace_bytes(M)), hidden.device)
    hb.hb_lmhead_argmax(hidden, weight, ids, mx, workspace)
    return ids, mx


def tree_accept(node_offset, parent, draft_ids, target_ids, max_path, max_nodes, prev_target=None):
    B = node_offset.numel() - 1
    dev = node_offset.device
    accept_len = torch.empty(B, dtype=torch.int32, device=dev)
    accept_path = torch.empty((B, max_path), dtype=torch.int32, device=dev)
    out_tokens = torch.empty((B, max_path), dtype=torch.int32, device=dev)
    bonus = torch.empty(B, dtype=torch.int32, device=dev)
    hb.hb_tree_accept(B, max_nodes, node_offset, parent, draft_ids, target_ids, max_path, accept_len,
                      accept_path, out_tokens, bonus, prev_target=prev_target)
    return accept_len, accept_path, out_tokens, bonus


def tree_accept_sample(node_offset, parent, draft_ids, p_target, q_draft, u_accept, u_bonus, max_path, max_nodes):
    """u_accept / u_bonus: int32 tensors holding the bit patterns of the 32-bit uniforms."""
    B = node_offset.numel() - 1
    dev = node_offset.device
    accept_len = torch.empty(B, dtype=torch.int32, device=dev)
    accept_path = torch.empty((B, max_path), dtype=torch.int32, device=dev)
    out_tokens = torch.empty((B, max_path), dtype=torch.int32, device=dev)
    bonus = torch.empty(B, dtype=torch.int32, device=dev)
    ws = alloc_workspace(max(4, hb.hb_tree_accept_sample_workspace_bytes(B, p_target.shape[1])), dev)
    hb.hb_tree_accept_sample(B, max_nodes, node_offset, parent, draft_ids, p_target, q_draft, u_accept, u_bonus,
                             max_path, accept_len, accept_path, out_tokens, bonus, ws)
    return accept_len, accept_path, out_tokens, bonus


def topk_logprob(logits, k):
    """ids int32 [M, k], logp float32 [M, k] of the k best tokens of every row."""
    M, V = logits.shape
    dev = logits.device
    ids = torch.empty((M, k), dtype=torch.int32, device=dev)
    logp = torch.empty((M, k), dtype=torch.float32, device=dev)
    ws = alloc_workspace(max(8, hb.hb_topk_logprob_workspace_bytes(M, V, k)), dev)
    hb.hb_topk_logprob(logits, k, ids, logp, ws)
    return ids, logp


class DraftTreeBuilder:
    """Device state of the draft tree's construction for a batch: the candidate pool and the
    frontier.  ``grow`` takes the top-k outputs of the rows the draft model just ran on (the
    root at level 0, then the frontier nodes in order); ``finalize`` emits the tree in the
    verification calls' layout."""

    def __init__(self, B: int, K: int, T: int, device="cuda"):
        self.B, self.K, self.T, self.level = B, K, T, 0
        C = hb.hb_draft_tree_candidates(K, T)
        if C <= 0:
            raise ValueError("unsupported K / T")
        self.C = C
        # what starts at zero is cleared by one launch
        zeros = torch.zeros(2 * B * (C + K), dtype=torch.int32, device=device).split([B * C, B * C, B * K, B * K])
        self.cand_score = zeros[0].view(torch.float32).view(B, C)
        self.cand_token = zeros[1].view(B, C)
        self.cand_parent = torch.full((B, C), -1, dtype=torch.int32, device=device)
        self.frontier = zeros[2].view(B, K)
        self.frontier_slot = zeros[3].view(B, K)

    def grow(self, child_ids, child_logp):
        hb.hb_tree_grow(self.B, self.K, self.T, self.level, child_ids, child_logp, self.cand_score, self.cand_token,
                        self.cand_parent, self.frontier, self.frontier_slot)
        self.level += 1
        return self.frontier, self.frontier_slot

    def finalize(self, n_nodes: int, root_token):
        B, dev = self.B, self.cand_score.device
        i32 = lambda *shape: torch.empty(shape, dtype=torch.int32, device=dev)
        out = dict(node_offset=i32(B + 1), parent=i32(B * n_nodes), draft_ids=i32(B * n_nodes), depth=i32(B * n_nodes),
                   anc_mask=torch.empty(B * n_nodes, dtype=torch.int64, device=dev), node_cand=i32(B * n_nodes),
                   node_score=torch.empty(B * n_nodes, dtype=torch.float32, device=dev))
        hb.hb_tree_finalize(B, self.K, self.T, n_nodes, self.cand_score, self.cand_token, self.cand_parent, root_token,
                            out["node_offset"], out["parent"], out["draft_ids"], out["depth"], out["anc_mask"],
                            out["node_cand"], out["node_score"])
        return out


def linear(x, w, residual, out):
    """out = x w^T (+ residual); small token counts take the split-K path (its workspace is allocated here)."""
    nbytes = hb.hb_proj_workspace_bytes(x.shape[0], x.shape[1], w.shape[0])
    ws = alloc_workspace(nbytes, x.device) if nbytes else None
    hb.hb_out_project_ws(x, w, residual, out, ws)


class MetaQueryLayer:
    """The draft model's intermediate layer up to fc1: meta-query cross-attention over the layer
    features of every token, output projection with the skip connection, fc1.  Weights bf16 in
    the y = x W^T layout; the key projection is folded into the queries at construction."""

    def __init__(self, f_q, w_q, w_k, w_v, w_o, w_fc1, H: int, residual_layers=None):
        self.Q, self.D = f_q.shape
        self.H, self.residual_layers = H, residual_layers
        self.w_v, self.w_o, self.w_fc1 = w_v, w_o, w_fc1
        dev = f_q.device
        self.a_fold = torch.empty(hb.hb_meta_query_fold_bytes(self.Q, self.D, H) // 2, dtype=torch.bfloat16, device=dev)
        ws = torch.empty(self.Q * self.D, dtype=torch.float32, device=dev)
        hb.hb_meta_query_fold(H, f_q, w_q, w_k, self.a_fold, ws)

    def run(self, feats):
        """feats bf16 [S, L, D] -> (F_c [S, Q * D], fc1 output [S, N1])."""
        S, L, D = feats.shape
        Q, dev = self.Q, feats.device
        bf = lambda *shape: torch.empty(shape, dtype=torch.bfloat16, device=dev)
        pre, f_c = bf(S * Q, D), bf(S * Q, D)
        res = bf(S * Q, D) if self.residual_layers is not None else None
        pre_, res_ = pre.view(S, Q, D), None if res is None else res.view(S, Q, D)
        if hb.hb_meta_query_attn_project_pays(S, L, D, self.H, Q):  # values projected after the mixing
            ws = alloc_workspace(hb.hb_meta_query_attn_project_workspace_bytes(S, D, self.H, Q), dev)
            hb.hb_meta_query_attn_project(self.H, Q, feats, self.w_v, self.a_fold, self.residual_layers, pre_, res_, ws)
        else:
            v_proj = bf(S * L, D)
            hb.hb_out_project(feats.view(S * L, D), self.w_v, None, v_proj)
            ws = torch.empty(hb.hb_meta_query_attn_workspace_bytes(S, D, self.H, Q) // 4, dtype=torch.float32, device=dev)
            hb.hb_meta_query_attn(self.H, Q, feats, v_proj.view(S, L, D), self.a_fold, self.residual_layers, pre_, res_, ws)
        linear(pre, self.w_o, res, f_c)
        f_c = f_c.view(S, Q * D)
        out = bf(S, self.w_fc1.shape[0])
        linear(f_c, self.w_fc1, None, out)
        return f_c, out


def fc_concat(a, b, w_a, w_b):
    """fc over the concatenation [a, b]: a w_a^T + b w_b^T (w_a, w_b: the two column blocks of the
    layer's weight, stored as separate matrices)."""
    T = a.shape[0]
    tmp = torch.empty((T, w_a.shape[0]), dtype=torch.bfloat16, device=a.device)
    out = torch.empty_like(tmp)
    if a.shape[1] != b.shape[1]:  # column blocks of different widths
        linear(a, w_a, None, tmp)
        linear(b, w_b, tmp, out)
        return out
    N, K = w_a.shape
    nbytes = max(hb.hb_proj_workspace_bytes(T, K, N), hb.hb_proj_workspace_bytes(T, 2 * K, N))
    hb.hb_out_project_two_ws(a, w_a, b, w_b, tmp, out, alloc_workspace(nbytes, a.device))
    return out


def kv_compact(desc, dev: DeviceInputs, accept_len, accept_path):
    B, max_path = accept_path.shape
    out_slots = torch.empty((B, max_path), dtype=torch.int32, device=accept_path.device)
    new_len = torch.empty(B, dtype=torch.int32, device=accept_path.device)
    hb.hb_kv_compact(desc, dev.k_tree, dev.v_tree, dev.k_pool, dev.v_pool, dev.block_table, dev.prefix_len,
                     dev.node_offset, accept_len, accept_path, max_path, out_slots, new_len)
    return out_slots, new_len


class Kv4Pool(NamedTuple):
    """One layer's 4-bit cache: codes [num_blocks, Hkv, page, D / 2] and scales [num_blocks, Hkv, page, D / 32] of K and V."""

    k_codes: torch.Tensor
    k_scales: torch.Tensor
    v_codes: torch.Tensor
    v_scales: torch.Tensor


def kv4_pool(num_blocks: int, Hkv: int, page: int, D: int, device="cuda") -> Kv4Pool:
    u8 = lambda n: torch.empty((num_blocks, Hkv, page, n), dtype=torch.uint8, device=device)
    return Kv4Pool(u8(D // 2), u8(D // 32), u8(D // 2), u8(D // 32))


class PagePool:
    """Who has which page of a cache: every sequence's pages and committed length, and the pages that are free, on the device.

    ``take`` gives pages to sequences that get ``row_offset[b+1] - row_offset[b]`` new positions (and ``reserve`` more, for a tree's
    accepted nodes) and says where the new rows go; ``length`` is advanced by ``advance``, when they are there.  A sequence that is not
    ``granted`` keeps its length, and its rows' slots are -1, which the append passes over.  ``give`` takes back what is behind
    ``keep_len`` positions (all: 0).  A sequence that ends has ``length`` set to -1 as well, an empty place, which takes no pages (0 is a
    sequence that has no positions yet: it is given those that ``reserve`` asks for); the next request there begins with 0.  A verification
    step's ``new_len`` is 0 for an empty place, which has to stay one.  Nothing is synchronised or allocated, so a HIP graph can hold it
    all."""

    def __init__(self, B: int, page: int, max_blocks: int, num_blocks: int, max_rows: int, reserve: int = 0, device="cuda"):
        i32 = lambda n, value=0: torch.full((n,), value, dtype=torch.int32, device=device)
        self.page, self.reserve = page, reserve
        self.block_table = i32(B * max_blocks, -1).view(B, max_blocks)
        self.length, self.pages, self.new_len, self.granted = i32(B), i32(B), i32(B), i32(B)
        self.free_pages = torch.arange(num_blocks - 1, -1, -1, dtype=torch.int32, device=device)  # page 0 is the first to go
        self.free_count = i32(1, num_blocks)
        self.slots = i32(max_rows, -1)
        self._pages, self._free = i32(B), i32(1)

    def take(self, row_offset):
        self.slots.fill_(-1)  # rows behind the last sequence have no place
        hb.hb_pages_take(self.page, self.reserve, self.length, row_offset, self.pages, self.free_pages, self.free_count, self.block_table,
                         self.slots, self.new_len, self._pages, self.granted, self._free)
        self._keep()

    def advance(self):
        self.length.copy_(self.new_len)

    def give(self, keep_len):
        hb.hb_pages_give(self.page, keep_len, self.pages, self.block_table, self.free_pages, self.free_count, self._pages, self._free)
        self._keep()

    def _keep(self):
        self.pages.copy_(self._pages)
        self.free_count.copy_(self._free)


def prompt_attn(desc: hb.AttnDesc, q, k_rows, v_rows, row_offset, k_pool=None, v_pool=None, block_table=None, prefix_len=None, want_lse=True,
                workspace=None, out=None):
    """Returns (out, lse).  Allocates what is not passed in."""
    if out is None:
        out = torch.empty_like(q)
    lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device) if want_lse else None
    if workspace is None:
        workspace = alloc_workspace(hb.hb_prompt_attn_workspace_bytes(desc), q.device)
    hb.hb_prompt_attn(desc, q, k_rows, v_rows, k_pool, v_pool, block_table, prefix_len, row_offset, out, lse, workspace)
    return out, lse


@dataclass
class SamplingRules:
    """What a batch's requests want of the next token (field names as in the C ABI); a field that is None is not there."""

    counts: Optional[torch.Tensor] = None       # int32 [B, V]
    rules: Optional[torch.Tensor] = None        # float32 [B, 4]: temperature, repetition, presence, frequency
    bias_offset: Optional[torch.Tensor] = None  # int32 [B + 1]
    bias_id: Optional[torch.Tensor] = None      # int32 [n_bias]
    bias_value: Optional[torch.Tensor] = None   # float32 [n_bias]
    mask: Optional[torch.Tensor] = None         # int32 [num_masks, ceil(V / 32)]
    mask_row: Optional[torch.Tensor] = None     # int32 [T]

    def fields(self):
        return self.counts, self.rules, self.bias_offset, self.bias_id, self.bias_value, self.mask, self.mask_row


def rules_probs(logits, rules: SamplingRules, node_offset=None, parent=None, draft_ids=None, max_nodes: int = 1, probs=None, workspace=None):
    """The probabilities of each row's next token.  ``node_offset`` None: one row a sequence.  Allocates what is not passed in."""
    if probs is None:
        probs = torch.empty(logits.shape, dtype=torch.float32, device=logits.device)
    if workspace is None:
        workspace = alloc_workspace(hb.hb_rules_probs_workspace_bytes(*logits.shape), logits.device)
    hb.hb_rules_probs(logits, max_nodes, node_offset, parent, draft_ids, *rules.fields(), probs, workspace)
    return probs


class VerifyStep:
    """Pre-allocated buffers for one full verification step (attention of one layer, LM head,
    acceptance, compaction); ``run`` only enqueues kernels."""

    def __init__(self, desc: hb.AttnDesc, dev: DeviceInputs, weight: torch.Tensor, draft_ids: torch.Tensor,
                 max_path: int):
        self.desc, self.dev, self.weight, self.draft_ids, self.max_path = desc, dev, weight, draft_ids, max_path
        d = dev.q.device
        T, Hq, D = dev.q.shape
        B = desc.batch
        self.out = torch.empty_like(dev.q)
        self.ws_attn = alloc_workspace(hb.hb_tree_verify_attn_workspace_bytes(desc), d)
        self.ws_lm = alloc_workspace(max(8, hb.hb_lmhead_argmax_workspace_bytes(T)), d)
        self.target_ids = torch.empty(T, dtype=torch.int32, device=d)
        self.accept_len = torch.empty(B, dtype=torch.int32, device=d)
        self.accept_path = torch.empty((B, max_path), dtype=torch.int32, device=d)
        self.out_tokens = torch.empty((B, max_path), dtype=torch.int32, device=d)
        self.bonus = torch.empty(B, dtype=torch.int32, device=d)
        self.out_slots = torch.empty((B, max_path), dtype=torch.int32, device=d)
        self.new_len = torch.empty(B, dtype=torch.int32, device=d)

    def run(self, compact=True):
        dev, desc = self.dev, self.desc
        hidden = self.out.view(self.out.shape[0], -1)  # [T, Hq*D]: attention output feeds the LM head
        hb.hb_tree_verify_attn_clearing(desc, dev.q, dev.k_tree, dev.v_tree, dev.k_pool, dev.v_pool, dev.block_table,
                                        dev.prefix_len, dev.node_offset, dev.parent, self.out, None, self.ws_attn,
                                        self.ws_lm, hidden.shape[0])
        hb.hb_lmhead_accept_cleared(desc, hidden, self.weight, self.draft_ids, dev.node_offset, dev.parent, self.max_path,
                                    self.target_ids, self.accept_len, self.accept_path, self.out_tokens, self.bonus, self.ws_lm,
                                    int(bool(compact)), (dev.k_tree, dev.v_tree, dev.k_pool, dev.v_pool), dev.block_table,
                                    dev.prefix_len, self.out_slots, self.new_len)


class SampledVerifyStep:
    """Buffers of a verification step whose tokens are sampled as each request wants them: attention of one layer, logits, their
    probabilities by the rules, acceptance by sampling, compaction, and the count of what came out.  ``q_draft`` is what the nodes were
    drawn from (float32 [T, V]); ``u_accept`` and ``u_bonus`` hold the step's random bits.  ``rules.counts`` holds the trees' roots when
    ``run`` is called, and what the step emitted when it is done.  ``run`` only enqueues kernels."""

    def __init__(self, desc: hb.AttnDesc, dev: DeviceInputs, weight: torch.Tensor, draft_ids, q_draft, u_accept, u_bonus, max_path: int,
                 rules: SamplingRules):
        self.desc, self.dev, self.weight, self.max_path, self.rules = desc, dev, weight, max_path, rules
        self.draft_ids, self.q_draft, self.u_accept, self.u_bonus = draft_ids, q_draft, u_accept, u_bonus
        d, B = dev.q.device, desc.batch
        (V, K), T = weight.shape, dev.q.shape[0]
        i32 = lambda *shape: torch.empty(shape, dtype=torch.int32, device=d)
        self.out = torch.empty_like(dev.q)
        self.logits = torch.empty((T, V), dtype=weight.dtype, device=d)
        self.probs = torch.empty((T, V), dtype=torch.float32, device=d)
        self.ws_attn = alloc_workspace(hb.hb_tree_verify_attn_workspace_bytes(desc), d)
        self.ws_proj = alloc_workspace(hb.hb_proj_workspace_bytes(T, K, V), d)
        self.ws_rules = alloc_workspace(hb.hb_rules_probs_workspace_bytes(T, V), d)
        self.ws_accept = alloc_workspace(max(4, hb.hb_tree_accept_sample_workspace_bytes(B, V)), d)
        self.accept_len, self.bonus, self.new_len = i32(B), i32(B), i32(B)
        self.accept_path, self.out_tokens, self.out_slots = i32(B, max_path), i32(B, max_path), i32(B, max_path)

    def run(self, compact=True):
        dev, desc = self.dev, self.desc
        hb.hb_tree_verify_attn(desc, dev.q, dev.k_tree, dev.v_tree, dev.k_pool, dev.v_pool, dev.block_table, dev.prefix_len,
                               dev.node_offset, dev.parent, self.out, None, self.ws_attn)
        hb.hb_out_project_ws(self.out.view(self.out.shape[0], -1), self.weight, None, self.logits, self.ws_proj)
        rules_probs(self.logits, self.rules, dev.node_offset, dev.parent, self.draft_ids, desc.max_nodes_per_tree, self.probs, self.ws_rules)
        hb.hb_tree_accept_sample(desc.batch, desc.max_nodes_per_tree, dev.node_offset, dev.parent, self.draft_ids, self.probs, self.q_draft,
                                 self.u_accept, self.u_bonus, self.max_path, self.accept_len, self.accept_path, self.out_tokens, self.bonus,
                                 self.ws_accept)
        if compact:
            hb.hb_kv_compact(desc, dev.k_tree, dev.v_tree, dev.k_pool, dev.v_pool, dev.block_table, dev.prefix_len, dev.node_offset,
                             self.accept_len, self.accept_path, self.max_path, self.out_slots, self.new_len)
        if self.rules.counts is not None:
            hb.hb_rules_count(self.out_tokens, self.rules.counts)


class Kv4VerifyStep:
    """Verification steps of one layer over a 4-bit cache that is kept within a budget.

    ``run`` enqueues one step: attention over the cache and the nodes' own keys, LM head and acceptance, the attention weight
    that the cached positions received from the accepted nodes, and the append of these nodes.  ``advance`` makes the step's
    lengths the next one's; ``evict`` cuts every head's positions back to ``budget`` (the last ``recent`` and the first
    ``sinks`` ones stay).  A program calls it when lengths come near the pages that the table maps, between steps.  ``dev.k_pool``
    and ``dev.v_pool`` are not used; ``dev.prefix_len`` is advanced in place."""

    def __init__(self, desc: hb.AttnDesc, dev: DeviceInputs, pool: Kv4Pool, weight: torch.Tensor, draft_ids: torch.Tensor,
                 max_path: int, budget: int, recent: int = 0, sinks: int = 0, decay: float = 1.0, seq_len=None):
        self.desc, self.dev, self.pool, self.weight, self.draft_ids, self.max_path = desc, dev, pool, weight, draft_ids, max_path
        self.budget, self.recent, self.sinks, self.decay = budget, recent, sinks, decay
        d, B, T = dev.q.device, desc.batch, desc.total_nodes
        i32 = lambda *shape: torch.empty(shape, dtype=torch.int32, device=d)
        slots = (B, desc.num_kv_heads, desc.max_blocks_per_seq * desc.page_size)
        self.seq_len = dev.prefix_len.clone() if seq_len is None else seq_len
        # what is cached already has no weight yet, and is where it was written
        self.slot_weight = torch.zeros(slots, dtype=torch.float32, device=d)
        self.slot_pos = torch.arange(slots[2], dtype=torch.int32, device=d).expand(slots).contiguous()
        self.out = torch.empty_like(dev.q)
        self.lse = torch.empty(dev.q.shape[:2], dtype=torch.float32, device=d)
        self.ws_attn = alloc_workspace(hb.hb_tree_verify_attn_kv4_workspace_bytes(desc), d)
        self.ws_lm = alloc_workspace(max(8, hb.hb_lmhead_argmax_workspace_bytes(T)), d)
        self.ws_evict = alloc_workspace(hb.hb_kv4_evict_workspace_bytes(desc, budget), d)
        self.target_ids, self.accept_len, self.bonus = i32(T), i32(B), i32(B)
        self.accept_path, self.out_tokens, self.out_slots = i32(B, max_path), i32(B, max_path), i32(B, max_path)
        self.new_len, self.kept = i32(B), i32(B, desc.num_kv_heads, budget)

    def run(self):
        dev, desc = self.dev, self.desc
        hb.hb_tree_verify_attn_kv4(desc, dev.q, dev.k_tree, dev.v_tree, *self.pool, dev.block_table, dev.prefix_len,
                                   dev.node_offset, dev.parent, self.out, self.lse, self.ws_attn)
        hb.hb_lmhead_accept(desc, self.out.view(self.out.shape[0], -1), self.weight, self.draft_ids, dev.node_offset, dev.parent,
                            self.max_path, self.target_ids, self.accept_len, self.accept_path, self.out_tokens, self.bonus,
                            self.ws_lm)
        hb.hb_kv4_attn_weight(desc, dev.q, self.pool.k_codes, self.pool.k_scales, dev.block_table, dev.prefix_len,
                              dev.node_offset, self.accept_len, self.accept_path, self.max_path, self.lse, self.decay,
                              self.slot_weight)
        hb.hb_kv4_compact(desc, dev.k_tree, dev.v_tree, *self.pool, dev.block_table, dev.prefix_len, dev.node_offset,
                          self.accept_len, self.accept_path, self.max_path, self.seq_len, self.slot_weight, self.slot_pos,
                          self.out_slots, self.new_len)

    def advance(self):
        self.dev.prefix_len.copy_(self.new_len)
        self.seq_len.add_(self.accept_len)

    def evict(self):
        dev = self.dev
        hb.hb_kv4_evict(self.desc, self.budget, self.recent, self.sinks, *self.pool, dev.block_table, dev.prefix_len, self.seq_len,
                        self.slot_weight, self.slot_pos, self.slot_weight, self.slot_pos, self.kept, self.new_len, self.ws_evict)
        dev.prefix_len.copy_(self.new_len)


class VerifyLayerStack:
    """Buffers and call chain of one verification step through ``n_layers`` decoder layers, then
    LM head with argmax, acceptance, and the append of the accepted nodes' K/V to every layer's
    pools.  Without ``mlp`` a layer is its attention half (QKV projection + rotary embedding ->
    tree-verify attention over that layer's KV pools -> output projection with residual).  With
    ``mlp = dict(norm1=[..], norm2=[..], w_gate_up=[..], w_down=[..], norm_f=.., eps=..)`` it is the
    whole pre-norm layer: RMSNorm in front of the attention half, then RMSNorm -> gated-SiLU
    projection -> down projection with residual, and a final RMSNorm in front of the LM head.
    ``run`` only enqueues kernels on the current stream (no allocation, no host synchronisation),
    so a step can be captured into a HIP graph once and replayed."""

    def __init__(self, desc: hb.AttnDesc, dev: DeviceInputs, pools, w_qkv, w_o, lm_weight, draft_ids, max_path: int,
                 hidden0: torch.Tensor, theta: float = 1e6, mlp=None):
        self.desc, self.dev, self.pools, self.w_qkv, self.w_o = desc, dev, pools, w_qkv, w_o
        self.lm_weight, self.draft_ids, self.max_path, self.theta = lm_weight, draft_ids, max_path, theta
        d = hidden0.device
        T, Hq, D = dev.q.shape
        Hkv = dev.k_tree.shape[1]
        B = desc.batch
        self.n_layers = len(pools)
        self.hidden = [hidden0] + [torch.empty_like(hidden0) for _ in range(2)]  # input, ping, pong
        self.mlp = mlp
        self.positions = torch.empty(T, dtype=torch.int32, device=d)
        self.cos = torch.empty((T, D // 2), dtype=torch.float32, device=d)
        self.sin = torch.empty_like(self.cos)
        self.q = torch.empty_like(dev.q)
        self.k_tree = [torch.empty_like(dev.k_tree) for _ in range(self.n_layers)]  # kept for the compaction
        self.v_tree = [torch.empty_like(dev.v_tree) for _ in range(self.n_layers)]
        self.attn_out = torch.empty_like(dev.q)
        self.ws_attn = alloc_workspace(hb.hb_tree_verify_attn_workspace_bytes(desc), d)
        self.ws_lm = alloc_workspace(max(8, hb.hb_lmhead_argmax_workspace_bytes(T)), d)
        K = hidden0.shape[1]
        proj_bytes = max(hb.hb_proj_workspace_bytes(T, K, w_qkv[0].shape[0]), hb.hb_proj_workspace_bytes(T, K, w_o[0].shape[0]))
        if mlp is not None:
            F = mlp["w_down"][0].shape[1]
            proj_bytes = max(proj_bytes, hb.hb_proj_workspace_bytes(T, K, 2 * F), hb.hb_proj_workspace_bytes(T, F, K))
            self.normed = torch.empty_like(hidden0)
            self.mid = torch.empty_like(hidden0)      # the layer's hidden state between its two halves
            self.act = torch.empty((T, F), dtype=hidden0.dtype, device=d)
        self.ws_proj = alloc_workspace(proj_bytes, d) if proj_bytes else None  # small token counts: split-K partials
        self.target_ids = torch.empty(T, dtype=torch.int32, device=d)
        self.accept_len = torch.empty(B, dtype=torch.int32, device=d)
        self.accept_path = torch.empty((B, max_path), dtype=torch.int32, device=d)
        self.out_tokens = torch.empty((B, max_path), dtype=torch.int32, device=d)
        self.bonus = torch.empty(B, dtype=torch.int32, device=d)
        self.out_slots = torch.empty((B, max_path), dtype=torch.int32, device=d)
        self.new_len = torch.empty(B, dtype=torch.int32, device=d)
        # tables of every layer's tensor addresses, for the compaction of all layers in one launch
        table = lambda ts: torch.tensor([t.data_ptr() for t in ts], dtype=torch.int64, device=d)
        self.ptr_tables = (table(self.k_tree), table(self.v_tree), table([p[0] for p in pools]),
                           table([p[1] for p in pools]))

    def run(self, compact=True, on_call=None):
        """``on_call(name)`` (optional) is invoked before every library call, e.g. to record events.  What a plain run does
        in one call (a projection and the normalisation of its result; LM head, acceptance and append) is then made by
        the calls it consists of, so that each has its name; the sum of a normalisation may round differently."""
        dev, desc = self.dev, self.desc
        T = self.q.shape[0]
        mark = on_call or (lambda name: None)

        def project(x, w, residual, out, norm):
            """Into the residual stream; norm: the weight that normalises it for the call that follows, or None."""
            if norm is None or on_call:
                hb.hb_out_project_ws(x, w, residual, out, self.ws_proj)
                if norm is not None:
                    mark("rmsnorm")
                    hb.hb_rmsnorm(out, norm, self.mlp["eps"], self.normed)
            else:
                hb.hb_out_project_norm_ws(x, w, residual, out, norm, self.mlp["eps"], self.normed, self.ws_proj)

        mark("positions")
        hb.hb_tree_positions(desc.batch, desc.max_nodes_per_tree, dev.node_offset, dev.parent, dev.prefix_len,
                             self.positions)
        hb.hb_rope_table(self.q.shape[2], self.theta, self.positions, self.cos, self.sin)
        x = self.hidden[0]
        mlp = self.mlp
        if mlp is not None and self.n_layers:
            mark("rmsnorm")
            hb.hb_rmsnorm(x, mlp["norm1"][0], mlp["eps"], self.normed)
        for l in range(self.n_layers):
            nxt = self.hidden[1 + (l & 1)]
            y = nxt if mlp is None else self.mid
            kp, vp = self.pools[l]
            a = x if mlp is None else self.normed
            mark("qkv_rope_project")
            hb.hb_qkv_rope_project_ws(a, self.w_qkv[l], None, self.cos, self.sin, self.q, self.k_tree[l],
                                      self.v_tree[l], self.ws_proj)
            mark("tree_verify_attn")
            # the last layer's also clears the LM head's keys
            hb.hb_tree_verify_attn_clearing(desc, self.q, self.k_tree[l], self.v_tree[l], kp, vp, dev.block_table,
                                            dev.prefix_len, dev.node_offset, dev.parent, self.attn_out, None, self.ws_attn,
                                            self.ws_lm, T if l == self.n_layers - 1 else 0)
            mark("out_project")
            project(self.attn_out.view(T, -1), self.w_o[l], x, y, None if mlp is None else mlp["norm2"][l])
            if mlp is not None:
                mark("swiglu_project")
                hb.hb_swiglu_project(self.normed, mlp["w_gate_up"][l], self.act, self.ws_proj)
                mark("down_project")
                project(self.act, mlp["w_down"][l], y, nxt, mlp["norm1"][l + 1] if l + 1 < self.n_layers else mlp.get("norm_f"))
            x = nxt
        if mlp is not None and mlp.get("norm_f") is not None:
            if not self.n_layers:
                mark("rmsnorm")
                hb.hb_rmsnorm(x, mlp["norm_f"], mlp["eps"], self.normed)
            x = self.normed
        self.final_hidden = x
        if on_call:
            mark("lmhead_argmax")
            hb.hb_lmhead_argmax(x, self.lm_weight, self.target_ids, None, self.ws_lm)
            mark("tree_accept")
            hb.hb_tree_accept(desc.batch, desc.max_nodes_per_tree, dev.node_offset, dev.parent, self.draft_ids,
                              self.target_ids, self.max_path, self.accept_len, self.accept_path, self.out_tokens,
                              self.bonus)
            if compact:
                mark("kv_compact")
                hb.hb_kv_compact_layers(desc, self.n_layers, *self.ptr_tables, dev.block_table, dev.prefix_len,
                                        dev.node_offset, self.accept_len, self.accept_path, self.max_path,
                                        self.out_slots, self.new_len)
            mark("end")
            return
        accept = hb.hb_lmhead_accept_cleared if self.n_layers else hb.hb_lmhead_accept  # no layer, no attention to clear the keys
        accept(desc, x, self.lm_weight, self.draft_ids, dev.node_offset, dev.parent, self.max_path, self.target_ids,
               self.accept_len, self.accept_path, self.out_tokens, self.bonus, self.ws_lm, self.n_layers if compact else 0,
               self.ptr_tables, dev.block_table, dev.prefix_len, self.out_slots, self.new_len)


class PromptLayerStack:
    """Buffers and call chain that take prompts, whole or in parts, through ``n_layers`` decoder layers (those of
    ``VerifyLayerStack``, with the same weights): pages for the new rows, then in each layer the rows' attention over what the cache
    holds and over each other, and their append; at the end each sequence's last row through the LM head.  ``first_ids[b]`` is the token
    that follows the rows by the largest logit, whatever rules the request has (-1: sequence b had none, or no pages); with rules, its
    row of ``final_hidden`` goes through the LM head's projection and ``rules_probs`` instead.  ``desc`` is a batch of at most
    ``desc.total_nodes`` rows; ``row_offset`` may say fewer.  Pools and pages are those that the verification steps go on with.  ``run`` only
    enqueues kernels."""

    def __init__(self, desc: hb.AttnDesc, pages: PagePool, pools, w_qkv, w_o, lm_weight, row_offset, hidden0: torch.Tensor,
                 theta: float = 1e6, mlp=None):
        self.desc, self.pages, self.pools, self.w_qkv, self.w_o, self.lm_weight = desc, pages, pools, w_qkv, w_o, lm_weight
        self.row_offset, self.hidden0, self.theta, self.mlp = row_offset, hidden0, theta, mlp
        d, (T, K), B = hidden0.device, hidden0.shape, desc.batch
        like = lambda *shape: torch.empty(shape, dtype=hidden0.dtype, device=d)
        self.rows = torch.arange(T, dtype=torch.int32, device=d)
        self.cos = torch.empty((T, desc.head_dim // 2), dtype=torch.float32, device=d)
        self.sin = torch.empty_like(self.cos)
        self.q, self.attn_out = like(T, desc.num_q_heads, desc.head_dim), like(T, desc.num_q_heads, desc.head_dim)
        self.k, self.v = like(T, desc.num_kv_heads, desc.head_dim), like(T, desc.num_kv_heads, desc.head_dim)
        self.hidden = [like(T, K), like(T, K)]
        shapes = [(K, w_qkv[0].shape[0]), (w_o[0].shape[1], K)]
        if mlp is not None:
            F = mlp["w_down"][0].shape[1]
            shapes += [(K, 2 * F), (F, K)]
            self.normed, self.mid, self.act = like(T, K), like(T, K), like(T, F)
        self.ws_proj = alloc_workspace(max(hb.hb_proj_workspace_bytes(T, k, n) for k, n in shapes), d)
        self.ws_attn = alloc_workspace(hb.hb_prompt_attn_workspace_bytes(desc), d)
        self.ws_lm = alloc_workspace(max(8, hb.hb_lmhead_argmax_workspace_bytes(B)), d)
        self.ids = torch.empty(B, dtype=torch.int32, device=d)
        self.first_ids = torch.empty_like(self.ids)

    def run(self):
        desc, pages, mlp, offset = self.desc, self.pages, self.mlp, self.row_offset
        T = self.hidden0.shape[0]
        pages.take(offset)
        # a row's position: behind what its sequence has in the cache
        seq = torch.bucketize(self.rows, offset[1:], right=True).clamp_(max=desc.batch - 1)
        hb.hb_rope_table(desc.head_dim, self.theta, self.rows + (pages.length - offset[:-1])[seq], self.cos, self.sin)

        def project(x, w, residual, out, norm):
            if norm is None:
                hb.hb_out_project_ws(x, w, residual, out, self.ws_proj)
            else:
                hb.hb_out_project_norm_ws(x, w, residual, out, norm, mlp["eps"], self.normed, self.ws_proj)

        x, n = self.hidden0, len(self.pools)
        if mlp is not None:
            first = mlp["norm1"][0] if n else mlp.get("norm_f")
            if first is not None:
                hb.hb_rmsnorm(x, first, mlp["eps"], self.normed)
        for l, (kp, vp) in enumerate(self.pools):
            nxt = self.hidden[l & 1]
            y = nxt if mlp is None else self.mid
            hb.hb_qkv_rope_project_ws(x if mlp is None else self.normed, self.w_qkv[l], None, self.cos, self.sin, self.q, self.k, self.v,
                                      self.ws_proj)
            hb.hb_prompt_attn(desc, self.q, self.k, self.v, kp, vp, pages.block_table, pages.length, offset, self.attn_out, None, self.ws_attn)
            hb.hb_kv_append(desc, self.k, self.v, pages.slots, kp, vp)
            project(self.attn_out.view(T, -1), self.w_o[l], x, y, None if mlp is None else mlp["norm2"][l])
            if mlp is not None:
                hb.hb_swiglu_project(self.normed, mlp["w_gate_up"][l], self.act, self.ws_proj)
                project(self.act, mlp["w_down"][l], y, nxt, mlp["norm1"][l + 1] if l + 1 < n else mlp.get("norm_f"))
            x = nxt
        self.final_hidden = self.normed if mlp is not None and mlp.get("norm_f") is not None else x
        hb.hb_lmhead_argmax(self.final_hidden[(offset[1:] - 1).clamp(min=0)], self.lm_weight, self.ids, None, self.ws_lm)
        self.first_ids.copy_(torch.where((offset[1:] > offset[:-1]) & (pages.granted > 0), self.ids, -1))
        pages.advance()
