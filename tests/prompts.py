"""Inputs of the tests of prompts, pages and sampling rules, and how far results may be from the oracle's."""
import numpy as np
import torch

import workloads as W
from oracle import prompt_attn_ref


class Prompts:
    """Packed prompts over a paged cache; slots that no sequence owns hold NaN."""

    def __init__(self, seed, dtype, Hq, Hkv, D, page, lens, rows, scale=None, sharp=1.0, spare=0):
        rng = np.random.default_rng(seed)
        self.dtype, self.Hq, self.Hkv, self.D, self.page = dtype, Hq, Hkv, D, page
        self.lens, self.rows, self.B = list(lens), list(rows), len(lens)
        self.scale = D ** -0.5 if scale is None else scale
        self.tdtype = torch.float32 if dtype == "f32" else torch.bfloat16
        r = lambda *shape: torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(self.tdtype)
        used = [-(-n // page) for n in lens]
        self.max_blocks = max(max(used), 1) + spare
        self.num_blocks = sum(used) + 2
        order = rng.permutation(self.num_blocks)
        self.table = np.full((self.B, self.max_blocks), -1, dtype=np.int32)
        self.k_pool, self.v_pool = (torch.full((self.num_blocks, Hkv, page, D), float("nan"), dtype=self.tdtype) for _ in range(2))
        at = 0
        for b, n in enumerate(lens):
            self.table[b, :used[b]] = order[at:at + used[b]]
            at += used[b]
            for p in range(n):
                self.k_pool[self.table[b, p // page], :, p % page] = r(Hkv, D)
                self.v_pool[self.table[b, p // page], :, p % page] = r(Hkv, D)
        self.offset = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
        self.T = int(self.offset[-1])
        self.q = (r(self.T, Hq, D).float() * sharp).to(self.tdtype)
        self.k, self.v = r(self.T, Hkv, D), r(self.T, Hkv, D)

    def desc(self, total=None, **kw):
        import paper_2509_18824_amd.step as S
        return S.make_desc(self.dtype, self.B, self.Hq, self.Hkv, self.D, self.page, self.max_blocks, self.num_blocks,
                           self.T if total is None else total, 1, self.scale, **kw)

    def device(self):
        i = lambda x: torch.from_numpy(np.asarray(x, dtype=np.int32)).cuda()
        return dict(q=self.q.cuda(), k=self.k.cuda(), v=self.v.cuda(), k_pool=self.k_pool.cuda(), v_pool=self.v_pool.cuda(),
                    table=i(self.table), lens=i(self.lens), offset=i(self.offset))

    def run(self, dev=None, lse=True, prefix=True, desc=None, workspace=None, **kw):
        """(out, lse), with a fill that shows what is not written."""
        import paper_2509_18824_amd as hb
        import paper_2509_18824_amd.step as S
        d = self.device() if dev is None else dev
        desc = self.desc(**kw) if desc is None else desc
        out = torch.full_like(d["q"], 7.0)
        ls = torch.full(out.shape[:2], 7.0, dtype=torch.float32, device="cuda") if lse else None
        if workspace is None:
            workspace = S.alloc_workspace(hb.hb_prompt_attn_workspace_bytes(desc))
        if workspace is not None:
            workspace.fill_(255)  # no result may depend on it
        cache = (d["k_pool"], d["v_pool"], d["table"], d["lens"]) if prefix else (None,) * 4
        hb.hb_prompt_attn(desc, d["q"], d["k"], d["v"], *cache, d["offset"], out, ls, workspace)
        return out, ls

    def reference(self, **given):
        w = {n: W.widen(getattr(self, n)) for n in ("q", "k", "v", "k_pool", "v_pool")}
        w.update(given)
        return prompt_attn_ref(w["q"], w["k"], w["v"], w["k_pool"], w["v_pool"], self.table, self.lens, self.offset, self.scale)

    def check(self, out, lse, ref=None, label=""):
        """Element by element.  mass = sum of weight times |value|.
        A score is a sum of D products: in float32, each step off by 2^-24 of a partial sum of magnitudes S, D 2^-24 S at most; on the
        bf16 matrix cores products are exact, and what lies 2^-14 below the largest one may be dropped in a sum of 32.  A weight is off
        by as much as its score, twice (its sum too), by two roundings more, and in bf16 by its own, 2^-8.  Sums of n weights: n 2^-24."""
        ref_out, ref_lse = self.reference() if ref is None else ref
        w = lambda t: np.abs(W.widen(t))
        mass, _ = self.reference(v=w(self.v), v_pool=w(self.v_pool)) if ref is None else (np.abs(ref_out).max() + 4.0, None)
        n = max((a + b for a, b in zip(self.lens, self.rows)), default=0)
        fin = lambda x: np.where(np.isfinite(x), x, 0)
        S = abs(self.scale) * float(np.linalg.norm(fin(w(self.q)), axis=-1).max(initial=0)) * max(
            float(np.linalg.norm(fin(w(x)), axis=-1).max(initial=0)) for x in (self.k, self.k_pool))  # Cauchy and Schwarz
        f32 = self.dtype == "f32"
        ds = S * (self.D * 2.0 ** -24 if f32 else 2.0 ** -14) + 8 * 2.0 ** -24 * (S + 1)
        tol = (2 * ds + (n + 16) * 2.0 ** -24) * mass + (2.0 ** -23 * np.abs(ref_out) if f32 else 2.0 ** -8 * (mass + np.abs(ref_out))) + 1e-30
        got = W.widen(out)
        there = np.zeros(got.shape[0], dtype=bool)
        there[:self.offset[-1]] = True
        far = np.abs(got - ref_out)[there]
        assert np.isfinite(got[there]).all(), label
        assert (far <= np.broadcast_to(tol, got.shape)[there]).all(), f"{label}: {(far / np.broadcast_to(tol, got.shape)[there]).max():.3g} of the tolerance"
        # the sums themselves are near: far less than the worst case in the mean
        rel = np.linalg.norm(far) / max(np.linalg.norm(ref_out), 1e-30)
        assert rel <= (2e-5 if f32 else 1e-2), f"{label}: rel {rel:.3g}"
        if lse is not None:
            off = np.abs(W.widen(lse) - ref_lse)[there].max(initial=0)
            assert off <= ds + (n + 16) * 2.0 ** -24 + 2.0 ** -22 * np.abs(ref_lse).max(initial=0), f"{label}: lse {off:.3g}"
