"""Inputs of the 4-bit cache tests: a verification workload whose pools the oracle has quantised."""
import numpy as np
import torch

import workloads as W
from oracle import kv4_quantise_ref, kv4_values_ref, tree_attn_ref


class Kv4Case:
    """``inp``'s tensors with the pools in 4 bits (numpy: ``pool``; what they stand for: ``k``, ``v``)."""

    def __init__(self, inp):
        self.inp = inp
        self.pool = [x for t in (inp.k_pool, inp.v_pool) for x in kv4_quantise_ref(W.widen(t))]
        self.k, self.v = kv4_values_ref(*self.pool[:2]), kv4_values_ref(*self.pool[2:])
        self.cap = inp.max_blocks * inp.page

    def desc(self, **kw):
        import paper_2509_18824_amd.step as S
        return S.desc_for(self.inp, **kw)

    def device(self):
        f = lambda t: t.cuda().contiguous()
        i = self.inp
        pool = [torch.from_numpy(x).cuda() for x in self.pool]
        return pool, dict(q=f(i.q), k_tree=f(i.k_tree), v_tree=f(i.v_tree), block_table=f(i.block_table), prefix_len=f(i.prefix_len),
                          node_offset=f(i.node_offset), parent=f(i.parent))

    def attend(self, q=None, v=None, k_tree=None, v_tree=None):
        """(out, lse) of the definition."""
        i = self.inp
        w = lambda given, t: W.widen(t) if given is None else given
        return tree_attn_ref(w(q, i.q), w(k_tree, i.k_tree), w(v_tree, i.v_tree), self.k, self.v if v is None else v,
                             i.block_table.numpy(), i.prefix_len.numpy(), i.node_offset.numpy(), i.parent.numpy(), i.softmax_scale)

    def largest_sum(self):
        """Over rows and keys: softmax_scale * sum_d |q_d k_d|, which rounding in a score goes by."""
        i, best = self.inp, 0.0
        q, kt, G = np.abs(W.widen(i.q)), np.abs(W.widen(i.k_tree)), i.Hq // i.Hkv
        for b in range(i.B):
            n0, n1, p = int(i.node_offset[b]), int(i.node_offset[b + 1]), np.arange(int(i.prefix_len[b]))
            k = np.abs(self.k[i.block_table.numpy()[b, p // i.page], :, p % i.page])
            for g in range(i.Hkv):
                keys = np.concatenate([k[:, g], kt[n0:n1, g]])
                if n1 > n0:
                    best = max(best, float((q[n0:n1, g * G:(g + 1) * G].reshape(-1, i.D) @ keys.T).max()))
        return abs(i.softmax_scale) * best

    def check_attention(self, out, lse, ref=None, label=""):
        """Against the definition, element by element.  float32: sums of D products and of the keys, 2^-24 each, on average far
        less: 1e-5 of sum p |v| and 4 * 2^-24 * sqrt(D) * sum |q k| in a score.  bf16: probabilities and results are rounded
        to 2^-9 of themselves; the matrix cores drop what lies 2^-14 below the largest product of a score."""
        ref_out, ref_lse = self.attend() if ref is None else ref
        mass, _ = self.attend(v=np.abs(self.v), v_tree=np.abs(W.widen(self.inp.v_tree)))
        got, got_lse, f32 = W.widen(out), W.widen(lse), self.inp.dtype == "f32"
        ds = self.largest_sum() * (4 * 2.0 ** -24 * self.inp.D ** 0.5 if f32 else 2.0 ** -14) + 1e-6
        tol = 2 * ds * mass + (1e-5 * mass if f32 else 2.0 ** -9 * np.abs(ref_out) * 1.01 + 2.0 ** -9 * mass) + 1e-30
        far = np.abs(got - ref_out)
        assert np.isfinite(got).all(), label
        assert (far <= tol).all(), f"{label}: {(far / tol).max():.3g} of the tolerance"
        lse_far = np.abs(got_lse - ref_lse).max()
        assert lse_far <= ds + 4e-6 * (1 + np.abs(ref_lse).max()), f"{label}: lse {lse_far:.3g}, {ds:.3g}"


def mixed_case(seed, dtype, Hq, Hkv, D, page, lens, nodes, **kw):
    trees = [W.chain_tree(n) if n < 12 else W.seeded_tree(seed + n, n_nodes=n, levels=min(6, n - 9), root_fanout=10) for n in nodes]
    return Kv4Case(W.make_verify_inputs(seed, dtype, Hq, Hkv, D, lens, trees, page=page, **kw))
