"""Pages, appends and sampling rules on the GPU against the oracle, and a request's whole way."""
import numpy as np
import pytest
import torch

import workloads as W
from oracle import pages_give_ref, pages_take_ref, rules_logits_ref, rules_probs_ref

pytestmark = pytest.mark.gpu
i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def _pages(seed, B, page, max_rows, max_len, short, reserve, max_blocks=None):
    rng = np.random.default_rng(seed)
    lens, rows = rng.integers(0, max_len + 1, B), rng.integers(0, max_rows + 1, B)
    have = -(-lens // page) + rng.integers(0, 2, B)  # some have a page that they do not use yet
    want = -(-(lens + rows + reserve) // page)
    max_blocks = max_blocks or int(max(have.max(), want.max())) + 1
    need = np.maximum(want - have, 0).sum()
    n_free = int(need * short) if short else int(need) + 7
    blocks = int(have.sum()) + n_free + 5
    order = rng.permutation(blocks)
    table, at = np.full((B, max_blocks), -1), 0
    for b, n in enumerate(have):
        table[b, :min(n, max_blocks)] = order[at:at + min(n, max_blocks)]
        at += n
    have = np.minimum(have, max_blocks)
    lens = np.minimum(lens, have * page)
    free = np.full(blocks, -1)
    free[:n_free] = order[at:at + n_free]
    return dict(B=B, page=page, blocks=blocks, max_blocks=max_blocks, lens=lens, rows=rows, have=have, table=table, free=free, n_free=n_free,
                offset=np.concatenate([[0], np.cumsum(rows)]), reserve=reserve)


def _take(c, extra=3):
    import paper_2509_18824_amd as hb
    T = int(c["offset"][-1])
    got = dict(table=i32(c["table"]), slots=i32([-2] * (T + extra)), new_len=i32([-9] * c["B"]), have=i32([-9] * c["B"]), granted=i32([-9] * c["B"]),
               left=i32([-9]), free=i32(c["free"]))
    hb.hb_pages_take(c["page"], c["reserve"], i32(c["lens"]), i32(c["offset"]), i32(c["have"]), got["free"], i32([c["n_free"]]), got["table"], got["slots"],
                     got["new_len"], got["have"], got["granted"], got["left"])
    return got


@pytest.mark.parametrize("B,page,max_rows,max_len,short,reserve,max_blocks", [
    (1, 16, 1, 0, 0, 0, None), (1, 16, 5000, 100, 0, 8, None), (3, 1, 7, 5, 0, 0, None), (16, 16, 8, 500, 0, 8, None), (16, 16, 100, 0, 0.5, 3, None),
    (64, 7, 60, 200, 0.3, 1, None), (256, 16, 1024, 0, 0.8, 8, None), (300, 32, 40, 400, 0, 0, None), (700, 16, 33, 90, 0.9, 2, 7), (5, 64, 3000, 10, 0, 0, 20),
])
def test_pages_taken_and_given(B, page, max_rows, max_len, short, reserve, max_blocks):
    import paper_2509_18824_amd as hb
    c = _pages(B + page, B, page, max_rows, max_len, short, reserve, max_blocks)
    got = _take(c)
    T = int(c["offset"][-1])
    table, slots, new_len, have, granted, left = pages_take_ref(page, c["max_blocks"], c["blocks"], reserve, c["lens"], c["offset"], c["have"],
                                                                c["free"][:c["n_free"]], c["table"], np.full(T + 3, -2))
    for name, want in (("table", table), ("slots", slots), ("new_len", new_len), ("have", have), ("granted", granted), ("left", [left])):
        assert np.array_equal(got[name].cpu().numpy(), np.asarray(want)), name
    # back again: as it was, and then what is behind shorter lengths
    rng = np.random.default_rng(B)
    for keep in (np.where(granted > 0, c["have"] * page, have * page), rng.integers(-3, c["max_blocks"] * page, B)):
        free, out, now = got["free"].clone(), i32([-9] * B), i32([-9])
        free[left:] = -3
        hb.hb_pages_give(page, i32(keep), got["have"], got["table"], free, got["left"], out, now)
        want, kept = pages_give_ref(page, keep, have, table, c["free"][:left])
        assert np.array_equal(free[:len(want)].cpu().numpy(), want) and (free[len(want):] == -3).all()
        assert np.array_equal(out.cpu().numpy(), kept) and int(now) == len(want)
    assert np.array_equal(got["free"].cpu().numpy(), c["free"])


def test_pages_without_slots_and_malformed():
    import paper_2509_18824_amd as hb
    c = _pages(3, 20, 16, 50, 60, 0, 2)
    want, got = _take(c), _take(c)
    hb.hb_pages_take(16, 2, i32(c["lens"]), i32(c["offset"]), i32(c["have"]), got["free"], i32([c["n_free"]]), got["table"], None, None, got["have"], None,
                     got["left"])
    assert all(torch.equal(got[n], want[n]) for n in want)
    for bad in (dict(lens=c["lens"] + (1 << 30)), dict(lens=c["lens"] - 100), dict(have=c["have"] + 10 ** 6), dict(have=c["have"] - 100),
                dict(n_free=1 << 30), dict(n_free=-4), dict(offset=c["offset"][::-1].copy()), dict(offset=c["offset"] + (1 << 29)), dict(free=c["free"] + 10 ** 8)):
        _take(c | bad, extra=int(c["offset"][-1]))
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype,Hkv,D,page,n", [("bf16", 4, 128, 16, 1), ("bf16", 4, 128, 16, 333), ("f32", 1, 64, 16, 100), ("f32", 3, 8, 5, 17),
                                                ("bf16", 2, 72, 48, 70), ("bf16", 10, 128, 32, 4099), ("f32", 2, 256, 1, 9)])
def test_append(dtype, Hkv, D, page, n):
    import paper_2509_18824_amd as hb
    import paper_2509_18824_amd.step as S
    rng = np.random.default_rng(n)
    blocks = -(-n // page) + 3
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    bits = lambda *s: torch.from_numpy(rng.integers(-2 ** 31, 2 ** 31, (*s[:-1], s[-1] * dt.itemsize // 4), dtype=np.int64).astype(np.int32)).view(dt)
    k, v, kp, vp = bits(n, Hkv, D), bits(n, Hkv, D), bits(blocks, Hkv, page, D), bits(blocks, Hkv, page, D)
    slots = rng.permutation(blocks * page)[:n].astype(np.int32)
    slots[::5] = [[-1, blocks * page, 2 ** 31 - 1][i % 3] for i in range(len(slots[::5]))]
    dev = [t.cuda() for t in (kp, vp)]
    hb.hb_kv_append(S.make_desc(dtype, 1, Hkv, Hkv, D, page, 1, blocks, 0, 1, 1.0), k.cuda(), v.cuda(), torch.from_numpy(slots).cuda(), *dev)
    for r, s in enumerate(slots):
        if 0 <= s < blocks * page:
            kp[s // page, :, s % page], vp[s // page, :, s % page] = k[r], v[r]
    for got, want in zip(dev, (kp, vp)):
        assert torch.equal(got.cpu().view(torch.int32), want.view(torch.int32))


# ---- sampling rules ---------------------------------------------------------------------------------

class Rules:
    def __init__(self, seed, dtype, nodes, V, biases, masks, temps=(0.7, 0.0, 1.3), path=True):
        rng = self.rng = np.random.default_rng(seed)
        self.B, self.nodes, self.V = len(nodes), list(nodes), V
        self.offset = np.concatenate([[0], np.cumsum(nodes)])
        T = self.T = int(self.offset[-1])
        dt = torch.float32 if dtype == "f32" else torch.bfloat16
        self.logits = torch.from_numpy((3 * rng.standard_normal((T, V))).astype(np.float32)).to(dt)
        self.parent = np.concatenate([[-1] + [int(rng.integers(0, i)) for i in range(1, n)] for n in nodes if n] or [[]]).astype(int)
        self.draft = rng.integers(0, min(V, 12), T)
        self.path = path
        self.counts = np.where(rng.random((self.B, V)) < 0.1, rng.integers(1, 5, (self.B, V)), 0) + (rng.random((self.B, V)) < 0.1) * (1 << 30)
        f = lambda lo, hi: rng.uniform(lo, hi, self.B)
        self.rules = np.stack([np.resize(temps, self.B), f(0.8, 1.5), f(-0.2, 0.6), f(-0.2, 0.6)], 1).astype(np.float32)
        self.biases = [[(int(rng.integers(0, V)), float(np.float32(rng.choice([-np.inf, 1.5, -2.25])))) for _ in range(biases)] for _ in range(self.B)]
        words = -(-V // 32)
        self.mask = rng.integers(0, 1 << 32, (masks, words), dtype=np.uint64).astype(np.uint32) if masks else None
        self.mask_row = rng.integers(-1, masks + 1, T) if masks else None

    def args(self):
        b = self.biases
        return (i32(self.offset), i32(self.parent) if self.path else None, i32(self.draft) if self.path else None, i32(self.counts),
                torch.from_numpy(self.rules).cuda(), i32(np.concatenate([[0], np.cumsum([len(x) for x in b])])),
                i32([t for x in b for t, _ in x]), torch.tensor([v for x in b for _, v in x], dtype=torch.float32, device="cuda"),
                torch.from_numpy(self.mask.view(np.int32)).cuda() if self.mask is not None else None,
                i32(self.mask_row) if self.mask_row is not None else None)

    def reference(self):
        z = rules_logits_ref(W.widen(self.logits), self.offset, self.parent if self.path else None, self.draft, self.counts, self.rules, self.biases,
                             self.mask, self.mask_row)
        with np.errstate(over="ignore"):
            return z, rules_probs_ref(z.astype(np.float32).astype(np.float64), self.offset, self.rules)

    def run(self, most=None):
        import paper_2509_18824_amd as hb
        import paper_2509_18824_amd.step as S
        logits, args, most = self.logits.cuda(), self.args(), most or max(self.nodes + [1])
        z, p = torch.full_like(logits, 5.0), torch.full(logits.shape, 5.0, device="cuda")
        hb.hb_rules_logits(logits, most, *args, z)
        ws = S.alloc_workspace(max(16, hb.hb_rules_probs_workspace_bytes(*logits.shape)))
        ws.fill_(255)
        hb.hb_rules_probs(logits, most, *args, p, ws)
        return z, p

    def check(self, z, p, ref=None):
        """z: five float32 operations, 2^-24 each of what they handle (the logit, penalties, the biases), and the rounding to the type.
        p: exp of (z - max) / T off by that of z over T twice, its own rounding, and a sum of V numbers joined pairwise."""
        rz, rp = self.reference() if ref is None else ref
        z, p = W.widen(z)[:self.T], W.widen(p)[:self.T]
        held = W.widen(torch.from_numpy(rz).float().to(self.logits.dtype))  # the type's lowest value times a penalty is beyond it
        same = (np.isneginf(z) == np.isneginf(held)).all() and (np.isposinf(z) == np.isposinf(held)).all()
        assert same
        fin = np.isfinite(held)
        size = np.abs(W.widen(self.logits)[np.isfinite(W.widen(self.logits))]).max(initial=0) * 2 + 6 + 0.6 * 80 + 3 * 8
        half = 2.0 ** -24 if self.logits.dtype == torch.float32 else 2.0 ** -8
        assert (np.abs(z[fin] - rz[fin]) <= 6 * 2.0 ** -24 * size + 1.01 * half * np.abs(rz[fin])).all()
        T = np.repeat(self.rules[:, 0], np.diff(self.offset))
        T = np.where(T > 0, T, 1)[:, None].astype(np.float64)
        rel = 2 * 6 * 2.0 ** -24 * size / T + 40 * 2.0 ** -24
        assert (np.abs(p - rp) <= rel * rp + 1e-37).all(), (np.abs(p - rp) / (rel * rp + 1e-37)).max()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("nodes,V,biases,masks", [([1], 8, 0, 0), ([1], 1, 1, 1), ([8], 1000, 3, 5), ([60, 0, 1], 1000, 40, 9), ([3, 2], 33, 5, 2),
                                                  ([64], 70, 10, 3), ([2] * 70, 257, 2, 20), ([5, 9], 40000, 1500, 3), ([1, 1], 100003, 7, 1), ([2], 65544, 0, 2)])
def test_rules_against_the_oracle(dtype, nodes, V, biases, masks):
    c = Rules(V + len(nodes), dtype, nodes, V, biases, masks)
    c.check(*c.run())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("nodes,V,biases,masks,had", [([60, 60, 60], 1000, 5, 7, 0.1), ([64, 0, 64, 33], 9001, 1100, 3, 0.5), ([1] * 130, 4000, 3, 5, 0.9),
                                                      ([43, 43, 43], 30000, 0, 0, 0.2), ([50, 50, 50], 20004, 2, 4, 0.0), ([44, 43, 43], 262148, 2, 1, 0.01)])
def test_rules_of_many_rows(dtype, nodes, V, biases, masks, had):
    """A workgroup a row: counts of a few tokens and of nearly all, shared by a tree's rows or not; rows that are too long for one."""
    c = Rules(V + len(nodes) + 1, dtype, nodes, V, biases, masks)
    rng = np.random.default_rng(V)
    c.counts = np.where(rng.random(c.counts.shape) < had, rng.integers(1, 4, c.counts.shape), 0) + (rng.random(c.counts.shape) < had / 2) * (1 << 30)
    c.check(*c.run())
    again = c.run()
    assert torch.equal(again[1], c.run()[1])  # the same bits


def test_rules_with_nothing_given():
    import paper_2509_18824_amd as hb
    import paper_2509_18824_amd.step as S
    x = torch.randn((5, 999), device="cuda")
    z, p, ws = torch.empty_like(x), torch.empty_like(x), S.alloc_workspace(hb.hb_rules_probs_workspace_bytes(5, 999))
    none = (None,) * 10
    hb.hb_rules_logits(x, 1, *none, z)
    hb.hb_rules_probs(x, 1, *none, p, ws)
    assert torch.equal(z, x) and (p.double() - torch.softmax(x.double(), 1)).abs().max() <= 1e-6
    hb.hb_rules_logits(x, 1, *none, x)  # in place
    assert torch.equal(z, x)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [64, 1001, 40000])
def test_rows_that_have_nothing_left_infinities_and_nan(dtype, V):
    c = Rules(3, dtype, [4, 4], V, 0, 3, temps=(0.5, 0.0))
    c.mask[:] = 0xffffffff
    c.mask[1] = 0
    c.mask_row = np.array([1, 0, 0, 0, 1, 0, 0, 0])
    inf = float("inf")
    c.logits[1] = -inf
    c.logits[2] = float("nan")
    c.logits[3, 5], c.logits[3, 9] = inf, inf
    c.logits[5] = torch.finfo(c.logits.dtype).min
    c.logits[6, ::2] = float("nan")
    c.logits[7, V - 1] = inf
    c.rules[:, 1:] = [1.25, 0.5, 0.25]
    c.counts[:] = 0
    c.draft[:] = 20
    z, p = c.run()
    c.check(z, p)
    p = W.widen(p)
    assert not p[0].any() and not p[1].any() and not p[2].any() and not p[4].any() and p[3, 5] == 0.5 and p[3, 9] == 0.5 and p[7, V - 1] == 1 and p[5].argmax() == 0


def test_temperatures_at_the_borders():
    V = 5000
    c = Rules(4, "f32", [1] * 7, V, 0, 0, temps=(1e-30, 1e-45, 1e30, float("inf"), -1.0, float("nan"), 1.0))
    c.rules[:, 1:] = [1, 0, 0]
    c.logits[:, 77] = c.logits[:, 4000] = 40.0
    c.logits[2:4, 99] = -float("inf")
    _, p = c.run()
    p = W.widen(p)
    for t in (0, 1):
        assert p[t, 77] == 0.5 and p[t, 4000] == 0.5
    for t in (2, 3):
        assert p[t, 99] == 0 and np.abs(np.delete(p[t], 99) * (V - 1) - 1).max() <= 1e-4
    for t in (4, 5):
        assert p[t, 77] == 1 and p[t].sum() == 1
    assert np.abs(p[6].sum() - 1) < 1e-5


def test_rows_that_nobody_has_and_malformed_trees():
    import paper_2509_18824_amd as hb
    c = Rules(6, "f32", [4, 0, 5], 300, 3, 4)
    c.logits = torch.cat((c.logits, c.logits[:3]))
    for name in ("parent", "draft", "mask_row"):
        setattr(c, name, np.concatenate([getattr(c, name), getattr(c, name)[:3]]))
    z, p = c.run()
    assert (z[9:] == 5).all() and (p[9:] == 5).all()
    c2 = Rules(6, "f32", [4, 0, 5], 300, 3, 4)
    c2.check(z[:9], p[:9])
    for name, value in (("parent", 10 ** 6), ("parent", -9), ("draft", -1), ("draft", 10 ** 9), ("offset", c.offset[::-1].copy()), ("offset", c.offset + 10 ** 8)):
        b = Rules(6, "f32", [4, 0, 5], 300, 3, 4)
        setattr(b, name, np.full_like(getattr(b, name), value) if np.isscalar(value) else value)
        b.run(most=5)
    torch.cuda.synchronize()


def test_equal_largest_values_go_to_the_lowest_token():
    V = 152064
    c = Rules(8, "bf16", [3], V, 0, 0, temps=(0.0,), path=False)
    c.counts[:] = 0
    c.logits[:, [151000, 70001, 70000]] = 50.0
    _, p = c.run()
    assert (p.argmax(1) == 70000).all() and (p.sum(1) == 1).all()


def test_counting():
    import paper_2509_18824_amd as hb
    counts = torch.zeros((3, 50), dtype=torch.int32, device="cuda")
    tokens = i32([[1, 1, 7, -1], [49, 50, 1 << 30, -1], [0, 0, 0, 0]])
    hb.hb_rules_count(tokens, counts)
    hb.hb_rules_count(i32([3, 3, 1, 49]), counts, row_offset=i32([0, 3, 3, 4]), prompt=True)
    want = np.zeros((3, 50), dtype=int)
    want[0, 1], want[0, 7], want[1, 49], want[2, 0] = 2, 1, 1, 4
    want[0, 3] += 1 << 30
    want[0, 1] += 1 << 30
    want[2, 49] += 1 << 30
    assert np.array_equal(counts.cpu().numpy(), want)
    many = torch.randint(0, 50, (3, 5000), dtype=torch.int32, device="cuda")
    counts.zero_()
    hb.hb_rules_count(many, counts)
    assert torch.equal(counts, torch.stack([torch.bincount(m, minlength=50) for m in many]).int())


def test_probabilities_make_the_greedy_rule_of_acceptance():
    """Temperature 0: sampling acceptance over these probabilities accepts what greedy acceptance accepts."""
    import paper_2509_18824_amd as hb
    import paper_2509_18824_amd.step as S
    c = Rules(12, "bf16", [12, 9], 3000, 4, 6, temps=(0.0,))
    _, p = c.run()
    args = c.args()
    target = p.argmax(1).to(torch.int32)
    draft = args[2].clone()
    for b in range(2):  # plant a path
        at = int(c.offset[b])
        node = at
        for n in range(at + 1, int(c.offset[b + 1])):
            if c.parent[n] == node - at:
                draft[n] = target[node]
                node = n
    q = torch.full_like(p, 1.0 / 3000)
    u = lambda n: torch.randint(-2 ** 31, 2 ** 31 - 1, (n,), dtype=torch.int32, device="cuda")
    sampled = S.tree_accept_sample(args[0], args[1], draft, p, q, u(c.T), u(2), 8, 12)
    greedy = S.tree_accept(args[0], args[1], draft, target, 8, 12)
    for a, b in zip(sampled, greedy):
        assert torch.equal(a, b)
